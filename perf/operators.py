"""The operators that a decoding loop runs beside the eviction pass, as cases that can be timed and compared.

Each case is one pass through one operator. With ``own`` the pass is the call that a user makes of the torch
layer (``paper_2609_08131_gb300.api``); without it the same formulas in elementary torch operations:

  rope    queries and keys turned by their tokens' positions           Rope.apply
  attend  drafted tokens (a chain or a tree; one token: an ordinary    CacheAttention.run
          decode step) over the cached tokens of each request
  weigh   the attention weight that each cached token received from    WeightEvictor.score
          a window of queries, alone or on top of earlier weights
  evict   the budget kept by those weights, first and last tokens      WeightEvictor.select_compact
          protected; rows and weights of the kept tokens copied out

Fields of a case: ``op``; ``layers``, ``hq``, ``hkv`` (query and KV heads); ``requests`` and ``n``, tokens of
each request's slot; ``live`` (attend), the cached tokens of each request as a text; ``drafts`` (attend) or
``window`` (weigh), queries per request; ``tree`` (attend), a tree of drafted tokens instead of a chain;
``given`` (weigh), the softmax normalisers known from the attention call and earlier weights to add to;
``budget``, ``sinks``, ``recent`` (evict); ``tokens`` (rope), tokens per request, ``first``, the largest
position of a request's first token, ``rot``, ``interleaved``, ``scaling``; ``dtype``, "bf16" or "f32".
"""

import math
import random

import torch

own = False

D = 128
_HEADS = ((32, 8), (32, 8), (40, 8), (28, 4), (8, 8), (16, 8), (12, 2), (8, 1))  # Llama-3-8B, Qwen3-14B, Nemotron-7B, ...


def _rope(name, requests, tokens, hq, hkv, first, rot=D, interleaved=False, scaling="none", dtype="bf16"):
    c = {"op": "rope", "requests": requests, "tokens": tokens, "hq": hq, "hkv": hkv, "first": first, "rot": rot,
         "interleaved": interleaved, "scaling": scaling, "dtype": dtype}
    return {"name": name, **c} if name else c


def _attend(name, hq, hkv, n, live, drafts, tree=False, dtype="bf16"):
    c = {"op": "attend", "layers": 1, "hq": hq, "hkv": hkv, "requests": len(live), "n": n,
         "live": " ".join(str(x) for x in live), "drafts": drafts, "tree": tree, "dtype": dtype}
    return {"name": name, **c} if name else c


def _weigh(name, layers, hq, hkv, requests, n, window, given=False, dtype="bf16"):
    c = {"op": "weigh", "layers": layers, "hq": hq, "hkv": hkv, "requests": requests, "n": n, "window": window,
         "given": given, "dtype": dtype}
    return {"name": name, **c} if name else c


def _evict(name, layers, hkv, requests, n, budget, sinks, recent, dtype="bf16"):
    c = {"op": "evict", "layers": layers, "hq": hkv, "hkv": hkv, "requests": requests, "n": n, "budget": budget,
         "sinks": sinks, "recent": recent, "dtype": dtype}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the new token of four requests, far into a long context: nothing but latency
        _rope("rope_step_4_requests", 4, 1, 32, 8, 131000, scaling="llama3"),
        # a long prompt's queries and keys of one layer
        _rope("rope_prompt_32k", 1, 32768, 32, 8, 0, scaling="yarn"),
        # one request, one token, a short cache: the smallest attention call
        _attend("attend_1_short", 32, 8, 640, (37,), 1),
        # a decode step of sixteen requests whose slots hold 2048 tokens and up to 128 more
        _attend("attend_16_slots", 32, 8, 2176, (2048, 2175, 2100, 2057, 2144, 2090, 2171, 2063, 2119, 2050, 2150,
                                                 2081, 2134, 2167, 2072, 2099), 1),
        # eight drafted tokens, one after another, over a whole document of 128K tokens
        _attend("attend_long_chain", 32, 8, 131072, (131011,), 8),
        # trees of 64 drafted tokens for sixteen requests of very different lengths, five query heads per KV head
        _attend("attend_16_trees", 40, 8, 16384, (6231, 987, 2304, 16383, 9020, 3391, 9600, 12502, 5111, 4097, 511, 13873,
                                                  7449, 2999, 46, 10533), 64, tree=True),
        # float32, multi-head, a short tree: a model evaluated in float32
        _attend("attend_f32_tree", 8, 8, 4096, (4096, 1377), 5, tree=True, dtype="f32"),
        # the prompt of one layer right after its prefill, an odd length
        _weigh("weigh_layer_4k", 1, 32, 8, 1, 4099, 32),
        # eight layers of a prompt of 32K tokens
        _weigh("weigh_8_layers_32k", 8, 32, 8, 1, 32768, 32),
        # after a decode step that took four drafted tokens: all layers' weights brought up to date, with the
        # normalisers that the attention calls returned
        _weigh("weigh_step_8_slots", 28, 28, 4, 8, 2176, 4, given=True),
        # one layer of a short prompt cut to its budget
        _evict("evict_layer_4k", 1, 8, 1, 4099, 512, 4, 32),
        # a whole model's cache of four prompts cut to a tenth
        _evict("evict_4_prompts_16k", 32, 8, 4, 16384, 1638, 4, 64),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "attend", "attend", "attend", "weigh", "weigh", "evict"))
    hq, hkv = rng.choice(_HEADS)
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if op == "rope":
        requests = rng.choice((1, 1, 2, 5, 16, 64))
        tokens = _between(rng, 1, 16384 // requests)
        return _rope("", requests, tokens, hq, hkv, _between(rng, 1, 131072 - tokens),
                     rot=rng.choice((128, 128, 64, 32, 96, 50, 20)), interleaved=rng.random() < 0.5,
                     scaling=rng.choice(("none", "linear", "ntk", "llama3", "yarn")), dtype=dtype)
    if op == "attend":
        requests = rng.choice((1, 1, 2, 3, 8, 16, 32))
        drafts = rng.choice((1, 1, 1, 2, 3, 5, 8, 13, 25, 33, 48, 64))
        longest = _between(rng, 1, min(131072, 262144 // requests // (4 if dtype == "f32" else 1)) // (1 + drafts // 9))
        live = [longest] + [max(1, int(longest * rng.uniform(0.05, 1.0))) for _ in range(requests - 1)]
        return _attend("", hq, hkv, longest + rng.choice((0, 1, 64, 128)), live, drafts,
                       tree=drafts > 1 and rng.random() < 0.6, dtype=dtype)
    if op == "weigh":
        given = rng.random() < 0.4
        requests = rng.choice((1, 2, 4, 8)) if given else rng.choice((1, 1, 2, 3))
        window = rng.choice((1, 2, 3, 5, 8)) if given else rng.choice((8, 16, 20, 32, 32, 64))
        layers = rng.choice((1, 2, 4, 8))
        n = _between(rng, max(window, 16), 131072 // requests // layers // (4 if dtype == "f32" else 1))
        return _weigh("", layers, hq, hkv, requests, n, window, given=given, dtype=dtype)
    layers, requests = rng.choice((1, 2, 8, 16)), rng.choice((1, 2, 4))
    n = _between(rng, 64, 400000 // requests // layers)
    budget = _between(rng, 32, max(33, n // 2))
    return _evict("", layers, hkv, requests, n, budget, rng.choice((0, 0, 4)), rng.choice((0, 1, 16)), dtype=dtype)


# ----------------------------------------------------------------- inputs ----
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# base, and the arguments of each kind of scaling: (kind, factor, original length, ...)
_SCALINGS = {"none": (10000.0, None), "linear": (10000.0, ("linear", 4.0)), "ntk": (10000.0, ("ntk", 4.0)),
             "llama3": (500000.0, ("llama3", 8.0, 1.0, 4.0, 8192)), "yarn": (1000000.0, ("yarn", 4.0, 32768, 32.0, 1.0))}


def _frequencies(rot, scaling):
    """The pairs' angles per position in 64 bits, and the factor on sine and cosine."""
    base, how = _SCALINGS[scaling]
    if scaling == "ntk":
        base = base * how[1] ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaling == "linear":
        return f / how[1], 1.0
    if scaling == "llama3":  # long wavelengths divided, short ones kept, a ramp between
        _, factor, low, high, length = how
        s = ((length * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return f * (s + (1 - s) / factor), 1.0
    if scaling == "yarn":  # the same by the number of turns over the original length, linear in the pair's number
        _, factor, length, fast, slow = how
        at = [rot * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (fast, slow)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        s = 1 - ((torch.arange(rot // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (s + (1 - s) / factor), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _prepare_rope(case, seed):
    g, S, T = _generator(seed), case["requests"], case["tokens"]
    q = torch.randn(S, T, case["hq"], D, generator=g, device="cuda").to(_type(case))
    k = torch.randn(S, T, case["hkv"], D, generator=g, device="cuda").to(_type(case))
    first = torch.randint(0, case["first"] + 1, (S, 1), generator=g, device="cuda")
    positions = (first + torch.arange(T, device="cuda")).to(torch.int32)
    freq, amplitude = _frequencies(case["rot"], case["scaling"])
    return {"case": case, "q": q, "k": k, "positions": positions, "freq": freq.cuda(), "amplitude": amplitude}


def _cache(case, seed):
    """Keys and values of slots of n tokens, [L, Hkv, S n, 128]: per-channel scales, and first tokens that draw
    the attention of every query. Returns those tokens' direction too."""
    g, L, Hkv, S, n = _generator(seed), case["layers"], case["hkv"], case["requests"], case["n"]
    scale = torch.exp(0.5 * torch.randn(2, L, Hkv, 1, 1, D, generator=g, device="cuda"))
    k = scale[0] * torch.randn(L, Hkv, S, n, D, generator=g, device="cuda")
    v = scale[1] * torch.randn(L, Hkv, S, n, D, generator=g, device="cuda")
    toward = torch.randn(L, Hkv, D, generator=g, device="cuda") / math.sqrt(D)
    k[:, :, :, :4] += 4.0 * math.sqrt(D) * toward[:, :, None, None]
    return k.to(_type(case)).view(L, Hkv, S * n, D), v.to(_type(case)).view(L, Hkv, S * n, D), toward, g


def _queries(case, toward, g, count):
    G = case["hq"] // case["hkv"]
    q = torch.randn(case["requests"], case["layers"], case["hq"], count, D, generator=g, device="cuda")
    return (q + 8.0 * toward.repeat_interleave(G, dim=1)[None, :, :, None]).to(_type(case))


def _starts(case):
    return torch.arange(0, (case["requests"] + 1) * case["n"], case["n"], dtype=torch.int32, device="cuda")


def _prepare_attend(case, seed):
    k, v, toward, g = _cache(case, seed)
    S, T = case["requests"], case["drafts"]
    state = {"case": case, "k": k, "v": v, "q": _queries(case, toward, g, T), "starts": _starts(case), "tree": None,
             "live": torch.tensor([int(x) for x in case["live"].split()], dtype=torch.int32, device="cuda")}
    drafts = torch.randn(2, S, case["layers"], case["hkv"], T, D, generator=g, device="cuda").to(_type(case))
    state["k_draft"], state["v_draft"] = drafts[0], drafts[1]
    if case["tree"]:  # bit j of a token's mask: it descends from drafted token j, or is it
        rng, masks = random.Random(seed), []
        for _ in range(S):
            row = []
            for t in range(T):
                parent = rng.randint(max(-1, t - 9), t - 1)
                row.append((row[parent] if parent >= 0 else 0) | 1 << t)
            masks.append([m - (1 << 64) if m >> 63 else m for m in row])
        state["tree"] = torch.tensor(masks, dtype=torch.int64, device="cuda")
    return state


def _prepare_weigh(case, seed):
    k, v, toward, g = _cache(case, seed)
    q = _queries(case, toward, g, case["window"])
    state = {"case": case, "k": k, "v": v, "q": q, "starts": _starts(case), "lse": None, "before": None}
    if case["given"]:
        state["before"] = 0.1 * torch.rand(k.shape[:3], generator=g, device="cuda")
        state["lse"] = _logits(case, q, k).logsumexp(-1).view(q.shape[1], case["hkv"], case["requests"], -1,
                                                              case["window"])
        state["lse"] = state["lse"].permute(2, 0, 1, 3, 4).reshape(q.shape[:4]).contiguous()
    return state


def _prepare_evict(case, seed):
    k, v, _, g = _cache(case, seed)
    # weights as attention leaves them: a few tokens hold most, many equal to nothing
    weights = torch.exp(3.0 * torch.randn(k.shape[:3], generator=g, device="cuda") - 6.0)
    weights[torch.rand(k.shape[:3], generator=g, device="cuda") < 0.05] = 0.0
    return {"case": case, "k": k, "v": v, "weights": weights, "starts": _starts(case)}


def prepare(case, seed):
    return {"rope": _prepare_rope, "attend": _prepare_attend, "weigh": _prepare_weigh,
            "evict": _prepare_evict}[case["op"]](case, seed)


# ------------------------------------------------------------ plain forms ----
def _plain_rope(state):
    case, rot = state["case"], state["case"]["rot"]
    angle = (state["positions"].double()[..., None] * state["freq"])[:, :, None]
    cos, sin = (state["amplitude"] * angle.cos()).float(), (state["amplitude"] * angle.sin()).float()

    def turn(x):
        y = x.float()
        if case["interleaved"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)

    return {"q": turn(state["q"]), "k": turn(state["k"])}


def _rows(case, x):
    """[L, Hkv, S n, 128] or [S, L, Hkv, n, 128] as float [S, L, Hkv, n, 128]."""
    if x.dim() == 4:
        x = x.view(x.shape[0], x.shape[1], case["requests"], case["n"], D).permute(2, 0, 1, 3, 4)
    return x.float()


def _plain_attend(state):
    case, q = state["case"], state["q"]
    S, L, Hq, T, _ = q.shape
    Hkv, n, dev = case["hkv"], case["n"], q.device
    k = torch.cat([_rows(case, state["k"]), state["k_draft"].float()], 3)
    v = torch.cat([_rows(case, state["v"]), state["v_draft"].float()], 3)
    s = (q.float().view(S, L, Hkv, -1, D) @ k.mT).view(S, L, Hkv, -1, T, n + T) / math.sqrt(D)
    cached = (torch.arange(n, device=dev) < state["live"][:, None])[:, None].expand(S, T, n)
    bit = torch.arange(T, device=dev)
    if state["tree"] is None:
        drafted = (bit <= bit[:, None]).expand(S, T, T)
    else:
        drafted = (state["tree"][..., None] >> bit & 1).bool()
    s = s.masked_fill(~torch.cat([cached, drafted], 2)[:, None, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = (p.view(S, L, Hkv, -1, n + T) @ v).view(S, L, Hkv, -1, T, D) / total
    return {"o": o.view(S, L, Hq, T, D).to(q.dtype), "lse": (top + total.log()).view(S, L, Hq, T)}


def _logits(case, q, k):
    """[L, Hkv, S, G w, n] logits of the window's queries; a token after a query's own is masked."""
    S, L, Hq, w, _ = q.shape
    n = case["n"]
    qs = q.float().view(S, L, case["hkv"], -1, D).permute(1, 2, 0, 3, 4)
    s = (qs @ k.float().view(L, case["hkv"], S, n, D).mT) / math.sqrt(D)
    late = torch.arange(n, device=q.device) > (n - w + torch.arange(w, device=q.device))[:, None]
    return s.view(L, case["hkv"], S, -1, w, n).masked_fill_(late, -math.inf).view(s.shape)


def _plain_weigh(state):
    case, q = state["case"], state["q"]
    S, L, Hq, w, _ = q.shape
    Hkv, n = case["hkv"], case["n"]
    s = _logits(case, q, state["k"])
    if state["lse"] is None:
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        weights = (p / total).sum(-2).view(L, Hkv, S * n)
        lse = (top + total.log()).view(L, Hkv, S, -1, w).permute(2, 0, 1, 3, 4).reshape(S, L, Hq, w)
        return {"weights": weights, "lse": lse}
    lse = state["lse"].view(S, L, Hkv, -1).permute(1, 2, 0, 3)[..., None]
    old = (torch.arange(n, device=q.device) < n - w) * state["before"].view(L, Hkv, S, n)
    return {"weights": (old + torch.exp(s - lse).sum(-2)).view(L, Hkv, S * n), "lse": None}


def _bits(x):
    """Copied rows are compared as the whole numbers that their bytes are."""
    return x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)


def _plain_evict(state):
    case = state["case"]
    L, Hkv, S, n, B = case["layers"], case["hkv"], case["requests"], case["n"], case["budget"]
    dev, kept = state["k"].device, min(case["budget"], case["n"])
    w = state["weights"].view(L, Hkv, S, n)
    at = torch.arange(n, device=dev)
    order = w.masked_fill((at < case["sinks"]) | (at >= n - case["recent"]), math.inf)
    idx = order.sort(dim=-1, descending=True, stable=True).indices[..., :kept].sort(dim=-1).values

    def rows(x):
        x = x.view(L, Hkv, S, n, -1)
        out = torch.zeros(L, Hkv, S, B, x.shape[-1], dtype=x.dtype, device=dev)
        out[..., :kept, :] = x.gather(3, idx[..., None].expand(-1, -1, -1, -1, x.shape[-1]))
        return out

    listed_idx = torch.full((L, Hkv, S, B), -1, dtype=torch.int32, device=dev)
    listed_idx[..., :kept] = idx
    return {"idx": listed_idx, "kept": torch.full((S,), kept, dtype=torch.int32, device=dev),
            "k_out": _bits(rows(state["k"])), "v_out": _bits(rows(state["v"])),
            "w_out": _bits(rows(state["weights"])[..., 0])}


# ------------------------------------------------- the framework's operators ----
def _kept(state, make):
    """What a user's program makes once and keeps: the plan, the workspace and the output buffers."""
    if "handle" not in state:
        from paper_2609_08131_gb300 import api
        state["handle"] = make(api)
    return state["handle"]


def _slots(api, state, q):
    case = state["case"]
    return api.Cache(q, state["k"], state["v"], state["starts"], [case["n"]] * case["requests"], case["hq"])


def _own_rope(state):
    case = state["case"]
    base, how = _SCALINGS[case["scaling"]]
    rope = _kept(state, lambda api: api.Rope(case["rot"], base=base, interleaved=case["interleaved"], scaling=how))
    q, k = rope.apply(state["q"], state["k"], state["positions"])
    return {"q": q, "k": k}


def _own_attend(state):
    att = _kept(state, lambda api: api.CacheAttention(_slots(api, state, state["q"])))
    o, lse = att.run(lengths=state["live"], k_draft=state["k_draft"], v_draft=state["v_draft"], tree=state["tree"])
    return {"o": o, "lse": lse}


def _own_weigh(state):
    ev = _kept(state, lambda api: api.WeightEvictor(_slots(api, state, state["q"]), 1))
    weights, lse = ev.score(lse=state["lse"], before=state["before"])
    return {"weights": weights, "lse": lse if state["lse"] is None else None}


def _own_evict(state):
    case = state["case"]

    def make(api):
        q = torch.zeros(case["requests"], case["layers"], case["hq"], 1, D, dtype=_type(case), device="cuda")
        return api.WeightEvictor(_slots(api, state, q), case["budget"], sinks=case["sinks"], recent=case["recent"])

    ev = _kept(state, make)
    ev.select_compact(weights=state["weights"])
    return {"idx": ev.idx, "kept": ev.kept, "k_out": _bits(ev.k_out), "v_out": _bits(ev.v_out),
            "w_out": _bits(ev.weights_out)}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"rope": _own_rope, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict}[op](state)
    return {"rope": _plain_rope, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[op](state)


# ------------------------------------------------------------------- work ----
def work(case):
    """Every input read once and every output written once; the logits once, and the values' sums (attend). A masked
    pair of a query and a token is no work."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rope":
        tokens, heads = case["requests"] * case["tokens"], case["hq"] + case["hkv"]
        return {"bytes": tokens * (2 * heads * D * es + 4), "flops": tokens * heads * case["rot"] * 3}
    L, S, Hq, Hkv, n = case["layers"], case["requests"], case["hq"], case["hkv"], case["n"]
    if case["op"] == "attend":
        live, T = sum(int(x) for x in case["live"].split()), case["drafts"]
        nbytes = L * ((live + S * T) * Hkv * 2 * D * es + 2 * S * Hq * T * D * es + S * Hq * T * 4)
        if case["tree"]:
            nbytes += S * T * 8
        return {"bytes": nbytes, "flops": L * Hq * (live * T + S * T) * 4 * D}
    if case["op"] == "weigh":
        w = case["window"]
        nbytes = L * (S * n * Hkv * (D * es + 4) + S * Hq * w * (D * es + 4)) + (L * S * n * Hkv * 4 if case["given"] else 0)
        return {"bytes": nbytes, "flops": L * S * Hq * (w * n - w * (w - 1) // 2) * 2 * D}
    units, kept = L * Hkv * S, min(case["budget"], n)
    return {"bytes": units * (4 * n + kept * (2 * 2 * D * es + 4) + case["budget"] * 4), "flops": units * n}


# ------------------------------------------------------------------ exact ----
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "evict":
        return None
    if case["op"] == "rope":
        freq, amplitude = _frequencies(case["rot"], case["scaling"])
        turn = amplitude * torch.exp(1j * state["positions"].double()[..., None] * freq.cuda())

        def turned(x):
            y, rot = x.double(), case["rot"]
            part = y[..., :rot]
            pairs = part.unflatten(-1, (-1, 2)) if case["interleaved"] else part.unflatten(-1, (2, -1)).mT
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, :, None])
            y[..., :rot] = (z if case["interleaved"] else z.mT).flatten(-2)
            return y

        return {"q": turned(state["q"]), "k": turned(state["k"])}
    q, n, G = state["q"], case["n"], case["hq"] // case["hkv"]
    S, L, Hq, T, _ = q.shape
    lse = torch.empty(S, L, Hq, T, dtype=torch.float64, device=q.device)
    if case["op"] == "attend":
        o = torch.empty(S, L, Hq, T, D, dtype=torch.float64, device=q.device)
        lives = [int(x) for x in case["live"].split()]
        for s in range(S):
            seen = [[True] * (t + 1) + [False] * (T - t - 1) for t in range(T)]
            if state["tree"] is not None:
                seen = [[bool(m >> j & 1) for j in range(T)] for m in state["tree"][s].tolist()]
            hidden = ~torch.tensor(seen, device=q.device)
            for l in range(L):
                for g in range(case["hkv"]):
                    at, h = slice(s * n, s * n + lives[s]), slice(g * G, (g + 1) * G)
                    ks = torch.cat([state["k"][l, g, at], state["k_draft"][s, l, g]]).double()
                    vs = torch.cat([state["v"][l, g, at], state["v_draft"][s, l, g]]).double()
                    x = q[s, l, h].double() @ ks.T / math.sqrt(D)
                    x[..., lives[s]:][hidden.expand(G, T, T)] = -math.inf
                    lse[s, l, h] = torch.logsumexp(x, -1)
                    o[s, l, h] = torch.softmax(x, -1) @ vs
        return {"o": o, "lse": lse}
    weights = torch.empty(state["k"].shape[:3], dtype=torch.float64, device=q.device)
    for l in range(L):
        for g in range(case["hkv"]):
            for s in range(S):
                at, h = slice(s * n, (s + 1) * n), slice(g * G, (g + 1) * G)
                x = q[s, l, h].double() @ state["k"][l, g, at].double().T / math.sqrt(D)
                x[..., n - T:] += torch.full((T, T), -math.inf, dtype=torch.float64, device=q.device).triu(1)
                lse[s, l, h] = torch.logsumexp(x, -1) if not case["given"] else state["lse"][s, l, h].double()
                weights[l, g, at] = torch.exp(x - lse[s, l, h][..., None]).sum((0, 1))
                if case["given"]:
                    weights[l, g, s * n:(s + 1) * n - T] += state["before"][l, g, s * n:(s + 1) * n - T].double()
    return {"weights": weights, "lse": None if case["given"] else lse}
