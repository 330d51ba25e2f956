"""GPU tests of the decoding loop's operators (rotary positions, attention of drafted tokens, weights received,
eviction by weights) against plain implementations in 64 bits.

Tolerances are bounds, from the roundings of each path (a rounding is off by half a step: 2^-24 relative in float32,
2^-8 in bf16):

* a logit is a sum of 128 products: |error| <= 136 2^-24 scale sum_c |q_c k_c| (the products, the additions - the
  tensor cores' truncate, a whole step each, but in blocks of 16 - and the scaling), so a softmax weight is off by
  twice that relative, plus 2^-20 for the exponential at its argument and the sums (float32, a few hundred terms at a
  time);
* an output adds the weights' roundings to bf16 (bf16 caches), 2^-8 of sum p |v|, and its own.
"""

import math

import pytest
import torch

import paper_2609_08131_gb300.api as api
from paper_2609_08131_gb300 import JACAP_ATTEND_ZERO_BYTES, JACAP_ERR_INVALID_ARG, JACAP_ERR_NONFINITE

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
D = 128
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
SCALE = 1 / math.sqrt(D)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def within(got, want, tol, what):
    got, tol = got.double(), torch.as_tensor(tol, dtype=torch.float64, device=got.device)
    assert got.shape == want.shape, what
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN in other places"
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]) and not got[~inf].isinf().any(), f"{what}: infinities in other places"
    fine = want.isfinite()
    off = ((got - want).abs() - tol)[fine]
    assert off.numel() == 0 or off.max() <= 0, f"{what}: {(off > 0).sum()} of {off.numel()} out of bounds, by {off.max():.3e}"


# ------------------------------------------------------------------- rope ----
def rope_plain(x, positions, freq, amplitude, rot, interleaved, inverse):
    """The turned x in 64 bits and its bound."""
    angle = positions.double()[..., None] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    if inverse:
        angle = -angle
    c, s = (amplitude * angle.cos())[..., None, :], (amplitude * angle.sin())[..., None, :]
    y, tol = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x.double()[..., at[0]], x.double()[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    # sine and cosine: 2^-23 by sincospif, 2^-25 by the turn's rounding, 2^-24 by the amplitude; 2^-24 for each product
    # and the sum
    tol[..., at[0]] = tol[..., at[1]] = (a.abs() + b.abs()) * amplitude * 2.0 ** -21.5
    return y, tol + y.abs() * (HALF[x.dtype] if x.dtype == BF16 else 0.0)


ROPES = [(128, False, None), (128, True, None), (64, False, ("linear", 4.0)), (96, True, ("ntk", 2.0)), (2, True, None),
         (50, False, ("llama3", 8.0, 1.0, 4.0, 8192)), (20, True, ("yarn", 4.0, 32768, 32.0, 1.0)), (6, False, None),
         (32, False, ("yarn", 16.0, 4096, 32.0, 1.0)), (16, False, None), (8, True, None)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rot,interleaved,scaling", ROPES)
def test_rope_against_64_bits(rot, interleaved, scaling, dtype):
    rope = api.Rope(rot, base=10000.0, interleaved=interleaved, scaling=scaling, device=DEV)
    freq, amplitude = api.rope_frequencies(rot, 10000.0, scaling)
    g = gen(rot)
    for lead, hq, hkv in (((1,), 1, 1), ((3, 7), 8, 2), ((2, 130), 5, 5), ((1300,), 28, 4), ((0, 4), 2, 2)):
        q, k = randn(g, *lead, hq, D, dtype=dtype), randn(g, *lead, hkv, D, dtype=dtype)
        positions = torch.randint(-5, 1 << 20, lead, generator=g, device=DEV, dtype=torch.int32)
        if positions.numel():
            positions.view(-1)[0] = 2 ** 31 - 1
            positions.view(-1)[-1] = 0
        for inverse in (False, True):
            for got, x in zip(rope.apply(q, k, positions, inverse=inverse), (q, k)):
                want, tol = rope_plain(x, positions, freq, amplitude, rot, interleaved, inverse)
                within(got, want, tol, f"rope {lead}")
                assert torch.equal(got[..., rot:], x[..., rot:])


def test_rope_strides_in_place_and_one_tensor():
    g, rope = gen(5), api.Rope(64, device=DEV)
    freq, amplitude = api.rope_frequencies(64)
    wide = randn(g, 3, 6, 9, 2 * D + 8, dtype=BF16)
    positions = torch.arange(27, device=DEV, dtype=torch.int32).view(9, 3).t()
    # [requests, heads, tokens, 128] turned around, rows inside wider ones; aligned and not
    for x in (wide[..., :D].transpose(1, 2), wide[..., 1:D + 1].transpose(1, 2), wide[:, :, :, 8:8 + D].transpose(1, 2)):
        want, tol = rope_plain(x, positions, freq, amplitude, 64, False, False)
        q, k = rope.apply(x, None, positions)
        assert k is None
        within(q, want, tol, "strided")
        within(rope.apply(None, x, positions)[1], want, tol, "strided keys")
    before = wide.clone()
    x = wide[..., 1:D + 1].transpose(1, 2)
    assert rope.apply(x, None, positions, inplace=True)[0] is x
    within(x, want_of(before, positions, freq, amplitude), tol_of(before, positions, freq, amplitude), "in place")
    outside = torch.ones_like(wide, dtype=torch.bool)
    outside[..., 1:D + 1] = False
    assert torch.equal(wide[outside], before[outside])
    # a key head shared by every query head: read with stride 0
    shared = randn(g, 5, 1, D).expand(5, 4, D)
    at = torch.arange(5, device=DEV, dtype=torch.int32)
    want, tol = rope_plain(shared, at, freq, amplitude, 64, False, False)
    within(rope.apply(shared, None, at)[0], want, tol, "shared head")
    with pytest.raises(api.JacapError):
        rope.apply(shared, None, at, inplace=True)


def want_of(before, positions, freq, amplitude):
    return rope_plain(before[..., 1:D + 1].transpose(1, 2), positions, freq, amplitude, 64, False, False)[0]


def tol_of(before, positions, freq, amplitude):
    return rope_plain(before[..., 1:D + 1].transpose(1, 2), positions, freq, amplitude, 64, False, False)[1]


def test_threads_share_a_rope():
    from concurrent.futures import ThreadPoolExecutor
    rope, g = api.Rope(device=DEV), gen(5)
    data = [(randn(g, 64, 4, D, dtype=BF16), torch.randint(0, 9000, (64,), generator=g, device=DEV, dtype=torch.int32))
            for _ in range(8)]
    want = [rope.apply(x, None, at)[0] for x, at in data]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream(device=DEV)):
            got = [rope.apply(*data[i][:1], None, data[i][1])[0] for _ in range(200)]
            torch.cuda.current_stream().synchronize()
        return all(torch.equal(x, want[i]) for x in got)

    with ThreadPoolExecutor(8) as pool:
        assert all(pool.map(work, range(8)))


def test_rope_turns_back_and_is_its_own_gradient():
    g, rope = gen(6), api.Rope(128, interleaved=True, device=DEV)
    x, y = randn(g, 50, 3, D), randn(g, 50, 3, D)
    at = torch.randint(0, 1 << 17, (50,), generator=g, device=DEV, dtype=torch.int32)
    there = rope.apply(x, None, at)[0]
    back = rope.apply(there, None, at, inverse=True)[0]
    assert (back - x).abs().max() <= 4 * x.abs().max() * 2.0 ** -21.5
    # d/dx <turn(x), y> = turn back(y): the map is linear, so a difference of any size is exact but for rounding
    step = randn(g, 50, 3, D)
    lhs = ((rope.apply(x + step, None, at)[0].double() - there.double()) * y.double()).sum()
    rhs = (step.double() * rope.apply(y, None, at, inverse=True)[0].double()).sum()
    bound = 2.0 ** -20 * ((x.abs() + step.abs()).double().sum() * y.abs().max())
    assert (lhs - rhs).abs() <= bound


# ----------------------------------------------------------------- attend ----
def make_cache(g, S, L, Hq, Hkv, T, lens, dtype, spread=1.0):
    N = max(1, sum(lens))
    k, v = (randn(g, L, Hkv, N, D, dtype=dtype) for _ in range(2))
    q = (spread * randn(g, S, L, Hq, T, D)).to(dtype)
    cu = torch.tensor([sum(lens[:i]) for i in range(S + 1)], dtype=torch.int32, device=DEV)
    return api.Cache(q, k, v, cu, list(lens), Hq)


def attend_plain(q, k, v, seen, dtype):
    """q [rows, D], k and v [n, D], seen [rows, n]: (o, lse, bounds) in 64 bits; what is not seen is left out."""
    q, k, v = q.double(), k.double(), v.double()
    x = torch.where(seen, q @ torch.where(seen.any(0)[:, None], k, 0).T * SCALE, -math.inf)
    size = torch.where(seen, (q.abs() @ k.abs().T) * SCALE, 0.0)
    size = torch.nan_to_num(size, 0.0, 0.0).amax(1, keepdim=True) if x.shape[1] else x.sum(1, keepdim=True)
    p = torch.exp(x - x.amax(1, keepdim=True)) if x.shape[1] else x
    p = torch.where(seen, p, 0.0)
    z = p.sum(1, keepdim=True)
    rows = []
    for r in range(q.shape[0]):
        at = seen[r]
        rows.append((p[r, at][:, None] * v[at]).sum(0) / z[r] if at.any() else torch.zeros(D, dtype=torch.float64, device=q.device))
    o = torch.stack(rows)
    lse = torch.where(seen.any(1), torch.logsumexp(torch.where(seen.any(1)[:, None], x, 0.0), 1) if x.shape[1] else 0.0, -math.inf)
    mass = torch.nan_to_num((p / z.clamp_min(1e-300)) @ torch.nan_to_num(v.abs(), 0.0, 0.0))
    logit = 136 * 2.0 ** -24 * size
    tol = (2 * logit + 2.0 ** -20 + (HALF[BF16] if dtype == BF16 else 0.0)) * mass + HALF[dtype] * torch.nan_to_num(o.abs())
    return o, lse, tol, (logit[:, 0] + 2.0 ** -20 + 2.0 ** -23 * torch.nan_to_num(lse.abs(), 0, 0, 0))


def check_attend(cache, o, lse, kd=None, vd=None, tree=None, lengths=None, draft_lens=None, untouched=None):
    S, L, Hq, T = lse.shape
    Hkv, cu = cache.k.shape[1], cache.cu_seqlens.tolist()
    G = Hq // Hkv
    for s in range(S):
        n = cache.seqlens[s] if lengths is None else lengths[s]
        rows = T if draft_lens is None else draft_lens[s]
        nd = 0 if kd is None else rows
        seen = torch.ones(rows, n + nd, dtype=torch.bool, device=DEV)
        if kd is not None:
            bits = torch.arange(nd, device=DEV)
            seen[:, n:] = bits <= bits[:, None] if tree is None else (tree[s, :rows, None] >> bits & 1).bool()
        for l in range(L):
            for h in range(Hq):
                g = h // G
                k, v = cache.k[l, g, cu[s]:cu[s] + n], cache.v[l, g, cu[s]:cu[s] + n]
                if kd is not None:
                    k, v = torch.cat([k, kd[s, l, g, :nd]]), torch.cat([v, vd[s, l, g, :nd]])
                if rows:
                    wo, wl, to, tl = attend_plain(cache_q(cache, s, l, h)[:rows], k, v, seen, cache.k.dtype)
                    within(o[s, l, h, :rows], wo, to, f"o of request {s}, head {h}")
                    within(lse[s, l, h, :rows], wl, tl, f"lse of request {s}, head {h}")
                if untouched is not None:
                    assert (o[s, l, h, rows:] == untouched).all() and (lse[s, l, h, rows:] == untouched).all()


def cache_q(cache, s, l, h):
    return cache.q_win[s, l, h]


def random_tree(seed, S, T):
    r = torch.Generator().manual_seed(seed)
    return [[int(torch.randint(-1, t, (1,), generator=r)) if t else -1 for t in range(T)] for _ in range(S)]


ATTEND = [
    # (L, Hq, Hkv, T, lens, drafted: None, "chain", "tree")
    (1, 4, 1, 1, (37,), "chain"),
    (1, 1, 1, 1, (1,), None),
    (1, 8, 8, 1, (64, 65, 63), "chain"),
    (2, 8, 2, 3, (128, 1, 129, 200), "tree"),
    (1, 28, 4, 5, (640, 17), "tree"),       # 35 rows
    (1, 32, 8, 8, (700,), "chain"),         # 32 rows
    (1, 16, 2, 8, (301,), "tree"),          # 64 rows
    (1, 10, 2, 13, (1000, 60), "tree"),     # 65 rows
    (1, 8, 1, 16, (500,), "chain"),         # 128 rows
    (1, 5, 1, 64, (257, 5), "tree"),        # 320 rows
    (1, 8, 1, 64, (130,), "tree"),          # 512 rows
    (1, 4, 4, 2, (2500, 900), "tree"),      # several splits
    (1, 2, 1, 33, (70,), None),
    (3, 3, 1, 1, (5, 2, 9), "chain"),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attend_against_64_bits(case, dtype):
    L, Hq, Hkv, T, lens, drafted = ATTEND[case]
    S, g = len(lens), gen(100 + case)
    cache = make_cache(g, S, L, Hq, Hkv, T, lens, dtype, spread=2.0)
    att = api.CacheAttention(cache)
    kd = vd = tree = None
    if drafted:
        kd, vd = (randn(g, S, L, Hkv, T, D, dtype=dtype) for _ in range(2))
    if drafted == "tree":
        tree = api.tree_masks(random_tree(case, S, T)).to(DEV)
    o, lse = att.run(k_draft=kd, v_draft=vd, tree=tree)
    att.check()
    check_attend(cache, o, lse, kd, vd, tree)
    first = (o.clone(), lse.clone())
    att.run(k_draft=kd, v_draft=vd, tree=tree)
    assert torch.equal(first[0], o) and torch.equal(first[1], lse)  # the order of every sum is fixed


@pytest.mark.parametrize("L,Hq,Hkv,T,lens,dtype", [
    (1, 4, 2, 1, (40000, 300, 9000), BF16), (2, 5, 1, 9, (17000, 3), BF16), (1, 5, 1, 20, (30000, 6000), BF16),
    (1, 5, 1, 64, (26000, 40, 7000), BF16), (1, 8, 1, 32, (70000,), BF16), (1, 4, 2, 1, (20000, 300), F32),
    (1, 5, 1, 9, (12000, 70), F32), (5, 16, 8, 3, (900, 100, 64, 400, 0, 1, 333, 640, 65), BF16),
    (2, 8, 1, 20, tuple(range(20, 2000, 23)), BF16), (1, 4, 1, 4, (5000, 30), F32), (2, 5, 1, 20, (9000, 300), F32),
    (1, 8, 1, 48, (3000,), F32)])
def test_attend_splits_joined_and_several_items_per_block(L, Hq, Hkv, T, lens, dtype):
    """Requests in many splits, and more items than the GPU takes at once. A split's sum takes at most some hundred
    additions one after the other (one per tile of 64 tokens), 2^-24 each: below a fifth of the logits' bound (their
    size is above 10 here, the bound 8e-5)."""
    S, g = len(lens), gen(300 + T)
    cache = make_cache(g, S, L, Hq, Hkv, T, lens, dtype, spread=2.0)
    kd, vd = (randn(g, S, L, Hkv, T, D, dtype=dtype) for _ in range(2))
    tree = api.tree_masks(random_tree(T, S, T)).to(DEV)
    att = api.CacheAttention(cache)
    o, lse = att.run(k_draft=kd, v_draft=vd, tree=tree)
    att.check()
    check_attend(cache, o, lse, kd, vd, tree)
    # shorter requests with the same workspace: other splits, and counters that the call before left at zero
    lengths = [n // 3 for n in lens]
    o, lse = att.run(k_draft=kd, v_draft=vd, tree=tree, lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV))
    att.check()
    check_attend(cache, o, lse, kd, vd, tree, lengths)


def test_caches_whose_offsets_pass_32_bits():
    """Two heads of 8.5 million tokens: the second head's last rows are past 2^31 elements. All keys are zero but the
    last 300 of a head, whose logits leave the others a share below 1e-2 of the least tolerance."""
    N, T, n = 8_500_000, 2, 300
    g = gen(31)
    k = torch.zeros((1, 2, N, D), dtype=BF16, device=DEV)
    v = torch.zeros_like(k)
    k[:, :, -n:], v[:, :, -n:] = 20 * randn(g, 1, 2, n, D, dtype=BF16), randn(g, 1, 2, n, D, dtype=BF16)
    q = randn(g, 1, 1, 4, T, D, dtype=BF16)
    assert (q[0, 0].view(2, 4, D) @ k[0, :, -n:].transpose(1, 2)).amax(2).min() * SCALE > 36 and k.numel() > 2 ** 31
    cache = api.Cache(q, k, v, torch.tensor([0, N], dtype=torch.int32, device=DEV), [N], 4)
    att = api.CacheAttention(cache)
    o, lse = att.run()
    att.check()
    seen = torch.ones(T, n, dtype=torch.bool, device=DEV)
    for h in range(4):
        wo, wl, to, tl = attend_plain(q[0, 0, h], k[0, h // 2, -n:], v[0, h // 2, -n:], seen, BF16)
        others = N * math.exp(-36)  # of the sum of exponentials, at most
        within(o[0, 0, h], wo, to + others * wo.abs(), "o")
        within(lse[0, 0, h], wl, tl + others, "lse")
    ev = api.WeightEvictor(cache, 64)
    ev.run()
    ev.check()
    small = api.Cache(q, k[:, :, -n:].contiguous(), v[:, :, -n:].contiguous(),
                      torch.tensor([0, n], dtype=torch.int32, device=DEV), [n], 4)
    weights, tol, *_ = weigh_plain(small)
    # (what is below float32's normal numbers, 2^-126, becomes zero: of four rows)
    within(ev.weights[:, :, -n:], weights, tol + 2 * others * weights + 4 * 2.0 ** -126, "weights")
    for h in range(2):
        keep = select_plain(ev.weights[0, h, -n:], n, 64, 0, 0)
        assert ev.idx[0, h, 0].tolist() == [N - n + i for i in keep]
        for out, x in ((ev.k_out, k), (ev.v_out, v)):
            assert torch.equal(out[0, h, 0], x[0, h, -n:][keep])
    del k, v, cache, att, ev
    x = torch.zeros((1_100_000, 16, D), dtype=BF16, device=DEV)
    x[-3:] = randn(g, 3, 16, D, dtype=BF16)
    assert x.numel() > 2 ** 31
    at = torch.arange(x.shape[0], dtype=torch.int32, device=DEV)
    y, _ = api.Rope(device=DEV).apply(x, None, at)
    freq, amplitude = api.rope_frequencies(D, 10000.0)
    want, tol = rope_plain(x[-3:], at[-3:], freq, amplitude, D, False, False)
    within(y[-3:], want, tol, "rope")
    assert not y[:-3].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attend_live_lengths_masks_and_rows_left_alone(dtype):
    S, L, Hq, Hkv, T, cap = 5, 2, 6, 2, 9, 200
    g = gen(7)
    cache = make_cache(g, S, L, Hq, Hkv, T, (cap,) * S, dtype)
    lengths, draft_lens = [0, 200, 64, 1, 0], [9, 0, 4, 1, 3]
    # what lies behind the live tokens and behind the drafted ones may be anything
    for s, n in enumerate(lengths):
        for t in (cache.k, cache.v):
            t[:, :, s * cap + n:(s + 1) * cap] = math.nan
    kd, vd = (randn(g, S, L, Hkv, T, D, dtype=dtype) for _ in range(2))
    for s, n in enumerate(draft_lens):
        kd[s, :, :, n:] = math.inf
        vd[s, :, :, n:] = math.nan
    tree = api.tree_masks(random_tree(3, S, T)).to(DEV)
    tree[0, 4] = 0           # sees nothing at all
    tree[2, 1] = 0           # cached tokens only
    tree[3, 0] = -1          # bits of tokens that are not there
    att = api.CacheAttention(cache)
    att.o.fill_(77.0)
    att.lse.fill_(77.0)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    o, lse = att.run(k_draft=kd, v_draft=vd, tree=tree, lengths=dev(lengths), draft_lens=dev(draft_lens))
    att.check()
    check_attend(cache, o, lse, kd, vd, tree, lengths, draft_lens, untouched=77.0)
    assert (lse[0, :, :, 4] == -math.inf).all() and (o[0, :, :, 4] == 0).all()
    o, lse = att.run(lengths=dev(lengths))  # no drafted tokens
    check_attend(cache, o, lse, lengths=lengths)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attend_drafted_values_that_are_not_finite(dtype):
    S, Hq, Hkv, T = 1, 8, 2, 6
    g = gen(8)
    cache = make_cache(g, S, 1, Hq, Hkv, T, (100,), dtype)
    kd, vd = (randn(g, S, 1, Hkv, T, D, dtype=dtype) for _ in range(2))
    tree = api.tree_masks([[-1, 0, 0, 1, 2, -1]]).to(DEV)
    vd[0, 0, 0, 1, 5] = math.nan    # seen by tokens 1 and 3
    vd[0, 0, 1, 2, 7] = -math.inf   # seen by tokens 2 and 4
    kd[0, 0, 1, 5, 0] = math.nan    # seen by token 5 only
    o, lse = api.CacheAttention(cache).run(k_draft=kd, v_draft=vd, tree=tree)
    check_attend(cache, o, lse, kd, vd, tree)


def test_attend_strides():
    g, S, L, Hq, Hkv, T, cap = gen(9), 3, 2, 8, 2, 4, 90
    # slots as [tokens, heads] rows (a head's rows apart), queries and drafts as [S, T, H, D]
    kv = randn(g, 2, L, S * cap, Hkv, D, dtype=BF16).transpose(2, 3)
    q = randn(g, S, L, T, Hq, D, dtype=BF16).transpose(2, 3)
    drafts = randn(g, 2, S, L, T, Hkv, D + 8, dtype=BF16)[..., :D].transpose(3, 4)
    cu = torch.arange(0, S * cap + 1, cap, dtype=torch.int32, device=DEV)
    cache = api.Cache(q, kv[0], kv[1], cu, [cap] * S, Hq)
    o, lse = api.CacheAttention(cache).run(k_draft=drafts[0], v_draft=drafts[1])
    check_attend(cache, o, lse, drafts[0], drafts[1])


def test_attend_large_logits():
    """Maxima that rise by far more than the lazy rescaling allows, and logits whose exponentials underflow."""
    g = gen(10)
    for dtype in (BF16, F32):
        cache = make_cache(g, 1, 1, 4, 1, 2, (900,), dtype, spread=4.0)
        cache.k[:, :, ::7] *= 6.0
        cache.k[:, :, 500] *= 20.0
        o, lse = api.CacheAttention(cache).run()
        check_attend(cache, o, lse)


def test_attend_reports_lengths_out_of_range():
    g = gen(11)
    cache = make_cache(g, 2, 1, 4, 1, 1, (50, 60), BF16)
    att = api.CacheAttention(cache)
    bad = torch.tensor([50, 61], dtype=torch.int32, device=DEV)
    o, lse = att.run(lengths=bad)  # clamped
    with pytest.raises(api.JacapError) as e:
        att.check()
    assert e.value.status == JACAP_ERR_INVALID_ARG
    check_attend(cache, o, lse)
    att.run()
    att.check()  # the word was cleared


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cu", [(0, 60, 50), (0, 50, 111), (-1, 50, 110)])
def test_attend_reports_ranges_that_are_none(cu, dtype):
    """A request whose range is not one of the cache's has no cached tokens, the other one its own."""
    g = gen(12)
    cache = make_cache(g, 2, 1, 4, 1, 3, (50, 60), dtype)
    cache.cu_seqlens.copy_(torch.tensor(cu, dtype=torch.int32))
    kd, vd = (randn(g, 2, 1, 1, 3, D, dtype=dtype) for _ in range(2))
    att = api.CacheAttention(cache)
    o, lse = att.run(k_draft=kd, v_draft=vd)
    with pytest.raises(api.JacapError) as e:
        att.check()
    assert e.value.status == JACAP_ERR_INVALID_ARG
    good = [0 <= cu[s] <= cu[s + 1] <= 110 for s in range(2)]
    lengths = [cu[s + 1] - cu[s] if good[s] else 0 for s in range(2)]
    cache.cu_seqlens.copy_(torch.tensor([max(0, c) for c in cu], dtype=torch.int32))
    check_attend(cache, o, lse, kd, vd, lengths=lengths)


# ------------------------------------------------------------------ weigh ----
def weigh_plain(cache, lengths=None, q_lens=None, q_rows=None, lse=None, before=None):
    """weights and lse of every unit in 64 bits, with their bounds; NaN where nothing is written."""
    S, L, Hq, w, _ = cache.q_win.shape
    Hkv, N = cache.k.shape[1:3]
    G, cu = Hq // Hkv, cache.cu_seqlens.tolist()
    weights = torch.full((L, Hkv, N), math.nan, dtype=torch.float64, device=DEV)
    tol, out, tol_lse = weights.clone(), torch.full((S, L, Hq, w), math.nan, dtype=torch.float64, device=DEV), None
    tol_lse = out.clone()
    for s in range(S):
        n = cache.seqlens[s] if lengths is None else lengths[s]
        ql = w if q_lens is None else q_lens[s]
        rows = list(range(ql)) if q_rows is None else [int(x) for x in q_rows[s, :ql]]
        for l in range(L):
            for g in range(Hkv):
                k = cache.k[l, g, cu[s]:cu[s] + n].double()
                sums, bound = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
                for h in range(g * G, (g + 1) * G):
                    for j, r in enumerate(rows):
                        if r < 0 or r >= w:
                            continue
                        last = n - ql + j
                        q = cache.q_win[s, l, h, r].double()
                        x = k[:max(0, last + 1)] @ q * SCALE
                        size = (k.abs() @ q.abs()).amax() * SCALE if n else torch.zeros(())
                        e = torch.logsumexp(x, 0) if x.numel() else torch.tensor(-math.inf, dtype=torch.float64)
                        d = 136 * 2.0 ** -24 * float(size) + 2.0 ** -20
                        out[s, l, h, r], tol_lse[s, l, h, r] = e, d + 2.0 ** -23 * (abs(float(e)) if x.numel() else 0.0)
                        if lse is not None:
                            e = lse[s, l, h, r].double()
                        if x.numel() and e > -math.inf:
                            p = torch.exp(x - e)
                            sums[:x.numel()] += p
                            # with e given its own rounding to float32 is the input's; e log2 e rounds again
                            bound[:x.numel()] += p * (2 * d + 2.0 ** -23 * abs(float(e)) + 2.0 ** -22 * x.abs())
                if before is not None:
                    old = max(0, n - ql)
                    sums[:old] += before[l, g, cu[s]:cu[s] + old].double()
                weights[l, g, cu[s]:cu[s] + n] = sums
                tol[l, g, cu[s]:cu[s] + n] = bound + sums * 2.0 ** -22
    return weights, tol, out, tol_lse


def check_weigh(cache, got, lse, want, filler=None):
    weights, tol, e, tol_e = want
    written = ~weights.isnan()
    within(got[written], weights[written], tol[written], "weights")
    if lse is not None:
        rows = ~e.isnan()
        within(lse[rows], e[rows], tol_e[rows], "lse")
    if filler is not None:
        assert (got[~written] == filler).all()
        if lse is not None:
            assert (lse[e.isnan()] == filler).all()


WEIGH = [  # (L, Hq, Hkv, w, lens)
    (1, 4, 1, 8, (300,)), (1, 1, 1, 1, (1,)), (2, 8, 2, 16, (129, 5, 128)), (1, 4, 4, 32, (20, 33, 32)),
    (1, 5, 1, 32, (400,)), (1, 7, 1, 32, (700, 40)), (1, 6, 1, 64, (300,)), (1, 8, 1, 64, (257,)), (1, 8, 1, 40, (150,)),
    (1, 3, 1, 3, (1100, 2, 1)), (1, 8, 2, 20, (513,)),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", range(len(WEIGH)))
def test_weigh_against_64_bits(case, dtype):
    L, Hq, Hkv, w, lens = WEIGH[case]
    cache = make_cache(gen(200 + case), len(lens), L, Hq, Hkv, w, lens, dtype, spread=2.0)
    ev = api.WeightEvictor(cache, 1)
    got, lse = ev.score()
    ev.check()
    want = weigh_plain(cache)
    check_weigh(cache, got, lse, want)
    first = got.clone()
    ev.score()
    assert torch.equal(first, got)
    # the same with the normalisers given, on top of earlier weights, into the same array
    before = torch.rand(got.shape, generator=gen(1), device=DEV)
    given = lse.clone()
    got.copy_(before)
    ev.score(lse=given, before=got)
    ev.check()
    check_weigh(cache, got, None, weigh_plain(cache, lse=given, before=before))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weigh_slots_queries_and_paths(dtype):
    S, L, Hq, Hkv, w, cap = 6, 2, 6, 2, 7, 300
    g = gen(13)
    cache = make_cache(g, S, L, Hq, Hkv, w, (cap,) * S, dtype)
    lengths, q_lens = [300, 0, 5, 130, 1, 200], [7, 3, 7, 0, 1, 4]
    for s, n in enumerate(lengths):
        cache.k[:, :, s * cap + n:(s + 1) * cap] = math.nan
    rows = torch.tensor([[6, 5, 4, 3, 2, 1, 0], [0, 1, 2, 3, 4, 5, 6], [0, 2, 4, 6, 1, 3, 5], [1] * 7, [3] + [-1] * 6,
                         [0, -1, 9, 2, 5, 5, 5]], dtype=torch.int32)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    ev = api.WeightEvictor(cache, 1)
    ev.weights.fill_(55.0)
    ev.lse.fill_(55.0)
    before = torch.rand(ev.weights.shape, generator=g, device=DEV)
    got, lse = ev.score(lengths=dev(lengths), q_lens=dev(q_lens), q_rows=rows.to(DEV), before=before)
    ev.check()
    check_weigh(cache, got, lse, weigh_plain(cache, lengths, q_lens, rows, before=before), filler=55.0)


def test_weigh_many_runs_and_requests():
    """Enough tokens that a unit's statistics come from several runs of several CTAs."""
    for dtype, lens in ((BF16, (30000, 17, 9000, 4097)), (F32, (9000, 100))):
        cache = make_cache(gen(14), len(lens), 1, 2, 1, 4, lens, dtype, spread=2.0)
        ev = api.WeightEvictor(cache, 1)
        got, lse = ev.score()
        ev.check()
        check_weigh(cache, got, lse, weigh_plain(cache))


def test_weigh_reports_what_is_not_finite_and_bad_lengths():
    cache = make_cache(gen(15), 1, 1, 4, 1, 4, (200,), BF16)
    cache.k[0, 0, 100, 3] = math.nan
    ev = api.WeightEvictor(cache, 8)
    ev.run()
    with pytest.raises(api.JacapError) as e:
        ev.check()
    assert e.value.status == JACAP_ERR_NONFINITE
    cache.k[0, 0, 100, 3] = 0.0
    ev.run()
    ev.check()
    for n in (-1, 201):
        ev.score(lengths=torch.tensor([n], dtype=torch.int32, device=DEV))
        with pytest.raises(api.JacapError) as e:
            ev.check()
        assert e.value.status == JACAP_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weights_of_all_of_a_prompt_s_queries(dtype):
    """Window by window from the first token on, each on top of the ones before: the causal softmax weights of every
    query, summed. Bounds as in weigh_plain, and a rounding for each window's addition."""
    S, Hq, Hkv, w, lens = 2, 6, 2, 32, (310, 75)
    g = gen(34)
    cache = make_cache(g, S, 1, Hq, Hkv, w, lens, dtype, spread=2.0)
    q = torch.zeros((S, 1, Hq, 320, D), dtype=dtype, device=DEV)
    q[:] = (2.0 * randn(g, *q.shape)).to(dtype)
    ev = api.WeightEvictor(cache, 1)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for c in range(10):
        q_lens = [min(max(n - w * c, 0), w) for n in lens]
        ev.score(q[:, :, :, w * c:w * (c + 1)], lengths=dev([min(n, w * (c + 1)) for n in lens]), q_lens=dev(q_lens),
                 before=ev.weights if c else None)
        ev.check()
    first = 0
    for s, n in enumerate(lens):
        for h in range(Hkv):
            k, sums, tol = cache.k[0, h, first:first + n].double(), 0.0, 0.0
            for hq in range(3 * h, 3 * h + 3):
                x = q[s, 0, hq, :n].double() @ k.t() * SCALE
                size = (q[s, 0, hq, :n].abs().double() @ k.abs().t()).amax(1, keepdim=True) * SCALE
                x = x.masked_fill(~torch.ones(n, n, dtype=torch.bool, device=DEV).tril(), -math.inf)
                p = torch.softmax(x, 1)
                sums = sums + p.sum(0)
                tol = tol + (p * (2 * (136 * 2.0 ** -24 * size + 2.0 ** -20) + 2.0 ** -22 * x.clamp(min=-1e4).abs())).sum(0)
            within(ev.weights[0, h, first:first + n], sums, tol + sums * (2.0 ** -22 + 10 * 2.0 ** -24), "weights")
        first += n


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("Hq,w", [(3, 3), (8, 40)])
def test_weigh_keys_that_no_query_sees(Hq, w, given, dtype):
    """NaN and infinities in K where no query of the request looks: earlier weights stay, nothing is reported."""
    cap, lengths = 500, [300, 500, 130, 200]
    q_lens, rows = [0, 3, 2, 3], [[0, 1, 2], [-1, 7 + w, -1], [0, 1, 2], [1, -1, -1]]
    g = gen(33)
    cache = make_cache(g, 4, 1, Hq, 1, w, (cap,) * 4, dtype)
    for s, (first, last) in enumerate(((10, 300), (0, 500), (130, 500), (198, 200))):  # request 2: behind its length
        cache.k[:, :, s * cap + first:s * cap + last, ::2] = math.nan
        cache.k[:, :, s * cap + first:s * cap + last, 1::4] = math.inf
    rows = torch.tensor([r + [-1] * (w - 3) for r in rows], dtype=torch.int32)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    ev = api.WeightEvictor(cache, 1)
    before = torch.rand(ev.weights.shape, generator=g, device=DEV)
    args = dict(lengths=dev(lengths), q_lens=dev(q_lens), q_rows=rows.to(DEV), before=before)
    got, lse = ev.score(**args)
    if given:
        got, _ = ev.score(lse=lse.clone(), **args)
    ev.check()
    plain = api.Cache(cache.q_win, cache.k.nan_to_num(0.0, 0.0, 0.0), cache.v, cache.cu_seqlens, cache.seqlens, Hq)
    check_weigh(plain, got, None, weigh_plain(plain, lengths, q_lens, rows, lse=lse if given else None, before=before))


# ------------------------------------------------------------------ evict ----
def select_plain(weights, n, budget, sinks, recent, tags=None):
    tag = torch.arange(n) if tags is None else tags.cpu().long()
    w = weights.double().cpu().clone()
    if n:
        w[(tag < sinks) | (tag > tag.max() - recent)] = math.inf
    order = sorted(range(n), key=lambda i: (-w[i].item(), i))
    return sorted(order[:budget])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("L,Hkv,lens,budget,sinks,recent", [
    (1, 1, (1,), 1, 0, 0), (2, 3, (100, 7, 33), 16, 2, 5), (1, 2, (4000, 900), 700, 4, 64), (1, 1, (5000,), 96, 96, 0),
    (1, 1, (40000,), 300, 0, 300), (3, 60, (50, 60), 20, 1, 1), (1, 2, (64, 64), 64, 3, 3)])
def test_select_by_weights(L, Hkv, lens, budget, sinks, recent, dtype):
    g = gen(16)
    cache = make_cache(g, len(lens), L, Hkv, Hkv, 1, lens, dtype)
    ev = api.WeightEvictor(cache, budget, sinks=sinks, recent=recent)
    weights = torch.exp(2 * randn(g, L, Hkv, sum(lens)))
    weights[torch.rand(weights.shape, generator=g, device=DEV) < 0.3] = 0.0   # many ties
    weights[torch.rand(weights.shape, generator=g, device=DEV) < 0.1] = 1e-30
    kept_weights = weights.clone()
    ev.select_compact(weights)
    ev.check()
    assert torch.equal(weights, kept_weights)
    at = 0
    for s, n in enumerate(lens):
        for l in range(L):
            for h in range(Hkv):
                want = select_plain(weights[l, h, at:at + n], n, budget, sinks, recent)
                got = ev.idx[l, h, s].tolist()
                assert got == want + [-1] * (budget - len(want))
                rows = torch.tensor(want, device=DEV, dtype=torch.long) + at
                for out, src in ((ev.k_out, cache.k), (ev.v_out, cache.v)):
                    assert torch.equal(out[l, h, s, :len(want)], src[l, h, rows]) and (out[l, h, s, len(want):] == 0).all()
                assert torch.equal(ev.weights_out[l, h, s, :len(want)], weights[l, h, rows])
                assert (ev.weights_out[l, h, s, len(want):] == 0).all()
        assert ev.kept[s] == min(n, budget)
        at += n


def test_select_by_weights_and_tags():
    g, n = gen(17), 500
    cache = make_cache(g, 1, 2, 2, 2, 1, (n,), BF16)
    ev = api.WeightEvictor(cache, 50, sinks=3, recent=20)
    weights = torch.rand((2, 2, n), generator=g, device=DEV)
    tags = torch.stack([torch.randperm(2 * n, generator=g, device=DEV)[:n] for _ in range(4)]).view(2, 2, n).to(torch.int32)
    ev.select_compact(weights, pos=tags)
    ev.check()
    for l in range(2):
        for h in range(2):
            assert ev.idx[l, h, 0].tolist() == select_plain(weights[l, h], n, 50, 3, 20, tags[l, h])


@pytest.mark.parametrize("bad", [math.nan, -1.0, math.inf])
def test_select_refuses_weights_that_are_none(bad):
    cache = make_cache(gen(18), 1, 1, 1, 1, 1, (100,), BF16)
    ev = api.WeightEvictor(cache, 10)
    ev.idx.fill_(-7)
    weights = torch.rand((1, 1, 100), device=DEV)
    weights[0, 0, 42] = bad
    ev.select_compact(weights)
    with pytest.raises(api.JacapError) as e:
        ev.check()
    assert e.value.status == JACAP_ERR_NONFINITE and (ev.idx == -7).all()
    weights[0, 0, 42] = 0.5
    ev.select_compact(weights)
    ev.check()
    assert ev.idx[0, 0, 0].tolist() == select_plain(weights[0, 0], 100, 10, 0, 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("ordered", [0, 1])
@pytest.mark.parametrize("lens", [(9000, 100, 5000), (100, 9000), (4096, 1, 4097, 8192), (40, 30), (8193, 4095, 50)])
def test_evict_by_weights_without_tags(lens, ordered, dtype):
    """In place and by row, over requests that end in different parts of the longest's tokens; what lies behind the
    arrays stays."""
    L, Hkv, budget, sinks, recent, guard = 2, 2, 48, 5, 9, 9216
    g, S, N = gen(27), len(lens), sum(lens)
    cache = make_cache(g, S, L, Hkv, Hkv, 1, lens, dtype)
    k0, v0 = cache.k.clone(), cache.v.clone()
    room = torch.full((L * Hkv * N + guard,), -77.0, device=DEV)  # (as a weight -77 is refused)
    keys = torch.full((L * Hkv * N + guard,), -77.0, device=DEV)
    weights = room[:L * Hkv * N].view(L, Hkv, N)
    weights.copy_(torch.rand(weights.shape, generator=g, device=DEV))
    weights[torch.rand(weights.shape, generator=g, device=DEV) < 0.3] = 0.25  # ties
    w0 = weights.clone()
    idx = torch.full((L, Hkv, S, budget), -7, dtype=torch.int32, device=DEV)
    kept = torch.zeros(S, dtype=torch.int32, device=DEV)
    ws = torch.zeros(64, dtype=torch.uint8, device=DEV)
    at = lambda t: t.data_ptr()  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream
    status = api.jacap_evict_weights(cache.layout(), at(weights), None, sinks, recent, budget, at(idx), at(kept),
                                     at(cache.k), at(cache.v), ordered, at(keys), at(ws), ws.numel(), stream)
    assert status == 0 and api.jacap_device_status(at(ws), stream) == 0
    assert (room[L * Hkv * N:] == -77.0).all() and (keys[L * Hkv * N:] == -77.0).all()
    first = 0
    for s, n in enumerate(lens):
        for l in range(L):
            for h in range(Hkv):
                want = select_plain(w0[l, h, first:first + n], n, budget, sinks, recent)
                assert idx[l, h, s].tolist() == want + [-1] * (budget - len(want))
                rows = torch.tensor(want, device=DEV) + first
                now = slice(first, first + len(want))
                for got, src in ((cache.k, k0), (cache.v, v0), (weights, w0)):
                    got, src = got[l, h, now].reshape(len(want), -1), src[l, h, rows].reshape(len(want), -1)
                    if not ordered:  # the kept rows from past the budget fill the holes
                        moved = sorted(r for r in want if r >= budget)
                        place = [r for r in range(len(want)) if r not in set(want)] if n > budget else []
                        order = {r: r for r in want if r < budget} | dict(zip(moved, place))
                        src = src[torch.tensor(sorted(range(len(want)), key=lambda i: order[want[i]]), device=DEV)]
                    assert torch.equal(got, src)
                # rows that were not moved into, and those behind the kept ones
                assert torch.equal(weights[l, h, first + len(want):first + n], w0[l, h, first + len(want):first + n])
        assert kept[s] == min(n, budget)
        first += n


# --------------------------------------------------- streams, graphs, refusals ----
def test_operators_on_another_stream_and_in_graphs():
    g, S, L, Hq, Hkv, T = gen(19), 2, 1, 8, 2, 3
    cache = make_cache(g, S, L, Hq, Hkv, T, (900, 1500), BF16)
    kd, vd = (randn(g, S, L, Hkv, T, D, dtype=BF16) for _ in range(2))
    lengths = torch.tensor([900, 1500], dtype=torch.int32, device=DEV)
    at = torch.arange(S * T, dtype=torch.int32, device=DEV).view(S, T)
    rope = api.Rope(device=DEV)
    att, ev = api.CacheAttention(cache), api.WeightEvictor(cache, 100, sinks=2, recent=10)

    def loop(stream=None):
        q, k = rope.apply(cache.q_win[:, 0].transpose(1, 2), kd[:, 0].transpose(1, 2), at, stream=stream)
        q, k = q.transpose(1, 2).unsqueeze(1), k.transpose(1, 2).unsqueeze(1)
        o, lse = att.run(q, k_draft=k, v_draft=vd, lengths=lengths, stream=stream)
        ev.score(q, lse=lse, lengths=lengths, stream=stream)
        ev.select_compact(stream=stream)
        return [t.clone() for t in (q, o, lse, ev.weights, ev.idx, ev.k_out)]

    ref = loop()
    side = torch.cuda.Stream(device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = loop()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(ref, out))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(torch.cuda.current_stream()):
        loop(side)
    side.synchronize()
    # two graphs that share the workspaces, replayed one after the other with other lengths
    graphs, results = [], []
    torch.cuda.synchronize()
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(loop())
        graphs.append(graph)
    for n in ([900, 1500], [1, 700], [450, 0]):
        lengths.copy_(torch.tensor(n, dtype=torch.int32))
        want = loop()
        for graph, got in zip(graphs, results):
            graph.replay()
        torch.cuda.synchronize()
        for got in results:
            for a, b in zip(want[:3], got[:3]):
                assert torch.equal(a, b)
            for s in range(2):
                a0 = 900 * s
                assert torch.equal(want[3][:, :, a0:a0 + n[s]], got[3][:, :, a0:a0 + n[s]])


def test_attentions_of_several_layouts_share_a_workspace():
    """Its start zeroed once, used by one layout after the other: many units in splits that the kernel joins by counting them,
    calls of one split, of more rows, of many splits, float32."""
    calls = []
    for i, (S, L, Hq, Hkv, T, n, dtype) in enumerate((
            (4, 4, 64, 16, 1, 600, BF16), (1, 2, 8, 8, 64, 450, BF16), (2, 1, 16, 2, 64, 1900, BF16), (3, 1, 4, 4, 2, 700, F32),
            (16, 1, 8, 1, 1, 40, BF16), (1, 1, 8, 2, 3, 30000, BF16), (1, 8, 32, 32, 1, 5000, BF16), (2, 1, 8, 1, 40, 3000, F32))):
        g = gen(60 + i)
        cache = make_cache(g, S, L, Hq, Hkv, T, (n,) * S, dtype)
        kd, vd = (randn(g, S, L, Hkv, T, D, dtype=dtype) for _ in range(2))
        att = api.CacheAttention(cache)
        want = [x.clone() for x in att.run(k_draft=kd, v_draft=vd)]
        calls.append((att, kd, vd, want))
    shared = torch.full((max(c[0].ws.numel() for c in calls),), 255, dtype=torch.uint8, device=DEV)
    shared[:JACAP_ATTEND_ZERO_BYTES].zero_()
    for c in calls:
        c[0].ws = shared
    for order in (range(8), (0, 1, 0, 2, 0, 3, 6, 4, 6, 5, 0, 7, 6, 3, 5, 1, 5)):
        for i in order:
            att, kd, vd, want = calls[i]
            att.o.fill_(7)
            att.lse.fill_(7)
            assert all(torch.equal(a, b) for a, b in zip(att.run(k_draft=kd, v_draft=vd), want)), i
            att.check()


def test_two_calls_at_once():
    """Two attentions and their weights on two streams, workspaces of their own: as one after the other."""
    work = []
    for i, (lens, T) in enumerate((((9000, 700, 3000), 3), ((20000,), 40))):
        g = gen(40 + i)
        cache = make_cache(g, len(lens), 2, 8, 2, T, lens, BF16)
        kd, vd = (randn(g, len(lens), 2, 2, T, D, dtype=BF16) for _ in range(2))
        att, ev = api.CacheAttention(cache), api.WeightEvictor(cache, 100, sinks=1, recent=3)

        def call(att=att, ev=ev, kd=kd, vd=vd):
            _, lse = att.run(k_draft=kd, v_draft=vd)
            ev.run()
            return [x.clone() for x in (att.o, lse, ev.weights, ev.lse, ev.idx, ev.v_out)]

        work.append((call, call(), torch.cuda.Stream(device=DEV)))
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for call, _, stream in work:
            with torch.cuda.stream(stream):
                got.append(call())
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(out, work[i % 2][1]))


# ------------------------------------------------------- the decoding loop ----
def _slot(ev, s, l, g):
    """{id: (k bits, v bits, weight)} of a slot."""
    n = ev.lengths[s]
    ids = ev.pos[s, l, g, :n].tolist()
    assert len(set(ids)) == n
    k, v = ev.k[s, l, g, :n].float().cpu(), ev.v[s, l, g, :n].float().cpu()
    w = ev.weights[s, l, g, :n].double().cpu() if ev.rule == "weight" else torch.zeros(n)
    return {i: (k[r], v[r], w[r].item()) for r, i in enumerate(ids)}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("ordered", [False, True])
@pytest.mark.parametrize("drafts", [1, 5])
def test_decoding_loop_by_weights(drafts, ordered, dtype):
    """Rotary positions, attention over the slots, the accepted path, weights and evictions together, against a plain
    simulation in 64 bits that keeps every request's tokens in dictionaries."""
    S, L, Hq, Hkv, B, I, T, w0 = 3, 2, 4, 2, 40, 6, drafts, 8
    G, g, lens = Hq // Hkv, gen(21 + drafts), [30, 45, 12]
    rope = api.Rope(64, base=1000.0, device=DEV)
    ev = api.DecodeEvictor(S, L, Hq, Hkv, B, I, dtype=dtype, device=DEV, preserve_order=ordered, rule="weight", sinks=2,
                           recent=4)
    k0, v0 = (randn(g, S, L, Hkv, max(lens), D, dtype=dtype) for _ in range(2))
    qw = randn(g, S, L, Hq, w0, D, dtype=dtype)
    ev.start(k0, v0, qw, lens)
    sim = {}
    for s, n in enumerate(lens):
        for l in range(L):
            for h in range(Hkv):
                rows = [[k0[s, l, h, i].double(), v0[s, l, h, i].double(), 0.0] for i in range(n)]
                for hq in range(h * G, (h + 1) * G):
                    for j in range(w0):
                        at = n - w0 + j
                        x = torch.stack([r[0] for r in rows[:at + 1]]) @ qw[s, l, hq, j].double() * SCALE
                        for r, p in zip(rows, torch.softmax(x, 0).tolist()):
                            r[2] += p
                sim[s, l, h] = dict(enumerate(rows))

    def same():
        for (s, l, h), rows in sim.items():
            got = _slot(ev, s, l, h)
            assert got.keys() == rows.keys(), (s, l, h)
            for i, (k, v, w) in got.items():
                assert torch.equal(k.double(), rows[i][0].cpu()) and torch.equal(v.double(), rows[i][1].cpu())
                # 2 (136 2^-24 size + 2^-20) of each weight added, sizes below 16: under 2.6e-4
                assert abs(w - rows[i][2]) <= 2.6e-4 * rows[i][2] + 1e-9

    same()
    r = torch.Generator().manual_seed(5)
    ids, evictions = list(lens), 0
    for step in range(14):
        parents = random_tree(step, S, T)
        tree = api.tree_masks(parents).to(DEV)
        depth = [[0] * T for _ in range(S)]
        for s in range(S):
            for t in range(T):
                depth[s][t] = 0 if parents[s][t] < 0 else depth[s][parents[s][t]] + 1
        depth = torch.tensor(depth, dtype=torch.int32, device=DEV)
        q, k, v = (randn(g, S, L, n, T, D, dtype=dtype) for n in (Hq, Hkv, Hkv))
        for l in range(L):
            q[:, l], k[:, l] = ev.rotate(rope, q[:, l], k[:, l], depth)
            o, lse = ev.attend(l, q[:, l], k[:, l], v[:, l], tree)
            for s in range(S):
                seen = torch.ones(T, ev.lengths[s] + T, dtype=torch.bool, device=DEV)
                seen[:, ev.lengths[s]:] = (tree[s, :, None] >> torch.arange(T, device=DEV) & 1).bool()
                for h in range(Hq):
                    n = ev.lengths[s]
                    kk = torch.cat([ev.k[s, l, h // G, :n], k[s, l, h // G]])
                    vv = torch.cat([ev.v[s, l, h // G, :n], v[s, l, h // G]])
                    wo, wl, to, tl = attend_plain(q[s, l, h], kk, vv, seen, dtype)
                    within(o[s, h], wo, to, "o")
                    within(lse[s, h], wl, tl, "lse")
        assert ev.next_id == ids
        # a path from the root: some requests take nothing, some all of a branch
        path = []
        for s in range(S):
            t = int(torch.randint(-1, T, (1,), generator=r))
            p = []
            while t >= 0:
                p.insert(0, t)
                t = parents[s][t]
            path.append(p)
        if T == 1:
            path = [[0]] * S
            gone = ev.step(k[:, :, :, 0], v[:, :, :, 0], q[:, :, :, 0])
        else:
            gone = ev.accept(k, v, q, path)
        ev.check()
        # the plain loop: rounds that end where a slot is full
        left, want_gone = [list(p) for p in path], set()
        seen_lse = {}
        for (s, l, h), rows in sim.items():
            for hq in range(h * G, (h + 1) * G):
                for t in path[s]:
                    chain = [t]
                    while parents[s][chain[0]] >= 0:
                        chain.insert(0, parents[s][chain[0]])
                    keys = torch.stack([x[0] for x in rows.values()] + [k[s, l, h, c].double() for c in chain])
                    seen_lse[s, l, hq, t] = torch.logsumexp(keys @ q[s, l, hq, t].double() * SCALE, 0)
        count = {s: len(sim[s, 0, 0]) for s in range(S)}
        for s in range(S):
            while left[s]:
                now = left[s][:B + I - count[s]]
                left[s] = left[s][len(now):]
                for l in range(L):
                    for h in range(Hkv):
                        rows = sim[s, l, h]
                        for i, t in enumerate(now):
                            rows[ids[s] + i] = [k[s, l, h, t].double(), v[s, l, h, t].double(), 0.0]
                        order = sorted(rows)
                        for hq in range(h * G, (h + 1) * G):
                            for i, t in enumerate(now):
                                see = [x for x in order if x <= ids[s] + i]
                                p = torch.exp(torch.stack([rows[x][0] for x in see]) @ q[s, l, hq, t].double() * SCALE
                                              - seen_lse[s, l, hq, t])
                                for x, e in zip(see, p.tolist()):
                                    rows[x][2] += e
                count[s] += len(now)
                ids[s] += len(now)
                if count[s] == B + I:
                    want_gone.add(s)
                    count[s] = B
                    for l in range(L):
                        for h in range(Hkv):
                            rows, last = sim[s, l, h], ids[s] - 1
                            stay = [x for x in rows if x < 2 or x > last - 4]
                            rest = sorted((x for x in rows if x not in stay), key=lambda x: -rows[x][2])
                            sim[s, l, h] = {x: rows[x] for x in stay + rest[:B - len(stay)]}
        assert sorted(want_gone) == list(gone)
        evictions += len(gone)
        same()
    assert evictions >= 3


def test_accepted_paths_keep_the_query_statistics():
    """The rule "jacap" with accepted paths: rows, ids and running statistics as one step at a time leaves them."""
    S, L, Hq, Hkv, T = 2, 2, 4, 2, 4
    g = gen(23)
    one = api.DecodeEvictor(S, L, Hq, Hkv, 20, 30, device=DEV)
    two = api.DecodeEvictor(S, L, Hq, Hkv, 20, 30, device=DEV)
    k0, v0 = (randn(g, S, L, Hkv, 10, D, dtype=BF16) for _ in range(2))
    qw = randn(g, S, L, Hq, 4, D, dtype=BF16)
    for ev in (one, two):
        ev.start(k0, v0, qw, [10, 10])
    for path in ([[0, 2, 3], [1, 2, 3]], [[], []], [[3, 0], [2, 2]]):
        k, v = (randn(g, S, L, T, Hkv, D, dtype=BF16).transpose(2, 3) for _ in range(2))
        q = randn(g, S, L, Hq, T, D, dtype=BF16)
        assert two.accept(k, v, q, path) == []
        for i in range(len(path[0])):
            pick = lambda x: torch.stack([x[s, :, :, path[s][i]] for s in range(S)]).contiguous()  # noqa: E731
            one.append(pick(k), pick(v), pick(q))
    assert one.lengths == two.lengths and one.next_id == two.next_id
    for a, b in ((one.k, two.k), (one.v, two.v), (one.pos, two.pos), (one.stats, two.stats), (one.counts, two.counts)):
        assert torch.equal(a, b)


def test_normalisers_are_those_of_the_step_they_belong_to():
    """Those that a call left for other tokens, another prompt or not for every token are not taken for the step's."""
    S, L, Hq, Hkv, T = 2, 2, 4, 2, 3
    g = gen(25)
    k0, v0, k1, v1 = (randn(g, S, L, Hkv, 12, D, dtype=BF16) for _ in range(4))
    qw = randn(g, S, L, Hq, 4, D, dtype=BF16)
    k, v, q = (randn(g, S, L, n, T, D, dtype=BF16) for n in (Hkv, Hkv, Hq))

    def enter(before):
        ev = api.DecodeEvictor(S, L, Hq, Hkv, 30, 10, device=DEV, rule="weight")
        before(ev)
        ev.accept(k, v, q, [[0, 1, 2], [0, 1]])
        ev.check()
        return ev.weights.clone()

    def attended(ev, **kw):
        ev.start(k0, v0, qw, [12, 9])
        for l in range(L):
            ev.attend(l, q[:, l], **{n: x[:, l] if x.dim() == 5 else x for n, x in kw.items()})

    want = enter(lambda ev: ev.start(k0, v0, qw, [12, 9]))
    assert torch.equal(enter(attended), want)  # over the cached tokens only
    short = torch.tensor([2, 1], dtype=torch.int32, device=DEV)
    assert torch.equal(enter(lambda ev: attended(ev, k_draft=k, v_draft=v, draft_lens=short)), want)

    def again(ev):  # another prompt in between
        attended(ev, k_draft=k, v_draft=v)
        ev.start(k1, v1, qw, [9, 12])

    assert torch.equal(enter(again), enter(lambda ev: ev.start(k1, v1, qw, [9, 12])))


def test_a_capture_alone_leaves_no_normalisers():
    """A captured attention that has not been replayed: the entered tokens' normalisers are computed."""
    S, L, Hq, Hkv, T = 2, 2, 4, 2, 3
    g = gen(31)
    k0, v0, k, v = (randn(g, S, L, Hkv, n, D, dtype=BF16) for n in (12, 12, T, T))
    qw, q = randn(g, S, L, Hq, 4, D, dtype=BF16), randn(g, S, L, Hq, T, D, dtype=BF16)
    evs = [api.DecodeEvictor(S, L, Hq, Hkv, 30, 10, device=DEV, rule="weight") for _ in range(2)]
    for ev in evs:
        ev.start(k0, v0, qw, [12, 9])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for l in range(L):
            evs[1].attend(l, q[:, l], k[:, l], v[:, l])
    for ev in evs:
        ev.accept(k, v, q, [[0, 1, 2], [0, 1]])
        ev.check()
    assert torch.equal(evs[0].weights, evs[1].weights)


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_a_captured_attention_follows_the_slots(rule):
    S, Hq, Hkv, T = 2, 4, 2, 1
    g = gen(26)
    ev = api.DecodeEvictor(S, 1, Hq, Hkv, 20, 4, device=DEV, rule=rule)
    rope = api.Rope(device=DEV)
    k0, v0 = (randn(g, S, 1, Hkv, 23, D, dtype=BF16) for _ in range(2))
    ev.start(k0, v0, randn(g, S, 1, Hq, 4, D, dtype=BF16), [23, 20])
    q, k, v = (randn(g, S, n, T, D, dtype=BF16) for n in (Hq, Hkv, Hkv))

    def layer():
        tq, tk = ev.rotate(rope, q, k)
        return (tq, tk, *ev.attend(0, tq, tk, v))

    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer()
    for step in range(7):
        for x in (q, k, v):
            x.copy_(randn(g, *x.shape, dtype=BF16))
        graph.replay()
        got = [x.clone() for x in captured]
        want = layer()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), step
        ev.step(want[1][:, None, :, 0].contiguous(), v[:, None, :, 0].contiguous(),
                want[0][:, None, :, 0].contiguous())
    ev.check()
    assert ev.events >= 3


@pytest.mark.parametrize("T", [1, 4])
def test_a_captured_loop_by_weights(T, monkeypatch):
    """Rotary positions and attention of all layers as a graph, its normalisers taken for the entered tokens: slots and
    weights as an eager loop leaves them, through evictions, with one pass over the keys in each weighing."""
    S, L, Hq, Hkv = 2, 3, 8, 2
    g = gen(32 + T)
    k0, v0 = (randn(g, S, L, Hkv, 150, D, dtype=BF16) for _ in range(2))
    q0, rope = randn(g, S, L, Hq, 8, D, dtype=BF16), api.Rope(device=DEV)
    k, v, q = (randn(g, S, L, n, T, D, dtype=BF16) for n in (Hkv, Hkv, Hq))
    evs = [api.DecodeEvictor(S, L, Hq, Hkv, 148, 6, device=DEV, rule="weight", sinks=2, recent=8) for _ in range(2)]
    for ev in evs:
        ev.start(k0, v0, q0, [150, 131])
    given, weigh = [], api.jacap_weigh
    monkeypatch.setattr(api, "jacap_weigh", lambda lay, how, *a: (given.append(how.lse_given), weigh(lay, how, *a))[1])

    def layers(ev):
        turned, out = [ev.rotate(rope, q[:, l], k[:, l]) for l in range(L)], []
        for l, (tq, tk) in enumerate(turned):
            out.append(ev.attend(l, tq, tk, v[:, l])[0])
        return torch.stack([x[0] for x in turned], 1), torch.stack([x[1] for x in turned], 1), torch.stack(out)

    layers(evs[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layers(evs[1])
    for step in range(8):
        for x in (q, k, v):
            x.copy_(randn(g, *x.shape, dtype=BF16))
        tq, tk, o = layers(evs[0])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(captured, (tq, tk, o))), step
        for ev, attended in zip(evs, (None, True)):
            if T == 1:
                ev.step(tk[:, :, :, 0], v[:, :, :, 0], tq[:, :, :, 0], attended=attended)
            else:
                ev.accept(tk, v, tq, [[0, 1, 2][:step % 4], [0, 1]], attended=attended)
            ev.check()
    assert evs[0].events >= 1 and evs[0].lengths == evs[1].lengths and set(given) == {1}
    for x in ("k", "v", "pos", "weights"):
        assert torch.equal(getattr(evs[0], x), getattr(evs[1], x)), x


@pytest.mark.parametrize("replays", [0, 1])
def test_the_first_attention_may_be_captured(replays):
    """Eager calls before or after the graph's first replay, and the replays, as without a graph. The slots are long
    enough for splits that the kernel joins by counting them."""
    S, L, Hq, Hkv, T, n = 4, 2, 8, 2, 3, 3000
    g = gen(29)
    k0, v0 = (randn(g, S, L, Hkv, n, D, dtype=BF16) for _ in range(2))
    q0, lens = randn(g, S, L, Hq, 4, D, dtype=BF16), [3000, 2111, 7, 1500]
    k, v, q = (randn(g, S, L, x, T, D, dtype=BF16) for x in (Hkv, Hkv, Hq))
    want, ev = (api.DecodeEvictor(S, L, Hq, Hkv, n, 64, device=DEV, rule="weight") for _ in range(2))
    for x in (want, ev):
        x.start(k0, v0, q0, lens)

    def attend(x):
        return [t.clone() for l in range(L) for t in x.attend(l, q[:, l], k[:, l], v[:, l])]

    ref = attend(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = attend(ev)
    for _ in range(replays):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(attend(ev), ref))
    for x in got:
        x.fill_(7)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    assert all(torch.equal(a, b) for a, b in zip(attend(ev), ref))
    ev.check()


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_start_on_another_stream_than_the_current_one(rule):
    """The slots and their statistics or weights as after a start on the current stream, which is busy here."""
    S, L, Hq, Hkv, n = 3, 2, 4, 2, 900
    g = gen(28)
    k0, v0 = (randn(g, S, L, Hkv, n, D, dtype=BF16) for _ in range(2))
    q, lens = randn(g, S, L, Hq, 16, D, dtype=BF16), [900, 411, 0]
    want = api.DecodeEvictor(S, L, Hq, Hkv, 800, 128, device=DEV, rule=rule)
    want.start(k0, v0, q, lens)
    side = torch.cuda.Stream(device=DEV)
    ev = api.DecodeEvictor(S, L, Hq, Hkv, 800, 128, device=DEV, rule=rule)
    for again in range(2):
        torch.cuda._sleep(20_000_000)  # some 10 ms
        ev.start(k0.clone(), v0.clone(), q.clone(), lens, stream=side)
        names = ("k", "v", "pos", "weights") if rule == "weight" else ("k", "v", "pos", "stats", "counts")
        for x in names:  # (k and v: the prompt's rows; those behind are left as they were)
            got, ref = getattr(ev, x), getattr(want, x)
            assert torch.equal(got[:, :, :, :n], ref[:, :, :, :n]) if x in "kv" else torch.equal(got, ref), (again, x)
        ev.check()
        for x in names:
            getattr(ev, x).fill_(3)


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_the_loop_on_another_stream_than_the_current_one(rule):
    """Every call of the loop with stream=, evictions among them, with the current stream busy: as on the current one."""
    S, L, Hq, Hkv, T = 3, 2, 8, 2, 3
    g = gen(30)
    rope = api.Rope(device=DEV)
    k0, v0 = (randn(g, S, L, Hkv, 600, D, dtype=BF16) for _ in range(2))
    q0, lens = randn(g, S, L, Hq, 16, D, dtype=BF16), [600, 597, 411]
    steps = [[randn(g, S, L, n, T, D, dtype=BF16) for n in (Hkv, Hkv, Hq)] for _ in range(6)]
    one = [[x[:, :, :, 0].contiguous() for x in step] for step in steps]
    side = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()

    def loop(stream):
        ev = api.DecodeEvictor(S, L, Hq, Hkv, 590, 16, device=DEV, rule=rule)
        out = []
        if stream is not None:
            torch.cuda._sleep(20_000_000)  # some 10 ms
        ev.start(k0, v0, q0, lens, stream=stream)
        for (k, v, q), token in zip(steps, one):
            if stream is not None:
                torch.cuda._sleep(2_000_000)
            turned = [ev.rotate(rope, q[:, l], k[:, l], stream=stream) for l in range(L)]
            out += [t for l, (tq, tk) in enumerate(turned) for t in ev.attend(l, tq, tk, v[:, l], stream=stream)[:1]]
            out += ev.accept(k, v, q, [[0, 1, 2], [0], []], stream=stream)
            out += ev.step(*token, stream=stream)
        ev.check(stream)
        torch.cuda.synchronize()
        assert ev.events >= 3
        return out + [ev.k, ev.v, ev.pos] + ([ev.weights] if rule == "weight" else [ev.stats, ev.counts])

    for a, b in zip(loop(side), loop(None)):
        assert torch.equal(a, b) if isinstance(a, torch.Tensor) else a == b


def test_steps_enqueued_ahead_of_the_device():
    """Lengths and paths that change many times while the device is busy: each step's own, as when it is waited for."""
    S, L, Hq, Hkv, T = 4, 1, 8, 2, 4
    g = gen(35)
    k0, v0 = (randn(g, S, L, Hkv, 100, D, dtype=BF16) for _ in range(2))
    q0 = randn(g, S, L, Hq, 8, D, dtype=BF16)
    k, v, q = (randn(g, S, L, n, T, D, dtype=BF16) for n in (Hkv, Hkv, Hq))
    r = torch.Generator().manual_seed(3)
    paths = [[sorted(torch.randperm(T, generator=r)[:int(torch.randint(0, T + 1, (1,), generator=r))].tolist())
              for _ in range(S)] for _ in range(60)]

    def loop(wait):
        ev = api.DecodeEvictor(S, L, Hq, Hkv, 110, 9, device=DEV, rule="weight", sinks=2, recent=4)
        ev.start(k0, v0, q0, [100, 97, 60, 1])
        torch.cuda.synchronize()
        out = []
        if not wait:
            torch.cuda._sleep(100_000_000)  # some 50 ms
        for path in paths:
            out.append(ev.attend(0, q[:, 0], k[:, 0], v[:, 0])[0])
            ev.accept(k, v, q, path, attended=False)
            if wait:
                torch.cuda.synchronize()
        ev.check()
        return out + [ev.k, ev.v, ev.pos, ev.weights], ev.lengths, ev.events

    (ahead, *end), (want, *other) = loop(False), loop(True)
    assert end == other and end[1] >= 8
    assert all(torch.equal(a, b) for a, b in zip(ahead, want))


def test_loop_refusals_on_the_device_side():
    ev = api.DecodeEvictor(2, 1, 4, 2, 8, 2, device=DEV, rule="weight")
    g = gen(24)
    k0 = randn(g, 2, 1, 2, 8, D, dtype=BF16)
    ev.start(k0, k0, randn(g, 2, 1, 4, 2, D, dtype=BF16), [8, 8])
    k, q = randn(g, 2, 1, 2, 3, D, dtype=BF16), randn(g, 2, 1, 4, 3, D, dtype=BF16)
    for path in ([[0]], [[0, 1, 2, 0], []], [[3], []], [[-1], []]):
        with pytest.raises(ValueError):
            ev.accept(k, k, q, path)
    with pytest.raises(ValueError):
        ev.attend(1, q[:, 0], k[:, 0], k[:, 0])
    with pytest.raises(ValueError):
        ev.attend(0, q[:, 0].float(), k[:, 0], k[:, 0])
    with pytest.raises(ValueError):
        ev.attend(0, q[:, 0], k[:, 0], None)
    with pytest.raises(api.JacapError):
        ev.attend(0, randn(g, 2, 4, 65, D, dtype=BF16))
    x = q[:, 0].clone().requires_grad_()
    with pytest.raises(ValueError):
        ev.attend(0, x, k[:, 0], k[:, 0])
    with pytest.raises(ValueError):
        api.Rope(device=DEV).apply(x, None, torch.zeros((2, 4), dtype=torch.int32, device=DEV))
    graph = torch.cuda.CUDAGraph()
    ev.attend(0, q[:, 0], k[:, 0], k[:, 0])
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(graph):
            ev.accept(k, k, q, [[0], [1]])
