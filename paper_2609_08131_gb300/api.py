"""Torch-facing convenience layer over the C ABI.

PyTorch supplies device memory and streams only; every step runs in
libjacap's kernels. Errors from the library raise ``JacapError``.
"""

from __future__ import annotations

import ctypes
import math
import threading
from dataclasses import dataclass

import torch

from . import (
    JACAP_ATTEND_ZERO_BYTES,
    JACAP_BF16,
    JACAP_F32,
    JACAP_OK,
    jacap_append,
    jacap_append_path,
    jacap_attend,
    jacap_attend_workspace,
    jacap_attention,
    jacap_compact,
    jacap_device_status,
    jacap_evict_host,
    jacap_evict_weights,
    jacap_host_buffer_size,
    jacap_layout,
    jacap_params,
    jacap_rope,
    jacap_rope_tensor,
    jacap_rotate,
    jacap_schedule_info,
    jacap_score,
    jacap_score_timed,
    jacap_score_out,
    jacap_score_stats,
    jacap_select,
    jacap_select_compact,
    jacap_select_compact_inplace,
    jacap_select_weights,
    jacap_stats_update,
    jacap_status_string,
    jacap_weigh,
    jacap_weigh_workspace,
    jacap_weighing,
    jacap_workspace_offsets,
    jacap_workspace_size,
)


class JacapError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {jacap_status_string(status)} (status {status})")


def _check(status: int, where: str):
    if status != JACAP_OK:
        raise JacapError(status, where)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


@dataclass
class Cache:
    """A KV cache in the library's layout plus the tensors that back it.

    k, v        [L, Hkv, N_tot, 128] (channel stride 1; K and V share strides)
    q_win       [S, L, Hq, w, 128]
    cu_seqlens  int32 [S + 1] on the device; seqlens: host list of n_s
    """

    q_win: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    cu_seqlens: torch.Tensor
    seqlens: list
    num_q_heads: int

    def layout(self) -> jacap_layout:
        k, q = self.k, self.q_win
        if k.dtype not in (torch.float32, torch.bfloat16) or q.dtype != k.dtype or self.v.dtype != k.dtype:
            raise ValueError("q_win, k and v must share dtype float32 or bfloat16")
        if k.stride() != self.v.stride() or k.shape != self.v.shape:
            raise ValueError("k and v must have the same shape and strides")
        if k.stride(-1) != 1 or q.stride(-1) != 1:
            raise ValueError("the channel axis must be contiguous")
        L, Hkv, N, d = k.shape
        S = len(self.seqlens)
        lay = jacap_layout()
        lay.num_seqs = S
        lay.cu_seqlens = self.cu_seqlens.data_ptr()
        lay.max_seqlen = max(1, max(self.seqlens))
        lay.total_tokens = N
        lay.num_layers = L
        lay.num_q_heads = self.num_q_heads
        lay.num_kv_heads = Hkv
        lay.head_dim = d
        lay.window = q.shape[3]
        lay.dtype = JACAP_BF16 if k.dtype == torch.bfloat16 else JACAP_F32
        lay.kv_stride_layer, lay.kv_stride_head, lay.kv_stride_token = k.stride(0), k.stride(1), k.stride(2)
        lay.q_stride_seq, lay.q_stride_layer, lay.q_stride_head, lay.q_stride_pos = (
            q.stride(0), q.stride(1), q.stride(2), q.stride(3))
        return lay


def _enqueue(device, stream, call):
    """call(handle of the stream) with the device current and the stream (the device's current one
    if None) current for what is allocated inside."""
    if stream is None and device.index == torch.cuda.current_device():
        return call(torch._C._cuda_getCurrentRawStream(device.index))
    with torch.cuda.device(device):
        if stream is None:
            stream = torch.cuda.current_stream(device)
        elif stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
        with torch.cuda.stream(stream):
            return call(stream.cuda_stream)


def _made(device):
    """An event behind what a constructor has enqueued, for the first call on another stream (None where there is no
    device; a capture's beginning waits for the device)."""
    if device.type != "cuda" or torch.cuda.is_current_stream_capturing():
        return None
    with torch.cuda.device(device):
        event = torch.cuda.Event()
        event.record()
    return event


def _wait_made(handle):
    """The current stream after what the handle's constructor enqueued (its first eager call waits)."""
    if handle._made is not None and not torch.cuda.is_current_stream_capturing():
        handle._made.wait()
        handle._made = None


def _tensor(name, t, device, dtype, shape, contiguous=False):
    """Checks a tensor argument; its address. None passes, as None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {device}")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this call does not give")
    if not t.is_contiguous():
        if contiguous:
            raise ValueError(f"{name} must be contiguous")
        if t.stride(-1) != 1:
            raise ValueError(f"the last axis of {name} must be contiguous")
    return t.data_ptr()


def _on_one_device(cache):
    """The cache's tensors are on one device and its ranges int32 there: the kernels read all of them."""
    if cache.v.device != cache.k.device or cache.q_win.device != cache.k.device:
        raise ValueError(f"q_win, k and v must be on one device, not {cache.q_win.device}, {cache.k.device} and "
                         f"{cache.v.device}")
    _tensor("cu_seqlens", cache.cu_seqlens, cache.k.device, torch.int32, (len(cache.seqlens) + 1,), True)
    return cache


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling=None):
    """(frequencies, amplitude): the rot_dim / 2 angles per position in 64 bits,
    base^(-2 i / rot_dim), changed for long contexts by ``scaling``:

      None
      ("linear", factor)    positions divided by factor
      ("ntk", factor)       base multiplied by factor^(rot_dim / (rot_dim - 2))
      ("llama3", factor, low, high, length)   pairs that turn fewer than `low` times over
                            the original `length` divided by factor, those that turn more
                            than `high` times kept, a ramp in the turns between
      ("yarn", factor, length, fast, slow)    pairs that turn `fast` times or more over
                            `length` kept, `slow` times or fewer divided by factor, a ramp
                            in the pair's number between; amplitude 0.1 ln(factor) + 1
    """
    if rot_dim < 2 or rot_dim > 128 or rot_dim % 2:
        raise ValueError("rot_dim must be even, 2 to 128")
    if not (base > 0 and math.isfinite(base)):
        raise ValueError("base must be positive")
    kind, args = (None, ()) if scaling is None else (scaling[0], tuple(scaling[1:]))
    wanted = {None: 0, "linear": 1, "ntk": 1, "llama3": 4, "yarn": 4}
    if kind not in wanted or len(args) != wanted[kind]:
        raise ValueError(f"unknown scaling {scaling!r}")
    if args and not args[0] > 0:
        raise ValueError("the scaling factor must be positive")
    half = rot_dim // 2
    if kind == "ntk":
        if rot_dim == 2:
            raise ValueError("ntk scaling needs more than one pair")
        base = base * args[0] ** (rot_dim / (rot_dim - 2))
    f = [base ** (-2.0 * i / rot_dim) for i in range(half)]
    if kind == "linear":
        f = [x / args[0] for x in f]
    elif kind == "llama3":
        factor, low, high, length = args
        if not high > low:
            raise ValueError("llama3 scaling needs low < high")
        keep = [min(max((length * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [x * (k + (1 - k) / factor) for x, k in zip(f, keep)]
    elif kind == "yarn":
        factor, length, fast, slow = args
        if not fast > slow > 0:
            raise ValueError("yarn scaling needs fast > slow > 0")
        at = [rot_dim * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (fast, slow)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot_dim - 1)
        keep = [1 - min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(half)]
        f = [x * (k + (1 - k) / factor) for x, k in zip(f, keep)]
        return f, 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return f, 1.0


class Rope:
    """Rotary positions (``jacap_rotate``): the first ``rot_dim`` channels of every
    head, in pairs (i, i + rot_dim / 2) or, interleaved, (2 i, 2 i + 1), turned by
    position times the pair's frequency (``rope_frequencies``). Keeps the frequencies on
    the device; exact to float32 for every int32 position."""

    def __init__(self, rot_dim: int = 128, base: float = 10000.0, interleaved: bool = False, scaling=None,
                 device="cuda"):
        freq, amplitude = rope_frequencies(rot_dim, base, scaling)
        self.rot_dim, self.amplitude, self.interleaved = int(rot_dim), float(amplitude), bool(interleaved)
        turns = [round(f / (2 * math.pi) * 2.0 ** 64) % (1 << 64) for f in freq]
        self.turns = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns], dtype=torch.int64, device=device)
        self.device = self.turns.device
        self._c = jacap_rope()
        self._c.head_dim, self._c.rot_dim, self._c.interleaved = 128, self.rot_dim, int(self.interleaved)
        self._c.amplitude, self._c.turns = self.amplitude, self.turns.data_ptr()
        self._calls = {}  # arguments of calls by the tensors' shapes and strides (not their addresses)
        self._last = None, None
        self._lock = threading.Lock()

    def apply(self, q, k, positions, inverse: bool = False, inplace: bool = False, stream=None):
        """q, k: [..., heads, 128] (one of them may be None) with one or two leading axes,
        of any strides but the last axis' (float32 or bfloat16); positions: int32 of the
        leading axes' shape. Returns the turned (q, k): new tensors, or the same ones
        with ``inplace``. ``inverse`` turns back (and is the gradient)."""
        key = (None if q is None else (q.dtype, q.shape, q.stride()),
               None if k is None else (k.dtype, k.shape, k.stride()), positions.dtype, positions.shape,
               positions.stride(), inplace)
        last, call = self._last
        if key != last:  # (comparing with the call before is cheaper than a look-up)
            call = self._calls.get(key)
            if call is None:
                call = self._arguments(q, k, positions, inplace)
                if len(self._calls) >= 64:
                    self._calls.clear()
                self._calls[key] = call
            self._last = key, call
        dev = self.device
        grad = torch.is_grad_enabled()
        if positions.device != dev or q is not None and (q.device != dev or grad and q.requires_grad) or \
                k is not None and (k.device != dev or grad and k.requires_grad):
            raise ValueError(f"the tensors must be on {dev} and require no gradient, which this call does not give")
        if stream is None and dev.index == torch._C._cuda_getDevice():
            return self._turn(call, q, k, positions, inverse, inplace, torch._C._cuda_getCurrentRawStream(dev.index))
        return _enqueue(dev, stream, lambda st: self._turn(call, q, k, positions, inverse, inplace, st))

    def _turn(self, call, q, k, positions, inverse, inplace, stream):
        S, T, qa, ka, ps, dtype = call
        qy = None if q is None else q if inplace else torch.empty_like(q)
        ky = None if k is None else k if inplace else torch.empty_like(k)
        if S and T:
            with self._lock:  # the addresses are this call's until it returns (threads may share a Rope)
                if q is not None:
                    qa.x, qa.y = q.data_ptr(), qy.data_ptr()
                if k is not None:
                    ka.x, ka.y = k.data_ptr(), ky.data_ptr()
                status = jacap_rotate(self._c, dtype, S, T, positions.data_ptr(), ps, inverse, qa, ka, stream)
            _check(status, "jacap_rotate")
        return qy, ky

    def _arguments(self, q, k, positions, inplace):
        """Checks shapes and strides; the call's arguments but for the addresses."""
        first = q if q is not None else k
        if first is None:
            raise ValueError("q or k must be given")
        lead, dtype = first.shape[:-2], first.dtype
        if len(lead) not in (1, 2) or dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("q and k must be float32 or bfloat16 [tokens, heads, 128] or [requests, tokens, heads, "
                             "128]")
        if positions.dtype is not torch.int32 or positions.shape != lead:
            raise ValueError(f"positions must be int32 of shape {tuple(lead)}")
        two, args = len(lead) == 2, [None, None]
        for i, (name, t) in enumerate((("q", q), ("k", k))):
            if t is None:
                continue
            if (t.dtype is not dtype or t.dim() != len(lead) + 2 or t.shape != (*lead, t.shape[-2], 128)
                    or t.stride(-1) != 1):
                raise ValueError(f"{name} must be {dtype} {(*lead, 'heads', 128)} with a contiguous last axis")
            if t.shape[-2] < 1:
                raise ValueError(f"{name} has no heads")
            xs, ys = t.stride()[:-1], (t if inplace else torch.empty_like(t, device="meta")).stride()[:-1]
            args[i] = jacap_rope_tensor(0, 0, t.shape[-2], xs if two else (0, *xs), ys if two else (0, *ys))
        S, T = lead if two else (1, lead[0])
        ps = (ctypes.c_int64 * 2)(*(positions.stride() if two else (0, positions.stride(0))))
        return S, T, args[0], args[1], ps, JACAP_BF16 if dtype == torch.bfloat16 else JACAP_F32


def tree_masks(parents):
    """The masks of drafted trees for ``CacheAttention``: ``parents[s][t]`` is the drafted
    token that token t of request s follows (before t), or -1 for the cached ones. Returns
    int64 [S, T] on the host: bit j of entry (s, t) says that token t sees token j."""
    rows = []
    for p in parents:
        row = []
        for t, at in enumerate(p):
            if not -1 <= at < t or t >= 64:
                raise ValueError("a token's parent is -1 or an earlier token, of at most 64")
            row.append((row[at] if at >= 0 else 0) | 1 << t)
        rows.append([m - (1 << 64) if m >> 63 else m for m in row])
    return torch.tensor(rows, dtype=torch.int64)


def _strides(t):
    """The strides of the four leading axes (that of an axis of one entry means nothing and may be anything)."""
    st, shape = t.stride(), t.shape
    return [st[i] if shape[i] > 1 else 128 for i in range(4)]


def _query_strides(lay, q):
    lay.q_stride_seq, lay.q_stride_layer, lay.q_stride_head, lay.q_stride_pos = _strides(q)
    return lay


class CacheAttention:
    """Attention of each request's last queries over its cached tokens and, if given, over
    drafted tokens that are not in the cache yet (``jacap_attend``): one token, a chain, or
    a tree (``tree_masks``). ``cache.q_win`` [S, L, Hq, T, 128] gives the shape of the
    queries (T at most 64) and the default ones. Owns the workspace and the outputs
    ``o`` [S, L, Hq, T, 128] and ``lse`` [S, L, Hq, T] (float32), which each run overwrites."""

    def __init__(self, cache: Cache, scale: float | None = None):
        self.cache = _on_one_device(cache)
        self.device, self.dtype = cache.k.device, cache.k.dtype
        q = cache.q_win
        if q.dim() != 5 or q.shape != (len(cache.seqlens), cache.k.shape[0], cache.num_q_heads, q.shape[3], 128):
            raise ValueError("q_win must be [S, L, Hq, T, 128]")
        S, L, Hq, T = q.shape[:4]
        self.lay = _query_strides(cache.layout(), q)
        nbytes = jacap_attend_workspace(self.lay)
        if nbytes == 0:
            raise JacapError(2 if T > 64 else 1, "jacap_attend_workspace")
        self.ws = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
        self.o = torch.empty((S, L, Hq, T, 128), dtype=self.dtype, device=self.device)
        self.lse = torch.empty((S, L, Hq, T), dtype=torch.float32, device=self.device)
        self._attn = jacap_attention()
        self._attn.scale = 1.0 / math.sqrt(128.0) if scale is None else float(scale)
        self._attn.o_strides[:] = self.o.stride()[:4]
        self._attn.lse_strides[:] = self.lse.stride()[:3]
        self._draft_at = self._q_at = None
        self._made = _made(self.device)

    def run(self, q=None, k_draft=None, v_draft=None, tree=None, lengths=None, draft_lens=None, stream=None):
        """q: [S, L, Hq, T, 128] (the cache's q_win if None); k_draft, v_draft: [S, L, Hkv,
        T, 128]; tree: int64 [S, T] masks (None: a chain); lengths: int32
        [S] cached tokens of each request (None: all); draft_lens: int32 [S] queries of
        each request (None: T; rows behind are left as they were). Returns (o, lse)."""
        c, a, dev, dt = self.cache, self._attn, self.device, self.dtype
        S, L, Hq, T = self.lse.shape
        if q is None:
            q = c.q_win
        qp = _tensor("q", q, dev, dt, (S, L, Hq, T, 128))
        a.lengths = _tensor("lengths", lengths, dev, torch.int32, (S,), True)
        a.draft_lens = _tensor("draft_lens", draft_lens, dev, torch.int32, (S,), True)
        a.tree = _tensor("tree", tree, dev, torch.int64, (S, T), True)
        if (k_draft is None) != (v_draft is None) or (tree is not None and k_draft is None):
            raise ValueError("k_draft and v_draft come together, and a tree with them")
        shape = (S, L, c.k.shape[1], T, 128)
        a.k_draft = _tensor("k_draft", k_draft, dev, dt, shape)
        a.v_draft = _tensor("v_draft", v_draft, dev, dt, shape)
        # (strides are written when they differ from the call before: of a call of 9 us on the device that saves 2)
        if k_draft is not None and (at := (k_draft.stride(), v_draft.stride())) != self._draft_at:
            a.draft_strides[:] = _strides(k_draft) + _strides(v_draft)
            self._draft_at = at
        lay = self.lay
        if (at := q.stride()) != self._q_at:
            _query_strides(lay, q)
            self._q_at = at

        def attend(st):
            _wait_made(self)
            _check(jacap_attend(lay, a, qp, c.k.data_ptr(), c.v.data_ptr(), self.o.data_ptr(), self.lse.data_ptr(),
                                self.ws.data_ptr(), self.ws.numel(), st), "jacap_attend")
            return self.o, self.lse

        return _enqueue(dev, stream, attend)

    def check(self, stream=None):
        _check_and_clear(self, self.ws, self.device, stream)


def _check_and_clear(handle, ws, device, stream):
    """Raises what the status word holds, clearing it: a later call starts anew."""
    def read(st):
        _wait_made(handle)
        status = jacap_device_status(ws.data_ptr(), st)
        if status != JACAP_OK:
            ws.zero_()
        return status

    _check(_enqueue(device, stream, read), "device status")


class WeightEvictor:
    """Eviction by accumulated attention: the tokens that received the most attention
    weight from the last queries stay, beside the first ``sinks`` and the last ``recent``
    ones (together at most ``budget``). ``cache.q_win`` [S, L, Hq, w, 128] are those
    queries (Hq / Hkv times w at most 512), the last w tokens' own.

    ``run()`` enqueues ``score()`` and ``select_compact()``. Buffers: ``weights``
    [L, Hkv, N] and ``lse`` [S, L, Hq, w] (float32); ``idx``, ``kept``, ``k_out``,
    ``v_out`` as ``Evictor``'s, and ``weights_out`` [L, Hkv, S, budget]."""

    def __init__(self, cache: Cache, budget: int, sinks: int = 0, recent: int = 0, scale: float | None = None):
        self.cache, self.budget = _on_one_device(cache), int(budget)
        self.sinks, self.recent = int(sinks), int(recent)
        if self.budget < 1 or self.sinks < 0 or self.recent < 0 or self.sinks + self.recent > self.budget:
            raise ValueError("the budget must be positive and hold the sinks and the recent tokens")
        self.device = cache.k.device
        L, Hkv, N, d = cache.k.shape
        S, q = len(cache.seqlens), cache.q_win
        if q.dim() != 5 or q.shape != (S, L, cache.num_q_heads, q.shape[3], 128):
            raise ValueError("q_win must be [S, L, Hq, w, 128]")
        w = q.shape[3]
        self.lay = _query_strides(cache.layout(), q)
        nbytes = jacap_weigh_workspace(self.lay)
        if nbytes == 0:
            raise JacapError(2 if cache.num_q_heads // Hkv * w > 512 else 1, "jacap_weigh_workspace")
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.ws[:64].zero_()
        self._how = jacap_weighing()
        self._how.scale = 1.0 / math.sqrt(128.0) if scale is None else float(scale)
        new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=self.device)  # noqa: E731
        self.weights = new((L, Hkv, N), torch.float32)
        self.lse = new((S, L, cache.num_q_heads, w), torch.float32)
        self.keys = None  # scratch of a selection by tags
        self.idx = new((L, Hkv, S, self.budget), torch.int32)
        self.kept = new((S,), torch.int32)
        self.k_out = new((L, Hkv, S, self.budget, d), cache.k.dtype)
        self.v_out = torch.empty_like(self.k_out)
        self.weights_out = new((L, Hkv, S, self.budget), torch.float32)
        self._made = _made(self.device)

    def score(self, q=None, lse=None, before=None, lengths=None, q_lens=None, q_rows=None, stream=None):
        """The weights (``jacap_weigh``) into ``weights``; returns (weights, lse).
        q: other queries of q_win's shape; lse: the rows' normalisers, as
        ``CacheAttention`` returned them for these queries (computed into ``lse`` if None);
        before: earlier weights to add to (``weights`` itself works); lengths, q_lens: int32
        [S] live tokens and queries of each request; q_rows: int32 [S, w] which query is
        the j-th. All of a prompt's queries: w at a time, from the first ones, with
        lengths the tokens up to the last of them and before=weights from the second call on."""
        c, h, dev = self.cache, self._how, self.device
        if q is None:
            q = c.q_win
        S, L, Hq, w = self.lse.shape
        qp = _tensor("q", q, dev, c.k.dtype, (S, L, Hq, w, 128))
        h.lse_given = int(lse is not None)
        if lse is None:
            lse = self.lse
        lp = _tensor("lse", lse, dev, torch.float32, self.lse.shape, True)
        bp = _tensor("before", before, dev, torch.float32, self.weights.shape, True)
        h.lengths = _tensor("lengths", lengths, dev, torch.int32, (S,), True)
        h.q_lens = _tensor("q_lens", q_lens, dev, torch.int32, (S,), True)
        h.q_rows = _tensor("q_rows", q_rows, dev, torch.int32, (S, w), True)
        lay = _query_strides(self.lay, q)

        def weigh(st):
            _wait_made(self)
            _check(jacap_weigh(lay, h, qp, c.k.data_ptr(), lp, bp, self.weights.data_ptr(), self.ws.data_ptr(),
                               self.ws.numel(), st), "jacap_weigh")
            return self.weights, lse

        return _enqueue(dev, stream, weigh)

    def select_compact(self, weights=None, pos=None, stream=None):
        """The selection by ``weights`` (None: those of ``score()``) and the retained
        cache (``jacap_select_weights``). ``pos``: int32 [L, Hkv, N] tags by which the
        first and the last tokens are told (None: by row)."""
        c, dev = self.cache, self.device
        if weights is None:
            weights = self.weights
        wp = _tensor("weights", weights, dev, torch.float32, self.weights.shape, True)
        pp = _tensor("pos", pos, dev, torch.int32, self.weights.shape, True)
        if pos is not None and not c.k.is_contiguous():
            raise ValueError("tags need a dense cache")

        def select(st):
            _wait_made(self)
            if pos is not None and self.keys is None:
                self.keys = torch.empty_like(self.weights)
            _check(jacap_select_weights(self.lay, wp, pp, self.sinks, self.recent, self.budget, self.idx.data_ptr(),
                                        self.kept.data_ptr(), c.k.data_ptr(), c.v.data_ptr(), self.k_out.data_ptr(),
                                        self.v_out.data_ptr(), self.weights_out.data_ptr(),
                                        None if pos is None else self.keys.data_ptr(),
                                        self.ws.data_ptr(), self.ws.numel(), st), "jacap_select_weights")

        _enqueue(dev, stream, select)

    def run(self, stream=None):
        self.score(stream=stream)
        self.select_compact(stream=stream)

    def check(self, stream=None):
        _check_and_clear(self, self.ws, self.device, stream)


class Evictor:
    """Owns the workspace and output buffers for repeated passes over caches
    of one shape; ``run()`` enqueues score, select and compact."""

    def __init__(self, cache: Cache, budget: int, params: jacap_params | None = None, out_factor=None,
                 layer_group: int | None = None):
        """``out_factor``: optional float32 [L][Hkv][128][128] device tensor of
        factors F with F^T F = W^T W for the output maps W (u_i = W v_i);
        None uses the proxy u_i = v_i.

        ``layer_group``: run the pass over groups of this many layers, one
        after the other on the same stream, with a workspace sized for one
        group instead of the whole cache (units are independent, so the kept
        sets are those of one pass up to near ties; the workspace takes ~36
        bytes per token and KV head of every layer it covers)."""
        self.cache = cache
        self.budget = int(budget)
        self.params = params if params is not None else jacap_params()
        if out_factor is not None:
            L, Hkv = cache.k.shape[0], cache.k.shape[1]
            if (out_factor.dtype != torch.float32 or tuple(out_factor.shape) != (L, Hkv, 128, 128)
                    or not out_factor.is_contiguous() or out_factor.device != cache.k.device):
                raise ValueError("out_factor must be a contiguous float32 [L][Hkv][128][128] tensor on the cache's device")
        self.out_factor = out_factor
        self.lay = cache.layout()
        dev = cache.k.device
        L = cache.k.shape[0]
        gl = L if layer_group is None else max(1, min(int(layer_group), L))
        self.groups = [(l0, min(gl, L - l0)) for l0 in range(0, L, gl)]
        self._glay = {}
        for _, n in self.groups:
            if n not in self._glay:
                lay = cache.layout()
                lay.num_layers = n
                self._glay[n] = lay
        nbytes = max(jacap_workspace_size(lay, self.budget) for lay in self._glay.values())
        if nbytes == 0:
            raise JacapError(1, "jacap_workspace_size")
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        L, Hkv, N, d = cache.k.shape
        S = len(cache.seqlens)
        self.scores = torch.empty((L, Hkv, N), dtype=torch.float32, device=dev)
        self.idx = torch.empty((L, Hkv, S, self.budget), dtype=torch.int32, device=dev)
        self.kept = torch.empty((S,), dtype=torch.int32, device=dev)
        self.k_out = torch.empty((L, Hkv, S, self.budget, d), dtype=cache.k.dtype, device=dev)
        self.v_out = torch.empty_like(self.k_out)

    def schedule_info(self):
        """(schedule, roles) of the scoring pass on the current device: 1 = separate kernels,
        2 = fused (roles = factor, Gram and score CTAs, V tiles per item kept in L2); see
        jacap_schedule_info. With output directions the pass always uses separate kernels."""
        if self.out_factor is not None:
            return 1, (0, 0, 0, 0)
        lay = self._glay[self.groups[0][1]]
        sched, roles = jacap_schedule_info(lay, self.params)
        if sched < 0:
            raise JacapError(-sched, "jacap_schedule_info")
        return sched, roles

    def bind_outputs(self, idx, kept, k_out, v_out):
        """Write the results into caller-owned device tensors (views into a
        larger buffer, for instance) of the shapes and dtypes of ``idx``,
        ``kept``, ``k_out`` and ``v_out``; each must be contiguous."""
        for name, t in (("idx", idx), ("kept", kept), ("k_out", k_out), ("v_out", v_out)):
            ref = getattr(self, name)
            if t.shape != ref.shape or t.dtype != ref.dtype or t.device != ref.device or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {ref.dtype} tensor of shape {tuple(ref.shape)} "
                                 f"on {ref.device}")
        self.idx, self.kept, self.k_out, self.v_out = idx, kept, k_out, v_out

    def score(self, stream=None, events=None):
        """jacap_score; with ``events`` (JACAP_SCORE_KERNELS + 1 torch.cuda.Event
        objects) the timed variant records them around the kernels of the pass."""
        c = self.cache
        if self.out_factor is not None:
            handles = [e.cuda_event for e in events] if events is not None else []
            _check(jacap_score_out(self.lay, self.params, _ptr(c.q_win), _ptr(c.k), _ptr(c.v), _ptr(self.out_factor),
                                   _ptr(self.scores), _ptr(self.ws), self.ws.numel(), _stream(stream), handles),
                   "jacap_score_out")
        elif events is None:
            _check(jacap_score(self.lay, self.params, _ptr(c.q_win), _ptr(c.k), _ptr(c.v), _ptr(self.scores),
                               _ptr(self.ws), self.ws.numel(), _stream(stream)), "jacap_score")
        else:
            handles = [e.cuda_event for e in events]
            _check(jacap_score_timed(self.lay, self.params, _ptr(c.q_win), _ptr(c.k), _ptr(c.v), _ptr(self.scores),
                                     _ptr(self.ws), self.ws.numel(), _stream(stream), handles), "jacap_score_timed")

    def select(self, stream=None):
        _check(jacap_select(self.lay, _ptr(self.scores), self.budget, _ptr(self.idx), _ptr(self.kept),
                            _ptr(self.ws), self.ws.numel(), _stream(stream)), "jacap_select")

    def compact(self, stream=None):
        c = self.cache
        _check(jacap_compact(self.lay, _ptr(c.k), _ptr(c.v), _ptr(self.idx), self.budget, _ptr(self.k_out),
                             _ptr(self.v_out), _stream(stream)), "jacap_compact")

    def select_compact(self, stream=None):
        """jacap_select and jacap_compact in one launch."""
        c = self.cache
        _check(jacap_select_compact(self.lay, _ptr(self.scores), self.budget, _ptr(self.idx), _ptr(self.kept),
                                    _ptr(c.k), _ptr(c.v), _ptr(self.k_out), _ptr(self.v_out), _ptr(self.ws),
                                    self.ws.numel(), _stream(stream)), "jacap_select_compact")

    def run(self, stream=None):
        if len(self.groups) == 1:
            self.score(stream)
            self.select_compact(stream)
            return
        # layer groups: the same calls on sub-layouts whose data pointers start
        # at the group's first layer, writing the group's slices of the outputs
        c, st = self.cache, _stream(stream)
        ek, eq = c.k.element_size(), c.q_win.element_size()
        ws, wn = _ptr(self.ws), self.ws.numel()
        for l0, n in self.groups:
            lay = self._glay[n]
            koff, qoff = l0 * self.lay.kv_stride_layer * ek, l0 * self.lay.q_stride_layer * eq
            k = ctypes.c_void_p(c.k.data_ptr() + koff)
            v = ctypes.c_void_p(c.v.data_ptr() + koff)
            q = ctypes.c_void_p(c.q_win.data_ptr() + qoff)
            scores = _ptr(self.scores[l0:l0 + n])
            if self.out_factor is not None:
                _check(jacap_score_out(lay, self.params, q, k, v, _ptr(self.out_factor[l0:l0 + n]), scores, ws, wn,
                                       st, []), "jacap_score_out")
            else:
                _check(jacap_score(lay, self.params, q, k, v, scores, ws, wn, st), "jacap_score")
            _check(jacap_select_compact(lay, scores, self.budget, _ptr(self.idx[l0:l0 + n]), _ptr(self.kept), k, v,
                                        _ptr(self.k_out[l0:l0 + n]), _ptr(self.v_out[l0:l0 + n]), ws, wn, st),
                   "jacap_select_compact")
            # a later group's first kernel clears the status word: surface a
            # problem of this group first
            if self.device_status(stream) != JACAP_OK:
                _check(self.device_status(stream), f"device status (layers {l0} .. {l0 + n - 1})")

    def device_status(self, stream=None) -> int:
        return jacap_device_status(_ptr(self.ws), _stream(stream))

    def check(self, stream=None):
        _check(self.device_status(stream), "device status")

    def intermediates(self):
        """Views of the workspace intermediates (see jacap_workspace_offsets)."""
        st, off = jacap_workspace_offsets(self.lay, self.budget)
        _check(st, "jacap_workspace_offsets")
        c = self.cache
        L, Hkv, N, d = c.k.shape
        S, Hq = len(c.seqlens), c.num_q_heads
        units = L * Hkv * S

        def view(o, shape):
            n = 1
            for s in shape:
                n *= s
            return self.ws[o:o + 4 * n].view(torch.float32).view(*shape)

        return {
            "mu_scaled": view(off.mu_scaled, (S, L, Hq, d)),
            "lambda": view(off.lambda_, (S, L, Hq, d)),
            "weights": view(off.weights, (L, Hkv, N)),
            "gram": view(off.gram, (L, Hkv, S, d, d)),
            "chol_inv": view(off.chol_inv, (L, Hkv, S, d, d)),
            "units": units,
        }


# Slots of the per-CTA time accounting of a JACAP_TRACE build (jacap_ws_offsets.trace_cta):
# kernel index -> (name, {slot: meaning}); "tiles" counts tiles, every other slot sums ns.
TRACE_CTA_SLOTS = {
    2: ("k_pass", {0: "producer: wait for a free stage", 1: "producer: loop", 2: "MMA: wait for the images",
                   3: "MMA: wait for a tile's operands and a free accumulator", 5: "MMA: loop", 6: "tiles",
                   7: "convert warp: wait for a K tile", 8: "convert warp: wait for a free operand buffer",
                   9: "convert warp: stores into tensor memory", 11: "convert warp: loop",
                   12: "readout warp: wait for an accumulator", 13: "readout warp: readout of a tile",
                   14: "readout warp: loop"}),
    0: ("gram", {0: "producer: wait for a free stage", 1: "producer: loop", 2: "MMA: wait for a scaled operand",
                 3: "MMA: wait for a free accumulator", 4: "MMA: loop", 5: "tiles", 6: "scaling warp: wait for V",
                 7: "scaling warp: wait for the weights", 8: "scaling warp: wait for a free operand buffer",
                 9: "scaling warp: scaling", 10: "scaling warp: loop", 11: "weight warp: wait for V",
                 12: "weight warp: weights of a tile", 13: "weight warp: loop"}),
    1: ("scores", {0: "producer: wait for a free stage", 1: "producer: loop", 2: "MMA: wait for an image",
                   3: "MMA: wait for a free accumulator", 4: "MMA: wait for a V tile", 5: "MMA: loop", 6: "tiles",
                   7: "epilogue warp: wait for an accumulator", 8: "epilogue warp: read, reduce and meet its partner",
                   9: "epilogue warp: weight and store", 10: "epilogue warp: loop"}),
    # slots 1 to 7: the factor role of the fused schedule; 11 to 14: the factor kernel of the separate ones
    3: ("factor", {0: "partial Grams summed into A", 1: "elimination of diagonal block 0",
                   2: "elimination of diagonal block 1", 3: "elimination of diagonal block 2",
                   4: "elimination of diagonal block 3", 5: "elimination warp: wait for the other warps",
                   6: "panels and look-ahead updates", 7: "last inverse phase", 8: "outputs", 9: "units",
                   10: "whole unit", 11: "elimination steps: wait for all vectors",
                   12: "elimination steps: vectors turned into u", 13: "elimination steps: update and vectors left",
                   14: "products before the elimination (output directions)"}),
    4: ("selection", {0: "scores loaded", 1: "boundary key found", 2: "emission", 3: "rows gathered", 4: "units",
                      5: "whole unit"}),
}


def cta_time_accounting(ev: Evictor) -> dict:
    """Per-CTA time accounting of the last pass of ``ev`` (a JACAP_TRACE build): for each
    streaming kernel and the factor, the mean over its CTAs (the first 1024) of every slot,
    in us per CTA and ns per 128-token tile (streaming kernels) or per unit (factor)."""
    st, off = jacap_workspace_offsets(ev.lay, ev.budget)
    _check(st, "jacap_workspace_offsets")
    if off.trace_cta == 0:
        raise RuntimeError("the library was not built with JACAP_TRACE=1")
    torch.cuda.synchronize(ev.ws.device)
    nk = len(TRACE_CTA_SLOTS)
    tc = ev.ws[off.trace_cta:off.trace_cta + nk * 1024 * 16 * 8].view(torch.int64).view(nk, 1024, 16).cpu().double()
    out = {}
    for k, (name, slots) in TRACE_CTA_SLOTS.items():
        # the streaming kernels count 128-token tiles, the factor units
        per = "tile" if "tiles" in slots.values() else "unit"
        count_slot = next(j for j, m in slots.items() if m == per + "s")
        a = tc[k]
        a = a[a[:, count_slot] > 0]
        if a.shape[0] == 0:
            continue
        cnt = a[:, count_slot].clamp(min=1)
        rep = {"ctas": int(a.shape[0]), per + "s_per_cta": float(cnt.mean())}
        for j, m in slots.items():
            if j != count_slot:
                rep[m] = {"us_per_cta": float(a[:, j].mean() / 1e3), "ns_per_" + per: float((a[:, j] / cnt).mean())}
        out[name] = rep
    return out


def evict(cache: Cache, budget: int, params: jacap_params | None = None, check: bool = True) -> Evictor:
    """One eviction pass over a device-resident cache; returns the Evictor
    whose scores / idx / kept / k_out / v_out hold the results."""
    ev = Evictor(cache, budget, params)
    ev.run()
    if check:
        ev.check()
    return ev


class _SlotAttention:
    """What ``DecodeEvictor.attend`` keeps for T tokens: its layer's layout and arguments, the workspace, and the
    normalisers ``lse`` of all layers."""

    def __init__(self, lay, nbytes):
        self.lay, self.nbytes, self.args = lay, nbytes, jacap_attention()
        self.ws = self.lse = None
        self._zeroed, self._filled = False, set()
        self.complete = set()  # layers whose last call, captured or not, was one that leaves every token's normalisers

    def ready(self, layer, shape, device):
        """The layer's part of ``lse``, with the workspace zeroed, on the current stream. Captured calls zero for
        themselves at every replay until an eager call has done so."""
        if self.ws is None:
            self.ws = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
            self.lse = torch.empty(shape, dtype=torch.float32, device=device)
        part = self.lse[:, layer]
        if not self._zeroed or layer not in self._filled:
            if not self._zeroed:
                self.ws[:JACAP_ATTEND_ZERO_BYTES].zero_()
            if layer not in self._filled:
                part.fill_(-math.inf)
            if not torch.cuda.is_current_stream_capturing():
                self._zeroed = True
                self._filled.add(layer)
        return part


class DecodeEvictor:
    """Decoding-stage eviction (Sec. 3.4: statistics from the queries seen so
    far; the decoding experiments of Sec. 4): one cache slot of
    ``budget + interval`` tokens per request and running query statistics.
    Whenever a request's cache reaches budget + interval tokens it is scored
    with those statistics and compacted in place back to ``budget`` tokens
    (by default by moving the kept rows from past the budget into the evicted
    rows, so the slot order is not the token order; ``pos`` records it).
    Requests that fill on the same decode step and sit next to each other are
    evicted together in one pass (one launch of each kernel for all of them).

    Buffers (device), stored [L, Hkv, S, cap(, 128)] so that neighbouring
    requests form one cache layout, exposed request-major:
      k, v    [S, L, Hkv, cap, 128] views, cap = budget + interval; request s
              holds its ``lengths[s]`` tokens in rows 0 .. lengths[s] - 1
      pos     int32 [S, L, Hkv, cap] view: the id of every cached token (the
              prefill tokens are 0 .. n0 - 1, decode step t of a request adds
              n0 + t); it moves with the rows
      stats   float32 [S, L, Hq, 2, 128] (mean, M2), counts int32 [S, L, Hq]
    After an eviction of requests a .. b - 1, ``scores`` [L, Hkv, (b - a) cap]
    and ``idx`` [L, Hkv, b - a, budget] hold that pass's scores and positions.
    A decode step's k, v, id and query go into the slot and the statistics in one
    launch (jacap_append; indexed copies and jacap_stats_update where that takes
    no such tensors); the scoring pass, the selection and the compaction run in
    libjacap's kernels too.

    A model's step reads the slots with ``attend`` (layer by layer, the step's own
    tokens passed as drafted ones: one, a chain, or a tree), with queries and keys turned
    by ``rotate`` where it uses rotary positions, and then enters its token with
    ``step`` or the accepted drafted tokens with ``accept``.
    """

    def __init__(self, num_seqs: int, num_layers: int, num_q_heads: int, num_kv_heads: int, budget: int,
                 interval: int, dtype=torch.bfloat16, params: jacap_params | None = None, device="cuda",
                 preserve_order: bool = False, rule: str = "jacap", sinks: int = 0, recent: int = 0,
                 scale: float | None = None):
        """``preserve_order``: keep the retained rows in ascending slot order
        (moves up to ``budget`` rows per eviction) instead of filling the
        evicted rows with the kept rows from past the budget (moves at most
        ``interval`` rows).

        ``rule``: "jacap", or "weight": the tokens that received the most attention so far
        stay, beside those with ids below ``sinks`` and the last ``recent`` ones. Every
        query adds its softmax weights (``scale``, 1 / sqrt(128) if None, in this rule and
        in ``attend``) to ``weights`` [S, L, Hkv, cap], which move with the rows; no query
        statistics are kept, and after an eviction ``scores`` holds the selection's keys
        (infinite for tokens that stay anyway)."""
        if budget < 1 or interval < 1:
            raise ValueError("budget and interval must be >= 1")
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("dtype must be bfloat16 or float32")
        self.S, self.L, self.Hq, self.Hkv = num_seqs, num_layers, num_q_heads, num_kv_heads
        self.budget, self.interval = int(budget), int(interval)
        self.cap = self.budget + self.interval
        self.dtype = dtype
        self.params = params if params is not None else jacap_params()
        self.preserve_order = bool(preserve_order)
        if rule not in ("jacap", "weight"):
            raise ValueError('rule must be "jacap" or "weight"')
        self.rule, self.sinks, self.recent = rule, int(sinks), int(recent)
        if self.sinks < 0 or self.recent < 0 or self.sinks + self.recent > (self.budget if rule == "weight" else 0):
            raise ValueError("sinks and recent tokens belong to the weight rule, and the budget must hold them")
        self.scale = 1.0 / math.sqrt(128.0) if scale is None else float(scale)
        dev = torch.device(device)
        S, L, Hq, Hkv, cap, d = self.S, self.L, self.Hq, self.Hkv, self.cap, 128
        self._k = torch.zeros((L, Hkv, S, cap, d), dtype=dtype, device=dev)
        self._v = torch.zeros_like(self._k)
        self._pos = torch.full((L, Hkv, S, cap), -1, dtype=torch.int32, device=dev)
        self.k = self._k.permute(2, 0, 1, 3, 4)
        self.v = self._v.permute(2, 0, 1, 3, 4)
        self.pos = self._pos.permute(2, 0, 1, 3)
        self.device = self._k.device
        self.stats = self.counts = None
        if rule == "jacap":
            self.stats = torch.zeros((S, L, Hq, 2, d), dtype=torch.float32, device=dev)
            self.counts = torch.zeros((S, L, Hq), dtype=torch.int32, device=dev)
        else:
            self._w = torch.zeros((L, Hkv, S, cap), dtype=torch.float32, device=dev)
            self.weights = self._w.permute(2, 0, 1, 3)
        self._ints = {}        # small int32 arrays on the device and what they hold
        self._attention = {}   # per number of drafted tokens
        self._attended = (0, set())
        self._weigh_ws = {}
        self.lengths = [0] * S
        self.next_id = [0] * S
        self.events = 0   # request evictions
        self.passes = 0   # scoring passes (one per group of neighbouring requests)
        self.cu = torch.arange(0, (S + 1) * cap, cap, dtype=torch.int32, device=dev)
        self._layouts = {}
        # one request's slot as a cache of cap tokens
        self.slot = self._group_layout(1)
        # one query per (request, layer, head), [S, L, Hq, 128] contiguous
        self.step_layout = self._layout(S, window=1, q_strides=(L * Hq * d, Hq * d, d, d))
        # one workspace serves every group size (the work-item size depends on it); the selection by
        # weights needs a status word
        sizes = [jacap_workspace_size(self._group_layout(n), self.budget) for n in range(1, S + 1)]
        if min(sizes) == 0:
            raise JacapError(1, "jacap_workspace_size")
        nbytes = max(sizes) if rule == "jacap" else 1024
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        self.ws[:64].zero_()  # the status word: nothing to report yet
        self._scores = torch.empty(L * Hkv * S * cap, dtype=torch.float32, device=dev)
        self._idx = torch.empty(L * Hkv * S * self.budget, dtype=torch.int32, device=dev)
        self._kept = torch.empty((S,), dtype=torch.int32, device=dev)
        self._views(1)
        self._made = _made(self.device)

    def _on(self, stream, call):
        """call(handle of the stream) with the device and the stream current, after what the constructor enqueued."""
        def after(st):
            _wait_made(self)
            return call(st)

        return _enqueue(self.device, stream, after if self._made is not None else call)

    def _views(self, n):
        L, Hkv = self.L, self.Hkv
        self.scores = self._scores[:L * Hkv * n * self.cap].view(L, Hkv, n * self.cap)
        self.idx = self._idx[:L * Hkv * n * self.budget].view(L, Hkv, n, self.budget)
        self.kept = self._kept[:n]

    def _layout(self, num_seqs, window, q_strides) -> jacap_layout:
        lay = jacap_layout()
        lay.num_seqs = num_seqs
        lay.cu_seqlens = self.cu.data_ptr()
        lay.max_seqlen = self.cap
        lay.total_tokens = num_seqs * self.cap
        lay.num_layers, lay.num_q_heads, lay.num_kv_heads, lay.head_dim = self.L, self.Hq, self.Hkv, 128
        lay.window = window
        lay.dtype = JACAP_BF16 if self.dtype == torch.bfloat16 else JACAP_F32
        st = self._k.stride()  # [L, Hkv, S, cap, 128]
        lay.kv_stride_layer, lay.kv_stride_head, lay.kv_stride_token = st[0], st[1], st[3]
        lay.q_stride_seq, lay.q_stride_layer, lay.q_stride_head, lay.q_stride_pos = q_strides
        return lay

    def _group_layout(self, n) -> jacap_layout:
        """n neighbouring requests' slots as one cache: request j of the group is
        tokens j cap .. (j + 1) cap - 1 (the storage puts them next to each
        other on the token axis of every (layer, KV head) plane)."""
        if n not in self._layouts:
            self._layouts[n] = self._layout(n, window=1, q_strides=(128, 128, 128, 128))
        return self._layouts[n]

    def _queries(self, q):
        if (q.dtype != self.dtype or q.device != self.device or q.dim() != 5 or q.stride(-1) != 1
                or tuple(q.shape) != (self.S, self.L, self.Hq, q.shape[3], 128)):
            raise ValueError("queries must be [S, L, Hq, m, 128] in the cache dtype, on its device")

    def _merge(self, q, reset: bool, stream=None):
        """q: [S, L, Hq, m, 128] queries (the slot dtype, channel contiguous)."""
        self._queries(q)
        lay = self._layout(self.S, q.shape[3], (q.stride(0), q.stride(1), q.stride(2), q.stride(3)))
        self._on(stream, lambda st: _check(jacap_stats_update(lay, _ptr(q), 1 if reset else 0, _ptr(self.stats),
                                                              _ptr(self.counts), st), "jacap_stats_update"))

    def start(self, k0, v0, q_win, lengths, stream=None):
        """Load the prefill caches (k0, v0: [S, L, Hkv, n, 128], request s using
        its first lengths[s] < cap rows) and start the statistics from the
        prefill window queries q_win [S, L, Hq, w, 128]. All of it runs on ``stream``,
        after what the current stream holds and before what it gets next."""
        if any(n < 0 or n >= self.cap for n in lengths):
            raise ValueError("a prefill cache must hold fewer than budget + interval tokens; evict it first")
        (self._weighing if self.rule == "weight" else self._queries)(q_win)  # refused before the slots change
        n = k0.shape[3]

        def load(_):
            self.k[:, :, :, :n].copy_(k0)
            self.v[:, :, :, :n].copy_(v0)
            ar = torch.arange(self.cap, dtype=torch.int32, device=self.pos.device)
            self.pos.copy_(torch.where(ar < torch.tensor(lengths, device=ar.device)[:, None], ar, -1)[:, None, None, :]
                           .expand_as(self.pos))
            self.lengths = list(lengths)
            self.next_id = list(lengths)
            self._attended = (0, set())
            self._follow(stream)
            if self.rule == "weight":
                self._w.zero_()
                self._weigh(q_win, None, None, stream)
            else:
                self._merge(q_win, reset=True, stream=stream)

        self._between(stream, load)

    def _between(self, stream, call):
        """call(handle) with its torch operations and kernels on `stream`, after what the current stream holds and
        before what it gets next."""
        if stream is None:
            return self._on(None, call)
        with torch.cuda.device(self.device):
            current = torch.cuda.current_stream(self.device)
        if stream != current:
            stream.wait_stream(current)
        out = self._on(stream, call)
        if stream != current:
            current.wait_stream(stream)
        return out

    def append(self, k_new, v_new, q_new, stream=None, attended=None):
        """One decode step for every request: k_new, v_new [S, L, Hkv, 128],
        q_new [S, L, Hq, 128]. Returns the requests whose cache is now full
        (each must be evicted before its next append). On another ``stream`` than the
        current one indexed copies enter the tokens of the rule "jacap", after what the
        current stream holds and before what it gets next. ``attended``: as in ``accept``."""
        full = [s for s in range(self.S) if self.lengths[s] >= self.cap]
        if full:
            raise RuntimeError(f"request {full[0]} is full; evict it first")
        if self.rule == "weight":
            known = self._normalisers(1, attended)
            self._take(k_new.unsqueeze(3), v_new.unsqueeze(3), q_new.unsqueeze(3), [[0]] * self.S, stream, known)
            self._attended = (0, set())  # the next step's normalisers are others
            return [s for s in range(self.S) if self.lengths[s] >= self.cap]
        if self._one_launch(k_new, v_new, q_new, stream):
            self._on(stream, lambda st: _check(
                jacap_append(self.step_layout, _ptr(k_new), _ptr(v_new), k_new.stride()[:3] + v_new.stride()[:3],
                             _ptr(q_new), self.lengths, self.next_id, _ptr(self._k), _ptr(self._v), _ptr(self._pos),
                             _ptr(self.stats), _ptr(self.counts), st), "jacap_append"))
            self.lengths = [n + 1 for n in self.lengths]
            self.next_id = [n + 1 for n in self.next_id]
            self._follow(stream)
            return [s for s in range(self.S) if self.lengths[s] >= self.cap]

        def copy(_):
            dev = self._k.device
            rows = torch.tensor(self.lengths, dtype=torch.long, device=dev)
            reqs = torch.arange(self.S, device=dev)
            # one indexed copy per tensor for all requests (each writes its next free row)
            self._k[:, :, reqs, rows] = k_new.permute(1, 2, 0, 3).to(self.dtype)
            self._v[:, :, reqs, rows] = v_new.permute(1, 2, 0, 3).to(self.dtype)
            ids = torch.tensor(self.next_id, dtype=torch.int32, device=dev)
            self._pos[:, :, reqs, rows] = ids.view(1, 1, self.S).expand(self.L, self.Hkv, self.S)
            self.lengths = [n + 1 for n in self.lengths]
            self.next_id = [n + 1 for n in self.next_id]
            self._follow(stream)
            self.merge_queries(q_new, stream)

        self._between(stream, copy)
        return [s for s in range(self.S) if self.lengths[s] >= self.cap]

    def _one_launch(self, k_new, v_new, q_new, stream) -> bool:
        """Whether jacap_append takes this step: plain tensors of the slots' dtype, device and exact
        shapes with 16-byte aligned rows, nothing to differentiate, and the stream that the indexed
        copies would run on. Otherwise the step is made of indexed copies and jacap_stats_update."""
        if stream is not None and stream != torch.cuda.current_stream(self._k.device):
            return False
        if torch.cuda.is_current_stream_capturing():  # the rows' numbers would be frozen in the graph
            return False
        el16 = 16 // self._k.element_size()
        for t, heads in ((k_new, self.Hkv), (v_new, self.Hkv), (q_new, self.Hq)):
            if (type(t) is not torch.Tensor or t.dtype != self.dtype or t.device != self._k.device or t.requires_grad
                    or tuple(t.shape) != (self.S, self.L, heads, 128) or t.stride(3) != 1 or t.data_ptr() % 16):
                return False
        return q_new.is_contiguous() and all(n % el16 == 0 for n in k_new.stride()[:3] + v_new.stride()[:3])

    def merge_queries(self, q_new, stream=None):
        """Merge one decode step's queries [S, L, Hq, 128] into the running statistics."""
        if (q_new.is_contiguous() and (q_new.dtype, q_new.device) == (self.dtype, self.device)
                and tuple(q_new.shape) == (self.S, self.L, self.Hq, 128)):
            self._on(stream, lambda st: _check(jacap_stats_update(self.step_layout, _ptr(q_new), 0, _ptr(self.stats),
                                                                  _ptr(self.counts), st), "jacap_stats_update"))
        else:
            self._merge(q_new.unsqueeze(3), reset=False, stream=stream)

    def evict(self, s: int, stream=None, events=None, tail=None):
        """Score request s's full slot with the running statistics, select the
        budget best tokens and compact them in place to rows 0 .. budget - 1.
        ``events``: JACAP_SCORE_KERNELS + 1 torch.cuda.Event recorded around
        the scoring kernels; ``tail``: one more, recorded after the selection
        with its in-place compaction (one launch)."""
        self._evict_group(s, s + 1, stream, events, tail)

    def evict_many(self, requests, stream=None):
        """Evict every listed (full) request; neighbouring requests go through
        one pass together. Returns the groups (first, end) that were evicted."""
        groups = []
        for s in sorted(set(requests)):
            if groups and groups[-1][1] == s:
                groups[-1][1] = s + 1
            else:
                groups.append([s, s + 1])
        for a, b in groups:
            self._evict_group(a, b, stream)
        return [tuple(g) for g in groups]

    def schedule_info(self, requests: int | None = None):
        """(schedule, roles) of the scoring pass (of the rule "jacap") over ``requests`` slots evicted together
        (default: all), as jacap_schedule_info reports it."""
        lay = self._group_layout(self.S if requests is None else int(requests))
        sched, roles = jacap_schedule_info(lay, self.params)
        if sched < 0:
            raise JacapError(-sched, "jacap_schedule_info")
        return sched, roles

    def _evict_group(self, a, b, stream=None, events=None, tail=None):
        if any(self.lengths[s] != self.cap for s in range(a, b)):
            raise RuntimeError("only full slots are evicted")
        n = b - a
        lay = self._group_layout(n)
        handles = [e.cuda_event for e in events] if events is not None else []
        k, v, pos = _ptr(self._k[0, 0, a]), _ptr(self._v[0, 0, a]), _ptr(self._pos[0, 0, a])
        if self.rule == "weight" and events is not None:
            raise ValueError("there are no scoring kernels to time: the weights are kept up step by step")
        self._views(n)

        def evict(st):
            if self.rule == "weight":
                _check(jacap_evict_weights(lay, _ptr(self._w[0, 0, a]), pos, self.sinks, self.recent, self.budget,
                                           _ptr(self.idx), _ptr(self.kept), k, v, self.preserve_order,
                                           _ptr(self.scores), _ptr(self.ws), self.ws.numel(), st),
                       "jacap_evict_weights")
                return
            _check(jacap_score_stats(lay, self.params, _ptr(self.stats[a]), _ptr(self.counts[a]), k, v,
                                     _ptr(self.scores), _ptr(self.ws), self.ws.numel(), st, handles),
                   "jacap_score_stats")
            _check(jacap_select_compact_inplace(lay, _ptr(self.scores), self.budget, _ptr(self.idx), _ptr(self.kept), k,
                                                v, pos, self.preserve_order, _ptr(self.ws), self.ws.numel(), st),
                   "jacap_select_compact_inplace")

        self._on(stream, evict)
        self._evicted(a, b, stream, tail)

    def _evicted(self, a, b, stream, tail):
        if tail is not None:
            self._on(stream, lambda _: tail[0].record())
        for s in range(a, b):
            self.lengths[s] = self.budget
        self._follow(stream)
        self.events += b - a
        self.passes += 1

    def step(self, k_new, v_new, q_new, stream=None, attended=None):
        """append() then evict every request that became full (neighbours together)."""
        full = self.append(k_new, v_new, q_new, stream, attended)
        self.evict_many(full, stream)
        return full

    def _int32(self, name, values):
        """The int32 array `name` on the device, holding `values` (copied when they changed)."""
        held, t = self._ints.get(name, (None, None))
        if held != values:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError(f"{name} changed: a graph would hold the old ones")
            host = torch.tensor(values, dtype=torch.int32)
            if t is None or t.shape != host.shape:
                t = torch.empty(host.shape, dtype=torch.int32, device=self.device)
            t.copy_(host, non_blocking=True)
            self._ints[name] = ([list(v) if isinstance(v, (list, tuple)) else v for v in values], t)
        return t

    def _follow(self, stream):
        """The arrays on the device that captured calls read follow the slots' lengths and next ids."""
        if self._ints and not torch.cuda.is_current_stream_capturing():
            now = (("lengths", self.lengths), ("next ids", self.next_id))
            self._on(stream, lambda _: [self._int32(k, x) for k, x in now if k in self._ints])

    def positions(self, tokens: int, depth=None):
        """int32 [S, tokens]: the ids that drafted tokens get if accepted; ``depth``: int32
        [S, tokens] how many drafted tokens come before each (a tree; None: a chain)."""
        first = self._int32("next ids", self.next_id)[:, None]
        if depth is None:
            depth = torch.arange(tokens, dtype=torch.int32, device=self.device)[None]
        return first + depth

    def rotate(self, rope: Rope, q, k, depth=None, stream=None):
        """q [S, Hq, T, 128] and k [S, Hkv, T, 128] of one layer's drafted tokens turned by
        their positions; returns new tensors."""
        T = (q if q is not None else k).shape[2]

        def turn(_):
            at = self.positions(T, depth)
            out = rope.apply(*(None if t is None else t.transpose(1, 2) for t in (q, k)), at)
            return tuple(None if t is None else t.transpose(1, 2) for t in out)

        return self._on(stream, turn)

    def attend(self, layer: int, q, k_draft=None, v_draft=None, tree=None, draft_lens=None, stream=None):
        """Attention of one layer's drafted tokens over the slots and over themselves:
        q [S, Hq, T, 128], k_draft and v_draft [S, Hkv, T, 128], tree int64 [S, T]
        (``tree_masks``; None: a chain; T = 1: the step's own token), draft_lens int32 [S] (rows
        behind are not written). Returns (o [S, Hq, T, 128], lse [S, Hq, T], a view of what the
        next call with as many tokens overwrites). Under the weight rule the normalisers are kept for ``step``,
        ``append`` or ``accept`` (not those of a call without drafted tokens or with draft_lens, which are
        computed again). A captured call follows the slots: its graph reads their lengths when it is replayed; say
        ``attended=True`` when its tokens are entered."""
        if not 0 <= layer < self.L:
            raise ValueError(f"layer must be 0 to {self.L - 1}")
        if not isinstance(q, torch.Tensor) or q.dim() != 4:
            raise ValueError("q must be [S, Hq, T, 128]")
        T = q.shape[2]
        if T not in self._attention:
            lay = self._layout(self.S, max(T, 1), (128, 128, 128, 128))
            lay.num_layers = 1
            nbytes = jacap_attend_workspace(lay)
            if nbytes == 0 or T == 0:
                raise JacapError(2 if T > 64 else 1, "jacap_attend_workspace")
            self._attention[T] = _SlotAttention(lay, nbytes)
        at = self._attention[T]
        lay, a = at.lay, at.args
        dev, S, Hq = self.device, self.S, self.Hq
        qp = _tensor("q", q, dev, self.dtype, (S, Hq, T, 128))
        if (k_draft is None) != (v_draft is None) or (tree is not None and k_draft is None):
            raise ValueError("k_draft and v_draft come together, and a tree with them")
        a.k_draft = _tensor("k_draft", k_draft, dev, self.dtype, (S, self.Hkv, T, 128))
        a.v_draft = _tensor("v_draft", v_draft, dev, self.dtype, (S, self.Hkv, T, 128))
        a.tree = _tensor("tree", tree, dev, torch.int64, (S, T), True)
        a.draft_lens = _tensor("draft_lens", draft_lens, dev, torch.int32, (S,), True)
        a.scale = self.scale
        if k_draft is not None:
            a.draft_strides[:] = _strides(k_draft.unsqueeze(1)) + _strides(v_draft.unsqueeze(1))
        _query_strides(lay, q.unsqueeze(1))

        def attend(st):
            part = at.ready(layer, (S, self.L, Hq, T), dev)
            a.lse_strides[:] = at.lse.stride()[:3]
            o = torch.empty((S, Hq, T, 128), dtype=self.dtype, device=dev)
            a.o_strides[:] = (o.stride(0), 0, o.stride(1), o.stride(2))
            a.lengths = self._int32("lengths", self.lengths).data_ptr()
            _check(jacap_attend(lay, a, qp, self._k[layer].data_ptr(), self._v[layer].data_ptr(), o.data_ptr(),
                                part.data_ptr(), at.ws.data_ptr(), at.ws.numel(), st), "jacap_attend")
            if self._attended[0] != T:
                self._attended = (T, set())
            # the normalisers of every token that may be entered, if a call by itself leaves them
            whole = k_draft is not None and draft_lens is None
            (at.complete.add if whole else at.complete.discard)(layer)
            whole = whole and not torch.cuda.is_current_stream_capturing()  # (else a replay does)
            (self._attended[1].add if whole else self._attended[1].discard)(layer)
            return o, part

        return self._on(stream, attend)

    def accept(self, k_draft, v_draft, q_draft, path, stream=None, attended=None):
        """Enter the accepted drafted tokens of a step: k_draft, v_draft [S, L, Hkv, T, 128],
        q_draft [S, L, Hq, T, 128] (turned, as ``attend`` took them), path[s]: which drafted
        tokens of request s, in order, each seen by those after it (none: an empty list). As in ``step`` a request whose
        slot becomes full is evicted, here in the middle of its path where that happens; returns the
        requests that were evicted.

        ``attended`` (the weight rule): whether the last ``attend`` of T tokens of every layer was that of these
        tokens, so that its normalisers serve for their weights; else they are computed, with another pass over the
        keys. None: as far as this object saw the calls. True: also the replays of captured ones, which it does not
        see (every layer's last call of T tokens, captured or not, must have been one with drafted tokens and without
        draft_lens). False: computed."""
        if len(path) != self.S:
            raise ValueError("one path per request")
        T = k_draft.shape[3]
        left = [[int(t) for t in p] for p in path]
        if any(len(p) > T or any(not 0 <= t < T for t in p) for p in left):
            raise ValueError(f"a path holds at most {T} tokens, 0 to {T - 1}")
        if any(n >= self.cap for n in self.lengths):
            raise RuntimeError("a request is full; evict it first")
        known = self._normalisers(T, attended)
        gone = set()
        while True:
            now = [p[:self.cap - n] for p, n in zip(left, self.lengths)]
            left = [p[len(x):] for p, x in zip(left, now)]
            self._take(k_draft, v_draft, q_draft, now, stream, known)
            full = [s for s in range(self.S) if self.lengths[s] >= self.cap]
            self.evict_many(full, stream)
            gone.update(full)
            if not any(left):
                self._attended = (0, set())  # the next step's normalisers are others
                return sorted(gone)

    def _normalisers(self, T, attended):
        """What the last attentions of T tokens left, where they are those of the tokens that are entered now."""
        if self.rule != "weight":
            return None
        at = self._attention.get(T)
        if attended and (at is None or len(at.complete) != self.L):
            raise ValueError(f"not every layer's last attention of {T} tokens left the normalisers of all of them")
        if attended is None:
            attended = self._attended[0] == T and len(self._attended[1]) == self.L
        return at.lse if attended else None

    def _take(self, k, v, q, path, stream, lse):
        """The drafted tokens `path` into the slots, and their queries into the statistics or weights (with the
        normalisers lse, or computed if None)."""
        S, L, Hq, Hkv, T = self.S, self.L, self.Hq, self.Hkv, k.shape[3]
        for name, t, heads in (("k", k, Hkv), ("v", v, Hkv), ("q", q, Hq)):
            _tensor(name, t, self.device, self.dtype, (S, L, heads, T, 128))
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the rows' numbers would be frozen in the graph")
        depth = max(len(p) for p in path)
        if depth == 0:
            return
        lay = self._layout(S, T, _strides(q))

        def append(st):
            _check(jacap_append_path(lay, _ptr(k), _ptr(v), _strides(k) + _strides(v), _ptr(q),
                                     [p + [0] * (depth - len(p)) for p in path], depth, [len(p) for p in path],
                                     self.lengths, self.next_id, _ptr(self._k), _ptr(self._v), _ptr(self._pos),
                                     _ptr(self.stats), _ptr(self.counts), st), "jacap_append_path")

        self._on(stream, append)
        self.lengths = [n + len(p) for n, p in zip(self.lengths, path)]
        self.next_id = [n + len(p) for n, p in zip(self.next_id, path)]
        self._follow(stream)
        if self.rule == "weight":
            self._weigh(q, lse, path, stream)

    def _weighing(self, q):
        """The layout of a weighing by the queries q and the bytes of its workspace; refuses what has none."""
        self._queries(q)
        lay = self._layout(self.S, q.shape[3], _strides(q))
        nbytes = jacap_weigh_workspace(lay)
        if nbytes == 0:
            raise JacapError(2 if self.Hq // self.Hkv * q.shape[3] > 512 else 1, "jacap_weigh_workspace")
        return lay, nbytes

    def _weigh(self, q, lse, path, stream):
        """Add the weights of the queries q [S, L, Hq, w, 128] (of `path` of them; None: the window of a
        prompt) to the slots' tokens; lse: their normalisers, or None."""
        w = q.shape[3]
        lay, nbytes = self._weighing(q)
        how = jacap_weighing()
        how.scale, how.lse_given = self.scale, int(lse is not None)

        def weigh(st):
            if w not in self._weigh_ws:  # (made on the stream that uses it)
                self._weigh_ws[w] = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
                self._weigh_ws[w][:64].zero_()
            ws = self._weigh_ws[w]
            how.lengths = self._int32("lengths", self.lengths).data_ptr()
            if path is not None and (w > 1 or any(not p for p in path)):
                how.q_lens = self._int32("taken", [len(p) for p in path]).data_ptr()
                how.q_rows = self._int32("path", [p + [-1] * (w - len(p)) for p in path]).data_ptr()
            wp = self._w.data_ptr()
            _check(jacap_weigh(lay, how, _ptr(q), _ptr(self._k), _ptr(lse), None if path is None else wp, wp, _ptr(ws),
                               ws.numel(), st), "jacap_weigh")

        self._on(stream, weigh)

    def check(self, stream=None):
        """Raises what the kernels reported so far."""
        if self.rule == "jacap":
            self._on(stream, lambda st: _check(jacap_device_status(_ptr(self.ws), st), "device status"))
        else:
            _check_and_clear(self, self.ws, self.device, stream)
        for ws in [x.ws for x in self._attention.values() if x.ws is not None] + list(self._weigh_ws.values()):
            _check_and_clear(self, ws, self.device, stream)


class HostEvictor:
    """Eviction of a cache held in pinned host memory (an offloaded cache),
    through ``jacap_evict_host``.

    The library moves the layers to the device in groups of ``group_layers``
    through two device buffers: while group g is scored, selected and
    compacted on the compute stream, group g + 1 is copied on a copy stream.
    Each ``run()`` returns when the kept positions (and, with ``copy_rows``,
    the retained K and V rows) are in host memory.

    q_win_h [S, L, Hq, w, 128], k_h and v_h [L, Hkv, N, 128]: contiguous
    tensors in pinned host memory; cu_seqlens: int32 [S + 1] (host or device),
    fixed with ``seqlens`` at construction like the layout; ``out_factor``:
    optional float32 [L][Hkv][128][128] device tensor, as for ``Evictor``.
    After ``run()``: ``idx_h`` [L, Hkv, S, B], ``kept_h`` [S] and, with
    ``copy_rows``, ``k_out_h``, ``v_out_h`` [L, Hkv, S, B, 128] (pinned host).
    The only device memory is one buffer of ``jacap_host_buffer_size`` bytes.
    """

    def __init__(self, q_win_h, k_h, v_h, cu_seqlens, seqlens, num_q_heads: int, budget: int,
                 params: jacap_params | None = None, group_layers: int = 8, device="cuda", out_factor=None,
                 copy_rows: bool = True):
        dev = torch.device(device)
        for name, t in (("q_win_h", q_win_h), ("k_h", k_h), ("v_h", v_h)):
            if t.device.type != "cpu" or not t.is_pinned() or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous tensor in pinned host memory")
        L, Hkv, N, d = k_h.shape
        S = len(seqlens)
        if v_h.shape != k_h.shape or q_win_h.shape[:2] != (S, L):
            raise ValueError("k_h and v_h must be [L, Hkv, N, 128] and q_win_h [S, L, Hq, w, 128]")
        if out_factor is not None and (out_factor.dtype != torch.float32 or tuple(out_factor.shape) != (L, Hkv, d, d)
                                       or not out_factor.is_contiguous() or out_factor.device != dev):
            raise ValueError("out_factor must be a contiguous float32 [L][Hkv][128][128] tensor on the device")
        self.out_factor = out_factor
        self.L, self.S, self.gl = L, S, max(1, min(int(group_layers), L))
        self.q_h, self.k_h, self.v_h = q_win_h, k_h, v_h
        self.budget = int(budget)
        self.params = params if params is not None else jacap_params()
        self.num_q_heads = num_q_heads
        self.seqlens = list(seqlens)
        self.copy_rows = bool(copy_rows)
        self.cu_h = torch.as_tensor(cu_seqlens, dtype=torch.int32).cpu().contiguous()
        self.lay = Cache(q_win_h, k_h, v_h, self.cu_h, self.seqlens, num_q_heads).layout()  # cu_seqlens: host
        nbytes = jacap_host_buffer_size(self.lay, self.budget, self.gl, 1 if self.copy_rows else 0)
        if nbytes == 0:
            raise JacapError(1, "jacap_host_buffer_size")
        self.dev_buf = torch.empty(nbytes + 1024, dtype=torch.uint8, device=dev)
        off = (-self.dev_buf.data_ptr()) % 1024
        self.dev_buf = self.dev_buf[off:off + nbytes]
        self.idx_h = torch.empty((L, Hkv, S, self.budget), dtype=torch.int32).pin_memory()
        self.kept_h = torch.empty((S,), dtype=torch.int32).pin_memory()
        self.k_out_h = self.v_out_h = None
        if self.copy_rows:
            self.k_out_h = torch.empty((L, Hkv, S, self.budget, d), dtype=k_h.dtype).pin_memory()
            self.v_out_h = torch.empty_like(self.k_out_h).pin_memory()
        self.copy_stream = torch.cuda.Stream(device=dev)

    @property
    def h2d_bytes(self) -> int:
        """Bytes one ``run()`` copies host->device (the cache and its window; cu_seqlens aside)."""
        return sum(t.numel() * t.element_size() for t in (self.q_h, self.k_h, self.v_h))

    @property
    def d2h_bytes(self) -> int:
        """Bytes one ``run()`` copies device->host: positions, kept counts and, with copy_rows, the rows."""
        rows = 0 if not self.copy_rows else 2 * self.k_out_h.numel() * self.k_out_h.element_size()
        return (self.idx_h.numel() + self.kept_h.numel()) * 4 + rows

    def run(self, stream=None):
        of = _ptr(self.out_factor) if self.out_factor is not None else ctypes.c_void_p(0)
        st = jacap_evict_host(self.lay, self.params, self.budget, self.gl, _ptr(self.q_h), _ptr(self.k_h),
                              _ptr(self.v_h), of, _ptr(self.idx_h), _ptr(self.kept_h),
                              _ptr(self.k_out_h), _ptr(self.v_out_h), _ptr(self.dev_buf), self.dev_buf.numel(),
                              _stream(stream), _stream(self.copy_stream))
        _check(st, "jacap_evict_host")

    def check(self, stream=None):
        """Errors are returned by ``run()`` itself (it raises); nothing more to read."""
        return None
