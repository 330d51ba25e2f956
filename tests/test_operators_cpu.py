"""The operators around the cached tokens' attention, as far as a host without a GPU goes: what the
calls refuse before they touch a device, the rotary frequencies, and the masks of drafted trees."""

import ctypes
import math

import pytest
import torch

import paper_2609_08131_gb300 as J
from paper_2609_08131_gb300 import api
from test_abi_cpu import good_layout

BAD, NO, WS = J.JACAP_ERR_INVALID_ARG, J.JACAP_ERR_UNSUPPORTED, J.JACAP_ERR_WORKSPACE
P, MIS8, MIS4, MIS2 = (ctypes.c_void_p(a) for a in (0x1000, 0x1008, 0x1004, 0x1002))
PASSED = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that passes the host's checks would run")


def refused(status, expect):
    assert status == expect, J.jacap_status_string(status)


# what a good call answers here: every check of the host passed, and there is no device
def passed(status):
    assert status not in (J.JACAP_OK, BAD, NO, WS), J.jacap_status_string(status)


# ------------------------------------------------------------------- rotate ----
def rotate(rope=None, dtype=J.JACAP_BF16, S=2, T=5, pos=P, ps=(5, 1), inverse=0, q=True, k=True, **kw):
    r = J.jacap_rope()
    r.head_dim, r.rot_dim, r.interleaved, r.amplitude, r.turns = 128, 128, 0, 1.0, 0x1000
    for n, v in (rope or {}).items():
        setattr(r, n, v)
    t = {"x": 0x1000, "y": 0x2000, "heads": 8, "x_strides": (5 * 1024, 1024, 128), "y_strides": (5 * 1024, 1024, 128), **kw}
    one = J.jacap_rope_tensor(t["x"], t["y"], t["heads"], t["x_strides"], t["y_strides"])
    two = J.jacap_rope_tensor(0x3000, 0x4000, 2, (1280, 256, 128), (1280, 256, 128))
    return J.jacap_rotate(r, dtype, S, T, pos, None if ps is None else (ctypes.c_int64 * 2)(*ps), inverse,
                          one if q else None, two if k else None, None)


@PASSED
@pytest.mark.parametrize("kw", [{}, {"q": False}, {"k": False}, {"S": 0}, {"T": 0}, {"rope": {"rot_dim": 2}},
                                {"rope": {"rot_dim": 66, "interleaved": 1}}, {"x": 0x1002}, {"x": 0x2000},
                                {"dtype": J.JACAP_F32}, {"ps": (0, 0)}, {"inverse": 1}])
def test_rotate_takes(kw):
    passed(rotate(**kw))


@pytest.mark.parametrize("kw,expect", [
    ({"rope": {"head_dim": 64}}, NO), ({"rope": {"rot_dim": 0}}, BAD), ({"rope": {"rot_dim": 63}}, BAD),
    ({"rope": {"rot_dim": 130}}, BAD), ({"rope": {"interleaved": 2}}, BAD), ({"rope": {"turns": None}}, BAD),
    ({"rope": {"turns": 0x1004}}, BAD), ({"rope": {"amplitude": math.nan}}, BAD), ({"rope": {"amplitude": math.inf}}, BAD),
    ({"dtype": 7}, BAD), ({"S": -1}, BAD), ({"T": -1}, BAD), ({"S": 1 << 16, "T": 1 << 15}, BAD), ({"pos": None}, BAD),
    ({"pos": MIS2}, BAD), ({"ps": None}, BAD), ({"ps": (-1, 1)}, BAD), ({"inverse": 2}, BAD), ({"q": False, "k": False}, BAD),
    ({"x": 0}, BAD), ({"y": 0}, BAD), ({"x": 0x1001}, BAD), ({"x": 0x1002, "dtype": J.JACAP_F32}, BAD), ({"heads": 0}, BAD),
    ({"x_strides": (5 * 1024, -128, 128)}, BAD), ({"y_strides": (0, 1024, 128)}, BAD),
    ({"y_strides": (4096, 1024, 64)}, BAD), ({"x": 0x2000, "x_strides": (8192, 1024, 128)}, BAD),
])
def test_rotate_refuses(kw, expect):
    refused(rotate(**kw), expect)


# ------------------------------------------------------------------- attend ----
def attend(lay=None, attn=None, q=P, k=P, v=P, o=P, lse=P, ws=P, less=0):
    layout = good_layout(**(lay or {}))
    T = layout.window
    a = J.jacap_attention()
    a.scale, a.k_draft, a.v_draft, a.lengths, a.draft_lens, a.tree = 0.1, 0x1000, 0x1000, 0x1000, 0x1000, 0x1000
    a.draft_strides[:] = [2 * 2 * T * 128, 2 * T * 128, T * 128, 128] * 2
    a.o_strides[:] = [2 * 8 * T * 128, 8 * T * 128, T * 128, 128]
    a.lse_strides[:] = [2 * 8 * T, 8 * T, T]
    for n, x in (attn or {}).items():
        if n.endswith("strides"):
            for i, new in enumerate(x):
                if new is not None:
                    getattr(a, n)[i] = new
        else:
            setattr(a, n, x)
    nbytes = J.jacap_attend_workspace(layout)
    return J.jacap_attend(layout, a, q, k, v, o, lse, ws, max(nbytes - less, 0), None)


@PASSED
@pytest.mark.parametrize("kw", [
    {}, {"lse": None}, {"attn": {"lengths": None, "draft_lens": None, "tree": None}},
    {"attn": {"tree": None, "k_draft": None, "v_draft": None}}, {"lay": {"window": 1}}, {"lay": {"window": 64}},
    {"lay": {"dtype": J.JACAP_F32}}, {"attn": {"lse_strides": (1 << 20, None, None)}}, {"attn": {"scale": 1e30}}])
def test_attend_takes(kw):
    passed(attend(**kw))


@pytest.mark.parametrize("kw,expect", [
    ({"lay": {"window": 65}}, NO), ({"lay": {"head_dim": 64}}, NO), ({"lay": {"num_q_heads": 7}}, BAD),
    ({"lay": {"cu_seqlens": 0}}, BAD), ({"q": None}, BAD), ({"k": None}, BAD), ({"v": None}, BAD), ({"o": None}, BAD),
    ({"ws": None}, BAD), ({"q": MIS8}, BAD), ({"k": MIS8}, BAD), ({"v": MIS8}, BAD), ({"o": MIS8}, BAD), ({"lse": MIS2}, BAD),
    ({"attn": {"scale": 0.0}}, BAD), ({"attn": {"scale": -1.0}}, BAD), ({"attn": {"scale": math.nan}}, BAD),
    ({"attn": {"scale": math.inf}}, BAD), ({"attn": {"scale": 1e-31}}, BAD), ({"attn": {"scale": 1e31}}, BAD),
    ({"attn": {"k_draft": None}}, BAD), ({"attn": {"v_draft": None}}, BAD),
    ({"attn": {"k_draft": None, "v_draft": None}}, BAD),  # a tree of nothing
    ({"attn": {"k_draft": 0x1008}}, BAD), ({"attn": {"v_draft": 0x1002}}, BAD), ({"attn": {"tree": 0x1004}}, BAD),
    ({"attn": {"lengths": 0x1002}}, BAD), ({"attn": {"draft_lens": 0x1001}}, BAD),
    ({"attn": {"draft_strides": (None, None, None, 132)}}, BAD), ({"attn": {"draft_strides": (None, 64)}}, BAD),
    ({"attn": {"draft_strides": (None,) * 7 + (0,)}}, BAD), ({"attn": {"draft_strides": (1 << 38,)}}, BAD),
    ({"attn": {"o_strides": (None, None, None, 64)}}, BAD), ({"attn": {"o_strides": (None, 1028)}}, BAD),
    ({"attn": {"o_strides": (-128,)}}, BAD), ({"attn": {"lse_strides": (None, None, 8)}}, BAD),
    ({"less": 1}, WS), ({"ws": ctypes.c_void_p(0x1010)}, WS),
])
def test_attend_refuses(kw, expect):
    refused(attend(**kw), expect)


def test_attend_workspace_follows_the_splits():
    def size(n, window=1):
        return J.jacap_attend_workspace(good_layout(num_seqs=1, max_seqlen=n, total_tokens=n, window=window,
                                                    kv_stride_head=n * 128, kv_stride_layer=2 * n * 128))
    assert J.jacap_attend_workspace(good_layout(window=65)) == 0
    assert 0 < size(64) <= size(256) < size(1024) < size(131072)
    # a split's sums are at most a quarter of the K and V that it reads
    for window in (1, 8, 64):
        assert size(131072, window) < 2 * 2 * 2 * 131072 * 256 / 4 + (1 << 16)


@pytest.mark.parametrize("window", [1, 8, 20, 64])
def test_attend_workspace_of_many_units(window):
    """bf16: what the borders between CTAs leave, however many units and tokens there are."""
    lay = good_layout(num_seqs=64, num_layers=28, num_q_heads=64, num_kv_heads=8, max_seqlen=131072, total_tokens=64 * 131072,
                      window=window)
    units = 64 * 28 * 8
    assert 0 < J.jacap_attend_workspace(lay) < 2 * 320 * 128 * (512 + 8) + 8 * units + (1 << 14)


# -------------------------------------------------------------------- weigh ----
def weigh(lay=None, how=None, q=P, k=P, lse=P, before=P, weights=P, ws=P, less=0):
    layout = good_layout(**(lay or {}))
    h = J.jacap_weighing()
    h.scale = 0.1
    for n, x in (how or {}).items():
        setattr(h, n, x)
    return J.jacap_weigh(layout, h, q, k, lse, before, weights, ws, max(J.jacap_weigh_workspace(layout) - less, 0), None)


@PASSED
@pytest.mark.parametrize("kw", [{}, {"lse": None}, {"before": None}, {"how": {"lse_given": 1}}, {"lay": {"window": 128}},
                                {"how": {"lengths": 0x1004, "q_lens": 0x1004, "q_rows": 0x1004}},
                                {"lay": {"dtype": J.JACAP_F32}}])
def test_weigh_takes(kw):
    passed(weigh(**kw))


@pytest.mark.parametrize("kw,expect", [
    ({"lay": {"window": 129}}, NO), ({"lay": {"head_dim": 64}}, NO), ({"lay": {"max_seqlen": 0}}, BAD), ({"q": None}, BAD),
    ({"k": None}, BAD), ({"weights": None}, BAD), ({"ws": None}, BAD), ({"q": MIS8}, BAD), ({"k": MIS8}, BAD),
    ({"lse": MIS2}, BAD), ({"before": MIS2}, BAD), ({"weights": MIS2}, BAD), ({"how": {"scale": 0.0}}, BAD),
    ({"how": {"scale": math.inf}}, BAD), ({"how": {"scale": math.nan}}, BAD), ({"how": {"lse_given": 2}}, BAD),
    ({"how": {"lse_given": 1}, "lse": None}, BAD), ({"how": {"lengths": 0x1002}}, BAD), ({"how": {"q_lens": 0x1002}}, BAD),
    ({"how": {"q_rows": 0x1002}}, BAD), ({"less": 1}, WS), ({"ws": ctypes.c_void_p(0x1010)}, WS),
])
def test_weigh_refuses(kw, expect):
    refused(weigh(**kw), expect)


# ----------------------------------------------------------- select and evict ----
def select(lay=None, weights=P, pos=None, sinks=2, recent=2, budget=8, idx=P, kept=P, k=P, v=P, k_out=P, v_out=P, w_out=P,
           keys=None, ws=P, nbytes=64):
    return J.jacap_select_weights(good_layout(**(lay or {})), weights, pos, sinks, recent, budget, idx, kept, k, v, k_out,
                                  v_out, w_out, keys, ws, nbytes, None)


def evict(lay=None, weights=P, pos=None, sinks=2, recent=2, budget=8, idx=P, kept=P, k=P, v=P, order=0,
          keys=ctypes.c_void_p(0x2000), ws=P, nbytes=64):
    return J.jacap_evict_weights(good_layout(**(lay or {})), weights, pos, sinks, recent, budget, idx, kept, k, v, order,
                                 keys, ws, nbytes, None)


BOTH = [({"weights": None}, BAD), ({"weights": MIS2}, BAD), ({"idx": None}, BAD), ({"idx": MIS2}, BAD), ({"kept": None}, BAD),
        ({"kept": MIS2}, BAD), ({"k": None}, BAD), ({"v": None}, BAD), ({"k": MIS8}, BAD), ({"v": MIS8}, BAD),
        ({"budget": 0}, BAD), ({"sinks": -1}, BAD), ({"recent": -1}, BAD), ({"sinks": 5, "recent": 4}, BAD),
        ({"sinks": (1 << 31) - 1, "recent": (1 << 31) - 1}, BAD), ({"ws": None}, BAD), ({"ws": ctypes.c_void_p(0x1040)}, WS),
        ({"nbytes": 63}, WS), ({"keys": P}, BAD), ({"pos": MIS2, "keys": ctypes.c_void_p(0x2000)}, BAD),
        ({"lay": {"head_dim": 64}}, NO)]


@pytest.mark.parametrize("kw,expect", BOTH + [({"pos": P}, BAD), ({"k_out": None}, BAD), ({"v_out": None}, BAD),
                                              ({"k_out": MIS8}, BAD), ({"w_out": MIS2}, BAD)])
def test_select_weights_refuses(kw, expect):
    refused(select(**kw), expect)


@pytest.mark.parametrize("kw,expect", BOTH + [({"keys": None}, BAD), ({"order": 2}, BAD),
                                              ({"lay": {"kv_stride_token": 136}}, BAD)])
def test_evict_weights_refuses(kw, expect):
    refused(evict(**kw), expect)


@PASSED
def test_select_and_evict_take():
    passed(select())
    passed(select(w_out=None))
    passed(select(pos=P, keys=ctypes.c_void_p(0x2000)))
    passed(evict())
    passed(evict(pos=P, order=1))
    passed(evict(lay={"kv_stride_token": 256}))  # a head's 500 x 128 elements are 250 of these strides


# ------------------------------------------------------ more than a launch takes ----
MANY = {"num_layers": 1 << 10, "num_q_heads": 1 << 10, "num_kv_heads": 1 << 10}
HUGE = {"num_layers": (1 << 31) - 1, "num_q_heads": (1 << 31) - 1, "num_kv_heads": (1 << 31) - 1}


@pytest.mark.parametrize("lay", [
    {**MANY, "num_seqs": 1 << 11}, {**HUGE, "num_seqs": (1 << 31) - 1}, {**HUGE, "num_seqs": 2},
    {"total_tokens": 1 << 30, "max_seqlen": 1 << 30, "num_layers": 32, "num_q_heads": 8, "num_kv_heads": 8},
    {**MANY, "num_seqs": 1 << 8, "window": 64}, {**MANY, "num_seqs": 1 << 8, "dtype": J.JACAP_F32}])
def test_attend_refuses_sizes_past_a_launch_s(lay):
    assert J.jacap_attend_workspace(good_layout(**lay)) == 0
    refused(attend(lay=lay), NO)


@pytest.mark.parametrize("lay", [
    {**MANY, "num_seqs": 1 << 11}, {**HUGE, "num_seqs": (1 << 31) - 1},
    {**MANY, "num_seqs": 1 << 8, "num_q_heads": 1 << 13, "window": 64},
    {**MANY, "total_tokens": 1 << 30, "max_seqlen": 1 << 30}])
def test_weigh_refuses_sizes_past_a_launch_s(lay):
    assert J.jacap_weigh_workspace(good_layout(**lay)) == 0
    refused(weigh(lay=lay), NO)


@pytest.mark.parametrize("lay", [{**MANY, "num_seqs": 1 << 11}, {**HUGE, "num_seqs": (1 << 31) - 1}])
def test_selections_refuse_more_units_than_a_launch_s(lay):
    refused(select(lay=lay), NO)
    refused(evict(lay=lay), NO)
    # the keys of long requests come from several blocks each
    refused(evict(lay={**MANY, "num_seqs": 1 << 8, "total_tokens": 1 << 20, "max_seqlen": 1 << 18}), NO)


# -------------------------------------------------------------- append_path ----
def append(lay=None, path=((0, 1), (2, 3)), depth=2, taken=(2, 1), lengths=(3, 0), ids=(3, 0), strides=None, k_new=P, v_new=P,
           q_new=P, k=P, v=P, pos=P, stats=P, counts=P):
    layout = good_layout(total_tokens=600, kv_stride_head=600 * 128, kv_stride_layer=2 * 600 * 128, **(lay or {}))
    return J.jacap_append_path(layout, k_new, v_new, strides or [8192, 4096, 2048, 128] * 2, q_new, path, depth, taken, lengths,
                               ids, k, v, pos, stats, counts, None)


@PASSED
def test_append_path_takes():
    passed(append())
    passed(append(stats=None, counts=None, q_new=None))
    passed(append(taken=(0, 0)))
    passed(append(path=((0, 99), (0, -5)), taken=(1, 1)))  # entries behind the accepted ones are not read
    passed(append(lengths=(298, 299)))


@pytest.mark.parametrize("kw", [
    {"path": ((0, 16), (2, 3))}, {"path": ((0, -1), (2, 3))}, {"taken": (3, 1)}, {"taken": (-1, 1)}, {"lengths": (-1, 0)},
    {"lengths": (299, 0)}, {"path": ((0,) * 17,) * 2, "depth": 17}, {"k_new": None}, {"v_new": None}, {"q_new": None},
    {"k": None}, {"v": None}, {"stats": None}, {"counts": None}, {"k_new": MIS8}, {"q_new": MIS8}, {"stats": MIS8},
    {"counts": MIS2}, {"pos": MIS2}, {"strides": [8192, 4096, 2048, 132] * 2}, {"strides": [-8, 0, 0, 128] * 2},
    {"lay": {"max_seqlen": 299}},
])
def test_append_path_refuses(kw):
    refused(append(**kw), BAD)


# ------------------------------------------------------------- frequencies ----
@pytest.mark.parametrize("rot", [2, 64, 126, 128])
def test_plain_frequencies(rot):
    freq, amplitude = api.rope_frequencies(rot, 500.0)
    assert amplitude == 1.0 and len(freq) == rot // 2
    for i, f in enumerate(freq):
        assert f == pytest.approx(500.0 ** (-2 * i / rot), rel=1e-15)


def test_scaled_frequencies():
    plain, _ = api.rope_frequencies(128, 10000.0)
    linear, a = api.rope_frequencies(128, 10000.0, ("linear", 4.0))
    assert a == 1.0 and all(x == pytest.approx(y / 4) for x, y in zip(linear, plain))
    ntk, _ = api.rope_frequencies(128, 10000.0, ("ntk", 4.0))
    # the slowest pair turns `factor` times slower, the fastest as before
    assert ntk[0] == plain[0] and ntk[-1] == pytest.approx(plain[-1] / 4, rel=1e-12)
    llama, _ = api.rope_frequencies(128, 10000.0, ("llama3", 8.0, 1.0, 4.0, 8192))
    yarn, amplitude = api.rope_frequencies(128, 10000.0, ("yarn", 8.0, 4096, 32.0, 1.0))
    assert amplitude == pytest.approx(0.1 * math.log(8.0) + 1)
    for scaled, length, fast in ((llama, 8192, 4.0), (yarn, 4096, 32.0)):
        for f, p in zip(scaled, plain):
            turns = length * p / (2 * math.pi)
            assert p / 8 * (1 - 1e-12) <= f <= p * (1 + 1e-12)
            if turns > fast * 1.2:
                assert f == pytest.approx(p)
            if turns < 0.8:
                assert f == pytest.approx(p / 8)
        ratio = [f / p for f, p in zip(scaled, plain)]
        assert all(x >= y - 1e-12 for x, y in zip(ratio, ratio[1:]))  # the ramp only falls


@pytest.mark.parametrize("args", [(0,), (3,), (130,), (128, 10000.0, ("spline", 2.0)), (128, 0.0), (128, -1.0),
                                  (128, math.nan), (128, 10000.0, ("linear", 0.0))])
def test_frequencies_refuse(args):
    with pytest.raises(ValueError):
        api.rope_frequencies(*args)


# ------------------------------------------------------------------- trees ----
def test_tree_masks():
    m = api.tree_masks([[-1, 0, 0, 2, 1], [-1, -1, -1, -1, -1]])
    assert m.tolist() == [[0b1, 0b11, 0b101, 0b1101, 0b10011], [1, 2, 4, 8, 16]]
    chain = api.tree_masks([list(range(-1, 63))])[0].tolist()
    assert [c % (1 << 64) for c in chain] == [(2 << t) - 1 for t in range(64)]


@pytest.mark.parametrize("parents", [[[0]], [[-1, 1]], [[-2]], [[-1, 2, 0]], [list(range(-1, 64))]])
def test_tree_masks_refuse(parents):
    with pytest.raises(ValueError):
        api.tree_masks(parents)


# -------------------------------------------------------------- torch layer ----
@pytest.mark.parametrize("kw", [{"rule": "other"}, {"sinks": 2}, {"rule": "weight", "sinks": 5, "recent": 4},
                                {"rule": "weight", "sinks": -1}, {"rule": "weight", "recent": -2}])
def test_decode_evictor_refuses(kw):
    with pytest.raises(ValueError):
        api.DecodeEvictor(1, 1, 2, 1, 8, 4, device="cpu", **kw)


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_decode_evictor_starts_with_nothing_to_report(rule, monkeypatch):
    """check() reads the status word, before the first pass writes one too."""
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: empty(*a, **kw).fill_(7))
    ev = api.DecodeEvictor(1, 1, 2, 1, 8, 4, device="cpu", rule=rule)
    monkeypatch.undo()
    assert (ev.ws[:64] == 0).all()


def cpu_cache(S=1, L=1, Hq=2, Hkv=1, w=4, n=32):
    k = torch.zeros((L, Hkv, S * n, 128), dtype=torch.bfloat16)
    return api.Cache(torch.zeros((S, L, Hq, w, 128), dtype=torch.bfloat16), k, torch.zeros_like(k),
                     torch.arange(0, (S + 1) * n, n, dtype=torch.int32), [n] * S, Hq)


@pytest.mark.parametrize("args,kw", [((0,), {}), ((8,), {"sinks": -1}), ((8,), {"recent": -1}),
                                     ((8,), {"sinks": 5, "recent": 4})])
def test_weight_evictor_refuses(args, kw):
    with pytest.raises(ValueError):
        api.WeightEvictor(cpu_cache(), *args, **kw)


def test_arguments_are_checked_before_anything_runs():
    att = api.CacheAttention(cpu_cache())
    good = torch.zeros((1, 1, 1, 4, 128), dtype=torch.bfloat16)
    for kw in ({"q": torch.zeros((1, 1, 2, 3, 128), dtype=torch.bfloat16)}, {"q": torch.zeros((1, 1, 2, 4, 128))},
               {"q": torch.zeros((1, 1, 2, 4, 128), dtype=torch.bfloat16, requires_grad=True)},
               {"q": torch.zeros((1, 1, 2, 128, 4), dtype=torch.bfloat16).transpose(3, 4)},
               {"k_draft": good}, {"v_draft": good}, {"tree": torch.zeros((1, 4), dtype=torch.int64)},
               {"k_draft": good, "v_draft": good[..., :3, :]}, {"k_draft": good, "v_draft": good.float()},
               {"k_draft": good, "v_draft": good, "tree": torch.zeros((1, 3), dtype=torch.int64)},
               {"k_draft": good, "v_draft": good, "tree": torch.zeros((1, 4), dtype=torch.int32)},
               {"lengths": torch.zeros(1)}, {"lengths": torch.zeros(2, dtype=torch.int32)}, {"lengths": [3]},
               {"draft_lens": torch.zeros((1, 1), dtype=torch.int32)}):
        with pytest.raises(ValueError):
            att.run(**kw)
    rope = api.Rope(64, device="cpu")
    x, at = torch.zeros((2, 3, 4, 128)), torch.zeros((2, 3), dtype=torch.int32)
    for args in ((None, None, at), (x, None, at[:1]), (x, None, at.long()), (x.half(), None, at), (x[..., :64], None, at),
                 (x, x.bfloat16(), at), (x.transpose(2, 3), None, at), (x, x[:1], at), (x.clone().requires_grad_(), None, at),
                 (x[:, :, :0], None, at), (x[0, 0], None, at[0, 0])):
        with pytest.raises(ValueError):
            rope.apply(*args)
    ev = api.WeightEvictor(cpu_cache(), 8)
    for kw in ({"lse": torch.zeros((1, 1, 2, 3))}, {"before": torch.zeros((1, 1, 31))}, {"q_rows": torch.zeros((1, 4))},
               {"q_lens": torch.zeros(3, dtype=torch.int32)}, {"lengths": torch.zeros(1, dtype=torch.int64)}):
        with pytest.raises(ValueError):
            ev.score(**kw)
    with pytest.raises(ValueError):
        ev.select_compact(weights=torch.zeros((1, 1, 31)))
    with pytest.raises(ValueError):
        ev.select_compact(pos=torch.zeros((1, 1, 32)))


@pytest.mark.parametrize("change", [
    {"cu_seqlens": torch.tensor([0, 32])}, {"cu_seqlens": torch.tensor([0, 16, 32], dtype=torch.int32)},
    {"cu_seqlens": torch.tensor([0, 0, 32, 0], dtype=torch.int32)[::2]}, {"cu_seqlens": [0, 32]},
    {"cu_seqlens": torch.tensor([0, 32], dtype=torch.int32, device="meta")},
    {"v": torch.zeros((1, 1, 32, 128), dtype=torch.bfloat16, device="meta")},
    {"q_win": torch.zeros((1, 1, 2, 4, 128), dtype=torch.bfloat16, device="meta")}])
def test_a_cache_is_on_one_device(change):
    cache = cpu_cache()
    for name, t in change.items():
        setattr(cache, name, t)
    with pytest.raises(ValueError):
        api.CacheAttention(cache)
    with pytest.raises(ValueError):
        api.WeightEvictor(cache, 8)


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_queries_are_refused_before_the_slots_change(rule):
    ev = api.DecodeEvictor(1, 1, 2, 1, 8, 4, device="cpu", rule=rule)
    k0 = torch.ones((1, 1, 1, 5, 128), dtype=torch.bfloat16)
    good = torch.zeros((1, 1, 2, 4, 128), dtype=torch.bfloat16)
    bad = [good.float(), good[..., :64], good[:, :, :1], good.to("meta"), good.transpose(3, 4).contiguous().transpose(3, 4)]
    for q in bad:
        with pytest.raises(ValueError):
            ev.start(k0, k0, q, [5])
        if rule == "jacap":
            with pytest.raises(ValueError):
                ev.merge_queries(q[:, :, :, 0])
    if rule == "weight":
        with pytest.raises(api.JacapError):
            ev.start(k0, k0, torch.zeros((1, 1, 2, 257, 128), dtype=torch.bfloat16), [5])
    assert ev.lengths == [0] and not ev.k.any()


@pytest.mark.parametrize("w,Hq", [(65, 2), (64, 64)])
def test_windows_past_the_limits_are_refused(w, Hq):
    cache = cpu_cache(w=w, Hq=Hq, Hkv=Hq // 2 if Hq < 64 else 4, n=80)
    with pytest.raises(api.JacapError):
        api.CacheAttention(cache) if w > 64 else api.WeightEvictor(cache, 8)
