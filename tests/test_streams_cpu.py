"""The decoding loop on a stream that is not the current one: every access of its buffers is ordered (stream_order.py
keeps the clocks; no GPU)."""

import pytest
import torch

from paper_2609_08131_gb300 import api
from stream_order import watch

S, L, HQ, HKV, D = 2, 2, 4, 2, 128


def rows(*shape):
    return torch.zeros((*shape, D), dtype=torch.bfloat16)


def cache():
    k = rows(L, HKV, S * 30)
    return api.Cache(rows(S, L, HQ, 3), k, k.clone(), torch.arange(0, 61, 30, dtype=torch.int32), [30, 30], HQ)


def slots(rule):
    return api.DecodeEvictor(S, L, HQ, HKV, 20, 4, device="cpu", rule=rule)


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_start_on_another_stream(rule, monkeypatch):
    """The prompt's rows, tags and zeroed weights are there when the window's weights are taken; what the current stream
    does with the slots afterwards comes after."""
    with watch(monkeypatch) as order:
        ev = slots(rule)
        k0, q = rows(S, L, HKV, 23), rows(S, L, HQ, 4)
        ev.start(k0, k0.clone(), q, [23, 20], stream=order.side)
        assert order.calls("jacap_weigh" if rule == "weight" else "jacap_stats_update")[0][1] == "side"
        assert order.races() == []
        ev.k.sum(), ev.pos.sum()
        if rule == "weight":
            ev.weights.sum()
        assert order.races() == []


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_first_calls_on_another_stream(rule, monkeypatch):
    """What the first attention and the first accepted tokens make for themselves is made on their stream."""
    with watch(monkeypatch) as order:
        ev = slots(rule)
        k0, q0, k, q = rows(S, L, HKV, 20), rows(S, L, HQ, 4), rows(S, L, HKV, 3), rows(S, L, HQ, 3)
        ev.start(k0, k0.clone(), q0, [20, 17], stream=order.side)
        for layer in range(L):
            ev.attend(layer, q[:, layer], k[:, layer], k[:, layer], stream=order.side)
        ev.accept(k, k, q, [[0, 1], [0]], stream=order.side)
        assert [len(order.calls(c)) for c in ("jacap_attend", "jacap_append_path")] == [L, 1]
        assert {a[1] for c in ("jacap_attend", "jacap_append_path", "jacap_weigh") for a in order.calls(c)} == {"side"}
        assert order.races() == []


def test_a_first_attention_that_is_captured_leaves_the_eager_ones_a_zeroed_workspace(monkeypatch):
    with watch(monkeypatch) as order:
        ev = slots("weight")
        k0, q0, k, q = rows(S, L, HKV, 20), rows(S, L, HQ, 4), rows(S, L, HKV, 3), rows(S, L, HQ, 3)
        ev.start(k0, k0.clone(), q0, [20, 17])
        order.capturing = True
        for layer in range(L):
            ev.attend(layer, q[:, layer], k[:, layer], k[:, layer])
        order.capturing = False
        for layer in range(L):
            ev.attend(layer, q[:, layer], k[:, layer], k[:, layer])
        ws = order.buffer(ev._attention[3].ws.data_ptr())
        calls = [(a[0], a[6]) for a in order.accesses if ws in a[5]]
        # every captured call zeroes for itself (a graph may be replayed before any other runs), the first eager one
        # for all
        captured, eager = [("zero_", True), ("jacap_attend", True)], ("jacap_attend", False)
        assert calls == captured * L + [("zero_", False)] + [eager] * L


@pytest.mark.parametrize("call", ["attend", "score", "select"])
def test_a_handle_s_first_call_on_another_stream(call, monkeypatch):
    """What the constructor zeroed is zero when the first call's kernels run."""
    with watch(monkeypatch) as order:
        c, kd = cache(), rows(S, L, HKV, 3)
        order.side.wait_stream(order.main)  # the caller's tensors are there
        ev = api.CacheAttention(c) if call == "attend" else api.WeightEvictor(c, 8)
        if call == "attend":
            ev.run(k_draft=kd, v_draft=kd, stream=order.side)
        else:
            (ev.score if call == "score" else ev.select_compact)(stream=order.side)
        assert order.races() == []


@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_slots_that_start_empty_on_another_stream(rule, monkeypatch):
    with watch(monkeypatch) as order:
        k, q = rows(S, L, HKV, 3), rows(S, L, HQ, 3)
        order.side.wait_stream(order.main)
        ev = slots(rule)
        ev.attend(0, q[:, 0], k[:, 0], k[:, 0], stream=order.side)
        ev.accept(k, k, q, [[0, 1], [0]], stream=order.side)
        assert order.races() == []


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rule", ["jacap", "weight"])
def test_steps_on_another_stream(rule, dtype, monkeypatch):
    """Tokens entered one by one (also those that indexed copies enter) and attended to; what the current stream does
    with the slots afterwards comes after."""
    with watch(monkeypatch) as order:
        ev = slots(rule)
        k0, q0, q1 = rows(S, L, HKV, 20), rows(S, L, HQ, 4), rows(S, L, HQ, 1)
        k, q = rows(S, L, HKV).to(dtype if rule == "jacap" else torch.bfloat16), rows(S, L, HQ)
        ev.start(k0, k0.clone(), q0, [20, 17], stream=order.side)
        for _ in range(3):
            ev.append(k, k, q, stream=order.side)
            for layer in range(L):
                ev.attend(layer, q1[:, layer], stream=order.side)
        assert order.races() == []


@pytest.mark.parametrize("rule", ["jacap", "weight"])
@pytest.mark.parametrize("side", [False, True])
def test_slots_on_another_device_than_the_current_one(rule, side, monkeypatch):
    """Every call of the loop, evictions among them, is made with the slots' device current and goes to one of its
    streams; on another stream nothing is left unordered."""
    with watch(monkeypatch) as order:
        ev = slots(rule)
        k0, q0, k, q = rows(S, L, HKV, 22), rows(S, L, HQ, 4), rows(S, L, HKV, 3), rows(S, L, HQ, 3)
        one = [x.contiguous() for x in (k[:, :, :, 0], k[:, :, :, 1], q[:, :, :, 0])]
        order.device = 5
        stream = order.side if side else None
        ev.start(k0, k0.clone(), q0, [22, 20], stream=stream)
        rope = api.Rope(device="cpu")
        order.side.wait_stream(order.main)
        for _ in range(2):
            ev.rotate(rope, q[:, 0], k[:, 0], stream=stream)
            for layer in range(L):
                ev.attend(layer, q[:, layer], k[:, layer], k[:, layer], stream=stream)
            ev.accept(k, k, q, [[0, 1], [0]], stream=stream)
            ev.step(*one, stream=stream)
        if rule == "jacap":
            ev.merge_queries(q[:, :, :, 2], stream=stream)
        assert ev.events >= 2 and order.races() == []


@pytest.mark.parametrize("enter", ["accept", "step"])
def test_captured_attentions_leave_no_normalisers_before_a_replay(enter, monkeypatch):
    """Tokens entered after a capture alone: their normalisers are computed."""
    with watch(monkeypatch) as order:
        ev, T = slots("weight"), 3 if enter == "accept" else 1
        k0, q0, k, q = rows(S, L, HKV, 17), rows(S, L, HQ, 4), rows(S, L, HKV, T), rows(S, L, HQ, T)
        ev.start(k0, k0.clone(), q0, [17, 17])

        def enters():
            if enter == "accept":
                ev.accept(k, k, q, [[0, 1], [0]])
            else:
                ev.step(k[:, :, :, 0], k[:, :, :, 0], q[:, :, :, 0])
            return order.calls("jacap_weigh")[-1][7][1].lse_given

        def attends():
            for layer in range(L):
                ev.attend(layer, q[:, layer], k[:, layer], k[:, layer])

        attends()
        assert enters() == 1
        assert enters() == 0  # (those were the step's before)
        order.capturing = True
        attends()
        order.capturing = False
        assert enters() == 0
        attends()
        order.capturing = True  # captured again after an eager step: its normalisers may be overwritten by a replay
        attends()
        order.capturing = False
        assert enters() == 0


def test_the_caller_says_that_a_replay_left_the_normalisers(monkeypatch):
    with watch(monkeypatch) as order:
        ev, T = slots("weight"), 3
        k0, q0, k, q = rows(S, L, HKV, 8), rows(S, L, HQ, 4), rows(S, L, HKV, T), rows(S, L, HQ, T)
        ev.start(k0, k0.clone(), q0, [8, 8])
        one = k[:, :, :, 0], k[:, :, :, 0], q[:, :, :, 0]

        def given():
            return order.calls("jacap_weigh")[-1][7][1].lse_given

        def attends(layers, **kw):
            for layer in layers:
                ev.attend(layer, q[:, layer], k[:, layer], k[:, layer], **kw)

        for refused in (lambda: ev.accept(k, k, q, [[0], [0]], attended=True), lambda: ev.step(*one, attended=True)):
            with pytest.raises(ValueError):
                refused()
        order.capturing = True
        attends(range(L - 1))
        order.capturing = False
        with pytest.raises(ValueError):  # a layer is missing
            ev.accept(k, k, q, [[0], [0]], attended=True)
        assert ev.lengths == [8, 8] and ev.next_id == [8, 8]
        order.capturing = True
        attends(range(L))
        order.capturing = False
        for attended, want in ((True, 1), (None, 0), (False, 0), (True, 1)):
            ev.accept(k, k, q, [[0], [0, 1]], attended=attended)
            assert given() == want
        attends(range(L))
        ev.accept(k, k, q, [[0], []], attended=False)
        assert given() == 0
        attends([1], draft_lens=torch.ones(S, dtype=torch.int32))
        with pytest.raises(ValueError):  # not every token's
            ev.accept(k, k, q, [[0], []], attended=True)
        with pytest.raises(ValueError):  # of other tokens
            ev.step(*one, attended=True)
        assert order.races() == []
