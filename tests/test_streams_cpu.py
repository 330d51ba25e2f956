"""The decoding loop on a stream that is not the current one: every access of its buffers is ordered (stream_order.py
keeps the clocks; no GPU)."""

import pytest
import torch

from paper_2609_08131_gb300 import api
from stream_order import watch

S, L, HQ, HKV, D = 2, 2, 4, 2, 128


def rows(*shape):
    return torch.zeros((*shape, D), dtype=torch.bfloat16)


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
