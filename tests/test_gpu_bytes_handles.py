"""GPU tests of handles of a cache held in 8 bits: their workspaces, parts of a cache, and slots of any length."""

import pytest
import torch

import paper_2609_08131_gb300.api as api
from paper_2609_08131_gb300 import JACAP_ATTEND_ZERO_BYTES
from test_gpu_bytes import BF16, D, DEV, gen, ints, randn, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 5, 40])
def test_a_workspace_of_few_queries_does_what_one_of_many_does(T):
    """Only the status word and the counters start at zero; the rest may hold anything."""
    g, S, Hq, Hkv, n = gen(800 + T), 3, 8, 2, 9088
    many = api.Cache8.empty(S, 2, Hq, Hkv, n, device=DEV)
    many.store(*(randn(g, S, 2, Hkv, 9000, D, dtype=BF16) for _ in range(2)), ints([9000, 70, 4000]))
    few = many.part(tokens=T)
    assert few.ws.numel() <= many.ws.numel()
    few.ws[JACAP_ATTEND_ZERO_BYTES + 4 * S:].fill_(0xFF)
    q, kd, vd = randn(g, S, 2, Hq, T, D, dtype=BF16), *(randn(g, S, 2, Hkv, T, D, dtype=BF16) for _ in range(2))
    masks = trees(g, S, T)
    for _ in range(2):
        for a, b in zip(many.attend(q, kd, vd, masks), few.attend(q, kd, vd, masks)):
            assert torch.equal(a, b)
    few.append(kd, vd, taken=ints([T, 0, 1]))
    assert many.lengths.tolist() == [9000 + T, 70, 4001]
    many.check(), few.check()


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_a_store_of_no_rows_empties_the_slots(dtype):
    g = gen(810)
    c = api.Cache8.empty(2, 1, 4, 2, 128, device=DEV)
    c.store(*(randn(g, 2, 1, 2, 100, D, dtype=BF16) for _ in range(2)))
    before = [x.clone() for x in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scales, c.v_scales)]
    none = torch.empty(2, 1, 2, 0, D, dtype=dtype, device=DEV)
    c.store(none, none, ints([0, 0]))
    assert c.lengths.tolist() == [0, 0]
    assert all(torch.equal(a, b) for a, b in zip(before, (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scales, c.v_scales)))
    c.check()
    c.append(*(randn(g, 2, 1, 2, 3, D, dtype=dtype) for _ in range(2)))
    c.store(none, none)
    assert c.lengths.tolist() == [0, 0]
    o, lse = c.attend(randn(g, 2, 1, 4, 1, D, dtype=BF16))
    assert (o == 0).all() and (lse == -float("inf")).all()
    c.store(none, none, ints([0, 1]))  # a length that there is no row for
    with pytest.raises(api.JacapError):
        c.check()


def test_rows_at_the_very_end_of_slots_whose_offsets_pass_32_bits():
    """5.4 GB: the last block of the last slot has what a small cache's has, and nothing else is touched."""
    S, L, Hkv, n, g = 2, 2, 8, 655360, gen(820)
    c = api.Cache8.empty(S, L, 8, Hkv, n, device=DEV, tokens=1)
    small = api.Cache8.empty(1, 1, 8, Hkv, 64, device=DEV, tokens=1)
    k, v = (randn(g, 1, 1, Hkv, 3, D, dtype=BF16) for _ in range(2))
    x, y = (torch.zeros(S, L, Hkv, 3, D, dtype=BF16, device=DEV) for _ in range(2))
    x[1:, 1:], y[1:, 1:] = k, v
    small.append(k, v, lengths=ints([61]))
    c.append(x, y, lengths=ints([n - 3] * S))
    assert c.lengths.tolist() == [n] * S
    for big, little in ((c.k.view(torch.uint8), small.k.view(torch.uint8)), (c.v.view(torch.uint8), small.v.view(torch.uint8)),
                        (c.k_scales, small.k_scales), (c.v_scales, small.v_scales)):
        last = big[1, :, 1]
        at = slice(-64, None) if big.dim() == 5 else slice(-1, None)
        assert torch.equal(last[:, at], little[0, :, 0]) and (little != 0).any()
        last[:, at].zero_()
        assert not any(big[l, h].any() for l in range(L) for h in range(Hkv))
    c.check(), small.check()


def test_a_step_entered_layer_by_layer():
    g, S, L, Hkv, T = gen(830), 3, 3, 2, 4
    whole, by_layer = (api.Cache8.empty(S, L, 4, Hkv, 128, device=DEV) for _ in range(2))
    k0, v0 = (randn(g, S, L, Hkv, 62, D, dtype=BF16) for _ in range(2))
    path, taken = ints([[0, 2, 3, -1], [1, -1, -1, -1], [-1] * 4]), ints([3, 1, 0])
    k, v = (3 * randn(g, S, L, Hkv, T, D, dtype=BF16) for _ in range(2))
    for c in (whole, by_layer):
        c.store(k0, v0, ints([62, 0, 30]))
    whole.append(k, v, path, taken)
    before = by_layer.lengths.clone()
    for l in range(L):
        at = slice(l, l + 1)
        by_layer.part(layers=at).append(k[:, at], v[:, at], path, taken, lengths=before)
    assert by_layer.lengths.tolist() == whole.lengths.tolist() == [65, 1, 30]
    for name in ("k", "v"):
        assert torch.equal(getattr(whole, name).view(torch.uint8), getattr(by_layer, name).view(torch.uint8))
        assert torch.equal(getattr(whole, name + "_scales"), getattr(by_layer, name + "_scales"))
    by_layer.check()
