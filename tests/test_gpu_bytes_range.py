"""GPU tests of attention over a cache held in 8 bits where its values, weights and queries differ by many orders of
magnitude, against a plain implementation in 64 bits.

The tolerances are bounds, from the roundings of the path (the bytes' values take part exactly):

* a query value is split into an e4m3 and an e5m2 part, at a power of two that brings the largest of its row to 224 ..
  448: exact from 2^-6 on, below that off by at most 2^-14 (half of e5m2's step where the remainder, 2^-10 at most, is
  largest), 2^-21.8 of the largest; the tensor cores' sums, the scaling and the reference as in test_gpu_bytes.py;
* a softmax weight is split alike: off by 2^-8 and, of the 16-bit value that it is split from, 2^-11 relative; from
  2^-6 down by at most 2^-14 and 2^-17. In those units the largest weight of a tile of 128 tokens, V's scale included, is at
  least 1, and at least 2^7 where one of the tile's quarters has none above 2^-6 of it (or no token at all); a tile that is
  far below others of its row keeps 2^-58 of the largest one;
* the output's own rounding, 2^-8, and half of bf16's lowest step.
"""

import math

import pytest
import torch

from test_gpu_bytes import BF16, BLOCK, D, DEV, F32, Slots, bad_values, gen, ints, randn, seen_by, trees, within

pytestmark = pytest.mark.gpu

LOG2E = 1.0 / math.log(2.0)


def plain(t, q, kd=None, vd=None, tree=None):
    """o, lse and their tolerances, in 64 bits; a cached value that passes float32 is infinite."""
    S, L, Hq, T, _ = q.shape
    Hkv, G = t.c.Hkv, t.c.Hq // t.c.Hkv
    K, V = (t.values(i).float().double() for i in (0, 1))
    seen = seen_by(S, T, tree, None)
    o, o_tol = (torch.zeros(S, L, Hq, T, D, dtype=torch.float64, device=DEV) for _ in range(2))
    lse, lse_tol = (torch.zeros(S, L, Hq, T, dtype=torch.float64, device=DEV) for _ in range(2))
    for s in range(S):
        n = t.n[s]
        mask = torch.ones(T, n + (T if kd is not None else 0), dtype=torch.bool, device=DEV)
        if kd is not None:
            mask[:, n:] = torch.tensor(seen[s], device=DEV)
        for l in range(L):
            for g in range(Hkv):
                k, v = K[s, l, g, :n], V[s, l, g, :n]
                if kd is not None:
                    k, v = torch.cat([k, kd[s, l, g].double()]), torch.cat([v, vd[s, l, g].double()])
                h = slice(g * G, (g + 1) * G)
                x = q[s, l, h].double()
                vv = torch.where(v.isfinite(), v, 0.0)
                vs = t.scales[1, l, g, s].repeat_interleave(BLOCK)[:n]
                logit = (t.c.scale * (x @ k.T)).masked_fill(~mask, -math.inf)
                mag = t.c.scale * (x.abs() @ k.abs().T)
                largest = x.abs().amax(-1, keepdim=True)
                small = t.c.scale * ((x.abs() < largest * 2.0 ** -13.8).double() @ k.abs().T) * largest * 2.0 ** -21.7
                off = (2.0 ** -19.8 + 2.0 ** -22) * mag + small + 2.0 ** -22 * logit.abs().nan_to_num(0.0, 0.0, 0.0)
                off[..., :n] += 2.0 ** -17 * mag[..., :n] * far(vs)  # (sums of float32, one by one)
                rel = 2 * torch.where(mask, off, 0.0).amax(-1) + 2.0 ** -20 + (n / 128 + 8) * 2.0 ** -24
                z, p = torch.logsumexp(logit, -1), torch.softmax(logit, -1)
                lse[s, l, h], lse_tol[s, l, h] = z, rel + 2.0 ** -23 * z.abs()
                o[s, l, h] = torch.stack([a @ vv for a in p]) + bad_values(mask, p, v)
                err = (p @ vv.abs()) * (rel + 2.0 ** -8 * (1 + 2.0 ** -3))[..., None]
                near = (vs > 0) & ~far(vs)
                kept = torch.where(near, vs, float(torch.where(near, vs, 2.0 ** -8).max()) if n else 0.0)
                y = (logit[..., :n] * LOG2E + torch.log2(kept)) if n else logit[..., :0]
                for b in range(0, n, 128):
                    e = min(b + 128, n)
                    top = y[..., b:e].amax(-1)
                    quarters = torch.stack([y[..., c:min(c + 32, e)].amax(-1) if c < e else torch.full_like(top, -math.inf)
                                            for c in range(b, b + 128, 32)])
                    wide = (top - quarters.amin(0) > 6.01) & near[b:e].all()
                    unit = torch.exp2(top - z * LOG2E) * torch.where(wide, 2.0 ** -7, 1.0)
                    unit = unit * 2.0 ** -14 * (1 + 2.0 ** -3) + torch.exp2(y.amax(-1) - z * LOG2E) * 2.0 ** -58
                    mags = torch.where(near[b:e, None], vv[b:e].abs() / vs[b:e, None], 0.0).sum(0)
                    err = err + unit[..., None] * mags
                o_tol[s, l, h] = err * (1 + 2.0 ** -8) + 2.0 ** -8 * o[s, l, h].abs().nan_to_num(0.0, 0.0, 0.0) + 2.0 ** -134
    return o, lse, o_tol, lse_tol


def far(vs):
    """Blocks whose V does not go through the tensor cores."""
    return (vs > 0) & ((vs < 2.0 ** -32) | (vs > 2.0 ** 16))


def check(t, q, *drafted):
    o, lse = t.c.attend(q, *drafted)
    wo, wl, to, tl = plain(t, q, *drafted)
    within(lse, wl, tl, "lse")
    within(o, wo, to, "o")
    t.c.check()


# ------------------------------------------------------------------- weights ----
def toward(g, S, L, Hq, Hkv, n, T=1):
    """Queries near one direction, and keys that are near 0 along it."""
    q = (torch.ones(S, L, Hq, T, D, device=DEV) + 0.05 * randn(g, S, L, Hq, T, D)).to(BF16)
    k = 0.3 * randn(g, S, L, Hkv, n, D)
    return q, k - k.mean(-1, keepdim=True)


@pytest.mark.parametrize("T", [1, 6, 40])
@pytest.mark.parametrize("n,share,worth", [(100, 0.9, 0.0), (100, 0.98, 0.0), (100, 0.99, 0.0), (100, 0.995, 0.0),
                                           (100, 0.998, 0.0), (512, 0.99, 0.02), (2048, 0.9, 0.02), (2048, 0.99, 0.02),
                                           (4000, 0.99, 0.0)])
def test_attend_one_token_with_most_of_the_weight_and_values_near_zero(n, share, worth, T):
    """What heads of language models do at a prompt's first token: the output is that of the others' small weights."""
    g, S, L, Hq, Hkv = gen(700 + n), 2, 1, 8, 2
    t = Slots(S, L, Hq, Hkv, n)
    q, k = toward(g, S, L, Hq, Hkv, n, T)
    v = randn(g, S, L, Hkv, n, D) + 0.5
    k[:, :, :, 0] = math.log(n * share / (1 - share)) / math.sqrt(D)  # its logit, the others' being near 0
    v[:, :, :, 0] *= worth
    t.store(k, v, [n, n - 3])
    check(t, q)
    kd, vd = (randn(g, S, L, Hkv, T, D, dtype=BF16) * 0.3 for _ in range(2))
    check(t, q, kd, vd, trees(g, S, T))


def test_attend_a_larger_token_in_every_tile():
    g, S, L, Hq, Hkv, n = gen(701), 1, 1, 8, 2, 4096
    t = Slots(S, L, Hq, Hkv, n)
    q, k = toward(g, S, L, Hq, Hkv, n)
    v = randn(g, S, L, Hkv, n, D) + 0.5
    for at, bits in ((slice(0, None, 128), 10.4), (slice(0, 1), 14.0)):  # 2^bits times the others'
        k[:, :, :, at] = bits / LOG2E / math.sqrt(D)
    v[:, :, :, ::128] = 0.0
    t.store(k, v)
    check(t, q)


# -------------------------------------------------------------------- scales ----
HEADS = [(1, 8, 2), (7, 8, 2), (30, 8, 2), (8, 4, 4)]  # queries, query and KV heads: 16, 32 and 64 rows at a time


def filled(g, S, Hq, Hkv, n, change, lengths=None, spread=0.7):
    """Slots whose V (float32) is what `change` makes of ordinary values."""
    t = Slots(S, 1, Hq, Hkv, n)
    k, v = spread * randn(g, S, 1, Hkv, n, D), randn(g, S, 1, Hkv, n, D) + 0.5
    change(v)
    t.store(k, v, lengths)
    return t


@pytest.mark.parametrize("T,Hq,Hkv", HEADS)
@pytest.mark.parametrize("size", [2.0 ** -118, 2.0 ** -100, 2.0 ** -60, 2.0 ** -31, 2.0 ** 22, 2.0 ** 40, 2.0 ** 102])
def test_attend_values_all_very_small_or_large(size, T, Hq, Hkv):
    """The logarithm of the sum of exponentials has nothing to do with V; scales from the least one on."""
    g = gen(720)
    t = filled(g, 2, Hq, Hkv, 640, lambda v: v.mul_(size), [640, 70])
    q = randn(g, 2, 1, Hq, T, D, dtype=BF16)
    check(t, q)
    kd, vd = (randn(g, 2, 1, Hkv, T, D, dtype=BF16) for _ in range(2))
    check(t, q, kd, (vd * size).to(BF16))


@pytest.mark.parametrize("T,Hq,Hkv", HEADS)
@pytest.mark.parametrize("n", [64, 640])
def test_attend_cached_values_that_are_not_finite(n, T, Hq, Hkv):
    """An infinite value is read as one, in its channel alone; the others, and the sum of exponentials, are as without it."""
    g = gen(721)

    def change(v):
        v[0, 0, 0, 5, 7], v[0, 0, -1, n - 1, 0] = math.inf, -math.inf
        v[1, 0, 0, 63, 100], v[1, 0, -1, 1, 3], v[1, 0, -1, n - 2, 3] = math.nan, math.inf, -math.inf

    t = filled(g, 3, Hq, Hkv, n, change)
    q = randn(g, 3, 1, Hq, T, D, dtype=BF16)
    check(t, q)
    kd, vd = (randn(g, 3, 1, Hkv, T, D, dtype=BF16) for _ in range(2))
    check(t, q, kd, vd, trees(g, 3, T))
    o, _ = t.c.attend(q)
    assert (o[0, 0, 0, :, 7] == math.inf).all() and (o[0, 0, -1, :, 0] == -math.inf).all()
    assert o[1, 0, 0, :, 100].isnan().all() and o[1, 0, -1, :, 3].isnan().all()
    assert (~o.isfinite()).sum() == 4 * T * (Hq // Hkv)


@pytest.mark.parametrize("T,Hq,Hkv", HEADS)
def test_attend_scales_that_differ_by_many_orders(T, Hq, Hkv):
    """Blocks whose few large values stand in channels of their own, blocks of small ones and of zeros: each channel has
    what its own values give."""
    g, n = gen(722), 64 * 14

    def change(v):
        for block, size in ((1, 2.0 ** 60), (4, 2.0 ** 100), (7, 2.0 ** 118), (12, 2.0 ** 30)):
            v[:, :, :, 64 * block + 3, block] = size
        for block, size in ((2, 2.0 ** -118), (5, 2.0 ** -70), (9, 0.0), (10, 2.0 ** -45)):
            v[:, :, :, 64 * block:64 * block + 64] *= size

    t = filled(g, 2, Hq, Hkv, n, change, [n, 64 * 8 - 5])
    q = randn(g, 2, 1, Hq, T, D, dtype=BF16)
    check(t, q)
    kd, vd = (randn(g, 2, 1, Hkv, T, D, dtype=BF16) for _ in range(2))
    check(t, q, kd, vd, trees(g, 2, T))


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 1), (40, 8, 1)])
def test_attend_far_scales_in_several_splits(T, Hq, Hkv):
    g, n = gen(723), 20032

    def change(v):
        v[:, :, :, 77, 5], v[:, :, :, 9000:9064, 6], v[:, :, :, n - 1, 7] = 2.0 ** 80, 2.0 ** 70, -math.inf
        v[:, :, :, 12800:13056] *= 2.0 ** -90

    t = filled(g, 1, Hq, Hkv, n, change, spread=0.4)
    q = randn(g, 1, 1, Hq, T, D, dtype=BF16)
    check(t, q)
    again = [x.clone() for x in t.c.attend(q)]
    for _ in range(3):
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(t.c.attend(q), again))



@pytest.mark.parametrize("T,Hq,Hkv", HEADS)
@pytest.mark.parametrize("n", [170, 426, 1300])
@pytest.mark.parametrize("size", [2.0 ** 60, 2.0 ** 85, 2.0 ** 105])
def test_attend_large_values_before_tokens_of_hardly_any_weight(size, n, T, Hq, Hkv):
    """A tile whose weights are far below those of the tiles before it, in the same split: the large value stays finite."""
    g = gen(725)
    t = Slots(1, 1, Hq, Hkv, n)
    q, k = toward(g, 1, 1, Hq, Hkv, n, T)
    v = randn(g, 1, 1, Hkv, n, D)
    k[:, :, :, n - 91] = 60.0 / math.sqrt(D)
    v[:, :, :, n - 91, 9] = size
    t.store(k, v)
    check(t, q)
    check(t, q, *(randn(g, 1, 1, Hkv, T, D, dtype=BF16) * 0.3 for _ in range(2)))


@pytest.mark.parametrize("T,Hq,Hkv,n", [(1, 4, 1, 20032), (6, 8, 2, 9000), (40, 8, 1, 20032), (1, 8, 2, 300)])
def test_attend_values_that_are_not_finite_at_tokens_of_hardly_any_weight(T, Hq, Hkv, n):
    """As plain sums have them: whichever splits there are, and however small their weight beside another's."""
    g = gen(724)
    t = Slots(1, 1, Hq, Hkv, n)
    q, k = toward(g, 1, 1, Hq, Hkv, n, T)
    v = randn(g, 1, 1, Hkv, n, D)
    k[:, :, :, 0] = 300.0 / math.sqrt(D)  # e^300 of the others' weight
    v[:, :, :, n // 2, 3], v[:, :, :, n - 1, 5], v[:, :, :, 7, 8], v[:, :, :, n - 2, 100] = (math.inf, -math.inf, math.inf,
                                                                                            math.nan)
    t.store(k, v)
    kd, vd = (randn(g, 1, 1, Hkv, T, D, dtype=BF16) * 0.3 for _ in range(2))
    for drafted in ((None, None), (kd, vd)):
        if drafted[0] is not None:
            vd[:, :, :, 0, 60], vd[:, :, :, 0, 61] = math.inf, math.nan  # of the first drafted token, which all see
        o, lse = t.c.attend(q, *drafted)
        assert lse.isfinite().all()
        for c, want in ((3, math.inf), (5, -math.inf), (8, math.inf)):
            assert (o[..., c] == want).all()
        assert o[..., 100].isnan().all()
        if drafted[0] is not None:
            assert (o[..., 60] == math.inf).all() and o[..., 61].isnan().all()
        assert (~o.isfinite()).sum() == o[..., 0].numel() * (4 if drafted[0] is None else 6)


# ------------------------------------------------------------------- queries ----
@pytest.mark.parametrize("T", [1, 6, 9, 40])
def test_attend_rows_of_very_different_sizes(T):
    """Heads and drafted tokens whose queries are small beside others of the same block of rows: a row's output has its own
    rounding, whatever stands beside it."""
    g, S, Hq, Hkv, n = gen(740 + T), 2, 8, 2, 320
    t = filled(g, S, Hq, Hkv, n, lambda v: v, [320, 77], spread=1.0)
    q = randn(g, S, 1, Hq, T, D, dtype=BF16)
    alone = q.clone()
    bits = torch.tensor([14, 0, 7, -1, 0, -30, 12, 20], dtype=F32, device=DEV)
    q *= torch.exp2(bits).to(BF16)[:, None, None]
    if T > 1:
        q[:, :, :, 1::3] *= 2.0 ** -9
        q[:, :, 1, 2::3], q[:, :, 4, 0] = 0.0, 2.0 ** -120
    check(t, q)
    kd, vd = (randn(g, S, 1, Hkv, T, D, dtype=BF16) for _ in range(2))
    check(t, q, kd, vd, trees(g, S, T))
    # rows that are the same give the same, to the last bit
    rows = [1, 4] if T == 1 else [1]
    at = [i for i in range(T) if i % 3 == 0 and (T == 1 or i > 0)]
    one, two = (x.clone() for x in t.c.attend(alone)), t.c.attend(q)
    for a, b in zip(one, two):
        assert torch.equal(a[:, :, rows][:, :, :, at], b[:, :, rows][:, :, :, at])
