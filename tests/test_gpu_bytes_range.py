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
    return (vs > 0) & ((vs < 2.0 ** -40) | (vs > 2.0 ** 16))


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
