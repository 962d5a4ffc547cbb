"""The 64-bit forms of cache_plain for sizes of many rows and slots: one (sequence,
head) at a time, all of its tokens in one product.  The bounds are those of
attn_plain and cache_plain, term for term.
"""

import torch

from attn_plain import ATTN_OUT, ATTN_WEIGHTED
from cache_plain import U, scores


def attend_head(q, k, v, visible, distance, sm, cap=0.0, slope=None):
    """q [T, D], k, v [N, D], visible and distance [T, N]: (out, its bound, lse, its
    bound).  A value that is not finite counts in the rows that see it, alone."""
    z, off = scores(q, k, distance, sm, cap, slope)
    z = torch.where(visible, z, -float("inf"))
    most = z.amax(1)
    p = torch.where(visible, torch.exp(z - most[:, None]), 0.0)
    total = p.sum(1)
    lse = most + torch.log(total)
    w = torch.where(visible, p / total[:, None], 0.0)
    v = v.double()
    fine = v.isfinite()
    kept = torch.where(fine, v, 0.0)
    out, weighted = w @ kept, w @ kept.abs()
    for n in (~fine).any(1).nonzero().flatten().tolist():
        out += torch.where(visible[:, n, None] & ~fine[n], v[n], 0.0)
    bound = ATTN_OUT * out.abs() + ATTN_WEIGHTED * weighted
    far = torch.where(visible, off, 0.0).amax(1) + 2.0 ** -15 + visible.sum(1) * U + 2.0 ** -22 * (lse.abs() + most.abs())
    return out, bound, lse, far


def check_head(got, sums, want, live):
    """One head's rows of the outputs [T, D] and log-sums [T] (or None), where live."""
    out, bound, lse, far = (x[live] for x in want)
    got = got[live].cpu().double()
    assert torch.equal(got.isnan(), out.isnan()) and torch.equal(got.isinf(), out.isinf())
    fine = out.isfinite()
    assert torch.equal(got[~fine & ~out.isnan()], out[~fine & ~out.isnan()])
    off = (got - out).abs()[fine]
    assert bool((off <= bound[fine]).all()), float((off / (bound[fine] + 1e-300)).max())
    if sums is not None:
        sums = sums[live].cpu().double()
        assert torch.equal(sums.isnan(), lse.isnan())
        some, none = lse.isfinite(), lse == -float("inf")
        assert torch.equal(sums[none], lse[none])
        off = (sums - lse).abs()[some]
        assert bool((off <= far[some]).all()), float((off / far[some]).max())


def weigh_head(q, k, lse, old, visible, distance, sm, decay, cap=0.0, slopes=None):
    """q [G, T, D] and lse [G, T] of a KV head's query heads, k [N, D], old [N]: the
    new weights of all N slots and their bound; `visible` [T, N] leaves out tokens
    that are not there and pages that are none."""
    total = torch.zeros(len(k), dtype=torch.float64)
    off = torch.zeros(len(k), dtype=torch.float64)
    for g in range(len(q)):
        z, far = scores(q[g], k, distance, sm, cap, None if slopes is None else slopes[g])
        L = lse[g].double()[:, None]
        use = visible & (L != -float("inf"))
        p = torch.where(use, torch.exp(z - L), 0.0)
        total += p.sum(0)
        off += torch.where(use, p * (far + 2.0 ** -22 * (z.abs() + L.abs()) + 2.0 ** -15), 0.0).sum(0)
    base = old.double() * decay if decay else torch.zeros_like(total)
    new = base + total
    return new, off + q.shape[0] * q.shape[1] * (U * total + 2.0 ** -126) + 2.0 ** -23 * (new.abs() + base.abs())
