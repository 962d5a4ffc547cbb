"""Plain 64-bit forms of the dense attention, the norm with rotation and the
paged store, one head or token at a time, and the bounds of the tests.

Bounds.  A bf16 result is off by half a step from what was rounded: 2^-8
relative.  A probability that enters the product with V is rounded to bf16 too,
so that the quotient sum(p v) / sum(p) is off by at most 2^-8 sum(w |v|), w the
exact weights.  Scores are fp32 sums of 128 exact products: off by at most
(128 + 8) 2^-24 S, S = sm_scale sum |q_i k_i|; the inputs here keep S below 64,
so that a weight is off by a factor of at most 1 + 2^-10 from its numerator and
as much from its sum, together under 2^-9 of sum(w |v|), half the bound above.
Capped scores add |cap| 2^-21 and biased ones |bias| 2^-23, both below 2^-10 for
the caps (up to 50) and distances (up to 2^13) here.  Together at most
2^-8 |out| + 2^-8 (1 + 1/2 + 1/4) sum(w |v|).
"""

import torch

ATTN_OUT = 2.0 ** -8
ATTN_WEIGHTED = 1.75 * 2.0 ** -8


def attend(q, K, V, visible, distance, sm_scale, cap=0.0, slopes=None):
    """q [B, Hq, T, D], K, V [B, Hkv, N, D] (CPU), visible and distance
    [B, T, N].  Returns (out, sum of w |v|), fp64; hidden keys are left out of
    every sum, not multiplied by zero."""
    q, K, V = q.double(), K.double(), V.double()
    B, Hq, T, D = q.shape
    G = Hq // K.shape[1]
    out, weighted = torch.zeros(B, Hq, T, D, dtype=torch.float64), torch.zeros(B, Hq, T, D, dtype=torch.float64)
    for b in range(B):
        for h in range(Hq):
            z = q[b, h] @ K[b, h // G].t() * sm_scale
            if cap:
                z = cap * torch.tanh(z / cap)
            if slopes is not None:
                z = z - slopes[h].double() * distance[b].double()
            for t in range(T):
                see = visible[b, t]
                if not bool(see.any()):
                    continue
                w = torch.softmax(z[t, see], 0)
                v = V[b, h // G][see]
                out[b, h, t] = (w[:, None] * v).sum(0)
                weighted[b, h, t] = (w[:, None] * v.abs()).sum(0)
    return out, weighted


def check_attend(got, want):
    out, weighted = want
    got = got.cpu().double()
    assert got.shape == out.shape
    fine = out.isfinite()
    assert torch.equal(got[~fine].isnan(), out[~fine].isnan())
    assert torch.equal(got[~fine & ~out.isnan()], out[~fine & ~out.isnan()])
    off = (got - out).abs()[fine]
    bound = (ATTN_OUT * out.abs() + ATTN_WEIGHTED * weighted)[fine]
    worst = ((off - bound) / (bound + 1e-300)).max().item() if off.numel() else -1.0
    assert bool((off <= bound).all()), f"off by {1 + worst:.3g} times the bound"


def ranges_visible(begin, end, N):
    n = torch.arange(N)
    return (n >= begin[..., None]) & (n < end[..., None])


def tree_view(lens, tree, T, N):
    """(visible, distance) [B, T, N] of drafts over a cache; tree: lists of
    T masks per sequence (Python integers), or None for a chain."""
    B = len(lens)
    visible, distance = torch.zeros(B, T, N, dtype=torch.bool), torch.zeros(B, T, N, dtype=torch.int64)
    for b in range(B):
        L = lens[b]
        bits = [[(tree[b][t] >> j) & 1 if tree is not None else int(j <= t) for j in range(T)] for t in range(T)]
        depth = [sum(bits[t]) - bits[t][t] for t in range(T)]
        place = torch.arange(N)
        for j in range(T):
            place[L + j] = L + depth[j]
        for t in range(T):
            visible[b, t, :L] = True
            for j in range(T):
                visible[b, t, L + j] = bool(bits[t][j])
            distance[b, t] = (L + depth[t] - place).abs()
    return visible, distance


def turn(x, w, table, pos, eps, interleaved):
    """Norm and rotation of rows x [..., 128] at positions pos [...] (CPU).
    Returns (y, |a| + |b| of the pair that made each coordinate), fp64."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    y, size = x.clone(), x.abs()
    if table is None:
        return y, size
    R = table.shape[1]
    cs = table.double()[pos.long()]
    c, s = cs[..., :R // 2], cs[..., R // 2:]
    i = torch.arange(R // 2)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size = size.clone()
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


def check_turn(got, want):
    """A bf16 rounding, and fp32 arithmetic: a norm's factor is off by under 12
    roundings (a sum of 128 squares in a tree of seven levels and eight terms, a
    root, two products), a rotation adds three: 2^-20 of |a| + |b| covers both."""
    y, size = want
    off = (got.cpu().double() - y).abs()
    assert bool((off <= 2.0 ** -8 * y.abs() + 2.0 ** -20 * size).all()), float((off / (size + 1e-300)).max())


def rope_table(rows, R):
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 1000.0 ** (-torch.arange(R // 2, dtype=torch.float64) * 2 / R)
    return torch.cat([angle.cos(), angle.sin()], -1).float()
