"""Plain 64-bit forms of the attention of a chunk, the weights that slots gather
and the eviction, one head and token at a time, and the bounds of the tests.

Scores.  A score is an fp32 sum of 128 exact products, times a scale: off by at
most 136 roundings of 2^-24, relative to S = sm_scale sum |q_i k_i|.  A cap's tanh
comes from an exponential and a reciprocal, each a rounding of 2^-23, whose
difference from the cap is off by |cap| 2^-21; a bias from a product and a sum, off
by |bias| 2^-23.  SCORE below is the sum of the three, an absolute error.

Log-sum-exp.  A factor of e^SCORE in each exponential moves the logarithm by SCORE
at most.  Every exponential is off by 2^-22 relative (its argument is one rounding
of at most 2^8 in log2, where it matters at all, off by 2^-16; its own error is
smaller), which 2^-15 covers; summing n of them by under n 2^-24; the logarithm and
its sum with the reference point by 2^-22 of the result and of the largest score.

Weights.  A term exp(s - lse) is off by SCORE + 2^-22 (|s| + |lse|) + 2^-15 relative,
a sum of n of them by at most n 2^-24 more, and adding to what was there is one
rounding of the result and one of the decayed old weight: 2^-23.  A term below the
smallest normal number, 2^-126, may come out as zero (the exponential of the hardware
has no subnormal results): n times that is off too.
"""

import torch

U = 2.0 ** -24


def chunk_visible(pos, count, T, N, window, sinks):
    """(visible, distance, live): [B, T, N] twice and [B, T]."""
    B = len(pos)
    n = torch.arange(N)
    p = torch.tensor(pos)[:, None] + torch.arange(T)
    away = p[..., None] - n
    visible = away >= 0
    if window:
        visible &= (away < window) | (n < sinks)
    count = torch.tensor([T] * B if count is None else count).clamp(0, T)
    live = torch.arange(T) < count[:, None]
    ok = (torch.tensor(pos) >= 0) & (torch.tensor(pos) + count <= N)
    return visible, away.abs(), live & ok[:, None]


def scores(q, k, distance, sm, cap, slope):
    """Scores [T, N] of one head and how far off they may be."""
    q, k = q.double(), k.double()
    z, size = q @ k.t() * sm, q.abs() @ k.abs().t() * sm
    off = 136 * U * size
    if cap:
        z = cap * torch.tanh(z / cap)
        off = off + cap * 2.0 ** -21
    if slope is not None:
        z = z - float(slope) * distance.double()
        off = off + abs(float(slope)) * distance.double() * 2.0 ** -23
    return z, off


def log_sums(q, K, visible, distance, sm, cap=0.0, slopes=None):
    """(lse [B, Hq, T], bound), 64 bits; -inf where nothing is visible."""
    B, Hq, T, _ = q.shape
    G = Hq // K.shape[1]
    lse, bound = torch.full((B, Hq, T), -float("inf"), dtype=torch.float64), torch.zeros(B, Hq, T, dtype=torch.float64)
    for b in range(B):
        for h in range(Hq):
            z, off = scores(q[b, h], K[b, h // G], distance[b], sm, cap, None if slopes is None else slopes[h])
            for t in range(T):
                see = visible[b, t]
                if bool(see.any()):
                    x = z[t, see]
                    lse[b, h, t] = torch.logsumexp(x, 0)
                    bound[b, h, t] = off[t, see].max() + 2.0 ** -15 + len(x) * U + 2.0 ** -22 * (lse[b, h, t].abs() + x.max().abs())
    return lse, bound


def check_log_sums(got, want, live):
    lse, bound = want
    got = got.cpu().double()
    live = live[:, None].expand_as(lse)
    gone = lse == -float("inf")
    assert torch.equal(got[live & gone], lse[live & gone])
    fine = live & lse.isfinite()
    off = (got - lse).abs()
    assert bool((off <= bound)[fine].all()), float((off / bound)[fine].max())


def gather_weights(q, K, lse, old, end, visible, live, distance, sm, decay, cap=0.0, slopes=None):
    """(weights [B, Hkv, N], bound): the old ones, decayed below end[b], with what
    the live tokens add."""
    B, Hq, T, _ = q.shape
    Hkv, N = old.shape[1:]
    G = Hq // Hkv
    new, bound = old.double().clone(), torch.zeros(old.shape, dtype=torch.float64)
    for b in range(B):
        if not end[b]:
            continue
        e = end[b]
        for h in range(Hkv):
            total, off = torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.float64)
            for j in range(h * G, h * G + G):
                z, far = scores(q[b, j], K[b, h], distance[b], sm, cap, None if slopes is None else slopes[j])
                L = lse[b, j].double()[:, None]
                use = visible[b] & live[b][:, None] & (L != -float("inf"))
                p = torch.where(use, torch.exp(z - L), 0.0)
                total += p.sum(0)
                off += torch.where(use, p * (far + 2.0 ** -22 * (z.abs() + L.abs()) + 2.0 ** -15), 0.0).sum(0)
            base = old[b, h, :e].double() * decay if decay else 0.0
            new[b, h, :e] = base + total[:e]
            bound[b, h, :e] = off[:e] + G * T * (U * total[:e] + 2.0 ** -126) + 2.0 ** -23 * (new[b, h, :e].abs() + (base.abs() if decay else 0.0))
    return new, bound


def kept_slots(w, n, keep, sinks, recent):
    """The slots of one head that stay, ascending: the first `sinks`, the last
    `recent`, and of the others the heaviest, the lower slot first among equals."""
    if n <= keep:
        return list(range(n))
    w = w.tolist()
    middle = list(range(sinks, n - recent))
    rank = sorted(middle, key=lambda i: (-w[i] if w[i] == w[i] else float("inf"), w[i] != w[i], i))
    return sorted(list(range(sinks)) + rank[:keep - sinks - recent] + list(range(n - recent, n)))


def paged(x, page, seed, spare=1, fill=float("nan")):
    """(pool, table) of [B, H, N, 128]: pages in shuffled order, `spare` that none has."""
    B, H, N, D = x.shape
    per = (N + page - 1) // page
    order = torch.randperm(B * per + spare, generator=torch.Generator().manual_seed(seed))[:B * per].view(B, per)
    pool = torch.full((B * per + spare, H, page, D), fill, dtype=x.dtype)
    for b in range(B):
        for i in range(per):
            rows = x[b, :, i * page:(i + 1) * page]
            pool[order[b, i], :, :rows.shape[1]] = rows
    return pool, order.to(torch.int32)
