"""key_weights' sums: terms and sums out of fp32's range, and what a sum over tens
of thousands of rows may lose."""

import math

import numpy as np
import pytest
import torch

import paper_2608_04405_amd as bpc

pytestmark = pytest.mark.gpu
DEV = "cuda"
# (B, Hq, Hkv, T, N): few rows (in one block, in two), many rows with 32 keys a wavefront and with 64
SIZES = [(1, 4, 2, 5, 200), (2, 4, 1, 13, 300), (1, 8, 2, 40, 300), (8, 16, 16, 70, 1100)]


def first_coordinate(values, *lead):
    x = torch.zeros(*lead, len(values), 128, dtype=torch.bfloat16)
    x[..., 0] = torch.as_tensor(values, dtype=torch.bfloat16)
    return x.to(DEV)


@pytest.mark.parametrize("decay", [0.0, 0.5])
@pytest.mark.parametrize("cap", [0.0, 300.0])
@pytest.mark.parametrize("sizes", SIZES)
def test_a_weight_past_the_range_is_infinite(sizes, cap, decay):
    """Log-sums that are not of the same call: exp(score - lse) of a slot may leave fp32's range, by itself or in the sum.
    Such a weight is infinite, no other is touched, and the eviction keeps its slot."""
    B, Hq, Hkv, T, N = sizes
    print(f"[weights range] {sizes} cap={cap} decay={decay}", flush=True)
    scores = torch.zeros(N)
    scores[3], scores[N - T - 20] = 200.0, 88.5  # e^200; e^88.5 = 2.7e38, in range, but not three times
    q, K = first_coordinate([1.0] * T, B, Hq), first_coordinate(scores, B, Hkv)
    lse = torch.zeros(B, Hq, T, device=DEV)
    weights = torch.full((B, Hkv, N), 2.0, device=DEV)
    pos = torch.full((B,), N - T, dtype=torch.int32, device=DEV)
    rows = T * (Hq // Hkv)
    assert rows >= 3
    got = bpc.key_weights(q, K, lse, weights, pos, sm_scale=1.0, softcap=cap, decay=decay)
    x = got.cpu()
    z = cap * math.tanh(200 / cap) if cap else 200.0
    assert z > 89 and (cap * math.tanh(88.5 / cap) if cap else 88.5) > 85
    heavy = torch.zeros(N, dtype=torch.bool)
    heavy[3] = True
    at = cap * math.tanh(88.5 / cap) if cap else 88.5
    heavy[N - T - 20] = math.exp(at) * rows > 2.0 ** 128
    assert bool((x[..., heavy] == float("inf")).all()), x[..., heavy].unique()
    assert bool(x[..., ~heavy].isfinite().all())
    plain = ~heavy
    plain[N - T - 20] = False
    seen = (N - torch.arange(N)).clamp(max=T).double() * (Hq // Hkv)  # rows that see each slot, a term of one each
    want = seen + 2 * decay
    # exp2 of zero is one; with a cap the score's zero is off by |cap| 2^-21
    assert bool(((x.double() - want).abs()[..., plain] <= want[plain] * (2.0 ** -15 + cap * 2.0 ** -21)).all())
    keep = 2
    K_out, V_out = (torch.empty(B, Hkv, keep, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lens = torch.full((B,), N, dtype=torch.int32, device=DEV)
    kept = bpc.evict_kv(K, K, got, lens, keep, K_out, V_out).cpu()
    assert bool((kept == torch.tensor([3, N - T - 20], dtype=torch.int32)).all())


@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, False), (0.0, True)])
@pytest.mark.parametrize("sizes", [(1, 64, 1, 640, 700), (8, 128, 16, 2050, 2200)])
def test_nothing_of_a_long_sum_is_lost(sizes, cap, bias):
    """Queries of zero and one log-sum for all rows: every term is the same fp32 number t, and the sum of the M rows that see
    a slot is M t.  Sums of 16 equal terms, by halves, are exact; the rest of the way is a sum of two numbers (what is added
    up, and what its roundings lost, itself off by (M / 32 2^-24)^2 relative to the sum at most: a lane adds M / 32 times), that
    of two halves and the store: three roundings.  Added up one tile after the other in fp32 the same numbers lose more, which is checked here too."""
    B, Hq, Hkv, T, N = sizes
    G = Hq // Hkv
    print(f"[weights long sum] {sizes} cap={cap} bias={bias}", flush=True)
    K = torch.randn(1, Hkv, N, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV).expand(B, Hkv, N, 128)
    slopes = torch.zeros(Hq, device=DEV) if bias else None
    lse = torch.full((B, Hq, T), 9.3, device=DEV)
    q = torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16, device=DEV).expand(B, Hq, T, 128)
    pos = torch.full((B,), N - T, dtype=torch.int32, device=DEV)
    got = bpc.key_weights(q, K, lse, torch.empty(B, Hkv, N, device=DEV), pos, decay=0.0, softcap=cap, slopes=slopes).cpu()
    # one row of one head: the term itself
    one = bpc.key_weights(q[:1, :1, :1], K[:1, :1], lse[:1, :1, :1], torch.empty(1, 1, N, device=DEV), torch.full((1,), N - 1, dtype=torch.int32, device=DEV),
                          decay=0.0, softcap=cap, slopes=None if slopes is None else slopes[:1]).cpu()
    t = float(one[0, 0, 0])
    assert bool((one == t).all()) and abs(t / math.exp(-9.3) - 1) < 2.0 ** -14
    rows = T * G
    bound = 3 * 2.0 ** -24 + ((rows / 32 + 1) * 2.0 ** -24) ** 2
    everyone = slice(0, N - T + 1)  # slots that all rows see
    off = (got[..., everyone].double() / (rows * t) - 1).abs().max()
    assert float(off) <= bound, float(off) / 2.0 ** -24
    naive, add = np.float32(0), np.float32(16 * t)
    for _ in range(rows // 32):
        naive += add
    assert abs(float(naive) / (rows // 32 * 16 * t) - 1) > bound


def test_rows_that_see_a_part_lose_no_more_than_16_terms():
    """As above, at the slots that only some rows see: of the 16 terms that a lane adds up at a time some are zero, which
    costs up to six roundings more."""
    B, Hq, Hkv, T, N = 1, 48, 2, 700, 800
    K = torch.randn(B, Hkv, N, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    lse = torch.full((B, Hq, T), 9.3, device=DEV)
    q = torch.zeros(B, Hq, T, 128, dtype=torch.bfloat16, device=DEV)
    pos = torch.full((B,), N - T, dtype=torch.int32, device=DEV)
    for window in (0, 300):
        got = bpc.key_weights(q, K, lse, torch.empty(B, Hkv, N, device=DEV), pos, decay=0.0, window=window).cpu()
        one = bpc.key_weights(q[:, :1, :1], K[:, :1], lse[:, :1, :1], torch.empty(1, 1, N, device=DEV), pos, decay=0.0).cpu()
        t = float(one[0, 0, 0])
        n, p = torch.arange(N), N - T + torch.arange(T)[:, None]
        see = ((n <= p) & ((p - n < window) | (window == 0))).sum(0).double() * (Hq // Hkv)
        off = (got.double() - see * t).abs()
        assert bool((off <= (9 * 2.0 ** -24 + ((T * 24 / 32 + 1) * 2.0 ** -24) ** 2) * see * t).all()), float((off / (see * t + 1e-300)).max() / 2.0 ** -24)
