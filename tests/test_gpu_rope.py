"""qk_norm_rope and append_kv_paged against the plain 64-bit form."""

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import check_turn, rope_table, turn

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-6


def rand(seed, *shape, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


@pytest.mark.parametrize("B,T,Hq,Hkv", [(1, 1, 1, 1), (1, 1, 32, 8), (2, 3, 5, 1), (3, 65, 8, 2), (1, 700, 40, 3), (5, 1, 0, 4), (1, 9, 7, 0)])
@pytest.mark.parametrize("R,inter", [(0, False), (16, False), (16, True), (96, False), (128, False), (128, True)])
def test_rows(B, T, Hq, Hkv, R, inter):
    print(f"[rope] {B} {T} {Hq} {Hkv} R={R} {inter}", flush=True)
    rows = T + 30
    table = rope_table(rows, R) if R else None
    pos = torch.randint(0, rows, (B, T), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    for form in ("heads", "fused"):
        for norm in (None, "one", "each"):
            if form == "heads":
                q, k = rand(1, B, Hq, T, 128, scale=3.0), rand(2, B, Hkv, T, 128)
            else:
                x = rand(3, B, T, Hq + 2 * Hkv, 128)
                q, k = x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:Hq + Hkv].transpose(1, 2)
            w = [None if norm is None or not H else 1 + rand(9, *((128,) if norm == "one" else (H, 128))) for H in (Hq, Hkv)]
            dq, dk = (x.to(DEV) if x.shape[1] else None for x in (q, k))
            got = bpc.qk_norm_rope(dq, dk, pos.to(DEV) if R else None, table.to(DEV) if R else None,
                                   wq=None if w[0] is None else w[0].to(DEV), wk=None if w[1] is None else w[1].to(DEV),
                                   eps=EPS, interleaved=inter)
            for g, x, wx in zip(got, (q, k), w):
                if not x.shape[1]:
                    assert g is None
                    continue
                wx = wx[:, None] if wx is not None and wx.dim() == 2 else wx
                at = pos[:, None].expand(B, x.shape[1], T)
                check_turn(g, turn(x, wx, table, at, EPS, inter))


@pytest.mark.parametrize("inter", [False, True])
def test_in_place_and_into_a_cache(inter):
    B, T, Hq, Hkv, Ncap, at = 2, 37, 8, 2, 100, 11
    table, pos = rope_table(64, 64), torch.arange(T, dtype=torch.int32).expand(B, T)
    q, k, w = rand(1, B, Hq, T, 128), rand(2, B, Hkv, T, 128), 1 + rand(3, 128)
    cache = rand(4, B, Hkv, Ncap, 128).to(DEV)
    before = cache.clone()
    dq = q.to(DEV)
    oq, ok = bpc.qk_norm_rope(dq, k.to(DEV), pos.to(DEV), table.to(DEV), wq=w.to(DEV), eps=EPS, interleaved=inter, q_out=dq,
                              k_out=cache[:, :, at:at + T])
    assert oq is dq
    check_turn(dq, turn(q, w, table, pos[:, None].expand(B, Hq, T), EPS, inter))
    check_turn(cache[:, :, at:at + T], turn(k, None, table, pos[:, None].expand(B, Hkv, T), EPS, inter))
    assert torch.equal(cache[:, :, :at], before[:, :, :at]) and torch.equal(cache[:, :, at + T:], before[:, :, at + T:])


def test_positions_outside_the_table_leave_their_rows():
    B, T, H = 2, 6, 5
    table = rope_table(10, 128)
    pos = torch.tensor([[0, -1, 9, 10, 3, 2 ** 31 - 1], [-2 ** 31, 1, 2, 3, 4, 5]], dtype=torch.int32)
    q = rand(1, B, H, T, 128)
    out = torch.full((B, H, T, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    bpc.qk_norm_rope(q.to(DEV), None, pos.to(DEV), table.to(DEV), q_out=out)
    good = (pos >= 0) & (pos < 10)
    want = turn(q, None, table, pos.clamp(0, 9)[:, None].expand(B, H, T), EPS, False)
    for b in range(B):
        for t in range(T):
            if good[b, t]:
                check_turn(out[b, :, t], (want[0][b, :, t], want[1][b, :, t]))
            else:
                assert bool((out[b, :, t] == 7).all())


def test_no_arithmetic_keeps_the_bits():
    q = rand(1, 1, 3, 5, 128).to(DEV)
    assert torch.equal(bpc.qk_norm_rope(q, None, None, None)[0], q)


def test_extreme_rows():
    q = torch.zeros(1, 1, 5, 128, dtype=torch.bfloat16)
    q[0, 0, 1] = 1e18  # squares near the top of fp32
    q[0, 0, 2, 3] = float("nan")
    q[0, 0, 3, 4] = float("inf")
    q[0, 0, 4] = 1e-30
    w = torch.ones(128, dtype=torch.bfloat16)
    out = bpc.qk_norm_rope(q.to(DEV), None, None, None, wq=w.to(DEV))[0].cpu()[0, 0]
    assert bool((out[0] == 0).all()) and bool((out[1] == 1).all()) and bool(out[2].isnan().all())
    assert bool(out[3, 4].isnan()) and bool((out[3, :4] == 0).all())
    check_turn(out[4], turn(q[0, 0, 4], w, None, None, 1e-6, False))


def paged(seed, B, Hkv, page, per, spare=2):
    """Pools of shuffled pages and a table of `per` pages a sequence."""
    n = B * per + spare
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))[:B * per].view(B, per).to(torch.int32)
    return rand(seed + 1, n, Hkv, page, 128), rand(seed + 2, n, Hkv, page, 128), order


def store(K, V, table, pos, count, k, v):
    """Row by row, in place, from finished keys k [B, Hkv, T, 128]; returns
    which rows were written [pages, page]."""
    hit = torch.zeros(K.shape[0], K.shape[2], dtype=torch.bool)
    B, _, T, _ = k.shape
    page = K.shape[2]
    for b in range(B):
        for t in range(min(T, count[b])):
            slot = pos[b] + t
            if slot < 0 or slot // page >= table.shape[1]:
                continue
            p = int(table[b, slot // page])
            if 0 <= p < K.shape[0]:
                K[p, :, slot % page], V[p, :, slot % page] = k[b, :, t], v[b, :, t]
                hit[p, slot % page] = True
    return hit


@pytest.mark.parametrize("B,Hkv,T,page", [(1, 1, 1, 16), (16, 8, 1, 16), (3, 2, 5, 32), (2, 8, 64, 64), (4, 3, 300, 256), (1, 8, 2500, 128)])
@pytest.mark.parametrize("R,inter,norm,depth", [(0, False, False, False), (128, False, True, False), (64, True, False, True), (32, False, True, True)])
def test_append_paged(B, Hkv, T, page, R, inter, norm, depth):
    print(f"[append paged] {B} {Hkv} {T} page={page} R={R} {inter} {norm} {depth}", flush=True)
    per = (T + 3 * page) // page + 1
    K, V, table = paged(7, B, Hkv, page, per)
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(0, 2 * page, (B,), generator=g, dtype=torch.int32)
    count = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
    count[0] = T
    x = rand(11, B, T, 2, Hkv, 128)
    k, v = x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2)  # strided, the two interleaved
    cs = rope_table(T + 3 * page, R) if R else None
    w = 1 + rand(12, Hkv, 128) if norm else None
    rope = torch.randint(0, T + 3 * page, (B, T), generator=g, dtype=torch.int32) if depth else None
    at = rope if depth else pos[:, None] + torch.arange(T)
    y, size = turn(k, None if w is None else w[:, None], cs, at[:, None].expand(B, Hkv, T).clamp(max=T + 3 * page - 1), EPS, inter)
    dK, dV = K.to(DEV), V.to(DEV)
    d = x.to(DEV)
    bpc.append_kv_paged(d[:, :, 0].transpose(1, 2), d[:, :, 1].transpose(1, 2), dK, dV, table.to(DEV), pos.to(DEV), count=count.to(DEV),
                        cos_sin=None if cs is None else cs.to(DEV), rope_pos=None if rope is None else rope.to(DEV),
                        wk=None if w is None else w.to(DEV), eps=EPS, interleaved=inter)
    wantK, wantV, sizes = K.double(), V.clone(), torch.zeros(K.shape, dtype=torch.float64)
    hit = store(wantK, wantV, table, pos.tolist(), count.tolist(), y, v)
    store(sizes, wantV, table, pos.tolist(), count.tolist(), size, v)
    assert torch.equal(dV.cpu(), wantV)
    rows = hit[:, None, :, None].expand(K.shape)
    assert torch.equal(dK.cpu()[~rows], K[~rows])
    check_turn(dK.cpu()[rows], (wantK[rows], sizes[rows]))
    if not R and not norm:
        assert torch.equal(dK.cpu().double(), wantK)


def test_append_paged_skips_what_has_no_place():
    B, Hkv, T, page = 4, 2, 40, 16
    K, V, table = paged(21, B, Hkv, page, 3)
    table[0, 1], table[1, 0] = -1, K.shape[0]  # unmapped, and past the pool
    pos, count = torch.tensor([0, 5, 30, -10], dtype=torch.int32), torch.tensor([40, 99, 40, 12], dtype=torch.int32)
    k, v = rand(22, B, Hkv, T, 128), rand(23, B, Hkv, T, 128)
    dK, dV = K.to(DEV), V.to(DEV)
    bpc.append_kv_paged(k.to(DEV), v.to(DEV), dK, dV, table.to(DEV), pos.to(DEV), count=count.to(DEV))
    store(K, V, table, pos.tolist(), count.tolist(), k, v)
    assert torch.equal(dK.cpu(), K) and torch.equal(dV.cpu(), V)


def test_append_into_a_contiguous_cache():
    """A contiguous cache is a pool of one page a sequence."""
    B, Hkv, T, Ncap = 3, 2, 7, 64
    K, V = rand(31, B, Hkv, Ncap, 128), rand(32, B, Hkv, Ncap, 128)
    pos = torch.tensor([0, 57, 60], dtype=torch.int32)
    k, v = rand(33, B, Hkv, T, 128), rand(34, B, Hkv, T, 128)
    dK, dV = K.to(DEV), V.to(DEV)
    bpc.append_kv_paged(k.to(DEV), v.to(DEV), dK, dV, torch.arange(B, dtype=torch.int32, device=DEV)[:, None], pos.to(DEV))
    store(K, V, torch.arange(B)[:, None], pos.tolist(), [T] * B, k, v)
    assert torch.equal(dK.cpu(), K) and torch.equal(dV.cpu(), V)


@pytest.mark.parametrize("inter", [False, True])
def test_more_rows_than_a_cache_holds(inter):
    """Rows past 256 MB (written past the caches), against the same rows in parts."""
    T, Hq, Hkv = 9001, 128, 5
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k = (torch.randn(1, H, T, 128, generator=g, device=DEV).to(torch.bfloat16) for H in (Hq, Hkv))
    table, w = rope_table(T, 128).to(DEV), (1 + rand(2, Hq, 128)).to(DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)[None]
    oq, ok = bpc.qk_norm_rope(q, k, pos, table, wq=w, eps=EPS, interleaved=inter)
    for a in range(0, T, 2500):
        pq, pk = bpc.qk_norm_rope(q[:, :, a:a + 2500], k[:, :, a:a + 2500], pos[:, a:a + 2500], table, wq=w, eps=EPS, interleaved=inter)
        assert torch.equal(oq[:, :, a:a + 2500], pq) and torch.equal(ok[:, :, a:a + 2500], pk)
