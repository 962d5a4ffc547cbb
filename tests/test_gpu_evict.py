"""evict_kv against the plain form: which slots stay, exactly, and their rows."""

import pytest
import torch

import paper_2608_04405_amd as bpc
from cache_plain import kept_slots, paged

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def gathered(seed, B, H, N):
    """A long tail, zeros, and equal weights."""
    x = torch.randn(B, H, N, generator=torch.Generator().manual_seed(seed)).mul_(2).exp_()
    return torch.where(x < 0.2, 0.0, torch.where(x < 0.7, 0.25, x))


def check(w, lens, keep, sinks, recent, page=0, out_page=0, W=0, N=None, same_pool=False, cap=None):
    B, H, N0 = w.shape
    N = N0 if N is None else N
    K, V = rand(1, B, H, N0, 128), rand(2, B, H, N0, 128)
    Kp, Vp, blocks, blocks_out = K, V, None, None
    if same_pool:  # one pool, the kept rows to pages that nothing has
        per, per_out = (N0 + page - 1) // page, (keep + page - 1) // page
        order = torch.randperm(B * (per + per_out) + 1, generator=torch.Generator().manual_seed(4)).to(torch.int32)
        blocks, blocks_out = order[:B * per].view(B, per), order[B * per:B * (per + per_out)].view(B, per_out)
        pools = torch.full((2, len(order), H, page, 128), 7.0, dtype=torch.bfloat16)
        for pool, x in zip(pools, (K, V)):
            for b in range(B):
                for i in range(per):
                    rows = x[b, :, i * page:(i + 1) * page]
                    pool[blocks[b, i], :, :rows.shape[1]] = rows
        Kp, Vp = (p.to(DEV) for p in pools)
        K_out, V_out = Kp, Vp
        before = Kp.cpu().clone(), Vp.cpu().clone()
    else:
        if page:
            (Kp, blocks), (Vp, _) = paged(K, page, 3), paged(V, page, 3)
        Kp, Vp = Kp.to(DEV), Vp.to(DEV)
        if out_page:
            per = (keep + out_page - 1) // out_page
            blocks_out = torch.randperm(B * per + 2, generator=torch.Generator().manual_seed(5))[:B * per].view(B, per).to(torch.int32)
            K_out, V_out = (torch.full((B * per + 2, H, out_page, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        else:
            K_out, V_out = (torch.full((B, H, keep + 5, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        before = K_out.cpu().clone(), V_out.cpu().clone()
    codes = codes_out = None
    if W:
        codes = torch.randint(-2 ** 31, 2 ** 31, (B, H, N0, W), generator=torch.Generator().manual_seed(6)).to(torch.int32)
        codes_out = torch.full((B, H, keep + 2, W), 7, dtype=torch.int32, device=DEV)
    cap = keep + 9 if cap is None else cap
    weights_out = torch.full((B, H, cap), 7.0, device=DEV)
    dev = lambda x: None if x is None else x.to(DEV)
    kept_out = torch.full((B, H, keep), 7, dtype=torch.int32, device=DEV)
    got = bpc.evict_kv(Kp, Vp, dev(w), ints(lens), keep, K_out, V_out, sinks=sinks, recent=recent, N=N, block_table=dev(blocks),
                       table_out=dev(blocks_out), codes=dev(codes), codes_out=codes_out, weights_out=weights_out, kept_out=kept_out)
    assert got is kept_out
    want_K, want_V = (x.clone() for x in before)
    for b in range(B):
        n = lens[b]
        for h in range(H):
            if not 0 <= n <= N:
                assert bool((got[b, h] == 7).all()) and bool((weights_out[b, h] == 7).all())
                continue
            slots = kept_slots(w[b, h], n, keep, sinks, recent)
            m = len(slots)
            assert got[b, h].tolist() == slots + [-1] * (keep - m), (b, h)
            at = torch.tensor(slots, dtype=torch.long)
            x, y = weights_out[b, h].cpu(), w[b, h, at]
            assert torch.equal(x[:m].nan_to_num(nan=3e38), y.nan_to_num(nan=3e38)) and bool((x[m:] == 0).all())
            if W:
                assert torch.equal(codes_out[b, h, :m].cpu(), codes[b, h, at]) and bool((codes_out[b, h, m:] == 7).all())
            for goal, x in ((want_K, K), (want_V, V)):
                if blocks_out is None:
                    goal[b, h, :m] = x[b, h, at]
                else:
                    op = goal.shape[2]
                    i = torch.arange(m)
                    goal[blocks_out[b].long()[i // op], h, i % op] = x[b, h, at]
    nan = lambda x: x.cpu().float().nan_to_num(nan=9e9)
    assert torch.equal(nan(K_out), nan(want_K)) and torch.equal(nan(V_out), nan(want_V))
    return got


@pytest.mark.parametrize("N,keep,sinks,recent", [(1, 1, 0, 0), (2, 1, 0, 0), (2, 1, 1, 0), (2, 1, 0, 1), (100, 100, 4, 4), (100, 99, 0, 0), (100, 50, 4, 46),
                                                 (100, 50, 4, 20), (1023, 300, 0, 0), (1025, 1024, 5, 1000), (4096, 2048, 4, 256), (5000, 17, 3, 3),
                                                 (9001, 4001, 16, 1024)])
@pytest.mark.parametrize("page,out_page,W", [(0, 0, 1), (16, 0, 0), (0, 32, 4), (64, 16, 2)])
def test_evict(N, keep, sinks, recent, page, out_page, W):
    print(f"[evict] {N} {keep} {sinks} {recent} page={page} {out_page} W={W}", flush=True)
    lens = [N, max(1, N - N // 3), N // 2]
    check(gathered(N, 3, 2, N), lens, keep, sinks, recent, page, out_page, W)


def test_other_pages_of_the_same_pool():
    check(gathered(1, 2, 3, 777), [777, 500], 300, 4, 100, page=16, same_pool=True)


@pytest.mark.parametrize("N", [64, 3000, 20000])
@pytest.mark.parametrize("what", ["equal", "zeros", "signed", "lowest bits", "nan", "infinite", "tiny"])
def test_weights_of_every_kind(what, N):
    g = torch.Generator().manual_seed(N)
    w = torch.randn(2, 2, N, generator=g)
    if what == "equal":
        w = torch.full_like(w, 0.75)
    elif what == "zeros":
        w = torch.where(w < 0.5, torch.where(w < 0, -0.0, 0.0), w)
    elif what == "lowest bits":
        w = (torch.randint(0, 40, w.shape, generator=g) + 0x3F800000).to(torch.int32).view(torch.float32)
    elif what == "nan":
        w = torch.where(w < 0.8, float("nan"), w)
        w[0, 0, ::3] = -float("inf")
    elif what == "infinite":
        w = torch.where(w > 1, float("inf"), torch.where(w < -1, -float("inf"), w))
    elif what == "tiny":
        w = w * 1e-42
    for keep, sinks, recent in ((N // 2, 0, 0), (N // 2, 3, N // 4), (N - 1, 2, 2), (max(1, N // 50), 0, 0)):
        check(w, [N, N - N // 4], keep, sinks, recent)


def test_lengths():
    """Empty sequences, sequences that stay whole, and ones that are skipped."""
    check(gathered(2, 6, 2, 300), [0, 1, 120, 121, 301, -1], 120, 10, 50, page=16, out_page=16, W=2)
    check(gathered(2, 3, 2, 300), [250, 251, 2 ** 31 - 1], 100, 0, 0, N=250, cap=100)


def test_bad_pages_are_left_out():
    """Rows of a page that is not in the pool, and rows that would go to one."""
    B, H, N, keep, page = 1, 2, 200, 100, 16
    K, V = rand(1, B, H, N, 128), rand(2, B, H, N, 128)
    (Kp, blocks), (Vp, _) = paged(K, page, 3), paged(V, page, 3)
    blocks[0, 1], blocks[0, 12] = -1, Kp.shape[0]
    out_blocks = torch.tensor([[0, 9, 2, -7, 4, 5, 6]], dtype=torch.int32)
    w = gathered(3, B, H, N)
    K_out, V_out = (torch.full((7, H, page, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    got = bpc.evict_kv(Kp.to(DEV), Vp.to(DEV), w.to(DEV), ints([N]), keep, K_out, V_out, sinks=20, recent=30, block_table=blocks.to(DEV), table_out=out_blocks.to(DEV))
    for h in range(H):
        slots = kept_slots(w[0, h], N, keep, 20, 30)
        assert got[0, h].tolist() == slots
        want = torch.full((2, 7, page, 128), 7.0, dtype=torch.bfloat16)
        for i, s in enumerate(slots):
            p = int(out_blocks[0, i // page])
            if 0 <= p < 7 and s // page not in (1, 12):
                want[0, p, i % page], want[1, p, i % page] = K[0, h, s], V[0, h, s]
        assert torch.equal(K_out[:, h].cpu(), want[0]) and torch.equal(V_out[:, h].cpu(), want[1])


def test_strides():
    """Keys and values of one pool, weights and results in larger buffers."""
    B, H, N, keep = 2, 2, 150, 70
    kv = rand(1, B, N, H, 2, 128).to(DEV)
    store = gathered(1, H, B, N + 9).to(DEV)
    w = store[:, :, 5:5 + N].transpose(0, 1)
    out = torch.full((B, keep, 2, H, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    weights_out = torch.full((B, 2, H, keep), 7.0, device=DEV)
    codes = torch.arange(B * H * (N + 4) * 2, dtype=torch.int32, device=DEV).view(B, H, N + 4, 2)
    codes_out = torch.zeros(B, H, keep + 2, 2, dtype=torch.int32, device=DEV)
    lens = ints([N, N - 40])
    kept = bpc.evict_kv(kv[..., 0, :].transpose(1, 2), kv[..., 1, :].transpose(1, 2), w, lens, keep, out[:, :, 0].transpose(1, 2),
                        out[:, :, 1].transpose(1, 2), sinks=2, recent=30, codes=codes, codes_out=codes_out, weights_out=weights_out[:, 1])
    for b in range(B):
        for h in range(H):
            slots = kept_slots(w[b, h].cpu(), int(lens[b]), keep, 2, 30)
            assert kept[b, h].tolist() == slots
            assert torch.equal(out[b, :, 0, h], kv[b, slots, h, 0]) and torch.equal(out[b, :, 1, h], kv[b, slots, h, 1])
            assert torch.equal(weights_out[b, 1, h], w[b, h, slots]) and torch.equal(codes_out[b, h, :keep], codes[b, h, slots])
    assert bool((weights_out[:, 0] == 7).all())


def test_long():
    """Many slots of few heads, and of many heads."""
    check(gathered(7, 1, 2, 131072), [131072], 65536, 4, 4096)
    check(gathered(8, 1, 1, 200001), [200001], 1000, 4, 96)
    check(gathered(9, 24, 16, 1500), [1500 - 7 * b for b in range(24)], 800, 16, 64, W=1)


@pytest.mark.parametrize("keep", [60, 17000])
def test_lengths_far_below_the_room(keep):
    """Sequences that use some of the segments, one, or none."""
    check(gathered(10, 6, 1, 50000), [50000, 16384, 16385, 100, 0, 33000], keep, 4, 16)
