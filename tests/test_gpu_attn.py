"""prefill_attention and tree_attention against the plain 64-bit form."""

import math

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import attend, check_attend, ranges_visible, tree_view

pytestmark = pytest.mark.gpu
DEV = "cuda"
SM = 1 / math.sqrt(128)


def rand(seed, *shape, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def slopes_of(H):
    return torch.tensor([2.0 ** (-(h % 8) - 1) for h in range(H)])


def prefill(q, K, V, pos0, begin, end, cap, slopes, **kw):
    """The call and its plain form; begin, end [B, T] CPU or None."""
    B, Hq, T, _ = q.shape
    N = K.shape[2]
    b0 = torch.zeros(B, T, dtype=torch.int32) if begin is None else begin
    e0 = (pos0 + 1 + torch.arange(T)).expand(B, T) if end is None else end
    dist = (pos0 + torch.arange(T)[:, None] - torch.arange(N)).abs().expand(B, T, N)
    want = attend(q, K, V, ranges_visible(b0, e0, N), dist, SM, cap, slopes)
    dev = lambda x: None if x is None else x.to(DEV)
    got = bpc.prefill_attention(dev(q), dev(K), dev(V), pos0=pos0, softcap=cap, slopes=dev(slopes), key_begin=dev(begin),
                                key_end=dev(end), **kw)
    return got, want


SIZES = [(1, 1, 1, 1, 1), (1, 4, 1, 1, 33), (2, 8, 2, 65, 65), (1, 3, 3, 31, 200), (1, 6, 2, 127, 129), (1, 16, 1, 64, 64), (1, 20, 1, 5, 40),
         (1, 2, 2, 17, 1500), (1, 8, 1, 3, 5000), (2, 4, 2, 300, 300), (1, 4, 4, 130, 777)]


@pytest.mark.parametrize("B,Hq,Hkv,T,N", SIZES)
@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, False), (0.0, True), (50.0, True)])
def test_prefill_causal(B, Hq, Hkv, T, N, cap, bias):
    print(f"[prefill] {B} {Hq} {Hkv} {T} {N} cap={cap} bias={bias}", flush=True)
    got, want = prefill(rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128), N - T, None, None, cap,
                        slopes_of(Hq) if bias else None)
    check_attend(got, want)


def masks(kind, B, T, N, pos0):
    at = pos0 + torch.arange(T).expand(B, T)
    g = torch.Generator().manual_seed(T + N)
    if kind == "documents":
        first = (torch.rand(B, N, generator=g) < 0.05).int() * torch.arange(N, dtype=torch.int32)
        begin = torch.cummax(first, 1).values[:, N - T:]
        return begin.int(), (at + 1).int()
    if kind == "prefix":
        return None, torch.maximum(at + 1, torch.randint(0, N + 1, (B, 1), generator=g)).int()
    if kind == "window":
        return (at - 9).int(), None
    # any ranges, empty ones and ones that leave [0, N) among them
    begin, end = torch.randint(-50, N + 50, (2, B, T), generator=g, dtype=torch.int32)
    begin[:, ::5], end[:, ::5] = -2 ** 31, 2 ** 31 - 1
    end[:, 1::7] = begin[:, 1::7]
    return begin, end


@pytest.mark.parametrize("kind", ["documents", "prefix", "window", "any"])
@pytest.mark.parametrize("B,Hq,Hkv,T,N", [(1, 1, 1, 1, 1), (2, 4, 2, 100, 100), (1, 8, 1, 40, 333), (1, 8, 2, 260, 300), (2, 2, 1, 4, 3001)])
def test_prefill_masks(kind, B, Hq, Hkv, T, N):
    print(f"[prefill masks] {kind} {B} {Hq} {Hkv} {T} {N}", flush=True)
    pos0 = N - T
    begin, end = masks(kind, B, T, N, pos0)
    for cap, bias in ((0.0, False), (30.0, True)):
        got, want = prefill(rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128), pos0, begin, end, cap,
                            slopes_of(Hq) if bias else None)
        check_attend(got, want)


def test_prefill_rows_without_keys_are_zero():
    q, K, V = rand(1, 2, 4, 70, 128), rand(2, 2, 2, 70, 128), rand(3, 2, 2, 70, 128)
    end = torch.zeros(2, 70, dtype=torch.int32)
    end[1, 3] = 5
    got, want = prefill(q, K, V, 0, None, end, 0.0, None)
    check_attend(got, want)
    assert bool((got[0] == 0).all()) and bool((got[1, :, 4:] == 0).all()) and bool((got[1, :, 3] != 0).any())


@pytest.mark.parametrize("T,N", [(40, 200), (2, 3000), (150, 150)])
@pytest.mark.parametrize("what", ["nan", "inf", "lowest"])
def test_prefill_hidden_keys_do_not_reach(T, N, what):
    """Each token's hidden keys hold anything; those it sees, finite or not, count."""
    q, K, V = rand(1, 1, 4, T, 128), rand(2, 1, 2, N, 128), rand(3, 1, 2, N, 128)
    bad = {"nan": float("nan"), "inf": float("inf"), "lowest": torch.finfo(torch.bfloat16).min}[what]
    end = (torch.arange(T, dtype=torch.int32) * 3 % (N - 20) + 10)[None]
    begin = (end - 8).contiguous()
    for n in (N - 1, N - 5, N // 2):  # hidden from most tokens
        V[0, :, n, ::3] = bad
    K[0, :, N - 1] = bad
    K[0, :, N - 2, 5] = -bad
    got, want = prefill(q, K, V, N - T, begin, end, 0.0, None)
    check_attend(got, want)
    assert bool(got.isfinite().any())
    # behind the last key
    big = torch.full((1, 2, N + 70, 128), bad, dtype=torch.bfloat16)
    bigK, bigV = big.clone(), big.clone()
    bigK[:, :, :N], bigV[:, :, :N] = rand(2, 1, 2, N, 128), rand(3, 1, 2, N, 128)
    a = bpc.prefill_attention(q.to(DEV), bigK.to(DEV), bigV.to(DEV), N=N)
    b = bpc.prefill_attention(q.to(DEV), rand(2, 1, 2, N, 128).to(DEV), rand(3, 1, 2, N, 128).to(DEV))
    assert torch.equal(a, b) and bool(a.isfinite().all())


def test_prefill_positions_past_the_keys():
    q, K, V = rand(1, 1, 2, 50, 128), rand(2, 1, 1, 20, 128), rand(3, 1, 1, 20, 128)
    got, want = prefill(q, K, V, 1000, None, None, 0.0, slopes_of(2) / 16)
    check_attend(got, want)


def test_prefill_strides():
    """Queries and results as [B, T, H, D], a cache with room, keys interleaved with values, a shared mask row."""
    B, Hq, Hkv, T, N, Ncap = 2, 8, 2, 90, 130, 160
    q = rand(1, B, T, Hq, 128).transpose(1, 2)
    kv = rand(2, B, Ncap, Hkv, 2, 128)
    K, V = kv[..., 0, :].transpose(1, 2), kv[..., 1, :].transpose(1, 2)
    end = (N - T + 1 + torch.arange(T, dtype=torch.int32))[None].expand(B, T)
    dkv = kv.to(DEV)
    out = torch.zeros(B, T, Hq, 128, dtype=torch.bfloat16, device=DEV)
    got = bpc.prefill_attention(q.to(DEV).transpose(1, 2).contiguous().transpose(1, 2), dkv[..., 0, :].transpose(1, 2),
                                dkv[..., 1, :].transpose(1, 2), N=N, key_end=end.to(DEV)[:1].expand(B, T), out=out.transpose(1, 2))
    assert got.data_ptr() == out.data_ptr()
    dist = torch.zeros(B, T, N, dtype=torch.int64)
    check_attend(out.transpose(1, 2), attend(q, K[:, :, :N], V[:, :, :N], ranges_visible(torch.zeros_like(end), end, N), dist, SM))


def tree_masks(seed, B, T):
    """Random trees, as lists of masks."""
    g = torch.Generator().manual_seed(seed)
    pick = torch.rand(B, T, generator=g).tolist()
    out = []
    for b in range(B):
        m = []
        for t in range(T):
            p = int(pick[b][t] * (t + 1)) - 1  # -1: a root
            m.append((m[p] if p >= 0 else 0) | 1 << t)
        out.append(m)
    return out


def as_int64(tree):
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in r] for r in tree], dtype=torch.int64)


def to_pages(x, page, seed, extra=1):
    """A cache [B, Hkv, N, D] cut into shuffled pages: (pool, table [B, pages])."""
    B, H, N, D = x.shape
    per = (N + page - 1) // page
    order = torch.randperm(B * per + extra, generator=torch.Generator().manual_seed(seed))
    pool = torch.full((B * per + extra, H, page, D), float("nan"), dtype=x.dtype)
    for b in range(B):
        for p in range(per):
            rows = x[b, :, p * page:(p + 1) * page]
            pool[order[b * per + p], :, :rows.shape[1]] = rows
    return pool, order[:B * per].view(B, per).to(torch.int32)


TREES = [(1, 1, 1, 1, [0], 1), (2, 8, 2, 1, [100, 0], 130), (3, 8, 2, 5, [0, 63, 250], 300), (1, 16, 1, 7, [1000], 1200), (2, 4, 4, 64, [129, 0], 200),
         (1, 32, 2, 24, [777], 801), (1, 6, 2, 33, [90], 200), (1, 2, 2, 3, [6000], 8000)]


@pytest.mark.parametrize("page", [0, 16, 64, 256])
@pytest.mark.parametrize("B,Hq,Hkv,T,lens,N", TREES)
def test_tree(B, Hq, Hkv, T, lens, N, page):
    print(f"[tree] {B} {Hq} {Hkv} {T} {lens} {N} page={page}", flush=True)
    q, K, V = rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128)
    for b in range(B):  # slots behind the drafts hold anything
        K[b, :, lens[b] + T:] = float("nan")
        V[b, :, lens[b] + T:] = float("inf")
    if page:
        (Kd, table), (Vd, _) = to_pages(K, page, 5), to_pages(V, page, 5)
        kw = dict(block_table=table.to(DEV), N=N)
    else:
        Kd, Vd, kw = K, V, {}
    for tree, cap, bias in ((None, 0.0, False), (tree_masks(T, B, T), 0.0, False), (tree_masks(T + 1, B, T), 30.0, True), (None, 0.0, True),
                            (tree_masks(T + 2, B, T), 50.0, False)):
        visible, dist = tree_view(lens, tree, T, N)
        want = attend(q, K, V, visible, dist, SM, cap, slopes_of(Hq) if bias else None)
        got = bpc.tree_attention(q.to(DEV), Kd.to(DEV), Vd.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                                 None if tree is None else as_int64(tree).to(DEV), softcap=cap, slopes=slopes_of(Hq).to(DEV) if bias else None, **kw)
        check_attend(got, want)


def test_tree_rows_without_keys_and_bits_past_the_drafts():
    B, T, N = 2, 3, 40
    q, K, V = rand(1, B, 4, T, 128), rand(2, B, 2, N, 128), rand(3, B, 2, N, 128)
    tree = [[0, 0b010, 0b1101 | 1 << 63], [0, 0, 0b111]]
    visible, dist = tree_view([0, 5], tree, T, N)
    got = bpc.tree_attention(q.to(DEV), K.to(DEV), V.to(DEV), torch.tensor([0, 5], dtype=torch.int32, device=DEV), as_int64(tree).to(DEV))
    check_attend(got, attend(q, K, V, visible, dist, SM))
    assert bool((got[0, :, 0] == 0).all())


@pytest.mark.parametrize("N", [64, 5000])
def test_tree_sequences_without_a_length_are_skipped(N):
    T = 4
    q, K, V = rand(1, 4, 4, T, 128), rand(2, 4, 2, N, 128), rand(3, 4, 2, N, 128)
    lens = [-1, N - T, N - T + 1, 2 ** 31 - 1]
    out = torch.full((4, 4, T, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    bpc.tree_attention(q.to(DEV), K.to(DEV), V.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out=out)
    assert all(bool((out[b] == 7).all()) for b in (0, 2, 3))
    visible, dist = tree_view([N - T], None, T, N)
    check_attend(out[1:2], attend(q[1:2], K[1:2], V[1:2], visible, dist, SM))


@pytest.mark.parametrize("T,N,page", [(1, 100, 16), (20, 300, 16), (5, 4000, 32), (64, 300, 64)])
def test_tree_bad_pages_hide_their_slots(T, N, page):
    q, K, V = rand(1, 2, 8, T, 128), rand(2, 2, 2, N, 128), rand(3, 2, 2, N, 128)
    lens = [N - T, N // 2]
    (Kd, table), (Vd, _) = to_pages(K, page, 6), to_pages(V, page, 6)
    visible, dist = tree_view(lens, None, T, N)
    for b, p, bad in ((0, 1, -1), (0, (N - 1) // page, Kd.shape[0]), (1, 0, 2 ** 31 - 1), (1, 2, -2 ** 31)):
        table[b, p] = bad
        visible[b, :, p * page:(p + 1) * page] = False
    got = bpc.tree_attention(q.to(DEV), Kd.to(DEV), Vd.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), block_table=table.to(DEV), N=N)
    check_attend(got, attend(q, K, V, visible, dist, SM))


def test_tree_hidden_drafts_do_not_reach():
    """A draft that its row does not see may hold anything, one that it sees counts."""
    T, N = 6, 80
    q, K, V = rand(1, 1, 4, T, 128), rand(2, 1, 2, N, 128), rand(3, 1, 2, N, 128)
    V[0, :, 50 + 2, 7] = float("nan")
    V[0, :, 50 + 4, 9] = float("inf")
    K[0, :, 50 + 4] = float("-inf")
    V[0, :, 50 + 5, 3] = float("-inf")
    tree = [[1, 2, 4, 8, 0, 0b100001]]
    visible, dist = tree_view([50], tree, T, N)
    got = bpc.tree_attention(q.to(DEV), K.to(DEV), V.to(DEV), torch.tensor([50], dtype=torch.int32, device=DEV), as_int64(tree).to(DEV))
    check_attend(got, attend(q, K, V, visible, dist, SM))


@pytest.mark.parametrize("Hq,Hkv,T", [(1, 1, 150), (4, 1, 70), (2, 2, 64), (8, 1, 4)])
def test_prefill_odd_values_reach_all_who_see_them(Hq, Hkv, T):
    """Values that are not finite in a tile that some rows see whole and others in part."""
    N = T + 200
    q, K, V = rand(1, 1, Hq, T, 128), rand(2, 1, Hkv, N, 128), rand(3, 1, Hkv, N, 128)
    V[0, :, 201, 5], V[0, :, 203, 6], V[0, :, N - 2, 7], V[0, :, 150, 9] = float("nan"), float("inf"), float("-inf"), float("nan")
    begin = torch.where(torch.arange(T) < 3, 160, 0)[None].int()
    got, want = prefill(q, K, V, N - T, begin, None, 0.0, None)
    check_attend(got, want)


@pytest.mark.parametrize("T,Hq", [(40, 4), (20, 2), (3, 8)])
def test_tree_odd_values_reach_all_who_see_them(T, Hq):
    N = 150
    q, K, V = rand(1, 1, Hq, T, 128), rand(2, 1, 1, N, 128), rand(3, 1, 1, N, 128)
    V[0, 0, 99, 5], V[0, 0, 101, 6], V[0, 0, 2, 7] = float("nan"), float("inf"), float("-inf")
    visible, dist = tree_view([100], None, T, N)
    got = bpc.tree_attention(q.to(DEV), K.to(DEV), V.to(DEV), torch.tensor([100], dtype=torch.int32, device=DEV))
    check_attend(got, attend(q, K, V, visible, dist, SM))


@pytest.mark.parametrize("cap", [2.0 ** -20, 0.01, 1.0, 1024.0])
@pytest.mark.parametrize("sm", [2.0 ** -40, 0.01, 1.0, 2.0 ** 10])
def test_prefill_caps_and_scales(cap, sm):
    """The ends of what is taken; scales at which scores saturate, all equal or one-hot."""
    q, K, V = rand(1, 1, 2, 9, 128), rand(2, 1, 1, 77, 128), rand(3, 1, 1, 77, 128)
    # one coordinate alone, a power of two per key: scores are exact, whatever their size
    q[..., 1:], K[..., 1:] = 0, 0
    q[..., 0], K[0, 0, :, 0] = 1, torch.tensor([2.0 ** (i % 5 - 2) * (-1) ** i for i in range(77)])
    got = bpc.prefill_attention(dev(q), dev(K), dev(V), sm, softcap=cap)
    visible = torch.ones(9, 77, dtype=torch.bool).tril(68)[None]
    check_attend(got, attend(q, K, V, visible, torch.zeros(1, 9, 77), sm, cap))


def dev(x):
    return x.to(DEV)
