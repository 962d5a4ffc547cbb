"""prefill_attention and tree_attention in each shape of their kernels: four and
eight row blocks a workgroup, the key axis whole and in pieces, keys streamed past
the caches; with the masks, hidden values and pages that can go wrong there.  Each
test says which cut its sizes are for and fails when a call of them is cut
otherwise.  Two query heads of every group are compared with the plain 64-bit form.
"""

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import attend, check_attend, ranges_visible, tree_view
from test_gpu_attn import as_int64, masks, rand, slopes_of, to_pages, tree_masks

pytestmark = pytest.mark.gpu
DEV = "cuda"
SM = 128 ** -0.5

# (sizes, row blocks of a workgroup, whether in pieces); the last workgroup of each is not full
PREFILLS = [((8, 20, 4, 100, 130), 4, False), ((3, 24, 2, 140, 700), 4, True), ((1, 32, 2, 67, 3000), 4, True), ((6, 40, 5, 130, 150), 8, False),
            ((1, 128, 1, 41, 5000), 8, True)]
TREES = [((16, 64, 8, 17, 300), 4, False), ((4, 64, 8, 33, 2000), 4, True), ((2, 128, 2, 9, 1500), 4, True)]
SCORES = [(0.0, False), (30.0, False), (0.0, True), (50.0, True)]


def dev(x):
    return None if x is None else x.to(DEV)


def cut_as(sizes, row_blocks, pieces, tree=False):
    got = bpc.attention_cut(*sizes, tree=tree)
    assert got[0] == row_blocks and (got[1] > 1) == pieces and not got[2], got


def inputs(B, Hq, Hkv, T, N):
    return rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128)


def check_some(got, q, K, V, visible, dist, cap, slopes):
    """Two heads of every group, others in each group."""
    B, Hq, T, _ = q.shape
    Hkv = K.shape[1]
    G = Hq // Hkv
    heads = [h * G + (g + 5 * h) % G for h in range(Hkv) for g in (T % G, T % G + G // 2)]
    check_attend(got[:, heads], attend(q[:, heads], K, V, visible, dist, SM, cap, None if slopes is None else slopes[heads]))


@pytest.mark.parametrize("kind", ["causal", "documents", "prefix", "window", "any"])
@pytest.mark.parametrize("sizes,row_blocks,pieces", PREFILLS)
def test_prefill_masks(sizes, row_blocks, pieces, kind):
    print(f"[prefill cut] {sizes} {kind}", flush=True)
    cut_as(sizes, row_blocks, pieces)
    B, Hq, Hkv, T, N = sizes
    q, K, V = inputs(*sizes)
    pos0 = N - T
    at = pos0 + torch.arange(T)
    begin, end = (None, None) if kind == "causal" else masks(kind, B, T, N, pos0)
    b0 = torch.zeros(B, T, dtype=torch.int32) if begin is None else begin
    e0 = (at + 1).int().expand(B, T) if end is None else end
    dist = (at[:, None] - torch.arange(N)).abs().expand(B, T, N)
    for cap, bias in SCORES if kind == "causal" else SCORES[::3]:
        slopes = slopes_of(Hq) if bias else None
        got = bpc.prefill_attention(dev(q), dev(K), dev(V), softcap=cap, slopes=dev(slopes), key_begin=dev(begin), key_end=dev(end))
        check_some(got, q, K, V, ranges_visible(b0, e0, N), dist, cap, slopes)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), torch.finfo(torch.bfloat16).min])
@pytest.mark.parametrize("sizes,row_blocks,pieces", PREFILLS)
def test_prefill_hidden_and_odd_values(sizes, row_blocks, pieces, what):
    """Values that are not finite in tiles that some rows see whole, others in part and others not at all."""
    print(f"[prefill cut, odd values] {sizes} {what}", flush=True)
    cut_as(sizes, row_blocks, pieces)
    B, Hq, Hkv, T, N = sizes
    q, K, V = inputs(*sizes)
    g = torch.Generator().manual_seed(T)
    end = (N - T - 3 + torch.arange(T, dtype=torch.int32))[None].expand(B, T).contiguous()
    begin = torch.where(torch.rand(B, T, generator=g) < 0.3, end - 40, torch.zeros_like(end)).int()
    begin[:, 2], end[:, 2] = 0, 0  # a row that sees nothing, and one that sees almost all
    begin[:, 3], end[:, 3] = 0, N - 4
    K[:, :, N - 1], K[:, :, N - 3, 5], V[:, :, N - 2:] = what, -what, what  # hidden from all
    odd = what if not abs(what) < float("inf") else 2.0 ** 100
    for b in range(B):
        for i, n in enumerate(torch.randint(0, N - 4, (6,), generator=g).tolist() + [N - T // 2]):
            V[b, i % Hkv, n, 3 * i:128:50] = odd if i % 2 else -odd
    if odd is what:
        K[B - 1, Hkv - 1, N - T // 3, 5] = what
    dist = torch.zeros(B, T, N)
    got = bpc.prefill_attention(dev(q), dev(K), dev(V), key_begin=dev(begin), key_end=dev(end))
    check_some(got, q, K, V, ranges_visible(begin, end, N), dist, 0.0, None)
    assert bool((got[:, :, 2] == 0).all())


def tree_call(q, K, V, lens, tree, page, spoil=None, **kw):
    """tree_attention over the contiguous cache, or over pages of it whose table `spoil` may change."""
    N = K.shape[2]
    tree = None if tree is None else dev(as_int64(tree))
    lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if not page:
        return bpc.tree_attention(dev(q), dev(K), dev(V), lens, tree, **kw)
    (Kd, table), (Vd, _) = to_pages(K, page, 5), to_pages(V, page, 5)
    if spoil:
        spoil(table, Kd.shape[0])
    return bpc.tree_attention(dev(q), dev(Kd), dev(Vd), lens, tree, block_table=dev(table), N=N, **kw)


def lengths(B, T, N):
    """From none to all that fit, ends of tiles of 64 among them."""
    return [(N - T, 0, 63, 64, 129, 64 - T % 64)[b] if b < 6 else (N - T) * b // B for b in range(B)]


@pytest.mark.parametrize("page", [0, 16, 64, 256])
@pytest.mark.parametrize("sizes,row_blocks,pieces", TREES)
def test_tree(sizes, row_blocks, pieces, page):
    """Trees and chains; slots behind the drafts hold anything."""
    print(f"[tree cut] {sizes} page={page}", flush=True)
    cut_as(sizes, row_blocks, pieces, tree=True)
    B, Hq, Hkv, T, N = sizes
    q, K, V = inputs(*sizes)
    lens = lengths(B, T, N)
    for b in range(B):
        K[b, :, lens[b] + T:], V[b, :, lens[b] + T:] = float("nan"), float("inf")
    for i, (cap, bias) in enumerate(SCORES):
        tree = None if i == page // 16 % 4 else tree_masks(T + i, B, T)
        visible, dist = tree_view(lens, tree, T, N)
        slopes = slopes_of(Hq) if bias else None
        got = tree_call(q, K, V, lens, tree, page, softcap=cap, slopes=dev(slopes))
        check_some(got, q, K, V, visible, dist, cap, slopes)


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("sizes,row_blocks,pieces", TREES)
def test_tree_hidden_and_odd_values(sizes, row_blocks, pieces, page):
    """Drafts that some rows do not see, and cached keys, with values that are not finite."""
    print(f"[tree cut, odd values] {sizes} page={page}", flush=True)
    cut_as(sizes, row_blocks, pieces, tree=True)
    B, Hq, Hkv, T, N = sizes
    q, K, V = inputs(*sizes)
    lens, tree = lengths(B, T, N), tree_masks(T, B, T)
    tree[0][1] = 0 if lens[0] == 0 else tree[0][1]
    for b in range(B):
        V[b, :, lens[b] + 2, 7], V[b, :, lens[b] + T - 1, 9], V[b, :, lens[b] + T // 2, 11] = float("nan"), float("inf"), float("-inf")
        if lens[b] > 9:
            V[b, 0, lens[b] - 5, 100], V[b, -1, 3, 101] = float("nan"), float("-inf")
    visible, dist = tree_view(lens, tree, T, N)
    check_some(tree_call(q, K, V, lens, tree, page), q, K, V, visible, dist, 0.0, None)


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("sizes,row_blocks,pieces", TREES)
def test_tree_bad_pages(sizes, row_blocks, pieces, page):
    """Pages outside the pool, beginning inside a tile, at its border, first and last."""
    print(f"[tree cut, bad pages] {sizes} page={page}", flush=True)
    cut_as(sizes, row_blocks, pieces, tree=True)
    B, Hq, Hkv, T, N = sizes
    q, K, V = inputs(*sizes)
    lens = lengths(B, T, N)
    visible, dist = tree_view(lens, None, T, N)
    last = (N - 1) // page
    bad = [(b, p, v) for b in range(B) for p, v in ((b % (last + 1), -1), ((3 * b + 1) % (last + 1), 2 ** 31 - 1), (last, None))]

    def spoil(table, pool):
        for b, p, v in bad:
            table[b, p] = pool if v is None else v

    for b, p, _ in bad:
        visible[b, :, p * page:(p + 1) * page] = False
    check_some(tree_call(q, K, V, lens, None, page, spoil), q, K, V, visible, dist, 0.0, None)


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("sizes,row_blocks,pieces", TREES)
def test_tree_skips_sequences(sizes, row_blocks, pieces, page):
    cut_as(sizes, row_blocks, pieces, tree=True)
    B, Hq, Hkv, T, N = sizes
    q, K, V = inputs(*sizes)
    lens = [(-1, N - T, N - T + 1, 2 ** 31 - 1)[b % 4] for b in range(B)]
    out = torch.full((B, Hq, T, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    tree_call(q, K, V, lens, None, page, out=out)
    on = [b for b in range(B) if b % 4 == 1]
    assert bool((out[[b for b in range(B) if b % 4 != 1]] == 7).all())
    visible, dist = tree_view([N - T] * len(on), None, T, N)
    check_some(out[on], q[on], K[on], V[on], visible, dist, 0.0, None)


@pytest.mark.parametrize("call", ["prefill", "tree", "paged"])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("full", [False, True])
def test_streamed(call, cap, bias, full):
    """A cache larger than the last-level cache, filled in part and whole."""
    print(f"[streamed] {call} cap={cap} bias={bias} full={full}", flush=True)
    T, Hq, N, page = (2, 1, 700000, 16) if full else (5, 3, 700000, 16)
    assert bpc.attention_cut(1, Hq, 1, T, N, tree=call != "prefill") == (1, 64, True)
    L = N - T if full else 3001  # cached tokens before the last T
    q, slopes = rand(1, 1, Hq, T, 128), slopes_of(Hq) / 1024 if bias else None
    seen = L + T
    if call == "paged":  # the sequence's pages are the pool's, over and over
        pool_k, pool_v = rand(2, 64, 1, page, 128), rand(3, 64, 1, page, 128)
        table = torch.randint(0, 64, (1, N // page), generator=torch.Generator().manual_seed(4), dtype=torch.int32)
        rows = table[0, :(seen + page - 1) // page].long()
        K, V = (x[rows, 0].reshape(1, 1, -1, 128)[:, :, :seen] for x in (pool_k, pool_v))
        got = bpc.tree_attention(dev(q), dev(pool_k), dev(pool_v), torch.tensor([L], dtype=torch.int32, device=DEV), block_table=dev(table), N=N,
                                 softcap=cap, slopes=dev(slopes))
    else:
        g = torch.Generator(device=DEV).manual_seed(5)
        dK, dV = (torch.randn(1, 1, N, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        dK[:, :, seen:], dV[:, :, seen:] = float("nan"), float("inf")
        K, V = dK[:, :, :seen].cpu(), dV[:, :, :seen].cpu()
        if call == "tree":
            got = bpc.tree_attention(dev(q), dK, dV, torch.tensor([L], dtype=torch.int32, device=DEV), softcap=cap, slopes=dev(slopes))
        else:
            got = bpc.prefill_attention(dev(q), dK, dV, pos0=L, softcap=cap, slopes=dev(slopes))
    at = L + torch.arange(T)[:, None]
    n = torch.arange(seen)
    check_attend(got, attend(q, K, V, (n <= at)[None], (at - n).abs()[None], SM, cap, slopes))
