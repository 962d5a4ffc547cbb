"""chunk_attention of many rows, four and eight row blocks a workgroup, where a call
leaves the straight path: more page entries than a wavefront holds, pages that are
none, slots that hold anything, values that are not finite, many first slots, scores
far from zero, wide strides.  Some heads of each call are compared with the 64-bit
form; calls are made twice."""

import math

import pytest
import torch

import paper_2608_04405_amd as bpc
from cache_plain import chunk_visible, paged
from cache_rows import attend_head, check_head

pytestmark = pytest.mark.gpu
DEV = "cuda"
SM = 1 / math.sqrt(128)


def rand(seed, *shape, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def slopes_of(H):
    return torch.tensor([2.0 ** (-(h % 8) - 1) for h in range(H)])


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def bits(x):
    return x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)


def call(q, K, V, pos, count, blocks=None, window=0, sinks=0, cap=0.0, slopes=None, sm=None, lse=True, N=None):
    B, Hq, T, _ = q.shape
    out = torch.full((B, Hq, T, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    sums = torch.full((B, Hq, T), 7.0, device=DEV) if lse else None
    bpc.chunk_attention(q, K, V, ints(pos), sm, N, count=ints(count), block_table=blocks, window=window, sinks=sinks, softcap=cap,
                        slopes=None if slopes is None else slopes.to(DEV), out=out, lse_out=sums)
    return out, sums


def check(q, K, V, pos, count, page=0, window=0, sinks=0, cap=0.0, slopes=None, sm=None, bad=(), repeat=True):
    """bad: (sequence, page of its table, value there)."""
    B, Hq, T, _ = q.shape
    Hkv, N = K.shape[1:3]
    G = Hq // Hkv
    Kp, Vp, blocks = K, V, None
    hidden = torch.zeros(B, N, dtype=torch.bool)
    if page:
        (Kp, blocks), (Vp, _) = paged(K, page, 11), paged(V, page, 11)
        for b, i, v in bad:
            blocks[b, i] = v
            hidden[b, i * page:(i + 1) * page] = True
        blocks = blocks.to(DEV)
    args = (q.to(DEV), Kp.to(DEV), Vp.to(DEV), pos, count, blocks, window, sinks, cap, slopes, sm)
    out, sums = call(*args, N=N)
    if repeat:
        again, same = call(*args, N=N)
        assert torch.equal(bits(again), bits(out)) and torch.equal(bits(same), bits(sums))
        bare, _ = call(*args, N=N, lse=False)
        assert torch.equal(bare.nan_to_num(9.0), out.nan_to_num(9.0))
    visible, away, live = chunk_visible(pos, count, T, N, window, sinks)
    rest = ~live[:, None].expand(B, Hq, T).to(DEV)
    assert bool((out[rest] == 7).all()) and bool((sums[rest] == 7).all())
    for b, j in sorted({(0, 0), (0, Hq // 2), (B // 2, Hq // 2 - 1), (B - 1, Hq - 1)}):
        want = attend_head(q[b, j], K[b, j // G], V[b, j // G], visible[b] & ~hidden[b], away[b], SM if sm is None else sm, cap, None if slopes is None else slopes[j])
        check_head(out[b, j], sums[b, j], want, live[b])
    return out, sums


def inputs(sizes):
    B, Hq, Hkv, T, N = sizes
    pos = [(N - T) * (2 * B - b) // (2 * B) for b in range(B)]
    return rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128), pos, [max(1, T - 13 * b) for b in range(B)]


def cut(sizes, window, sinks, row_blocks, pieces):
    got = bpc.chunk_cut(*sizes, window, sinks)
    assert got[0] == row_blocks and (got[1] > 1) == pieces and not got[2], got
    return got[1]


# sizes, window, first slots, row blocks, in pieces or not.  Pieces (the third number: tiles of 64 slots) are longer than a
# wavefront's 64 entries reach: 16 tiles with pages of 16, 32 with 32, 64 with more (16 in all pages with four row blocks).
CUTS = [((2, 64, 1, 130, 6000), 0, 0, 8, True, 32), ((1, 64, 1, 300, 9000), 0, 0, 8, True, 47), ((1, 256, 2, 520, 4500), 0, 0, 8, False, 71),
        ((3, 20, 1, 520, 8200), 0, 0, 8, True, 65), ((1, 64, 1, 130, 9000), 2500, 700, 8, True, 24), ((4, 64, 8, 260, 5000), 1000, 600, 8, False, 26),
        ((2, 32, 2, 260, 3000), 500, 600, 4, False, 18), ((6, 40, 2, 130, 3000), 1500, 1000, 4, True, 20)]


@pytest.mark.parametrize("page", [0, 16, 32, 64, 128])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (50.0, True)])
@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces,tiles", CUTS)
def test_more_tiles_than_entries_are_held(sizes, window, sinks, row_blocks, pieces, tiles, cap, bias, page):
    print(f"[chunk rows] {sizes} {window} {sinks} page={page} cap={cap} bias={bias}", flush=True)
    n = cut(sizes, window, sinks, row_blocks, pieces)
    if not window:
        assert ((sizes[4] + 63) // 64 + n - 1) // n == tiles
    q, K, V, pos, count = inputs(sizes)
    check(q, K, V, pos, count, page, window, sinks, cap, slopes_of(sizes[1]) if bias else None)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, True)])
@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces,tiles", CUTS)
def test_bad_pages(sizes, window, sinks, row_blocks, pieces, tiles, cap, bias, page):
    """Pages that are none, in the first, a middle and the last hold of entries, two at a hold's border, among the first slots
    and in the window."""
    print(f"[chunk rows, bad pages] {sizes} {window} {sinks} page={page} cap={cap} bias={bias}", flush=True)
    cut(sizes, window, sinks, row_blocks, pieces)
    q, K, V, pos, count = inputs(sizes)
    bad = []
    for b in range(len(pos)):
        last = (pos[b] + count[b] - 1) // page
        first = max(0, pos[b] - window) // page if window else 0
        for i, v in ((1, -1), (63, 2 ** 31 - 1), (64, -2 ** 31), ((first + last) // 2, 2 ** 31 - 1), (first + 2, -7), (last - 1 - b % 2, 10 ** 6)):
            if 0 <= i < last:
                bad.append((b, i, v))
    check(q, K, V, pos, count, page, window, sinks, cap, slopes_of(sizes[1]) if bias else None, bad=bad)


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("what", ["nan", "inf", "lowest"])
@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces,tiles", [CUTS[0], CUTS[3], CUTS[4], CUTS[5], CUTS[6], CUTS[7]])
def test_what_is_not_seen_does_not_reach(sizes, window, sinks, row_blocks, pieces, tiles, what, page):
    """Slots behind the last, and between the first ones and every window, hold anything; the last token's own key and value
    reach it alone."""
    print(f"[chunk rows, hidden] {sizes} {window} {sinks} page={page} {what}", flush=True)
    cut(sizes, window, sinks, row_blocks, pieces)
    q, K, V, pos, count = inputs(sizes)
    x = {"nan": float("nan"), "inf": float("inf"), "lowest": torch.finfo(torch.bfloat16).min}[what]
    for b, (p, c) in enumerate(zip(pos, count)):
        K[b, :, p + c:], V[b, :, p + c:] = x, x
        if window:
            K[b, :, sinks:p - window + 1], V[b, :, sinks:p - window + 1] = x, x
        if what == "nan":
            K[b, :, p + c - 1], V[b, :, p + c - 1, ::3] = x, x
    out, sums = check(q, K, V, pos, count, page, window, sinks)
    for b, c in enumerate(count):
        assert bool(out[b, :, :c - 1].isfinite().all()) and bool(sums[b, :, :c - 1].isfinite().all())
        if what == "nan":
            assert bool(out[b, :, c - 1].isnan().all()) and bool(sums[b, :, c - 1].isnan().all())


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, True)])
@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces,tiles", [CUTS[0], CUTS[3], CUTS[4], CUTS[5], CUTS[6], CUTS[7]])
def test_values_that_are_not_finite(sizes, window, sinks, row_blocks, pieces, tiles, cap, bias, page):
    """A value that is not finite reaches the rows that see it, and no others: among the new tokens (tiles that rows see in part),
    at the border of a window and of the first slots, next to one another and in the last place."""
    print(f"[chunk rows, odd values] {sizes} {window} {sinks} page={page} cap={cap} bias={bias}", flush=True)
    cut(sizes, window, sinks, row_blocks, pieces)
    q, K, V, pos, count = inputs(sizes)
    inf = float("inf")
    for b, (p, c) in enumerate(zip(pos, count)):
        h = b % K.shape[1]
        V[b, :, p + c // 2, 3], V[b, :, p + c // 2 + 1, 3], V[b, h, p + c - 1, 127] = inf, inf, -inf
        V[b, :, p + c // 3, 64:70], V[b, h, p, 5] = float("nan"), -inf
        V[b, :, p - 1, 9] = inf
        if window:
            V[b, :, p - window + c // 2, 17], V[b, :, p - window + c // 4, 17], V[b, :, sinks - 1, 30], V[b, :, 0, 31] = inf, -inf, inf, -inf
            V[b, :, p - window, 40], V[b, :, sinks, 41] = float("nan"), float("nan")  # (not seen, where the window is past the first slots)
    # biases under which no weight of a visible slot, at most 9000 away, rounds to zero in fp32
    check(q, K, V, pos, count, page, window, sinks, cap, slopes_of(sizes[1]) / 128 if bias else None)


def line(values, *lead):
    """Rows whose first coordinate alone is not zero."""
    x = torch.zeros(*lead, len(values), 128, dtype=torch.bfloat16)
    x[..., 0] = torch.tensor(values, dtype=torch.bfloat16)
    return x


@pytest.mark.parametrize("sm", [2.0 ** -40, 1.0, 2.0 ** 10, 2.0 ** 27, 2.0 ** 40])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces", [((1, 64, 1, 130, 5000), 0, 0, 8, True), ((6, 40, 5, 130, 400), 60, 10, 8, False),
                                                                  ((2, 32, 2, 260, 3000), 500, 600, 4, False)])
def test_scores_of_every_scale(sizes, window, sinks, row_blocks, pieces, sign, sm):
    """Products are exact here, and the weights go from all equal to one-hot (the bounds take the scores as exact)."""
    B, Hq, Hkv, T, N = sizes
    cut(sizes, window, sinks, row_blocks, pieces)
    q = line([sign * (1 + t % 64) for t in range(T)], B, Hq)
    K, V = line([1 + (7 * n) % 5 for n in range(N)], B, Hkv), rand(3, B, Hkv, N, 128)
    check(q, K, V, [N - T - 5 * b for b in range(B)], [T] * B, 0, window, sinks, sm=sm)


@pytest.mark.parametrize("base", [2.0 ** 14, -2.0 ** 14, 2.0 ** 22])
@pytest.mark.parametrize("sizes,row_blocks,pieces", [((1, 64, 1, 130, 5000), 8, True), ((8, 20, 4, 100, 130), 4, False)])
def test_scores_that_differ_little_far_from_zero(sizes, row_blocks, pieces, base):
    B, Hq, Hkv, T, N = sizes
    cut(sizes, 0, 0, row_blocks, pieces)
    q, K, V = torch.zeros(B, Hq, T, 128, dtype=torch.bfloat16), torch.zeros(B, Hkv, N, 128, dtype=torch.bfloat16), rand(3, B, Hkv, N, 128)
    q[..., 0], q[..., 1] = 1, 1
    K[..., 0], K[..., 1] = base, torch.arange(N) % 7 if base < 2 ** 20 else 0
    check(q, K, V, [N - T] * B, [T] * B, sm=1.0)


@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces,tiles", [CUTS[0], CUTS[5], CUTS[6]])
def test_strides(sizes, window, sinks, row_blocks, pieces, tiles):
    """Keys and values in one pool, token by token, queries among others' rows, an interleaved output: the bits of a dense call."""
    B, Hq, Hkv, T, N = sizes
    page = 32
    cut(sizes, window, sinks, row_blocks, pieces)
    q, K, V, pos, count = inputs(sizes)
    (Kp, blocks), (Vp, _) = paged(K, page, 5, fill=0.0), paged(V, page, 5, fill=0.0)
    want, want_sums = call(q.to(DEV), Kp.to(DEV), Vp.to(DEV), pos, count, blocks.to(DEV), window, sinks, N=N)
    x = torch.zeros(B, T, Hq + 2, 128, dtype=torch.bfloat16)
    x[:, :, :Hq] = q.transpose(1, 2)
    kv = torch.stack([Kp, Vp], 3).transpose(1, 2).contiguous().to(DEV)  # pages, rows, heads, two
    out = torch.full((B, T, Hq, 2, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    sums = torch.full((B, Hq, T + 5), 7.0, device=DEV)
    bpc.chunk_attention(x.to(DEV)[:, :, :Hq].transpose(1, 2), kv[..., 0, :].transpose(1, 2), kv[..., 1, :].transpose(1, 2), ints(pos), N=N, count=ints(count),
                        block_table=blocks.to(DEV), window=window, sinks=sinks, out=out[..., 0, :].transpose(1, 2), lse_out=sums[:, :, 2:2 + T])
    assert torch.equal(out[..., 0, :].transpose(1, 2), want) and bool((out[..., 1, :] == 7).all())
    assert torch.equal(sums[:, :, 2:2 + T], want_sums) and bool((sums[:, :, :2] == 7).all()) and bool((sums[:, :, 2 + T:] == 7).all())


@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces,tiles", [CUTS[0], CUTS[6]])
def test_offsets_past_32_bits(sizes, window, sinks, row_blocks, pieces, tiles):
    """Pages, and rows a megabyte apart, that lie further than 4 GiB from the pool's or the cache's first: the bits of a dense
    call."""
    B, Hq, Hkv, T, N = sizes
    page = 64
    cut(sizes, window, sinks, row_blocks, pieces)
    q, K, V, pos, count = inputs(sizes)
    q = q.to(DEV)
    (Kp, blocks), (Vp, _) = paged(K, page, 5, fill=0.0), paged(V, page, 5, fill=0.0)
    Kp, Vp = Kp.to(DEV), Vp.to(DEV)
    want, want_sums = call(q, Kp, Vp, pos, count, blocks.to(DEV), window, sinks, N=N)
    few = Kp.shape[0]
    pages = (5 << 30) // (Hkv * page * 256)
    pools = [torch.empty(pages, Hkv, page, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for pool, x in zip(pools, (Kp, Vp)):
        pool[pages - few:] = x
    out, sums = call(q, *pools, pos, count, (blocks + (pages - few)).to(DEV), window, sinks, N=N)
    assert torch.equal(out, want) and torch.equal(sums, want_sums)
    del pools
    if Hkv == 1:
        row = 1 << 19
        far = [torch.empty(N * row, dtype=torch.bfloat16, device=DEV).as_strided((1, 1, N, 128), (0, 0, row, 1)) for _ in range(2)]
        for x, y in zip(far, (K, V)):
            x[0, 0] = y[0, 0].to(DEV)
        want, want_sums = call(q[:1], K[:1].to(DEV), V[:1].to(DEV), pos[:1], count[:1], None, window, sinks, N=N)
        out, sums = call(q[:1], *far, pos[:1], count[:1], None, window, sinks, N=N)
        assert torch.equal(out, want) and torch.equal(sums, want_sums)
