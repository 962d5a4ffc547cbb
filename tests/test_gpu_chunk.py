"""chunk_attention against the plain 64-bit form: ragged chunks, windows with first
slots that stay visible, paged and contiguous caches, log-sum-exps, and whatever
lies in slots and rows that are not there."""

import math

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import attend, check_attend
from cache_plain import check_log_sums, chunk_visible, log_sums, paged

pytestmark = pytest.mark.gpu
DEV = "cuda"
SM = 1 / math.sqrt(128)
SCORES = [(0.0, False), (30.0, False), (0.0, True), (50.0, True)]


def rand(seed, *shape, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def slopes_of(H):
    return torch.tensor([2.0 ** (-(h % 8) - 1) for h in range(H)])


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def dev(x):
    return None if x is None else x.to(DEV)


def call(q, K, V, pos, count=None, page=0, window=0, sinks=0, cap=0.0, slopes=None, lse=True, N=None):
    """(out, lse) of the call, rows that it leaves filled with 7."""
    B, Hq, T, _ = q.shape
    out = torch.full((B, Hq, T, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    sums = torch.full((B, Hq, T), 7.0, device=DEV) if lse else None
    blocks = None
    N = K.shape[2] if N is None else N
    if page:
        (K, blocks), (V, same) = paged(K, page, 11), paged(V, page, 11)
        assert torch.equal(blocks, same)
    got = bpc.chunk_attention(dev(q), dev(K), dev(V), ints(pos), N=N, count=ints(count), block_table=dev(blocks), window=window, sinks=sinks,
                              softcap=cap, slopes=dev(slopes), out=out, lse_out=sums)
    assert got is out
    return out, sums


def check(q, K, V, pos, count=None, window=0, sinks=0, cap=0.0, slopes=None, heads=None, hidden=None, **kw):
    """The call against its plain form, on the given heads or all."""
    B, Hq, T, _ = q.shape
    G = Hq // K.shape[1]
    out, sums = call(q, K, V, pos, count, window=window, sinks=sinks, cap=cap, slopes=slopes, **kw)
    visible, away, live = chunk_visible(pos, count, T, K.shape[2], window, sinks)
    if hidden is not None:
        visible &= ~hidden[:, None]
    heads = list(range(Hq)) if heads is None else heads
    seen = visible & live[..., None]
    Kh, Vh = K[:, [h // G for h in heads]], V[:, [h // G for h in heads]]
    sl = None if slopes is None else slopes[heads]
    want = attend(q[:, heads], Kh, Vh, seen, away, SM, cap, sl)
    got = out[:, heads].cpu()
    lv = live[:, None, :, None].expand_as(got)
    check_attend(torch.where(lv, got, 0.0), want)
    assert bool((out.cpu()[~live[:, None, :, None].expand_as(out)] == 7).all())
    if sums is not None:
        check_log_sums(sums[:, heads], log_sums(q[:, heads], Kh, seen, away, SM, cap, sl), live)
        assert bool((sums.cpu()[~live[:, None].expand_as(sums)] == 7).all())
    return out, sums


# (B, Hq, Hkv, T, pos, count, N)
SIZES = [(1, 1, 1, 1, [0], None, 1), (1, 4, 1, 1, [32], None, 40), (2, 8, 2, 1, [130, 5], None, 150), (2, 8, 2, 65, [0, 40], [65, 3], 110),
         (1, 3, 3, 31, [169], None, 200), (3, 6, 2, 40, [100, 0, 57], [40, 0, 17], 150), (1, 16, 1, 64, [0], None, 64), (1, 20, 1, 5, [35], None, 40),
         (2, 4, 4, 130, [647, 0], [130, 129], 777), (1, 8, 1, 3, [4000], None, 4003), (2, 16, 1, 1, [2999, 1500], None, 3000)]


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("B,Hq,Hkv,T,pos,count,N", SIZES)
@pytest.mark.parametrize("cap,bias", SCORES)
def test_causal(B, Hq, Hkv, T, pos, count, N, cap, bias, page):
    print(f"[chunk] {B} {Hq} {Hkv} {T} {pos} {count} {N} page={page} cap={cap} bias={bias}", flush=True)
    check(rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128), pos, count, cap=cap,
          slopes=slopes_of(Hq) if bias else None, page=page)


@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (64, 0), (100, 33), (128, 64), (100000, 3), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("B,Hq,Hkv,T,pos,count,N", [(2, 4, 1, 1, [0, 900], None, 901), (2, 8, 2, 70, [0, 500], [70, 66], 600),
                                                      (1, 2, 2, 300, [200], None, 500), (1, 4, 1, 3, [2990], None, 3001)])
def test_window(B, Hq, Hkv, T, pos, count, N, window, sinks, page):
    print(f"[chunk window] {B} {Hq} {Hkv} {T} {pos} {count} {N} page={page} {window} {sinks}", flush=True)
    for cap, bias in ((0.0, False), (30.0, True)):
        check(rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128), pos, count, window, sinks, cap,
              slopes_of(Hq) if bias else None, page=page)


# sizes, window and sinks for each cut: row blocks of a workgroup, in pieces or not
CUTS = [((1, 8, 2, 9, 120), 0, 0, 1, False), ((1, 4, 1, 7, 3000), 0, 0, 1, True), ((8, 20, 4, 100, 130), 0, 0, 4, False),
        ((3, 24, 2, 140, 700), 0, 0, 4, True), ((6, 40, 5, 130, 150), 0, 0, 8, False), ((1, 128, 1, 41, 5000), 0, 0, 4, True), ((1, 64, 1, 130, 5000), 0, 0, 8, True),
        ((6, 40, 5, 130, 400), 60, 10, 8, False), ((1, 40, 2, 130, 3000), 2000, 70, 4, True), ((1, 64, 1, 130, 5000), 2500, 70, 8, True)]


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("cap,bias", SCORES)
@pytest.mark.parametrize("sizes,window,sinks,row_blocks,pieces", CUTS)
def test_cuts(sizes, window, sinks, row_blocks, pieces, cap, bias, page):
    B, Hq, Hkv, T, N = sizes
    print(f"[chunk cut] {sizes} {window} {sinks} page={page} cap={cap} bias={bias}", flush=True)
    got = bpc.chunk_cut(*sizes, window, sinks)
    assert got[0] == row_blocks and (got[1] > 1) == pieces and not got[2], got
    pos = [(N - T) * (b + 1) // B for b in range(B)]
    count = [max(1, T - 13 * b) for b in range(B)]
    G = Hq // Hkv
    heads = [h * G + (g + 5 * h) % G for h in range(Hkv) for g in (T % G, T % G + G // 2)]
    slopes = slopes_of(Hq) if bias else None
    args = (rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128), pos, count, window, sinks, cap, slopes)
    out, _ = check(*args, heads=heads, page=page)
    bare, _ = call(*args[:5], window=window, sinks=sinks, cap=cap, slopes=slopes, page=page, lse=False)
    assert torch.equal(bare, out)  # with or without the log-sum-exps


def test_streamed():
    """Keys and values that pass the last-level cache by: more than 320 MiB of them."""
    B, Hq, Hkv, T, N = 16, 32, 8, 1, 6000
    assert bpc.chunk_cut(B, Hq, Hkv, T, N)[2]
    pos = [N - 1 - 300 * b for b in range(B)]
    q, K, V = rand(1, B, Hq, T, 128, scale=1.5), rand(2, 1, Hkv, N, 128).expand(B, Hkv, N, 128), rand(3, 1, Hkv, N, 128).expand(B, Hkv, N, 128)
    check(q, K, V, pos, heads=[0, 13, 31])
    check(q, K, V, pos, heads=[5, 30], page=64)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("T,pos,window,sinks", [(40, 160, 0, 0), (2, 2900, 50, 5), (150, 0, 0, 0), (70, 100, 33, 2)])
@pytest.mark.parametrize("what", ["nan", "inf", "lowest"])
def test_hidden_slots_do_not_reach(T, pos, window, sinks, what, page):
    """Slots behind a token, out of its window, and behind the last hold anything."""
    N = pos + T + 30
    q, K, V = rand(1, 1, 4, T, 128), rand(2, 1, 2, N, 128), rand(3, 1, 2, N, 128)
    bad = {"nan": float("nan"), "inf": float("inf"), "lowest": torch.finfo(torch.bfloat16).min}[what]
    K[:, :, pos + T:], V[:, :, pos + T:] = bad, bad
    K[:, :, pos + T - 1], V[:, :, pos + T - 1, ::3] = bad, bad  # the last token alone sees this one
    if window:
        K[:, :, sinks:pos - window], V[:, :, sinks:pos - window] = bad, bad
    out, sums = call(q, K, V, [pos], window=window, sinks=sinks, page=page)
    visible, away, live = chunk_visible([pos], None, T, N, window, sinks)
    want = attend(q[:, :, :T - 1], K, V, visible[:, :T - 1], away[:, :T - 1], SM)
    check_attend(out[:, :, :T - 1], want)
    assert bool(want[0].isfinite().all())
    check_log_sums(sums[:, :, :T - 1], log_sums(q[:, :, :T - 1], K, visible[:, :T - 1], away[:, :T - 1], SM), live[:, :T - 1])
    if what == "nan":
        assert bool(out[:, :, T - 1].isnan().all()) and bool(sums[:, :, T - 1].isnan().all())


def test_visible_infinite_values_count():
    """A value of V that is infinite reaches the tokens that see it, and no others."""
    N, T = 200, 60
    q, K, V = rand(1, 1, 4, T, 128), rand(2, 1, 2, N, 128), rand(3, 1, 2, N, 128)
    V[0, :, 150, 7], V[0, :, 3, 9], V[0, 1, 180, 100] = float("inf"), -float("inf"), float("nan")
    for page in (0, 16):
        check(q, K, V, [140], window=20, sinks=4, page=page)
        check(q, K, V, [140], page=page)


def test_bad_pages_hide_their_slots():
    B, T, N, page = 2, 5, 150, 16
    q, K, V = rand(1, B, 4, T, 128, scale=1.5), rand(2, B, 2, N, 128), rand(3, B, 2, N, 128)
    (Kp, blocks), (Vp, _) = paged(K, page, 3), paged(V, page, 3)
    pos = [140, 20]
    hidden = torch.zeros(B, N, dtype=torch.bool)
    for b, i, v in ((0, 2, -1), (0, 8, Kp.shape[0]), (1, 0, 2 ** 31 - 1), (1, 1, -2 ** 31)):
        blocks[b, i] = v
        hidden[b, i * page:(i + 1) * page] = True
    for window, sinks in ((0, 0), (30, 3)):
        out, sums = torch.full((B, 4, T, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((B, 4, T), 7.0, device=DEV)
        bpc.chunk_attention(dev(q), dev(Kp), dev(Vp), ints(pos), N=N, block_table=dev(blocks), window=window, sinks=sinks, out=out, lse_out=sums)
        visible, away, live = chunk_visible(pos, None, T, N, window, sinks)
        visible &= ~hidden[:, None]
        check_attend(out, attend(q, K, V, visible, away, SM))
        check_log_sums(sums, log_sums(q, K, visible, away, SM), live)
        assert bool((out[1] == 0).all()) and bool((sums[1] == -float("inf")).all())  # sequence 1 sees nothing


def test_sequences_that_do_not_fit_are_left():
    N, T = 100, 8
    q, K, V = rand(1, 6, 4, T, 128), rand(2, 6, 2, N, 128), rand(3, 6, 2, N, 128)
    pos, count = [-1, 93, 92, 2 ** 31 - 1, -2 ** 31, 97], [8, 8, 8, 8, 8, 3]
    out, _ = check(q, K, V, pos, count)
    rows = [bool((out[b] == 7).all()) for b in range(6)]
    assert rows == [True, True, False, True, True, False]
    out, _ = check(q, K, V, [0] * 6, [-5, 0, 1, 8, 9, 2 ** 31 - 1])
    assert bool((out[:2] == 7).all()) and bool((out[2, :, 1:] == 7).all()) and bool((out[3:] != 7).any())


def test_slots_of_the_default_extent():
    """Without N: the cache's rows, or what the table holds."""
    q, K, V = rand(1, 2, 4, 3, 128), rand(2, 2, 2, 90, 128), rand(3, 2, 2, 90, 128)
    pos = ints([80, 87])
    a = bpc.chunk_attention(dev(q), dev(K), dev(V), pos)
    (Kp, blocks), (Vp, _) = paged(K, 16, 3), paged(V, 16, 3)
    b = bpc.chunk_attention(dev(q), dev(Kp), dev(Vp), pos, block_table=dev(blocks))
    assert torch.equal(a, b)


def test_strides():
    """Views of a projection's rows, an interleaved output, pools of keys and values in one."""
    B, Hq, Hkv, T, page, per = 2, 8, 2, 37, 16, 6
    x = rand(1, B, T, Hq + 2, 128)
    kv = rand(2, B * per, page, Hkv, 2, 128)
    blocks = torch.randperm(B * per, generator=torch.Generator().manual_seed(2)).view(B, per).to(torch.int32)
    out = torch.full((B, T, Hq, 2, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    sums = torch.full((B, Hq, T + 5), 7.0, device=DEV)
    dx, dkv = dev(x), dev(kv)
    Kp, Vp = dkv[..., 0, :].transpose(1, 2), dkv[..., 1, :].transpose(1, 2)
    bpc.chunk_attention(dx[:, :, :Hq].transpose(1, 2), Kp, Vp, ints([50, 3]), count=ints([37, 20]), block_table=dev(blocks),
                        out=out[..., 0, :].transpose(1, 2), lse_out=sums[:, :, 2:2 + T])
    K, V = (t.cpu()[blocks.long()].transpose(1, 2).flatten(2, 3) for t in (Kp, Vp))
    q = x[:, :, :Hq].transpose(1, 2)
    want, want_sums = call(q, K, V, [50, 3], [37, 20])
    assert torch.equal(out[..., 0, :].transpose(1, 2), want) and bool((out[..., 1, :] == 7).all())
    assert torch.equal(sums[:, :, 2:2 + T], want_sums) and bool((sums[:, :, :2] == 7).all()) and bool((sums[:, :, 2 + T:] == 7).all())


def test_it_is_the_prefill_and_the_tree():
    """Without window and ragged lengths: what the others compute."""
    q, K, V = rand(1, 2, 8, 50, 128), rand(2, 2, 2, 170, 128), rand(3, 2, 2, 170, 128)
    a, _ = call(q, K, V, [120, 120])
    visible, away, _ = chunk_visible([120, 120], None, 50, 170, 0, 0)
    check_attend(bpc.prefill_attention(dev(q), dev(K), dev(V)), attend(q, K, V, visible, away, SM))
    assert float((a.float() - bpc.prefill_attention(dev(q), dev(K), dev(V)).float()).abs().max()) <= 2.0 ** -6
    b = bpc.tree_attention(dev(q), dev(K), dev(V), ints([120, 120]))
    assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -6
