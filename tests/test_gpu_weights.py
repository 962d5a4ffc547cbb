"""key_weights against the plain 64-bit form: chunks and single tokens, windows,
caps and biases, decays, and whatever lies where nothing is to be read."""

import math

import pytest
import torch

import paper_2608_04405_amd as bpc
from cache_plain import chunk_visible, gather_weights, log_sums, paged

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


def check(q, K, pos, count=None, window=0, sinks=0, cap=0.0, slopes=None, decay=1.0, page=0, lse=None, hidden=None, bad=()):
    B, Hq, T, _ = q.shape
    Hkv, N = K.shape[1:3]
    visible, away, live = chunk_visible(pos, count, T, N, window, sinks)
    if lse is None:
        lse = log_sums(q, K, visible & live[..., None], away, SM, cap, slopes)[0].float()
    if hidden is not None:
        visible = visible & ~hidden[:, None]
    old = torch.rand(B, Hkv, N + 3, generator=torch.Generator().manual_seed(5)) * 3
    blocks, Kp = None, K
    if page:
        Kp, blocks = paged(K, page, 11)
        for b, i, v in bad:
            blocks[b, i] = v
    weights = dev(old)
    got = bpc.key_weights(dev(q), dev(Kp), dev(lse), weights, ints(pos), N=N, count=ints(count), block_table=dev(blocks), window=window, sinks=sinks,
                          softcap=cap, slopes=dev(slopes), decay=decay)
    assert got is weights
    counts = [T if count is None else min(max(c, 0), T) for c in (count or [T] * B)]
    end = [p + c if p >= 0 and p + c <= N else 0 for p, c in zip(pos, counts)]
    want, bound = gather_weights(q, K, lse, old[:, :, :N], end, visible, live, away, SM, decay, cap, slopes)
    got = weights.cpu()
    assert torch.equal(got[:, :, N:], old[:, :, N:])
    for b in range(B):
        assert torch.equal(got[b, :, end[b]:], old[b, :, end[b]:])
    off = (got[:, :, :N].double() - want).abs()
    assert bool((off <= bound).all()), float(((off - bound) / (bound + 1e-300)).max())
    return got


SIZES = [(1, 1, 1, 1, [0], None, 1), (1, 4, 1, 1, [32], None, 40), (2, 8, 2, 1, [130, 5], None, 150), (2, 8, 2, 65, [0, 40], [65, 3], 110),
         (1, 3, 3, 31, [169], None, 200), (3, 6, 2, 40, [100, 0, 57], [40, 0, 17], 150), (1, 20, 1, 5, [35], None, 40),
         (2, 4, 4, 130, [647, 0], [130, 129], 777), (1, 8, 1, 3, [4000], None, 4003), (2, 128, 1, 2, [299, 150], None, 310),
         (16, 8, 8, 2, [1000 - 50 * b for b in range(16)], None, 1100)]


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("B,Hq,Hkv,T,pos,count,N", SIZES)
@pytest.mark.parametrize("cap,bias", SCORES)
def test_weights(B, Hq, Hkv, T, pos, count, N, cap, bias, page):
    print(f"[weights] {B} {Hq} {Hkv} {T} {pos} {count} {N} page={page} cap={cap} bias={bias}", flush=True)
    check(rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), pos, count, cap=cap, slopes=slopes_of(Hq) if bias else None, page=page)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (64, 0), (100, 33), (300, 64), (100000, 3), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("B,Hq,Hkv,T,pos,count,N", [(2, 4, 1, 1, [0, 900], None, 901), (2, 8, 2, 70, [0, 500], [70, 66], 600), (1, 2, 2, 300, [200], None, 500)])
def test_window(B, Hq, Hkv, T, pos, count, N, window, sinks):
    print(f"[weights window] {B} {Hq} {Hkv} {T} {pos} {count} {N} {window} {sinks}", flush=True)
    for decay, page in ((1.0, 0), (0.5, 16), (0.0, 32)):
        for cap, bias in ((0.0, False), (30.0, True)):
            check(rand(1, B, Hq, T, 128, scale=1.5), rand(2, B, Hkv, N, 128), pos, count, window, sinks, cap, slopes_of(Hq) if bias else None, decay, page)


@pytest.mark.parametrize("decay", [0.0, 0.25, 0.98, 1.0, 3.0])
def test_decay(decay):
    got = check(rand(1, 2, 4, 9, 128), rand(2, 2, 2, 300, 128), [100, 0], [9, 0], decay=decay)
    assert bool(got.isfinite().all())


def test_decay_zero_does_not_read():
    q, K = rand(1, 1, 4, 3, 128), rand(2, 1, 2, 200, 128)
    w = torch.full((1, 2, 200), float("nan"), device=DEV)
    lse = torch.zeros(1, 4, 3, device=DEV) + 5
    bpc.key_weights(dev(q), dev(K), lse, w, ints([150]), decay=0.0)
    assert bool(w[:, :, :153].isfinite().all()) and bool(w[:, :, 153:].isnan().all())


def test_many_rows():
    """A slot that 40000 rows look at, a small share each: nothing of the sum is lost."""
    B, Hq, Hkv, T, N = 1, 64, 1, 640, 700
    q, K = rand(1, B, Hq, T, 128, scale=0.2), rand(2, B, Hkv, N, 128)
    check(q, K, [60])


def test_weights_sum_to_the_rows():
    """Every row's weights add up to one."""
    B, Hq, Hkv, T, N = 2, 8, 2, 33, 500
    q, K, V = dev(rand(1, B, Hq, T, 128, scale=1.5)), dev(rand(2, B, Hkv, N, 128)), dev(rand(3, B, Hkv, N, 128))
    lse = torch.empty(B, Hq, T, device=DEV)
    pos = ints([460, 100])
    bpc.chunk_attention(q, K, V, pos, window=90, sinks=3, lse_out=lse)
    w = bpc.key_weights(q, K, lse, torch.zeros(B, Hkv, N, device=DEV), pos, window=90, sinks=3)
    total = w.double().sum(-1).cpu()
    # lse and every term are off by scores' errors (136 roundings of S < 64) and less
    assert float((total / (Hq // Hkv * T) - 1).abs().max()) <= 2 * (136 * 64 * 2.0 ** -24 + 2.0 ** -14)


@pytest.mark.parametrize("what", ["nan", "inf", "lowest"])
@pytest.mark.parametrize("T,pos,window,sinks", [(40, 160, 0, 0), (2, 900, 50, 5), (70, 100, 33, 2)])
def test_hidden_slots_and_rows_do_not_reach(T, pos, window, sinks, what):
    """Slots that no token sees, rows behind the last, and their lse hold anything."""
    N = pos + T + 30
    q, K = rand(1, 1, 4, T + 5, 128), rand(2, 1, 2, N, 128)
    bad = {"nan": float("nan"), "inf": float("inf"), "lowest": torch.finfo(torch.bfloat16).min}[what]
    visible, away, live = chunk_visible([pos], [T], T + 5, N, window, sinks)
    lse = log_sums(q, K, visible & live[..., None], away, SM)[0].float()
    q[:, :, T:], lse[:, :, T:] = bad, bad
    seen = (visible & live[..., None]).any(1)[0]
    K[:, :, ~seen] = bad
    old = torch.rand(1, 2, N)
    clean = torch.where(seen[:, None], K, 0.0)
    want, bound = gather_weights(torch.where(live[:, None, :, None], q, 0.0), clean, lse, old, [pos + T], visible, live, away, SM, 0.5)
    got = bpc.key_weights(dev(q), dev(K), dev(lse), dev(old), ints([pos]), count=ints([T]), window=window, sinks=sinks, decay=0.5).cpu()
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), float((off - bound).max())


def test_a_nan_row_reaches_the_slots_it_sees_alone():
    N, T = 300, 40
    q, K = rand(1, 1, 2, T, 128), rand(2, 1, 2, N, 128)
    visible, away, live = chunk_visible([200], None, T, N, 20, 4)
    lse = log_sums(q, K, visible, away, SM)[0].float()
    q[0, 1, 7, 3] = float("nan")
    w = bpc.key_weights(dev(q), dev(K), dev(lse), torch.zeros(1, 2, N, device=DEV), ints([200]), window=20, sinks=4).cpu()
    assert torch.equal(w[0, 1].isnan(), visible[0, 7]) and bool(w[0, 0].isfinite().all())


def test_rows_that_saw_nothing_add_nothing():
    q, K = rand(1, 1, 4, 6, 128), rand(2, 1, 2, 50, 128)
    visible, away, live = chunk_visible([40], None, 6, 50, 0, 0)
    lse = log_sums(q, K, visible, away, SM)[0].float()
    lse[:, 1:3, 2:5] = -float("inf")
    check(q, K, [40], lse=lse)


def test_bad_pages_gather_nothing():
    hidden = torch.zeros(2, 150, dtype=torch.bool)
    hidden[0, 32:48] = hidden[0, 128:144] = hidden[1, :16] = True
    for decay in (1.0, 0.5):
        check(rand(1, 2, 4, 5, 128), rand(2, 2, 2, 150, 128), [140, 20], page=16, hidden=hidden, decay=decay, bad=((0, 2, -1), (0, 8, 99), (1, 0, 2 ** 31 - 1)))


def test_sequences_that_do_not_fit_are_left():
    check(rand(1, 6, 4, 8, 128), rand(2, 6, 2, 100, 128), [-1, 93, 92, 2 ** 31 - 1, -2 ** 31, 97], [8, 8, 8, 8, 8, 3], decay=0.5)
    check(rand(1, 6, 4, 8, 128), rand(2, 6, 2, 100, 128), [0] * 6, [-5, 0, 1, 8, 9, 2 ** 31 - 1], decay=0.5)


def test_strides_and_repeats():
    """Views of a projection's rows, of longer log-sum-exps and of interleaved weights; equal calls, equal bits."""
    B, Hq, Hkv, T, N = 2, 8, 2, 37, 200
    x, K = dev(rand(1, B, T, Hq + 2, 128)), dev(rand(2, B, N, Hkv, 128))
    lse = torch.randn(B, Hq, T + 9, generator=torch.Generator().manual_seed(3)).to(DEV) + 8
    store = torch.ones(Hkv, B, 2, N + 7, device=DEV)
    view = store[:, :, 0, :N].transpose(0, 1)
    pos = ints([150, 7])
    q = x[:, :, :Hq].transpose(1, 2)
    bpc.key_weights(q, K.transpose(1, 2), lse[:, :, 4:4 + T], view, pos)
    want = bpc.key_weights(q.contiguous(), K.transpose(1, 2).contiguous(), lse[:, :, 4:4 + T].contiguous(), torch.ones(B, Hkv, N, device=DEV), pos)
    assert torch.equal(view, want) and bool((store[:, :, 1] == 1).all()) and bool((store[:, :, 0, N:] == 1).all())
    again = bpc.key_weights(q.contiguous(), K.transpose(1, 2).contiguous(), lse[:, :, 4:4 + T].contiguous(), torch.ones(B, Hkv, N, device=DEV), pos)
    assert torch.equal(again, want)
    # the last tokens alone: views, and the position moved on
    tail = bpc.key_weights(q[:, :, 30:], K.transpose(1, 2), lse[:, :, 34:4 + T], torch.zeros(B, Hkv, N, device=DEV), pos + 30)
    head = bpc.key_weights(q[:, :, :30], K.transpose(1, 2), lse[:, :, 4:34], torch.zeros(B, Hkv, N, device=DEV), pos)
    assert float((tail + head + 1 - want).abs().max()) <= 2.0 ** -20 * float(want.max())
