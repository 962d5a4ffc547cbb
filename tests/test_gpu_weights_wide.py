"""key_weights at sizes whose kernels small calls do not reach: 64 keys a wavefront,
runs of many pages and keys, keys that pass the last-level cache by.  Some heads of
each call are compared with the 64-bit form, and every call is made twice."""

import math

import pytest
import torch

import paper_2608_04405_amd as bpc
from cache_plain import chunk_visible
from cache_rows import weigh_head

pytestmark = pytest.mark.gpu
DEV = "cuda"
SM = 1 / math.sqrt(128)


def rand(seed, *shape, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def slopes_of(H):
    return torch.tensor([2.0 ** (-(h % 8) - 1) for h in range(H)])


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def check(sizes, pos, count, page, window, sinks, decay, cap, bias, bad=False):
    B, Hq, Hkv, T, N = sizes
    G = Hq // Hkv
    print(f"[weights wide] {sizes} page={page} window={window} sinks={sinks} decay={decay} cap={cap} bias={bias} bad={bad}", flush=True)
    q = rand(1, B, Hq, T, 128, scale=1.5)
    hidden = torch.zeros(B, N, dtype=torch.bool)
    blocks = None
    if page:  # pages that several sequences share
        per = (N + page - 1) // page
        K = rand(2, 40, Hkv, page, 128)
        blocks = torch.randint(0, 40, (B, per), generator=torch.Generator().manual_seed(3)).to(torch.int32)
        whole = blocks.clone()
        if bad:
            for b in range(B):
                for i, v in ((1 + b % 3, -1), (per // 2 - b % 5, 40), ((pos[b] + count[b] - 1) // page, 2 ** 31 - 1)):
                    blocks[b, i] = v
                    hidden[b, i * page:(i + 1) * page] = True
        keys = lambda b, h: K[whole[b].long(), h].flatten(0, 1)[:N]
    else:
        K = rand(2, 1, Hkv, N, 128).expand(B, Hkv, N, 128)
        keys = lambda b, h: K[b, h]
    slopes = slopes_of(Hq) if bias else None
    # near the largest score of 1000 random ones, so that terms are of every size
    lse = (torch.randn(B, Hq, T, generator=torch.Generator().manual_seed(4)) + 8).float()
    old = torch.rand(B, Hkv, N, generator=torch.Generator().manual_seed(5)) * 3
    args = dict(N=N, count=ints(count), block_table=None if blocks is None else blocks.to(DEV), window=window, sinks=sinks, softcap=cap,
                slopes=None if slopes is None else slopes.to(DEV), decay=decay)
    qd, Kd, ld = q.to(DEV), K.to(DEV) if page else K[:1].to(DEV).expand(B, Hkv, N, 128), lse.to(DEV)
    got = bpc.key_weights(qd, Kd, ld, old.clone().to(DEV), ints(pos), **args)
    assert torch.equal(got, bpc.key_weights(qd, Kd, ld, old.clone().to(DEV), ints(pos), **args))
    got = got.cpu()
    visible, away, live = chunk_visible(pos, count, T, N, window, sinks)
    for b in sorted({0, B // 2, B - 1}):
        assert torch.equal(got[b, :, pos[b] + count[b]:], old[b, :, pos[b] + count[b]:])
    for b, h in sorted({(0, 0), (B // 2, Hkv // 2), (B - 1, Hkv - 1)}):
        e = pos[b] + count[b]
        heads = slice(h * G, h * G + G)
        see = visible[b] & live[b][:, None] & ~hidden[b]
        want, bound = weigh_head(q[b, heads], keys(b, h), lse[b, heads], old[b, h], see, away[b], SM, decay, cap, None if slopes is None else slopes[heads])
        off = (got[b, h].double() - want).abs()[:e]
        assert bool((off <= bound[:e]).all()), (b, h, float((off / bound[:e]).max()))


def ragged(B, T, N):
    return [max(0, N - T - 317 * b) for b in range(B)], [max(0, T - 3 * b) for b in range(B)]


# 64 keys a wavefront: more than 64 rows, at least 1024 blocks of 128 keys, of a multiple of eight heads, of many, and of few
MANY = [(4, 32, 8, 40, 4200), (4, 24, 8, 50, 4100), (5, 14, 7, 90, 3700), (3, 8, 1, 30, 17000)]


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("window,sinks,decay,cap,bias", [(0, 0, 1.0, 0.0, False), (700, 300, 0.5, 0.0, False), (100, 5, 0.0, 30.0, False), (0, 0, 0.5, 0.0, True),
                                                         (900, 64, 1.0, 50.0, True)])
@pytest.mark.parametrize("sizes", MANY)
def test_many_rows_of_many_keys(sizes, window, sinks, decay, cap, bias, page):
    B, Hq, Hkv, T, N = sizes
    assert T * Hq // Hkv > 64 and (B * Hkv + 7) // 8 * 8 * ((N + 127) // 128) >= 1024
    pos, count = ragged(B, T, N)
    check(sizes, pos, count, page, window, sinks, decay, cap, bias)


# runs of 512 keys and more, up to 2048; with more than 320 MiB of keys these are read once
LONG = [(4, 32, 8, 1, 20000), (8, 80, 8, 5, 20001), (16, 32, 8, 2, 20000), (16, 64, 16, 15, 17000)]


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("window,sinks,decay,cap,bias", [(0, 0, 0.5, 0.0, False), (5000, 3000, 1.0, 0.0, False), (3001, 5, 0.0, 30.0, False), (9000, 64, 0.98, 0.0, True)])
@pytest.mark.parametrize("sizes", LONG)
def test_few_rows_of_long_runs(sizes, window, sinks, decay, cap, bias, page):
    B, Hq, Hkv, T, N = sizes
    assert T * Hq // Hkv <= 64 and B * Hkv * N > 1 << 19
    pos, _ = ragged(B, T, N)
    check(sizes, pos, [T - b % T for b in range(B)], page, window, sinks, decay, cap, bias)


@pytest.mark.parametrize("decay", [1.0, 0.5])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("sizes", [MANY[0], LONG[0], LONG[3]])
def test_bad_pages_in_the_first_a_middle_and_the_last_place(sizes, page, decay):
    B, Hq, Hkv, T, N = sizes
    pos, count = ragged(B, T, N)
    check(sizes, pos, [max(1, c) for c in count], page, 0, 0, decay, 0.0, False, bad=True)
