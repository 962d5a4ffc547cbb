"""evict_kv over so many slots that the segments' counts are added up between its
launches: which slots stay, exactly, and that the time grows with the slots."""

import pytest
import torch

import paper_2608_04405_amd as bpc

pytestmark = pytest.mark.gpu
DEV = "cuda"
PAGE = 1024


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def gathered(seed, *shape):
    x = torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).mul_(2).exp_()
    return torch.where(x < 0.2, 0.0, torch.where(x < 0.7, 0.25, x))


def kept_slots(w, n, keep, sinks, recent):
    """As the plain form has them: NaN behind everything, the lower slot first among equals."""
    if n <= keep:
        return torch.arange(n)
    middle = w[sinks:n - recent] + 0.0
    nan = middle.isnan()
    some = (~nan).nonzero().flatten()
    order = torch.cat([some[torch.sort(middle[some], stable=True, descending=True).indices], nan.nonzero().flatten()])
    return torch.cat([torch.arange(sinks), (order[:keep - sinks - recent] + sinks).sort().values, torch.arange(n - recent, n)])


def call(w, lens, keep, sinks, recent, **kw):
    """Pages that the sequences share, so that the cache itself is small."""
    B, H, N = w.shape
    K = torch.randn(7, H, PAGE, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    blocks = (torch.arange(B * ((N + PAGE - 1) // PAGE)) % 7).to(torch.int32).view(B, -1).to(DEV)
    out = torch.full((2, B, H, keep, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    weights_out = torch.full((B, H, keep), 7.0, device=DEV)
    kept = torch.full((B, H, keep), 7, dtype=torch.int32, device=DEV)
    run = lambda: bpc.evict_kv(K, K, w, lens, keep, *out, sinks=sinks, recent=recent, N=N, block_table=blocks, weights_out=weights_out, kept_out=kept, **kw)
    return run, K, blocks, out, weights_out, kept


def check(w, lens, keep, sinks, recent):
    B, H, N = w.shape
    run, K, blocks, out, weights_out, kept = call(w.to(DEV), ints(lens), keep, sinks, recent)
    run()
    first = kept.clone()
    run()
    assert torch.equal(kept, first)
    for b in range(B):
        for h in range(H):
            if not 0 <= lens[b] <= N:
                assert bool((kept[b, h] == 7).all()) and bool((out[:, b, h] == 7).all())
                continue
            slots = kept_slots(w[b, h], lens[b], keep, sinks, recent)
            m = len(slots)
            assert torch.equal(kept[b, h, :m].cpu().long(), slots) and bool((kept[b, h, m:] == -1).all()), (b, h)
            x, y = weights_out[b, h].cpu(), w[b, h, slots]
            assert torch.equal(x[:m].nan_to_num(nan=3e38), y.nan_to_num(nan=3e38)) and bool((x[m:] == 0).all())
            at = slots.to(DEV)
            assert torch.equal(out[0, b, h, :m], K[blocks[b].long()[at // PAGE], h, at % PAGE]) and bool((out[:, b, h, m:] == 7).all())
            assert torch.equal(out[0, b, h], out[1, b, h])


# 31 segments of 16384 slots, 32, and 33: on either side of the rule
@pytest.mark.parametrize("N", [31 * 16384, 31 * 16384 + 1, 32 * 16384 + 77])
def test_around_the_rule(N):
    check(gathered(N, 2, 2, N), [N, N - 200001], 30000, 4, 1000)


@pytest.mark.parametrize("what", ["equal", "zeros", "lowest bits", "nan", "infinite", "ascending"])
def test_weights_of_every_kind(what):
    N = 900000
    g = torch.Generator().manual_seed(3)
    w = torch.randn(1, 2, N, generator=g)
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
    else:
        w = torch.arange(2 * N, dtype=torch.float32).view(1, 2, N)
    for keep, sinks, recent in ((N // 2, 3, N // 4), (N - 1, 2, 2), (20000, 0, 0), (500, 300, 200)):
        check(w, [N], keep, sinks, recent)


def test_lengths():
    """Sequences that fill the room, some segments, one or none, and ones that are skipped."""
    N, keep = 700000, 20000
    check(gathered(5, 9, 1, N), [N, 16384 * 32, 16384 * 40 + 1, keep, keep + 1, 0, N + 1, -1, 100], keep, 4, 16)


def test_captured_and_replayed():
    w = gathered(6, 1, 2, 600000).to(DEV)
    workspace = torch.empty(bpc.evict_workspace_bytes(1, 2, 600000, 9000), dtype=torch.uint8, device=DEV)
    lens = ints([600000])
    run, *_, kept = call(w, lens, 9000, 4, 100, workspace=workspace)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i, n in enumerate((600000, 540000, 20000, 599999)):
        w.copy_(gathered(10 + i, 1, 2, 600000))
        lens.fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        for h in range(2):
            assert torch.equal(kept[0, h].cpu().long(), kept_slots(w[0, h].cpu(), n, 9000, 4, 100))


def test_time_grows_with_the_slots():
    """Four times the slots take no more than 5.5 times as long (each workgroup adding up all segments' counts: 8)."""
    def time(N):
        w = torch.rand(1, 8, N, generator=torch.Generator().manual_seed(1)).to(DEV)
        workspace = torch.empty(bpc.evict_workspace_bytes(1, 8, N, 1000), dtype=torch.uint8, device=DEV)
        run, *_ = call(w, ints([N]), 1000, 4, 100, workspace=workspace)
        run()
        torch.cuda.synchronize()
        best = float("inf")
        for _ in range(20):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(3):
                run()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b) / 3)
        return best

    small, large = time(64 * 16384), time(256 * 16384)
    print(f"{small * 1000:.0f} us, {large * 1000:.0f} us", flush=True)
    assert large <= 5.5 * small
