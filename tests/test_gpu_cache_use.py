"""chunk_attention, key_weights and evict_kv as a program uses them: together with the
append and the hashed step, captured into graphs, on streams, with workspaces of
their own, and at offsets past 32 bits."""

import math

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import attend, check_attend, rope_table
from cache_plain import check_log_sums, chunk_visible, gather_weights, kept_slots, log_sums
from test_gpu_attn import rand

pytestmark = pytest.mark.gpu
DEV = "cuda"
SM = 1 / math.sqrt(128)


def dev(x):
    return None if x is None else x.to(DEV)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_serve_with_a_budget():
    """Prompts of two lengths piece by piece into pages, the weights of their slots, the cut to a budget on other pages,
    and steps behind a window over what is left."""
    B, Hq, Hkv, page, per, keep, sinks, recent = 2, 8, 2, 16, 12, 60, 4, 20
    lens, chunk = [150, 97], 64
    table = rope_table(400, 128)
    order = torch.randperm(B * per * 2, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    blocks, other = dev(order[:B * per].view(B, per)), dev(order[B * per:].view(B, per))
    pools = [torch.full((B * per * 2, Hkv, page, 128), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    q, k, v = rand(2, B, Hq, 192, 128), rand(3, B, Hkv, 192, 128), rand(4, B, Hkv, 192, 128)
    weights = torch.zeros(B, Hkv, per * page, device=DEV)
    outs, sums = [], []
    for at in range(0, 192, chunk):
        count = ints([min(max(n - at, 0), chunk) for n in lens])
        pos = ints([at] * B)
        part = slice(at, at + chunk)
        bpc.append_kv_paged(dev(k[:, :, part]), dev(v[:, :, part]), *pools, blocks, pos, count=count, cos_sin=dev(table))
        lse = torch.full((B, Hq, chunk), float("nan"), device=DEV)
        outs.append(bpc.chunk_attention(dev(q[:, :, part]), *pools, pos, count=count, block_table=blocks, lse_out=lse, out=torch.zeros(B, Hq, chunk, 128, dtype=torch.bfloat16, device=DEV)))
        bpc.key_weights(dev(q[:, :, part]), pools[0], lse, weights, pos, count=count, block_table=blocks)
        sums.append(lse)
    K, V = (p[blocks.long()].transpose(1, 2).flatten(2, 3).cpu() for p in pools)
    out, lse = torch.cat(outs, 2), torch.cat(sums, 2).cpu()
    visible, away, live = chunk_visible([0] * B, lens, 192, per * page, 0, 0)
    seen = visible & live[..., None]
    check_attend(out, attend(q, K.nan_to_num(), V.nan_to_num(), seen, away, SM))
    check_log_sums(lse.nan_to_num(), log_sums(q, K.nan_to_num(), seen, away, SM), live)
    want, bound = gather_weights(q, K.nan_to_num(), lse.nan_to_num(), torch.zeros(weights.shape), lens, visible, live, away, SM, 1.0)
    assert bool(((weights.cpu().double() - want).abs() <= 3 * bound + 1e-300).all())  # three calls, a rounding of each on the way
    # the cut, to other pages of the same pools
    left = torch.full((B, Hkv, per * page), 7.0, device=DEV)
    kept = bpc.evict_kv(*pools, weights, ints(lens), keep, *pools, sinks=sinks, recent=recent, block_table=blocks, table_out=other, weights_out=left)
    now = [min(n, keep) for n in lens]
    K2, V2 = (p[other.long()].transpose(1, 2).flatten(2, 3).cpu() for p in pools)
    w = weights.cpu()
    for b in range(B):
        for h in range(Hkv):
            slots = kept_slots(w[b, h, :lens[b]], lens[b], keep, sinks, recent)
            assert kept[b, h].tolist() == slots
            assert torch.equal(K2[b, h, :keep], K[b, h, slots]) and torch.equal(V2[b, h, :keep], V[b, h, slots])
            assert torch.equal(left[b, h, :keep].cpu(), w[b, h, slots]) and bool((left[b, h, keep:] == 0).all())
    # steps go on behind the kept slots, at the tokens' own positions
    K2, V2 = K2.nan_to_num(), V2.nan_to_num()
    for t in range(3):
        q1, k1, v1 = rand(10 + t, B, Hq, 1, 128), rand(20 + t, B, Hkv, 1, 128), rand(30 + t, B, Hkv, 1, 128)
        pos = ints(now)
        bpc.append_kv_paged(dev(k1), dev(v1), *pools, other, pos, cos_sin=dev(table), rope_pos=ints([[n + t] for n in lens]))
        K2, V2 = (p[other.long()].transpose(1, 2).flatten(2, 3).cpu().nan_to_num() for p in pools)
        lse1 = torch.empty(B, Hq, 1, device=DEV)
        got = bpc.chunk_attention(dev(q1), *pools, pos, block_table=other, window=25, sinks=sinks, lse_out=lse1)
        visible, away, live = chunk_visible(now, None, 1, per * page, 25, sinks)
        check_attend(got, attend(q1, K2, V2, visible, away, SM))
        old = left.cpu().clone()
        bpc.key_weights(dev(q1), pools[0], lse1, left, pos, block_table=other, window=25, sinks=sinks, decay=0.5)
        want, bound = gather_weights(q1, K2, lse1.cpu(), old, [n + 1 for n in now], visible, live, away, SM, 0.5)
        assert bool(((left.cpu().double() - want).abs() <= bound).all())
        now = [n + 1 for n in now]


def test_a_hashed_cache_is_cut():
    """The codes go with their keys: the sparse step over what is left selects among the kept slots."""
    B, Hq, Hkv, N, L, keep, k = 2, 8, 2, 1000, 64, 400, 50
    K, V, q = dev(rand(1, B, Hkv, N, 128)), dev(rand(2, B, Hkv, N, 128)), dev(rand(3, B, Hq, 128))
    P, codes, _ = bpc.build_hash(K, torch.randn(L, 128, generator=torch.Generator().manual_seed(4)).to(DEV))
    lse = torch.empty(B, Hq, 16, device=DEV)
    last = dev(rand(5, B, Hq, 16, 128))
    pos = ints([N - 16] * B)
    bpc.chunk_attention(last, K, V, pos, lse_out=lse)
    weights = bpc.key_weights(last, K, lse, torch.empty(B, Hkv, N, device=DEV), pos, decay=0.0)
    K2, V2 = (torch.full((B, Hkv, keep + 100, 128), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    codes2 = torch.zeros(B, Hkv, keep + 100, L // 32, dtype=torch.int32, device=DEV)
    kept = bpc.evict_kv(K, V, weights, ints([N] * B), keep, K2, V2, sinks=4, recent=64, codes=codes, codes_out=codes2)
    at = kept.long()[..., None]
    assert torch.equal(codes2[:, :, :keep], torch.gather(codes, 2, at.expand(-1, -1, -1, L // 32)))
    idx = torch.empty(B, Hkv, k, dtype=torch.int32, device=DEV)
    got = bpc.decode_attention(q, K2, V2, codes2, P, k, N=keep, idx_out=idx)
    K3, V3 = (torch.gather(x, 2, at.expand(-1, -1, -1, 128)) for x in (K, V))
    idx3 = torch.empty_like(idx)
    want = bpc.decode_attention(q, K3, V3, torch.gather(codes, 2, at.expand(-1, -1, -1, L // 32)), P, k, idx_out=idx3)
    assert torch.equal(idx, idx3) and torch.equal(got, want)


def test_a_prompt_in_pieces_is_the_whole_prompt():
    B, Hq, Hkv, N = 1, 8, 2, 700
    q, K, V = rand(1, B, Hq, N, 128), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128)
    parts = [bpc.chunk_attention(dev(q[:, :, a:a + n]), dev(K), dev(V), ints([a])) for a, n in ((0, 1), (1, 63), (64, 256), (320, 380))]
    visible, away, _ = chunk_visible([0], None, N, N, 0, 0)
    check_attend(torch.cat(parts, 2)[:, [0, 5]], attend(q[:, [0, 5]], K, V, visible, away, SM))


def calls(seed=0):
    """One call of each operator on fixed buffers, with what they write."""
    B, Hq, Hkv, T, N, page, keep = 2, 8, 2, 6, 20000, 32, 500
    q, K, V = dev(rand(seed, B, Hq, T, 128)), dev(rand(seed + 3, 1, Hkv, N, 128)).expand(B, Hkv, N, 128), dev(rand(seed + 4, 1, Hkv, N, 128)).expand(B, Hkv, N, 128)
    Kp, Vp = (dev(rand(seed + s, 60, Hkv, page, 128)) for s in (5, 6))
    blocks = dev(torch.arange(2 * 22, dtype=torch.int32).view(2, 22))
    other = dev(torch.arange(44, 60, dtype=torch.int32).view(2, 8))
    pos, far, lens = ints([5, 600]), ints([19000, 12000]), ints([N, 15000])
    out, lse, out2 = torch.empty_like(q), torch.empty(B, Hq, T, device=DEV), torch.empty_like(q)
    w = torch.rand(B, Hkv, N, generator=torch.Generator().manual_seed(seed)).to(DEV)
    w0, w_out = w.clone(), torch.empty(B, Hkv, keep + 7, device=DEV)
    K_out, V_out = (torch.empty(B, Hkv, keep, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    kept, kept2 = (torch.empty(B, Hkv, keep, dtype=torch.int32, device=DEV), torch.empty(B, Hkv, 250, dtype=torch.int32, device=DEV))

    def run(stream=None):
        bpc.chunk_attention(q, Kp, Vp, pos, block_table=blocks, window=50, sinks=3, out=out2, stream=stream)
        bpc.chunk_attention(q, K, V, far, lse_out=lse, out=out, softcap=20.0, stream=stream)
        bpc.key_weights(q, K, lse, w, far, softcap=20.0, decay=0.0, stream=stream)
        bpc.evict_kv(K, V, w, lens, keep, K_out, V_out, sinks=4, recent=50, weights_out=w_out, kept_out=kept, stream=stream)
        bpc.evict_kv(Kp, Vp, w[:, :, :704], pos, 250, Kp, Vp, block_table=blocks, table_out=other, kept_out=kept2, stream=stream)

    return run, (out, lse, out2, w, w_out, K_out, V_out, kept, kept2, Kp, Vp), (q, w, w0)


def test_captured_and_replayed():
    run, outs, (q, w, w0) = calls()
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(4):
        q.copy_(dev(rand(100 + i, *q.shape)))
        w.copy_(w0)
        g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        w.copy_(w0)
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), i


def test_two_graphs_in_turn_and_on_two_streams():
    """Each call has a workspace of its own unless it is given one."""
    (run_a, outs_a, _), (run_b, outs_b, _) = calls(0), calls(50)
    run_a(), run_b()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs_a + outs_b]
    graphs = []
    for run in (run_a, run_b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        graphs.append(g)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for o in (*outs_a[:3], *outs_a[4:9], *outs_b[:3], *outs_b[4:9]):
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(sa):
            graphs[0].replay()
        with torch.cuda.stream(sb):
            graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs_a + outs_b))
        run_a(stream=sa), run_b(stream=sb)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs_a + outs_b))


def test_given_workspaces():
    q, K, V = dev(rand(1, 1, 8, 16, 128)), dev(rand(2, 1, 2, 30000, 128)), dev(rand(3, 1, 2, 30000, 128))
    pos = ints([29000])
    need = bpc.chunk_workspace_bytes(1, 8, 2, 16, 30000)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)  # any contents
    want = bpc.chunk_attention(q, K, V, pos)
    assert torch.equal(bpc.chunk_attention(q, K, V, pos, workspace=ws), want) and torch.equal(bpc.chunk_attention(q, K, V, pos, workspace=ws), want)
    with pytest.raises(bpc.BPCError):
        bpc.chunk_attention(q, K, V, pos, workspace=ws[:256])
    w = torch.rand(1, 2, 30000, generator=torch.Generator().manual_seed(1)).to(DEV)
    K_out, V_out = torch.empty(1, 2, 9000, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 2, 9000, 128, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((bpc.evict_workspace_bytes(1, 2, 30000, 9000),), 255, dtype=torch.uint8, device=DEV)
    want = bpc.evict_kv(K, V, w, ints([30000]), 9000, K_out, V_out)
    for _ in range(2):
        assert torch.equal(bpc.evict_kv(K, V, w, ints([30000]), 9000, K_out, V_out, workspace=ws), want)
    with pytest.raises(bpc.BPCError):
        bpc.evict_kv(K, V, w, ints([30000]), 9000, K_out, V_out, workspace=ws[:256])


def test_what_is_allocated_belongs_to_the_stream():
    s = torch.cuda.Stream()
    q, K, V = dev(rand(1, 1, 8, 16, 128)), dev(rand(2, 1, 2, 30000, 128)), dev(rand(3, 1, 2, 30000, 128))
    w = torch.rand(1, 2, 30000, generator=torch.Generator().manual_seed(1)).to(DEV)
    K_out, V_out = torch.empty(1, 2, 9000, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 2, 9000, 128, dtype=torch.bfloat16, device=DEV)
    pos, lens = ints([29000]), ints([30000])
    want, kept = bpc.chunk_attention(q, K, V, pos), bpc.evict_kv(K, V, w, lens, 9000, K_out, V_out)
    torch.cuda.synchronize()
    got = []
    for _ in range(6):
        got.append((bpc.chunk_attention(q, K, V, pos, stream=s), bpc.evict_kv(K, V, w, lens, 9000, K_out, V_out, stream=s)))
        torch.empty(1 << 22, dtype=torch.uint8, device=DEV).fill_(255)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) and torch.equal(y, kept) for x, y in got)


def test_results_repeat():
    """No atomics on results: the same call gives the same bits."""
    run, outs, (_, w, w0) = calls(7)
    run()
    want = [o.clone() for o in outs]
    for _ in range(4):
        w.copy_(w0)
        run()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


@pytest.mark.parametrize("kind", ["head", "row", "page"])
def test_offsets_past_32_bits(kind):
    """A cache whose heads, rows or pool's pages lie more than 4 GiB apart."""
    T, n, keep = 70, 500, 100
    q, k, v = rand(1, 1, 2, T, 128), rand(2, 1, 2, n, 128), rand(3, 1, 2, n, 128)
    visible, away, live = chunk_visible([n - T], None, T, n, 0, 0)
    want = attend(q, k, v, visible, away, SM)
    blocks = None
    if kind == "head":
        store = torch.empty(2, (1 << 32) // 256 + 5000, 128, dtype=torch.bfloat16, device=DEV)
        K, V = store[:, -n:].unsqueeze(0), dev(v)
        K.copy_(dev(k))
    elif kind == "row":
        store = torch.empty(n, 1 << 23, dtype=torch.bfloat16, device=DEV)
        K, V = store[:, :256].view(n, 2, 128).transpose(0, 1).unsqueeze(0), dev(v)
        K.copy_(dev(k))
    else:
        page, per = 64, 8
        K = torch.empty((1 << 32) // (2 * page * 256) + 3 * per, 2, page, 128, dtype=torch.bfloat16, device=DEV)
        V = torch.empty_like(K)
        blocks = torch.tensor([[K.shape[0] - 1 - 2 * i if i % 2 else i for i in range(per)]], dtype=torch.int32).to(DEV)
        bpc.append_kv_paged(dev(k), dev(v), K, V, blocks, ints([0]))
    lse = torch.empty(1, 2, T, device=DEV)
    check_attend(bpc.chunk_attention(dev(q), K, V, ints([n - T]), N=n, block_table=blocks, lse_out=lse), want)
    w = bpc.key_weights(dev(q), K, lse, torch.zeros(1, 2, n, device=DEV), ints([n - T]), N=n, block_table=blocks)
    exact, bound = gather_weights(q, k, lse.cpu(), torch.zeros(1, 2, n), [n], visible, live, away, SM, 1.0)
    assert bool(((w.cpu().double() - exact).abs() <= bound).all())
    few = bpc.key_weights(dev(q[:, :, -3:]), K, lse[:, :, -3:], torch.zeros(1, 2, n, device=DEV), ints([n - 3]), N=n, block_table=blocks)
    exact, bound = gather_weights(q[:, :, -3:], k, lse[:, :, -3:].cpu(), torch.zeros(1, 2, n), [n], visible[:, -3:], live[:, -3:], away[:, -3:], SM, 1.0)
    assert bool(((few.cpu().double() - exact).abs() <= bound).all())
    K_out, V_out = (torch.empty(1, 2, keep, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    kept = bpc.evict_kv(K, V, w, ints([n]), keep, K_out, V_out, N=n, block_table=blocks)
    for h in range(2):
        slots = kept_slots(w[0, h].cpu(), n, keep, 0, 0)
        assert kept[0, h].tolist() == slots
        assert torch.equal(K_out[0, h].cpu(), k[0, h, slots]) and torch.equal(V_out[0, h].cpu(), v[0, h, slots])


def test_scores_far_from_zero():
    """Scores of thousands keep their weights, and their logarithm."""
    q, K, V = rand(1, 1, 2, 20, 128, scale=30.0), rand(2, 1, 2, 300, 128, scale=30.0), rand(3, 1, 2, 300, 128)
    visible, away, live = chunk_visible([280], None, 20, 300, 0, 0)
    lse = torch.empty(1, 2, 20, device=DEV)
    bpc.chunk_attention(dev(q), dev(K), dev(V), ints([280]), lse_out=lse)
    check_log_sums(lse, log_sums(q, K, visible, away, SM), live)
    w = bpc.key_weights(dev(q), dev(K), lse, torch.zeros(1, 2, 300, device=DEV), ints([280])).cpu()
    exact, bound = gather_weights(q, K, lse.cpu(), torch.zeros(1, 2, 300), [300], visible, live, away, SM, 1.0)
    assert bool(((w.double() - exact).abs() <= bound).all())


def test_one_token_everywhere():
    """The smallest calls: one head, one token, one slot."""
    q, v, zero = dev(rand(1, 1, 1, 1, 128, scale=0.1)), dev(rand(2, 1, 1, 1, 128)), ints([0])
    lse = torch.empty(1, 1, 1, device=DEV)
    assert torch.equal(bpc.chunk_attention(q, q, v, zero, lse_out=lse), v)
    assert abs(float(lse) - float((q.double() ** 2).sum() * SM)) <= 2.0 ** -15
    w = bpc.key_weights(q, q, lse, torch.zeros(1, 1, 1, device=DEV), zero)
    assert abs(float(w) - 1) <= 2.0 ** -14
    K_out, V_out = torch.zeros_like(q), torch.zeros_like(v)
    assert bpc.evict_kv(q, v, w, ints([1]), 1, K_out, V_out).tolist() == [[[0]]] and torch.equal(K_out, q) and torch.equal(V_out, v)


def test_wrong_device_and_stream():
    q, K, zero = dev(rand(1, 1, 1, 1, 128)), dev(rand(2, 1, 1, 5, 128)), ints([0])
    with pytest.raises(ValueError, match="GPU"):
        bpc.chunk_attention(q, K, K.cpu(), zero)
    with pytest.raises(ValueError, match="GPU"):
        bpc.key_weights(q, K, torch.zeros(1, 1, 1), torch.zeros(1, 1, 5, device=DEV), zero)
    with pytest.raises(TypeError, match="stream"):
        bpc.chunk_attention(q, K, K, zero, stream=3)
    with pytest.raises(bpc.BPCError, match="overlaps"):  # a cache is not cut in place
        bpc.evict_kv(K, K.clone(), torch.zeros(1, 1, 5, device=DEV), ints([5]), 3, K[:, :, :3], torch.zeros(1, 1, 3, 128, dtype=torch.bfloat16, device=DEV))


@pytest.mark.parametrize("T", [1, 20, 100, 300])
@pytest.mark.parametrize("N", [300, 5000])
def test_sequences_without_new_tokens(T, N):
    """No tokens: the slots before decay, nothing else changes; and chunks that end at the last slot, or one behind."""
    q, K = dev(rand(1, 3, 8, T, 128)), dev(rand(2, 3, 2, N, 128))
    lse, h = torch.full((3, 8, T), 5.0, device=DEV), N // 2
    out, sums = torch.full((3, 8, T, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((3, 8, T), 7.0, device=DEV)
    pos, count = ints([h, 0, N + 1]), ints([0, -3, 0])
    for decay in (0.5, 0.0):
        w = bpc.key_weights(q, K, lse, torch.ones(3, 2, N, device=DEV), pos, count=count, decay=decay)
        assert bool((w[0, :, :h] == decay).all()) and bool((w[0, :, h:] == 1).all()) and bool((w[1:] == 1).all())
    bpc.chunk_attention(q, K, K, pos, count=count, out=out, lse_out=sums)
    assert bool((out == 7).all()) and bool((sums == 7).all())
    bpc.chunk_attention(q, K, K, ints([N - T, N - T + 1, -1]), out=out, lse_out=sums)
    assert bool((out[1:] == 7).all()) and bool((sums[1:] == 7).all()) and bool((sums[0] != 7).all())
