"""qk_norm_rope, append_kv_paged, prefill_attention and tree_attention as a
program uses them: together with the hashed cache, captured into graphs, on
streams, with workspaces of their own, and at offsets past 32 bits."""

import math

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import attend, check_attend, check_turn, rope_table, tree_view, turn
from test_gpu_attn import as_int64, rand, tree_masks

pytestmark = pytest.mark.gpu
DEV = "cuda"
SM = 1 / math.sqrt(128)
EPS = 1e-6


def dev(x):
    return None if x is None else x.to(DEV)


def test_prefill_hash_draft_verify():
    """A prompt through the projections' rows, the prefill and the hash build; drafts by the sparse step; their
    verification over the same cache, contiguous and in pages."""
    B, Hq, Hkv, T0, T, Ncap, L, k, page = 2, 8, 2, 300, 5, 384, 64, 40, 64
    table = rope_table(Ncap, 128)
    wq, wk = 1 + rand(1, 128) * 0.1, 1 + rand(2, 128) * 0.1
    x = rand(3, B, T0, Hq + 2 * Hkv, 128)
    q, kk, v = (x[:, :, a:b].transpose(1, 2) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    pos = torch.arange(T0, dtype=torch.int32).expand(B, T0)
    K = torch.full((B, Hkv, Ncap, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    V = torch.full_like(K, float("nan"))
    dx = x.to(DEV)
    q_out, _ = bpc.qk_norm_rope(dx[:, :, :Hq].transpose(1, 2), dx[:, :, Hq:Hq + Hkv].transpose(1, 2), dev(pos), dev(table), wq=dev(wq), wk=dev(wk),
                                k_out=K[:, :, :T0])
    V[:, :, :T0] = dev(v)
    heads = pos[:, None]
    check_turn(q_out, turn(q, wq, table, heads.expand(B, Hq, T0), EPS, False))
    check_turn(K[:, :, :T0], turn(kk, wk, table, heads.expand(B, Hkv, T0), EPS, False))
    out = bpc.prefill_attention(q_out, K, V, N=T0)
    visible = torch.ones(T0, T0, dtype=torch.bool).tril().expand(B, T0, T0)
    check_attend(out, attend(q_out.cpu(), K[:, :, :T0].cpu(), V[:, :, :T0].cpu(), visible, visible, SM))
    P, codes, _ = bpc.build_hash(K, torch.randn(L, 128, generator=torch.Generator().manual_seed(4)).to(DEV), N=T0)
    # the same cache in pages
    per = Ncap // page
    blocks = torch.randperm(B * per, generator=torch.Generator().manual_seed(5)).view(B, per).to(torch.int32)
    Kp, Vp = (torch.full((B * per, Hkv, page, 128), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    zero = torch.zeros(B, dtype=torch.int32, device=DEV)
    bpc.append_kv_paged(dx[:, :, Hq:Hq + Hkv].transpose(1, 2), dx[:, :, Hq + Hkv:].transpose(1, 2), Kp, Vp, dev(blocks), zero, cos_sin=dev(table),
                        wk=dev(wk))
    for p in range(T0 // page):
        for b in range(B):
            assert torch.equal(Kp[blocks[b, p]], K[b, :, p * page:(p + 1) * page]) and torch.equal(Vp[blocks[b, p]], V[b, :, p * page:(p + 1) * page])
    # draft token by token with the sparse step, then verify all drafts with one dense pass
    n, drafts = T0, []
    for t in range(T):
        y = rand(10 + t, B, 1, Hq + 2 * Hkv, 128).to(DEV)
        at = torch.full((B, 1), n, dtype=torch.int32, device=DEV)
        qt, kt = bpc.qk_norm_rope(y[:, :, :Hq].transpose(1, 2), y[:, :, Hq:Hq + Hkv].transpose(1, 2), at, dev(table), wq=dev(wq), wk=dev(wk))
        vt = y[:, :, Hq + Hkv:].transpose(1, 2)
        bpc.append_kv(kt, vt.contiguous(), K, V, codes, P, n)
        bpc.append_kv_paged(y[:, :, Hq:Hq + Hkv].transpose(1, 2), vt, Kp, Vp, dev(blocks), at[:, 0].contiguous(), cos_sin=dev(table), wk=dev(wk))
        n += 1
        drafts.append(qt)
        sparse = bpc.decode_attention(qt[:, :, 0].contiguous(), K, V, codes, P, k, N=n)
        assert bool(sparse.isfinite().all())
        # all keys selected: the sparse step is dense attention
        full = bpc.decode_attention(qt[:, :, 0].contiguous(), K, V, codes, P, n, N=n)
        lens = torch.full((B,), n - 1, dtype=torch.int32, device=DEV)
        dense = bpc.tree_attention(qt, K, V, lens)
        assert float((dense[:, :, 0].float() - full).abs().max()) <= 2.0 ** -6 * float(full.abs().max())
    qd = torch.cat(drafts, 2)
    lens = torch.full((B,), T0, dtype=torch.int32, device=DEV)
    got = bpc.tree_attention(qd, K, V, lens)
    visible, dist = tree_view([T0] * B, None, T, n)
    check_attend(got, attend(qd.cpu(), K[:, :, :n].cpu(), V[:, :, :n].cpu(), visible, dist, SM))
    assert torch.equal(bpc.tree_attention(qd, Kp, Vp, lens, block_table=dev(blocks)), got)
    # a chain of drafts is the tail of a prefill
    check_attend(bpc.prefill_attention(qd, K, V, N=n), attend(qd.cpu(), K[:, :, :n].cpu(), V[:, :, :n].cpu(), visible, dist, SM))


def calls(seed=0):
    """One call of each operator on fixed buffers, with what it writes."""
    B, Hq, Hkv, T, N, page = 2, 8, 2, 6, 700, 32
    q, k, v = dev(rand(seed, B, Hq, T, 128)), dev(rand(seed + 1, B, Hkv, T, 128)), dev(rand(seed + 2, B, Hkv, T, 128))
    K, V = dev(rand(seed + 3, B, Hkv, N, 128)), dev(rand(seed + 4, B, Hkv, N, 128))
    Kp, Vp = (dev(rand(seed + s, 50, Hkv, page, 128)) for s in (5, 6))
    blocks = dev(torch.arange(2 * 22, dtype=torch.int32).view(2, 22))
    pos, table = dev(torch.arange(T, dtype=torch.int32).expand(B, T).contiguous()), dev(rope_table(800, 128))
    at, lens = dev(torch.tensor([5, 600], dtype=torch.int32)), dev(torch.tensor([5, 600], dtype=torch.int32))
    tree = dev(as_int64(tree_masks(seed, B, T)))
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    po, to, co = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)

    def run(stream=None):
        bpc.qk_norm_rope(q, k, pos, table, q_out=qo, k_out=ko, stream=stream)
        bpc.append_kv_paged(ko, v, Kp, Vp, blocks, at, stream=stream)
        bpc.prefill_attention(qo, K, V, out=po, softcap=20.0, stream=stream)
        bpc.tree_attention(qo, Kp, Vp, lens, tree, block_table=blocks, out=to, stream=stream)
        bpc.tree_attention(qo, K, V, lens, out=co, stream=stream)

    return run, (qo, ko, Kp, Vp, po, to, co), q


def test_captured_and_replayed():
    run, outs, q = calls()
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(4):
        q.copy_(dev(rand(100 + i, *q.shape)))
        for o in outs[4:]:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs[4:]:
            o.zero_()
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
        for o in outs_a[4:] + outs_b[4:]:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(sa):
            graphs[0].replay()
        with torch.cuda.stream(sb):
            graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs_a + outs_b))
    for _ in range(3):
        for o in outs_a[4:] + outs_b[4:]:
            o.zero_()
        torch.cuda.synchronize()
        run_a(stream=sa), run_b(stream=sb)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs_a + outs_b))


def test_what_is_allocated_belongs_to_the_stream():
    """Results and workspaces that a call allocates are not handed out again while its kernels run."""
    s = torch.cuda.Stream()
    q, K, V = dev(rand(1, 1, 8, 16, 128)), dev(rand(2, 1, 2, 9000, 128)), dev(rand(3, 1, 2, 9000, 128))
    want = bpc.prefill_attention(q, K, V)
    torch.cuda.synchronize()
    got = []
    for _ in range(8):
        got.append(bpc.prefill_attention(q, K, V, stream=s))
        torch.empty(1 << 22, dtype=torch.uint8, device=DEV).fill_(255)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_given_workspaces():
    q, K, V = dev(rand(1, 1, 8, 16, 128)), dev(rand(2, 1, 2, 9000, 128)), dev(rand(3, 1, 2, 9000, 128))
    need = bpc.prefill_workspace_bytes(1, 8, 2, 16, 9000)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)  # any contents
    want = bpc.prefill_attention(q, K, V)
    assert torch.equal(bpc.prefill_attention(q, K, V, workspace=ws), want)
    assert torch.equal(bpc.prefill_attention(q, K, V, workspace=ws), want)
    lens = dev(torch.tensor([8000], dtype=torch.int32))
    ws = torch.full((bpc.tree_workspace_bytes(1, 8, 2, 16, 9000),), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(bpc.tree_attention(q, K, V, lens, workspace=ws), bpc.tree_attention(q, K, V, lens))
    with pytest.raises(bpc.BPCError):
        bpc.prefill_attention(q, K, V, workspace=ws[:256])


def test_results_repeat():
    """No atomics: the same call gives the same bits."""
    q, K, V = dev(rand(1, 2, 8, 40, 128)), dev(rand(2, 2, 2, 5000, 128)), dev(rand(3, 2, 2, 5000, 128))
    lens = dev(torch.tensor([4960, 77], dtype=torch.int32))
    a, b = bpc.prefill_attention(q, K, V), bpc.tree_attention(q, K, V, lens)
    for _ in range(5):
        assert torch.equal(bpc.prefill_attention(q, K, V), a) and torch.equal(bpc.tree_attention(q, K, V, lens), b)


@pytest.mark.parametrize("kind", ["head", "row", "page"])
def test_offsets_past_32_bits(kind):
    """A cache whose heads, rows or pool's pages lie more than 4 GiB apart."""
    T, n = 3, 500
    q, k, v = rand(1, 1, 2, T, 128), rand(2, 1, 2, n, 128), rand(3, 1, 2, n, 128)
    visible, dist = tree_view([n - T], None, T, n)
    want = attend(q, k, v, visible, dist, SM)
    lens = dev(torch.tensor([n - T], dtype=torch.int32))
    if kind == "head":
        Ncap = (1 << 32) // 256 + 5000  # rows of one head: past 4 GiB of bytes
        store = torch.empty(2, Ncap, 128, dtype=torch.bfloat16, device=DEV)
        K = store[:, -n:].unsqueeze(0)
        K.copy_(dev(k))
        V = dev(v)
        check_attend(bpc.tree_attention(dev(q), K, V, lens), want)
        check_attend(bpc.prefill_attention(dev(q), K, V), want)
        return
    if kind == "row":
        store = torch.empty(n, 1 << 23, dtype=torch.bfloat16, device=DEV)
        K = store[:, :256].view(n, 2, 128).transpose(0, 1).unsqueeze(0)
        K.copy_(dev(k))
        V = dev(v)
        check_attend(bpc.tree_attention(dev(q), K, V, lens), want)
        check_attend(bpc.prefill_attention(dev(q), K, V), want)
        return
    page, per = 64, 8
    pool = torch.empty((1 << 32) // (2 * page * 256) + 3 * per, 2, page, 128, dtype=torch.bfloat16, device=DEV)
    blocks = torch.tensor([[pool.shape[0] - 1 - 2 * i if i % 2 else i for i in range(per)]], dtype=torch.int32)
    Vp = torch.empty_like(pool)
    zero = dev(torch.zeros(1, dtype=torch.int32))
    bpc.append_kv_paged(dev(k), dev(v), pool, Vp, dev(blocks), zero)
    far = int(blocks[0, 1])
    assert torch.equal(pool[far].cpu(), k[0, :, page:2 * page]) and torch.equal(Vp[far].cpu(), v[0, :, page:2 * page])
    check_attend(bpc.tree_attention(dev(q), pool, Vp, lens, block_table=dev(blocks), N=n), want)


@pytest.mark.parametrize("N,T,pos0", [(70000, 2, None), (40000, 5, 39000)])
def test_prefill_few_rows_many_keys(N, T, pos0):
    q, K, V = rand(1, 1, 2, T, 128), rand(2, 1, 1, N, 128), rand(3, 1, 1, N, 128)
    p0 = N - T if pos0 is None else pos0
    n = torch.arange(N)
    at = p0 + torch.arange(T)[:, None]
    got = bpc.prefill_attention(dev(q), dev(K), dev(V), pos0=pos0)
    check_attend(got, attend(q, K, V, (n <= at)[None], (at - n).abs()[None], SM))


def test_one_token_everywhere():
    """The smallest calls: one head, one token, one key."""
    q = dev(rand(1, 1, 1, 1, 128))
    v = dev(rand(2, 1, 1, 1, 128))
    assert torch.equal(bpc.prefill_attention(q, q, v), v)
    zero = dev(torch.zeros(1, dtype=torch.int32))
    assert torch.equal(bpc.tree_attention(q, q, v, zero), v)


def test_wrong_device_and_stream():
    q, K = dev(rand(1, 1, 1, 1, 128)), dev(rand(2, 1, 1, 5, 128))
    with pytest.raises(ValueError, match="GPU"):
        bpc.prefill_attention(q, K, K.cpu())
    with pytest.raises(ValueError, match="GPU"):
        bpc.tree_attention(q, K, K, torch.zeros(1, dtype=torch.int32))
