"""qk_norm_rope: results in the buffer of the inputs, coordinates outside the
rotation.  prefill_attention and tree_attention: strides that no element uses."""

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import rope_table
from test_gpu_attn import rand

pytestmark = pytest.mark.gpu
DEV = "cuda"


def dev(x):
    return None if x is None else x.to(DEV)


@pytest.mark.parametrize("inter", [False, True])
def test_fused_projection_in_place(inter):
    """Queries and keys of one buffer, each in its own place, or moved to that of the values and behind it."""
    B, T, Hq, Hkv = 2, 9, 8, 2
    x = rand(5, B, T, Hq + 2 * Hkv, 128)
    table, pos, w = rope_table(T, 128), torch.arange(T, dtype=torch.int32).expand(B, T), 1 + rand(6, 128)
    y = dev(x)
    q, k, v = y[:, :, :Hq].transpose(1, 2), y[:, :, Hq:Hq + Hkv].transpose(1, 2), y[:, :, Hq + Hkv:].transpose(1, 2)
    want_q, want_k = bpc.qk_norm_rope(q, k, dev(pos), dev(table), wq=dev(w), wk=dev(w), interleaved=inter)
    moved = v.clone()
    bpc.qk_norm_rope(q, k, dev(pos), dev(table), wq=dev(w), wk=dev(w), interleaved=inter, q_out=q, k_out=v)  # k_out: where v was
    assert torch.equal(q, want_q) and torch.equal(v, want_k)
    y = dev(x)
    q, k, v = y[:, :, :Hq].transpose(1, 2), y[:, :, Hq:Hq + Hkv].transpose(1, 2), y[:, :, Hq + Hkv:].transpose(1, 2)
    bpc.qk_norm_rope(q, k, dev(pos), dev(table), wq=dev(w), wk=dev(w), interleaved=inter, q_out=q, k_out=k)
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(v, moved)
    with pytest.raises(bpc.BPCError, match="overlaps"):
        bpc.qk_norm_rope(q, k, dev(pos), dev(table), q_out=q, k_out=q[:, :Hkv])
    assert torch.equal(q, want_q)


@pytest.mark.parametrize("R,inter", [(16, False), (64, False), (96, False), (64, True), (112, True)])
def test_coordinates_outside_the_rotation_are_their_own(R, inter):
    """No partner reaches them, by its value or its weight, and without weights they keep their bits."""
    B, H, T = 2, 5, 7
    q = rand(1, B, H, T, 128)
    q[..., ::9] = -0.0
    table, pos = rope_table(T, R), torch.arange(T, dtype=torch.int32).expand(B, T)
    plain = bpc.qk_norm_rope(dev(q), None, dev(pos), dev(table), interleaved=inter)[0].cpu()
    assert torch.equal(plain[..., R:].view(torch.int16), q[..., R:].contiguous().view(torch.int16))
    w = torch.ones(128, dtype=torch.bfloat16)
    w[R + 1], w[R + 6] = float("inf"), float("nan")
    q[..., R + 1] = 2.0
    for weights in (w, w.expand(H, 128).contiguous()):
        got = bpc.qk_norm_rope(dev(q), None, dev(pos), dev(table), wq=dev(weights), interleaved=inter)[0].cpu()
        odd = torch.zeros(128, dtype=torch.bool)
        odd[R + 1], odd[R + 6] = True, True
        assert bool((got[..., R + 1] == float("inf")).all()) and bool(got[..., R + 6].isnan().all())
        assert bool(got[..., ~odd].isfinite().all())


def test_strides_of_single_extents_do_not_matter():
    """A cache of one sequence, one head, one key: whatever stride its view has there."""
    N, T = 40, 3
    q, k, v = rand(1, 1, 4, T, 128), rand(2, 1, 1, N, 128), rand(3, 1, 1, N, 128)
    lens = torch.tensor([N - T], dtype=torch.int32)
    K, V = (dev(x).as_strided((1, 1, N, 128), (7, 3, 128, 1)) for x in (k, v))
    assert torch.equal(bpc.prefill_attention(dev(q), K, V), bpc.prefill_attention(dev(q), dev(k), dev(v)))
    assert torch.equal(bpc.tree_attention(dev(q), K, V, dev(lens)), bpc.tree_attention(dev(q), dev(k), dev(v), dev(lens)))
    K, V = (dev(x)[:, :, :1].as_strided((1, 1, 1, 128), (7, 3, 5, 1)) for x in (k, v))
    assert torch.equal(bpc.prefill_attention(dev(q), K, V, pos0=0), bpc.prefill_attention(dev(q), dev(k), dev(v), N=1, pos0=0))


@pytest.mark.parametrize("R,inter", [(0, False), (128, False), (64, False), (96, True)])
@pytest.mark.parametrize("weights", ["none", "one", "each"])
def test_rows_past_the_caches(R, inter, weights):
    """More rows than the last-level cache holds, against the same rows in parts that it does hold."""
    T, Hq, Hkv = 9001, 128, 5
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k = (torch.randn(1, H, T, 128, generator=g, device=DEV).to(torch.bfloat16) for H in (Hq, Hkv))
    table, pos = (dev(rope_table(T, R)), torch.arange(T, dtype=torch.int32, device=DEV)[None]) if R else (None, None)
    w = {"none": {}, "one": dict(wq=dev(1 + rand(2, 128)), wk=dev(1 + rand(3, 128))),
         "each": dict(wq=dev(1 + rand(2, Hq, 128)), wk=dev(1 + rand(3, Hkv, 128)))}[weights]
    oq, ok = bpc.qk_norm_rope(q, k, pos, table, interleaved=inter, **w)
    for a in range(0, T, 2500):
        pq, pk = bpc.qk_norm_rope(q[:, :, a:a + 2500], k[:, :, a:a + 2500], pos[:, a:a + 2500] if R else None, table, interleaved=inter, **w)
        assert torch.equal(oq[:, :, a:a + 2500], pq) and torch.equal(ok[:, :, a:a + 2500], pk)


def test_pools_in_one_buffer():
    """Keys and values as the two halves of each page, and of each head's page."""
    B, Hkv, T, page, pages = 2, 2, 5, 16, 7
    k, v, table, pos = rand(1, B, Hkv, T, 128), rand(2, B, Hkv, T, 128), torch.tensor([[3, 0], [6, 2]], dtype=torch.int32), torch.tensor([13, 0], dtype=torch.int32)
    K, V = (torch.zeros(pages, Hkv, page, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    bpc.append_kv_paged(dev(k), dev(v), K, V, dev(table), dev(pos))
    assert torch.equal(K[3, :, 13:].cpu(), k[0, :, :3]) and torch.equal(V[0, :, :2].cpu(), v[0, :, 3:]) and torch.equal(K[6, :, :5].cpu(), k[1])
    by_page, by_head = torch.zeros(pages, 2, Hkv, page, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(pages, Hkv, 2, page, 128, dtype=torch.bfloat16, device=DEV)
    for a, b in ((by_page[:, 0], by_page[:, 1]), (by_head[:, :, 1], by_head[:, :, 0])):
        bpc.append_kv_paged(dev(k), dev(v), a, b, dev(table), dev(pos))
        assert torch.equal(a, K) and torch.equal(b, V)
    with pytest.raises(bpc.BPCError, match="overlaps"):
        bpc.append_kv_paged(dev(k), dev(v), K, K, dev(table), dev(pos))
