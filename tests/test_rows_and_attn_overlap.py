"""Rows that a call writes lie apart, on the CPU: what the binding and the C
entries refuse (fake pointers; every call fails a check)."""

import pytest
import torch

from test_rows_and_attn_refusals import (APPEND, EINVAL, FAKE, PREFILL, ROPE, TREE, append, bpc, call, expect, lib, prefill,  # noqa: F401
                                         pytestmark, rope, tree, z)

# strides of a [2, 8, 5, 128] tensor whose rows meet, though each is 128 or more
MEET = [(128, 128, 128), (640, 640, 128), (5120, 640, 640), (5120, 128, 512), (5112, 640, 128), (4480, 640, 128), (128, 1024, 1024)]


def rows(strides):
    return torch.zeros(40 * 1024, dtype=torch.bfloat16).as_strided((2, 8, 5, 128), strides + (1,))


def nearest(strides):
    """The smallest distance of two of its rows."""
    at = sorted(i * strides[0] + j * strides[1] + k * strides[2] for i in range(2) for j in range(8) for k in range(5))
    return min(b - a for a, b in zip(at, at[1:]))


@pytest.mark.parametrize("strides", MEET)
def test_binding_refuses_rows_that_meet(bpc, strides):
    x = rows(strides)
    assert nearest(strides) < 128
    for call_it in (lambda: rope(bpc, q_out=x), lambda: prefill(bpc, out=x), lambda: tree(bpc, out=x)):
        expect(call_it, "overlap")
    expect(lambda: append(bpc, K=torch.zeros(99999, dtype=torch.bfloat16).as_strided((7, 2, 16, 128), (2176, 2048, 128, 1))), "overlap")


@pytest.mark.parametrize("strides", [(5120, 640, 128), (5120, 128, 1024), (640, 1280, 128), (128, 1280, 256), (8192, 1024, 136), (256, 512, 4096)])
def test_binding_takes_rows_in_any_order(bpc, strides):
    x = rows(strides)
    assert nearest(strides) >= 128
    for call_it in (lambda: rope(bpc, q_out=x), lambda: prefill(bpc, out=x), lambda: tree(bpc, out=x)):
        expect(call_it, "GPU")


@pytest.mark.parametrize("b,h,t", MEET)
def test_entries_refuse_rows_that_meet(lib, b, h, t):
    for name, spec, out in (("bpc_qk_norm_rope", ROPE, "qo"), ("bpc_prefill_attention", PREFILL, "o"), ("bpc_tree_attention", TREE, "o")):
        assert call(lib, name, spec, {out + "_b": b, out + "_h": h, out + "_t": t}) == EINVAL
        assert b"overlap" in lib.bpc_last_error()


@pytest.mark.parametrize("kw", [dict(K_b=2176, K_h=2048), dict(V_b=2176, V_h=2048), dict(K_b=1 << 62, K_h=2048)])
def test_append_refuses_pools_whose_rows_meet(lib, kw):
    good = dict(K_b=4096, K_h=2048, V_b=4096, V_h=2048)
    assert call(lib, "bpc_append_kv_paged", APPEND, {**good, **kw}) == EINVAL
    assert b"overlap" in lib.bpc_last_error()


# q and k of a fused projection [2, 5, 12, 128] (8 heads of q, 2 of k, 2 of v), in elements from its start
FUSED = dict(q_b=7680, q_h=128, q_t=1536, qo_b=7680, qo_h=128, qo_t=1536, k_b=7680, k_h=128, k_t=1536, ko_b=7680, ko_h=128, ko_t=1536)
FAR = 1 << 24


def fused(q, qo, k, ko, **kw):
    return {**FUSED, **{n: FAKE + 2 * at for n, at in (("q", q), ("qo", qo), ("k", k), ("ko", ko))}, **kw}


@pytest.mark.parametrize("kw,word", [
    (fused(0, 128, 1024, FAR), b"q_out overlaps q"),  # a head on
    (fused(0, 1536, 1024, FAR), b"q_out overlaps q"),  # a token on
    (fused(0, 7680 * 2 - 512, 1024, FAR), b"q_out overlaps k"),  # from the last token's k on
    (fused(0, 8, 1024, FAR), b"q_out overlaps q"),
    (fused(0, 0, 1024, 1024 - 256), b"k_out overlaps q"),  # the last heads of q
    (fused(0, 128, 1024 + FAR, 2 * FAR), b"q_out overlaps q"),
    (fused(0, FAR, 1024, FAR + 1024 - 128), b"q_out overlaps k_out"),
    (fused(0, FAR, 1024, 1024 + 128), b"k_out overlaps k"),
    (fused(0, 1024, FAR, 2 * FAR), b"q_out overlaps q"),  # eight heads from the k of a token on reach its next token's q
    (fused(0, FAR, 2 * FAR, 0), b"k_out overlaps q"),
])
def test_results_on_their_inputs(lib, kw, word):
    """Neither in place nor apart: another wavefront may not have read what a row replaces."""
    assert call(lib, "bpc_qk_norm_rope", ROPE, kw) == EINVAL
    assert word in lib.bpc_last_error()


@pytest.mark.parametrize("away", [0, 8, 2048, 8192, 6 * 8192 - 2048])
def test_append_refuses_pools_that_share_rows(lib, away):
    """K and V as views of a pool [7, 2, 2, 16, 128] whose pages meet."""
    pool = dict(K_b=8192, K_h=2048, V_b=8192, V_h=2048)
    assert call(lib, "bpc_append_kv_paged", APPEND, dict(pool, K=FAKE, V=FAKE + 2 * away)) == EINVAL
    assert b"K overlaps V" in lib.bpc_last_error()
