"""What the C entries of the rows and the attention refuse beyond the ends of
their arguments' ranges, on the CPU (fake pointers; every call fails a check)."""

import ctypes

import pytest

from test_rows_and_attn_refusals import APPEND, EINVAL, EUNSUP, OK, PREFILL, ROPE, bpc, call, lib, pytestmark  # noqa: F401


@pytest.mark.parametrize("T", [(1 << 25) - 1, 1 << 25, 1 << 28])
def test_more_tokens_than_a_launch_has_wavefronts(lib, T):
    for name, spec in (("bpc_qk_norm_rope", ROPE), ("bpc_append_kv_paged", APPEND)):
        assert call(lib, name, spec, dict(B=2, T=T)) == EUNSUP
        assert b"tokens" in lib.bpc_last_error()


@pytest.mark.parametrize("kw", [dict(B=8, Hq=2, Hkv=2, T=1 << 28), dict(B=64, Hq=8, Hkv=2, T=1 << 26), dict(B=1 << 12, Hq=1, Hkv=1, T=1 << 20, N=16)])
def test_more_rows_than_a_launch_has_threads(lib, kw):
    assert call(lib, "bpc_prefill_attention", PREFILL, kw) == EUNSUP
    assert b"workgroups" in lib.bpc_last_error()


def test_attention_cut(bpc, lib):
    """The timed cases' cuts, and what the entry refuses."""
    assert bpc.attention_cut(2, 32, 8, 8192, 8192) == (8, 1, False)
    assert bpc.attention_cut(1, 8, 2, 257, 257) == (1, 1, False)
    assert bpc.attention_cut(8, 32, 8, 24, 32768, tree=True)[0] == 4
    row_blocks, pieces, streamed = bpc.attention_cut(16, 32, 8, 8, 131072, tree=True)
    assert row_blocks == 1 and streamed
    # in pieces where there is a workspace, and only there
    for sizes in ((1, 32, 8, 64, 65536), (2, 32, 8, 8192, 8192), (1, 8, 2, 16, 9000), (1, 8, 2, 257, 257)):
        assert (bpc.attention_cut(*sizes)[1] > 1) == (bpc.prefill_workspace_bytes(*sizes) > 0)
    out = [ctypes.byref(ctypes.c_int()) for _ in range(3)]
    cut = lib.bpc_attention_cut
    assert cut(1, 8, 2, 65, 4096, 128, 0, *out) == OK and cut(1, 8, 2, 65, 4096, 128, 1, *out) == EUNSUP
    assert cut(1, 8, 2, 9, 8, 128, 0, *out) == OK and cut(1, 8, 2, 9, 8, 128, 1, *out) == EINVAL
    assert cut(1, 9, 2, 9, 80, 128, 0, *out) == EINVAL and cut(1, 8, 2, 9, 80, 64, 0, *out) == EUNSUP
    assert cut(1, 8, 2, 9, 80, 128, 0, None, *out[1:]) == EINVAL
