"""What the C entries of the rows and the attention refuse beyond the ends of
their arguments' ranges, on the CPU (fake pointers; every call fails a check)."""

import pytest

from test_rows_and_attn_refusals import APPEND, EUNSUP, PREFILL, ROPE, call, lib, pytestmark  # noqa: F401


@pytest.mark.parametrize("T", [(1 << 25) - 1, 1 << 25, 1 << 28])
def test_more_tokens_than_a_launch_has_wavefronts(lib, T):
    for name, spec in (("bpc_qk_norm_rope", ROPE), ("bpc_append_kv_paged", APPEND)):
        assert call(lib, name, spec, dict(B=2, T=T)) == EUNSUP
        assert b"tokens" in lib.bpc_last_error()


@pytest.mark.parametrize("kw", [dict(B=8, Hq=2, Hkv=2, T=1 << 28), dict(B=64, Hq=8, Hkv=2, T=1 << 26), dict(B=1 << 12, Hq=1, Hkv=1, T=1 << 20, N=16)])
def test_more_rows_than_a_launch_has_threads(lib, kw):
    assert call(lib, "bpc_prefill_attention", PREFILL, kw) == EUNSUP
    assert b"workgroups" in lib.bpc_last_error()
