"""The binding's sizes of chunk_attention calls whose windows are longer than any cache, on the CPU."""

import pytest

from test_rows_and_attn_refusals import bpc, pytestmark  # noqa: F401


@pytest.mark.parametrize("far", [2 ** 30 + 1, 2 ** 31, 2 ** 31 + 5, 2 ** 32 + 1, 2 ** 40])
def test_windows_longer_than_any_cache(bpc, far):
    """The call takes them as 2^30; its workspace and its cut are of the same window."""
    sizes = (1, 32, 8, 1, 16384)
    assert bpc.chunk_workspace_bytes(*sizes, far, 4) == bpc.chunk_workspace_bytes(*sizes, 1 << 30, 4) > bpc.chunk_workspace_bytes(*sizes, 1024, 4)
    assert bpc.chunk_workspace_bytes(*sizes, 1024, far) == bpc.chunk_workspace_bytes(*sizes, 1024, 1 << 30)
    assert bpc.chunk_cut(*sizes, far, far) == bpc.chunk_cut(*sizes, 1 << 30, 1 << 30)


def test_negative_ones(bpc):
    for window, sinks in ((-1, 0), (0, -1), (-2 ** 33, 0), (5, -2 ** 40)):
        assert bpc.chunk_workspace_bytes(1, 32, 8, 1, 16384, window, sinks) == 0
        with pytest.raises((ValueError, RuntimeError)):
            bpc.chunk_cut(1, 32, 8, 1, 16384, window, sinks)
