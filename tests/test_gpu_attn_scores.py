"""prefill_attention and tree_attention where fp32 needs care: scores far from
zero, distances that are large against what they differ in, and weights that
leave fp32's range.

The bounds are those of attn_plain: where scores are large the inputs have one or
two coordinates that count, so that products are exact, and a bias enters by its
difference from the nearest visible key's, below 2^9 here.
"""

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import attend, check_attend, ranges_visible, tree_view
from test_gpu_attn import rand, slopes_of

pytestmark = pytest.mark.gpu
DEV = "cuda"


def dev(x):
    return None if x is None else x.to(DEV)


def line(values, *lead):
    """Rows [*lead, len(values), 128] whose first coordinate alone is not zero."""
    x = torch.zeros(*lead, len(values), 128, dtype=torch.bfloat16)
    x[..., 0] = torch.tensor(values, dtype=torch.bfloat16)
    return x


SCALES = [2.0 ** -40, 1.0, 100.0, 2.0 ** 10, 2.0 ** 20, 2.0 ** 27, 2.0 ** 30, 2.0 ** 40]


@pytest.mark.parametrize("sm", SCALES)
@pytest.mark.parametrize("T,N", [(64, 64), (3, 5000)])
@pytest.mark.parametrize("sign", [1, -1])
def test_uncapped_scales(sm, T, N, sign):
    """Every scale that is taken: weights from all equal to one-hot, the largest score of either sign."""
    q = line([sign * (1 + t % 64) for t in range(T)], 1, 2)
    K, V = line([1 + (7 * n) % 5 for n in range(N)], 1, 1), rand(3, 1, 1, N, 128)
    visible = torch.ones(T, N, dtype=torch.bool).tril(N - T)[None]
    want = attend(q, K, V, visible, torch.zeros(1, T, N), sm)
    check_attend(bpc.prefill_attention(dev(q), dev(K), dev(V), sm), want)
    # the cache from the drafts on counts as hidden, and holds anything
    lens, more = torch.tensor([N - T], dtype=torch.int32), torch.full((1, 1, 9, 128), float("nan"), dtype=torch.bfloat16)
    got = bpc.tree_attention(dev(q), dev(torch.cat([K, more], 2)), dev(torch.cat([V, more], 2)), dev(lens), sm_scale=sm)
    check_attend(got, want)


@pytest.mark.parametrize("sm", SCALES)
@pytest.mark.parametrize("score", [3.0, -5.0, 2.0 ** 60])
def test_a_single_visible_key(sm, score):
    """Its weight is one, whatever its score."""
    q, K, V = line([score], 1, 1), line([1.0], 1, 1), rand(3, 1, 1, 1, 128)
    assert torch.equal(bpc.prefill_attention(dev(q), dev(K), dev(V), sm).cpu(), V)
    zero = torch.zeros(1, dtype=torch.int32)
    assert torch.equal(bpc.tree_attention(dev(q), dev(K), dev(V), dev(zero), sm_scale=sm).cpu(), V)


@pytest.mark.parametrize("base", [0.0, 2.0 ** 14, -2.0 ** 14, 2.0 ** 22])
def test_scores_that_differ_little_far_from_zero(base):
    """The weights follow the differences of exact scores, however far from zero these lie."""
    T, N = 40, 300
    q, K, V = torch.zeros(1, 2, T, 128, dtype=torch.bfloat16), torch.zeros(1, 1, N, 128, dtype=torch.bfloat16), rand(3, 1, 1, N, 128)
    q[..., 0], q[..., 1] = 1, 1
    K[..., 0], K[..., 1] = base, torch.arange(N) % 7 if base < 2 ** 20 else 0
    visible = torch.ones(T, N, dtype=torch.bool).tril(N - T)[None]
    check_attend(bpc.prefill_attention(dev(q), dev(K), dev(V), 1.0), attend(q, K, V, visible, torch.zeros(1, T, N), 1.0))


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("pos0", [300, 2 ** 20, 2 ** 24 - 7, 2 ** 30 - 40, 2 ** 30])
def test_bias_of_positions_past_all_keys(pos0, cap):
    """Every key lies far back: only the differences of the distances count."""
    B, Hq, Hkv, T, N = 1, 4, 2, 40, 300
    q, K, V, slopes = rand(1, B, Hq, T, 128), rand(2, B, Hkv, N, 128), rand(3, B, Hkv, N, 128), slopes_of(Hq)
    visible = torch.ones(B, T, N, dtype=torch.bool)
    dist = (pos0 + torch.arange(T)[:, None] - torch.arange(N))[None]
    got = bpc.prefill_attention(dev(q), dev(K), dev(V), pos0=pos0, softcap=cap, slopes=dev(slopes))
    check_attend(got, attend(q, K, V, visible, dist, 128 ** -0.5, cap, slopes))


@pytest.mark.parametrize("N,pos0,begin,end", [(2 ** 20, 2 ** 20 - 9, 50, 170), (2 ** 20, 0, 2 ** 20 - 130, 2 ** 20 - 10), (2 ** 20, 2 ** 19, 2 ** 19 - 60, 2 ** 19 + 40)])
def test_bias_of_a_far_window(N, pos0, begin, end):
    """A row's window behind, ahead of and around its position, a million keys long the cache."""
    Hq, T = 4, 9
    first, last = torch.full((1, T), begin, dtype=torch.int32), (end + torch.arange(T, dtype=torch.int32))[None]
    a, b = begin, end + T  # the keys that any row sees; the others hold anything
    q, k, v, slopes = rand(1, 1, Hq, T, 128), rand(2, 1, 1, b - a, 128), rand(3, 1, 1, b - a, 128), slopes_of(Hq)
    K, V = (torch.full((1, 1, N, 128), float("nan"), dtype=torch.bfloat16) for _ in range(2))
    K[:, :, a:b], V[:, :, a:b] = k, v
    dist = (pos0 + torch.arange(T)[:, None] - torch.arange(a, b)).abs()[None]
    want = attend(q, k, v, ranges_visible(first - a, last - a, b - a), dist, 128 ** -0.5, 0.0, slopes)
    got = bpc.prefill_attention(dev(q), dev(K), dev(V), pos0=pos0, slopes=dev(slopes), key_begin=dev(first), key_end=dev(last))
    check_attend(got, want)


@pytest.mark.parametrize("tree", [False, True])
def test_a_visible_nan_counts_in_a_piece_of_no_weight(tree):
    """A value that is not a number, at a key whose weight fp32 rounds to zero beside those of the axis' other pieces."""
    T, N = 2, 9000
    q, K, V = line([1.0] * T, 1, 2), line([0.0] * N, 1, 1), rand(3, 1, 1, N, 128)
    K[0, 0, N - 5, 0], V[0, 0, 5, 7] = 200.0, float("nan")
    if tree:
        assert bpc.tree_workspace_bytes(1, 2, 1, T, N) > 0  # the axis is in pieces
        visible, dist = tree_view([N - T], None, T, N)
        got = bpc.tree_attention(dev(q), dev(K), dev(V), dev(torch.tensor([N - T], dtype=torch.int32)), sm_scale=1.0)
    else:
        assert bpc.prefill_workspace_bytes(1, 2, 1, T, N) > 0
        visible, dist = ranges_visible(torch.zeros(1, T), torch.full((1, T), N), N), torch.zeros(1, T, N)
        got = bpc.prefill_attention(dev(q), dev(K), dev(V), 1.0, key_end=dev(torch.full((1, T), N, dtype=torch.int32)))
    want = attend(q, K, V, visible, dist, 1.0)
    assert bool(want[0][..., 7].isnan().all())
    check_attend(got, want)
