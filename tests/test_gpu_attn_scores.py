"""prefill_attention and tree_attention where fp32 needs care: scores far from
zero.

The bounds are those of attn_plain: the inputs have one or two coordinates that
count, so that products are exact.
"""

import pytest
import torch

import paper_2608_04405_amd as bpc
from attn_plain import attend, check_attend
from test_gpu_attn import rand

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
