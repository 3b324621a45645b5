"""sdp_route on the GPU with NaN among the logits or biases: larger than everything, the
lowest index first, and NaN in the weights and gradients that depend on it."""
import itertools

import pytest

from test_gpu_layer_route import BF16, F32, check, ctx, logits  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sigmoid,renormalize", list(itertools.product([False, True], [False, True])))
@pytest.mark.parametrize("e,top", [(8, 2), (32, 4), (60, 4), (128, 8), (256, 1), (512, 10), (2000, 8)])
def test_nan_logits_come_first(ctx, e, top, sigmoid, renormalize, dtype):  # noqa: F811
    z = logits(12, e, dtype, e)
    z[2, e // 3] = NAN
    z[4, 0], z[4, e - 1] = NAN, -NAN
    z[5, ::2] = NAN
    z[6] = NAN
    z[7], z[7, 3] = float("-inf"), NAN
    index, w, _, _ = check(ctx, z, top, None, sigmoid, renormalize=renormalize)
    assert int(index[2, 0]) == e // 3 and torch.isnan(w[2, 0])


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("e,groups", [(32, 1), (64, 8), (256, 4), (2000, 8)])
def test_nan_scores_with_a_bias_and_groups(ctx, e, groups, sigmoid):  # noqa: F811
    z = logits(6, e, F32, e)
    z[2, 9], z[4, e - 3] = NAN, NAN
    bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(e))
    for best in (1, 2):
        check(ctx, z, 4, bias.cuda(), sigmoid, groups, max(1, groups // 2), best)
        bad = bias.clone()
        bad[e // 2], bad[11] = NAN, float("-inf")
        check(ctx, z, 4, bad.cuda(), sigmoid, groups, max(1, groups // 2), best)
