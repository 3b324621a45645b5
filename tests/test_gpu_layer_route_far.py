"""sdp_route and its backward on the GPU where a token's chosen scores lie far apart, or far
below the row's best: renormalised weights are ratios that FP32 holds, whatever the scores are."""
import pytest

from test_gpu_layer_route import BF16, F32, check, ctx, logits  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("e,top,groups", [(8, 4, 1), (60, 6, 1), (256, 8, 8), (300, 64, 1), (1100, 8, 10), (2048, 16, 1)])
def test_ratios_of_scores_far_apart(ctx, e, top, groups, dtype, sigmoid):  # noqa: F811
    gen = torch.Generator().manual_seed(e)
    bias = (16.0 * torch.randn(e, generator=gen)).cuda()  # which decides, far from the scores
    for sigma in (10.0, 30.0, 60.0):
        z = logits(25, e, dtype, e, sigma=sigma)
        check(ctx, z, top, bias, sigmoid, groups, max(1, groups // 2), 2, renormalize=True)


@pytest.mark.parametrize("e", [8, 60, 300, 1100])
def test_ratios_of_small_sigmoids(ctx, e):  # noqa: F811
    """All chosen scores between 1 and what FP32 does not hold."""
    gen = torch.Generator().manual_seed(e)
    bias = torch.zeros(e)
    bias[:4] = 5.0
    for best in (-2.0, -10.0, -17.0, -19.0, -30.0, -60.0, -68.0, -70.0, -85.0, -100.0):
        z = torch.randn((30, e), generator=gen)
        z[:, :4] = best - 25.0 * torch.rand((30, 4), generator=gen)
        z[:, 0] = best
        if e == 60:
            z[:, 3] = best - 72.0 * torch.rand(30, generator=gen)  # down to ratios that FP32 ends at
        check(ctx, z.cuda(), 4, bias.cuda(), True, renormalize=True)
