"""sdp_route on the GPU where the choice of groups hangs on little: biases of both signs
that cancel in a group's worth."""
import pytest

from test_gpu_layer_route import BF16, F32, check, ctx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def opposite(e, groups, size, seed, tokens=300):
    """Logits and a bias: of each group one expert has about +size, one about -size, the others less; the groups'
    worths differ by a few millionths of size."""
    gen = torch.Generator().manual_seed(seed)
    each = e // groups
    bias = torch.full((groups, each), -2.0 * size)
    for g in range(groups):
        at = torch.randperm(each, generator=gen)
        bias[g, at[0]], bias[g, at[1]] = size, 0.4 - size
    z = 0.3 + 1e-6 * size * torch.randn((tokens, e), generator=gen)
    return z.cuda(), bias.view(-1).cuda()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("size", [2.0, 7.9, 16.0, 100.0, 5000.0])
@pytest.mark.parametrize("e,groups,top_groups,top", [(64, 8, 3, 6), (256, 8, 4, 8), (16, 8, 2, 4), (24, 2, 1, 2)])
def test_biases_of_both_signs(ctx, e, groups, top_groups, top, size, sigmoid):  # noqa: F811
    z, bias = opposite(e, groups, size, e)
    check(ctx, z, top, bias, sigmoid, groups, top_groups, 2, renormalize=True)
    # the bias in another place of each lane
    check(ctx, z, top, bias.flip(0), sigmoid, groups, top_groups, 2, renormalize=True)
    check(ctx, z, top, -bias, sigmoid, groups, top_groups, 2)
