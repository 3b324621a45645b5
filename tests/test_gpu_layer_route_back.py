"""sdp_route_backward on the GPU with indexes of 64 bits whose lower half names an expert."""
import itertools

import pytest

import layer_ref as ref
from test_gpu_layer_route import F32, ctx, logits  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e", [8, 60, 256, 2000])
@pytest.mark.parametrize("sigmoid,renormalize", list(itertools.product([False, True], [False, True])))
def test_far_negative_indexes_are_places_left_over(ctx, e, sigmoid, renormalize):  # noqa: F811
    from paper_2609_34162_amd import ops
    z = logits(3, e, F32, e)
    far = -(1 << 32)
    index = torch.tensor([[0, far + 5, 3], [far + 1, 2, -(1 << 63)], [far, far + 7, far + 4]]).cuda()
    dw = torch.randn((3, 3), device="cuda")
    dw[0, 0], dw[1, 1] = float("nan"), float("inf")
    dz = torch.full_like(z, 7.0)
    ops.sdp_route_backward(ctx, z, index, dw, dz, sigmoid=sigmoid, renormalize=renormalize)
    ref.check(dz, *ref.route_back(z, index, dw, sigmoid, renormalize, 1.0, F32), "dlogits")
