"""sdp_route on the GPU where logits are zeros of either sign: -0 counts as 0, and equals
go to the lowest index."""
import pytest

import layer_ref as ref  # noqa: F401
from test_gpu_layer_route import BF16, F32, I64, check, ctx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def zeros_of_both_signs(e, seed):
    """Rows of -0, of both zeros, of zeros among negative, positive and any logits, and masked ones."""
    gen = torch.Generator().manual_seed(seed)
    z = torch.randn((48, e), generator=gen)
    some = torch.rand((48, e), generator=gen) < 0.5
    z[0] = -0.0
    z[1] = 0.0
    z[2, ::2], z[2, 1::2] = -0.0, 0.0
    z[3, ::2], z[3, 1::2] = 0.0, -0.0
    z[4] = torch.where(some[4], -0.0, -z[4].abs())
    z[5] = torch.where(some[5], -0.0, z[5].abs())
    z[6] = torch.where(some[6], -0.0, float("-inf"))
    z[7], z[7, e - 1] = -1.0, -0.0
    z[8:24] = z[8:24] * some[8:24]           # what a mask of zeros leaves of random logits
    z[24:32] = -z[24:32].abs() * some[24:32]
    z[32:40] = -z[32:40].abs() * 0.0         # tokens that a mask takes out
    return z


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("e,top", [(1, 1), (2, 2), (4, 2), (8, 2), (8, 8), (16, 4), (31, 6), (60, 4), (63, 8), (64, 8),
                                   (65, 8), (100, 6), (128, 8), (250, 8), (256, 8), (256, 1), (384, 8), (512, 10),
                                   (500, 9), (1000, 64), (2048, 8)])
def test_zeros_of_both_signs(ctx, e, top, dtype):  # noqa: F811
    z = zeros_of_both_signs(e, e).to(dtype).cuda()
    for sigmoid in (False, True):
        check(ctx, z, top, None, sigmoid, renormalize=sigmoid)
        check(ctx, z, top, None, sigmoid, renormalize=not sigmoid, itype=I64, wtype=BF16)


@pytest.mark.parametrize("e", [8, 60, 128, 512])
def test_masked_tokens_have_experts_of_the_layer(ctx, e):  # noqa: F811
    """Logits times a mask of 0, to the sorted rows and to the gradient: every entry has its expert."""
    from paper_2609_34162_amd import ops
    t, top = 70, 4
    z = (torch.randn((t, e), generator=torch.Generator().manual_seed(e)) * 0.0).to(BF16).cuda()
    assert torch.signbit(z).any() and (z == 0).all()
    index, w = torch.full((t, top), 77, dtype=torch.int32, device="cuda"), torch.empty((t, top), device="cuda")
    ops.sdp_route(ctx, z, index, w)
    assert torch.equal(index.cpu(), torch.arange(top, dtype=torch.int32).expand(t, top))
    ends, place = torch.empty(e, dtype=torch.int32, device="cuda"), torch.empty_like(index)
    ops.sdp_expert_order(ctx, index, ends, place)
    assert int(ends[-1]) == t * top and int(place.min()) == 0
    dz = torch.empty_like(z)
    ops.sdp_route_backward(ctx, z, index, torch.ones_like(w), dz)
    assert not torch.isnan(dz).any()
