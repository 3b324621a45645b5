"""Sums over nothing: gradients of sdp_block_norm_backward without tokens."""
import pytest

from test_gpu_layer_norm import BF16, F32, ctx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h", [8, 1003, 9001])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_no_tokens_leave_zeros_whatever_the_weights_hold(ctx, h, dtype, sigmoid):  # noqa: F811
    """Neither the weight nor the gate is looked at."""
    from paper_2609_34162_amd import ops
    none = torch.empty((0, h), dtype=dtype, device="cuda")
    gate, w = torch.randn(h, device="cuda").to(dtype), torch.randn(h, device="cuda")
    gate[0], gate[3], w[1], w[2], w[3] = float("nan"), float("inf"), float("inf"), float("nan"), float("-inf")
    dgate, dpost, dpre = torch.full_like(gate, 7.0), torch.full_like(w, 7.0), torch.full_like(w, 7.0)
    ops.sdp_block_norm_backward(ctx, none, none, none, none, none.clone(), none.clone(), gate=gate, dgate=dgate,
                                gate_sigmoid=sigmoid, post_norm=True, post_weight=w, dpost_weight=dpost, pre_weight=w,
                                dpre_weight=dpre)
    for t in (dgate, dpost, dpre):
        assert (t == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("stride", [1, 3])
@pytest.mark.parametrize("t", [0, 1, 7, 1000])
def test_no_channels_leave_a_tokens_gate_zeros(ctx, t, stride, dtype):  # noqa: F811
    from paper_2609_34162_amd import ops
    none = torch.empty((t, 0), dtype=dtype, device="cuda")
    gate, room = torch.randn((t, 1), device="cuda").to(dtype), torch.full((t, stride), 7.0, dtype=dtype, device="cuda")
    ops.sdp_block_norm_backward(ctx, none, none, none, none, none.clone(), none.clone(), gate=gate, dgate=room[:, :1],
                                gate_sigmoid=True, post_norm=True)
    assert (room[:, 0] == 0).all() and (room[:, 1:] == 7.0).all()
