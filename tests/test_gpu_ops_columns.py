"""The training operators on blocks of columns of one buffer, inputs and outputs side by
side: the bits of the call on tensors of their own, and nothing else written."""
import pytest

import gpu_util

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    sdp = gpu_util.need_gpu()
    from paper_2609_34162_amd import ops
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield sdp, ops, c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


@pytest.mark.parametrize("n_in,n_out,gap", [(64, 96, 0), (96, 64, 8), (33, 70, 5)])
def test_grouped(lib, n_in, n_out, gap):
    sdp, ops, ctx = lib
    rows = 300
    buf = torch.randn((rows, n_in + 2 * (gap + n_out) + gap + n_in), device="cuda").to(BF16)
    at = [0, n_in + gap, n_in + gap + n_out + gap, n_in + 2 * (gap + n_out) + gap]
    x, y, dy, dx = (buf[:, a:a + n] for a, n in zip(at, (n_in, n_out, n_out, n_in)))
    w = torch.randn((3, n_out, n_in), device="cuda").to(BF16)
    ends = torch.tensor([100, 130, 290], device="cuda")
    own = x.clone(), torch.empty_like(y.contiguous()), dy.clone(), torch.empty_like(x.contiguous())
    ops.sdp_grouped_matmul(ctx, own[0], w, ends, own[1])
    ops.sdp_grouped_matmul_backward(ctx, None, w, ends, own[2], own[3], None)
    ops.sdp_grouped_matmul(ctx, x, w, ends, y)
    ops.sdp_grouped_matmul_backward(ctx, None, w, ends, dy, dx, None)
    for got, want in zip((x, y, dy, dx), own):
        assert torch.equal(got, want)
    with pytest.raises(ops.SdpError, match="y overlaps x"):
        ops.sdp_grouped_matmul(ctx, x, w, ends, buf[:, n_in - 1:n_in - 1 + n_out])


def test_distill(lib):
    sdp, ops, ctx = lib
    buf = torch.randn((5, 2 * 1000 + 24), device="cuda")
    z, d = buf[:, :1000], buf[:, 1016:2016]
    labels, g = torch.arange(5, device="cuda"), torch.ones(5, device="cuda")
    loss, want, alone = torch.empty(5, device="cuda"), torch.empty(5, 1000, device="cuda"), torch.empty(5, device="cuda")
    kept = buf.clone()
    ops.sdp_distill_loss(ctx, z.clone(), alone, labels=labels, label_weight=1.0, row_grad=g, dlogits=want)
    ops.sdp_distill_loss(ctx, z, loss, labels=labels, label_weight=1.0, row_grad=g, dlogits=d)
    assert torch.equal(d, want) and torch.equal(loss, alone)
    assert torch.equal(buf[:, :1016], kept[:, :1016]) and torch.equal(buf[:, 2016:], kept[:, 2016:])
