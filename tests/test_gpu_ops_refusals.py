"""What the training operators refuse, with a context and device tensors: the
status, that nothing was written, and that the next call works."""
import ctypes

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


def refused(ops, status, text, call, *args, **kw):
    with pytest.raises(ops.SdpError) as e:
        call(*args, **kw)
    assert e.value.status == status, (e.value.name, e.value.detail)
    assert text in e.value.detail, e.value.detail


def test_qk(lib):
    sdp, ops, ctx = lib
    bad, mem, align = sdp.SDP_ERR_INVALID_ARGUMENT, sdp.SDP_ERR_NOT_DEVICE_MEMORY, sdp.SDP_ERR_ALIGNMENT
    q, k = torch.randn(2, 6, 4, 16, device="cuda"), torch.randn(2, 6, 2, 16, device="cuda")
    qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
    cos, sin = torch.ones(8, 8, device="cuda"), torch.zeros(8, 8, device="cuda")
    f = ops.sdp_qk_norm_rope
    refused(ops, mem, "q (", f, ctx, q.cpu(), k, qo, ko, cos, sin)
    refused(ops, mem, "cos", f, ctx, q, k, qo, ko, cos.cpu(), sin.cpu())
    room = torch.randn(q.numel() + 64, device="cuda")
    refused(ops, bad, "q_out overlaps q", f, ctx, room[:q.numel()].view(q.shape), k, room[64:].view(q.shape), ko, cos, sin)
    refused(ops, bad, "overlaps", f, ctx, q, k, qo, qo[:, :, 1:3], cos, sin)
    refused(ops, bad, "overlaps itself", f, ctx, q, k, torch.zeros(16, device="cuda").expand(2, 6, 4, 16), ko, cos, sin)
    refused(ops, bad, "eps", f, ctx, q, k, qo, ko, cos, sin, eps=float("nan"))
    refused(ops, bad, "eps", f, ctx, q, k, qo, ko, cos, sin, eps=-1.0)
    wide = torch.ones(8, 9, device="cuda")
    refused(ops, bad, "rotary_dim", f, ctx, q, k, qo, ko, wide, wide)
    big = torch.zeros(1, 1, 1, 1026, device="cuda")
    refused(ops, bad, "head_dim", f, ctx, big, big, torch.zeros_like(big), torch.zeros_like(big))
    # a tensor said to be longer than its memory
    d = ops.sdp_qk_norm_rope_desc()
    d.batch, d.tokens, d.q_heads, d.head_dim, d.position_type = 1, 1 << 30, 4, 16, ops.SDP_TYPE_I32
    h = ops.sdp_heads(q.data_ptr(), 0, 64, 16)
    o = ops.sdp_heads(qo.data_ptr(), 0, 64, 16)
    call = lambda: sdp._check(sdp._lib.sdp_qk_norm_rope(ctx, ctypes.byref(d), ctypes.byref(h), ctypes.byref(h),
                                                        ctypes.byref(o), ctypes.byref(o), None))
    refused(ops, mem, "overrun", call)
    d.tokens = 6
    h.token_stride = -64
    refused(ops, bad, "stride", call)
    h.token_stride, h.data = 64, q.data_ptr() + 2
    refused(ops, align, "aligned", call)
    d.type = 9
    refused(ops, bad, "type", call)
    assert (qo == 7).all() and (ko == 7).all()
    f(ctx, q, k, qo, ko, cos, sin)
    torch.cuda.synchronize()
    want = q * (q.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    assert torch.allclose(qo, want, rtol=1e-5, atol=1e-6)


def test_grouped(lib):
    sdp, ops, ctx = lib
    bad, mem = sdp.SDP_ERR_INVALID_ARGUMENT, sdp.SDP_ERR_NOT_DEVICE_MEMORY
    x, w = torch.randn(10, 16, device="cuda").to(BF16), torch.randn(2, 24, 16, device="cuda").to(BF16)
    ends = torch.tensor([4, 10], device="cuda")
    y = torch.full((10, 24), 7.0, dtype=BF16, device="cuda")
    f = ops.sdp_grouped_matmul
    refused(ops, mem, "ends", f, ctx, x, w, ends.cpu(), y)
    refused(ops, mem, "w (", f, ctx, x, w.cpu(), ends, y)
    refused(ops, bad, "overlaps", f, ctx, x, w, ends, w.view(-1)[:240].view(10, 24))
    refused(ops, bad, "overlaps itself", f, ctx, x, w, ends, y[:1].expand(10, 24))
    many = torch.zeros(5000, 1, 1, dtype=BF16, device="cuda")
    refused(ops, bad, "groups", f, ctx, x[:, :1], many, torch.zeros(5000, dtype=torch.int32, device="cuda"), y[:, :1])
    dy, dx = torch.randn(10, 24, device="cuda").to(BF16), torch.full((10, 16), 7.0, dtype=BF16, device="cuda")
    refused(ops, bad, "x is NULL", ops.sdp_grouped_matmul_backward, ctx, None, w, ends, dy, None, torch.empty_like(w))
    refused(ops, bad, "overlaps", ops.sdp_grouped_matmul_backward, ctx, x, w, ends, dy, x, torch.empty_like(w))
    assert (y == 7).all() and (dx == 7).all()
    f(ctx, x, w, ends, y)
    torch.cuda.synchronize()
    assert torch.allclose(y[:4].float(), x[:4].float() @ w[0].float().t(), rtol=1e-2, atol=1e-2)


def test_distill(lib):
    sdp, ops, ctx = lib
    bad, mem = sdp.SDP_ERR_INVALID_ARGUMENT, sdp.SDP_ERR_NOT_DEVICE_MEMORY
    z = torch.randn(4, 100, device="cuda")
    labels = torch.zeros(4, dtype=torch.int64, device="cuda")
    loss, g, d = torch.full((4,), 7.0, device="cuda"), torch.ones(4, device="cuda"), torch.full_like(z, 7)
    f = ops.sdp_distill_loss
    one = dict(labels=labels, label_weight=1.0)
    refused(ops, mem, "logits", f, ctx, z.cpu(), loss, **one)
    refused(ops, mem, "labels", f, ctx, z, loss, labels=labels.cpu())
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-9):
        refused(ops, bad, "temperature", f, ctx, z, loss, temperature=tau, **one)
    refused(ops, bad, "finite", f, ctx, z, loss, labels=labels, label_weight=float("inf"))
    refused(ops, bad, "row_grad", f, ctx, z, loss, dlogits=d, **one)
    refused(ops, bad, "overlaps", f, ctx, z[:2], loss[:2], dlogits=z[1:3], row_grad=g[:2], labels=labels[:2])
    refused(ops, bad, "loss overlaps row_grad", f, ctx, z, loss, row_grad=loss, dlogits=d, **one)
    many = torch.zeros(4, 1025, dtype=torch.int64, device="cuda")
    refused(ops, bad, "teacher_k", f, ctx, z, loss, teacher_logits=many.float(), teacher_index=many)
    refused(ops, bad, "dlogits is NULL", lambda: ops._check(sdp._lib.sdp_distill_loss_backward(
        ctx, ctypes.byref(ops._distill_desc(z, None, None, labels, 1.0, 1.0, 1.0)), loss.data_ptr(), g.data_ptr(),
        None, 0, None)))
    assert (loss == 7).all() and (d == 7).all()
    f(ctx, z, loss, row_grad=g, dlogits=d, **one)
    torch.cuda.synchronize()
    assert torch.allclose(loss, torch.nn.functional.cross_entropy(z, labels, reduction="none"), rtol=1e-5, atol=1e-5)


def test_empty_sizes(lib):
    sdp, ops, ctx = lib
    e = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda")
    ops.sdp_qk_norm_rope(ctx, e(0, 4, 2, 8), e(0, 4, 1, 8), e(0, 4, 2, 8), e(0, 4, 1, 8), e(4, 4), e(4, 4))
    ops.sdp_grouped_matmul(ctx, e(0, 8, dtype=BF16), e(2, 4, 8, dtype=BF16), torch.zeros(2, dtype=torch.int32, device="cuda"),
                           e(0, 4))
    dw = torch.full((2, 4, 8), 7.0, device="cuda")
    ops.sdp_grouped_matmul_backward(ctx, e(0, 8, dtype=BF16), e(2, 4, 8, dtype=BF16),
                                    torch.zeros(2, dtype=torch.int32, device="cuda"), e(0, 4, dtype=BF16),
                                    e(0, 8, dtype=BF16), dw)
    assert (dw == 0).all()
    y = torch.full((3, 4), 7.0, device="cuda")
    ops.sdp_grouped_matmul(ctx, e(3, 0, dtype=BF16), e(2, 4, 0, dtype=BF16),
                           torch.tensor([1, 3], dtype=torch.int32, device="cuda"), y)
    assert (y == 0).all()
    ops.sdp_distill_loss(ctx, e(0, 10), e(0), labels=torch.zeros(0, dtype=torch.int64, device="cuda"))
    torch.cuda.synchronize()
