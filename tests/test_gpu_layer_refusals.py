"""What the training operators around the experts' products refuse, with a context
and device tensors: the status, that nothing was written, and that the next call
works."""
import ctypes

import pytest

import gpu_util

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


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


def seven(*shape, dtype=F32):
    return torch.full(shape, 7, dtype=dtype, device="cuda")


def test_embed(lib):
    sdp, ops, ctx = lib
    bad, mem, align = sdp.SDP_ERR_INVALID_ARGUMENT, sdp.SDP_ERR_NOT_DEVICE_MEMORY, sdp.SDP_ERR_ALIGNMENT
    table, ids, out = torch.randn(10, 16, device="cuda"), torch.arange(6, device="cuda"), seven(6, 16)
    f, b = ops.sdp_embed, ops.sdp_embed_backward
    refused(ops, mem, "table (", f, ctx, table.cpu(), ids, out)
    refused(ops, mem, "ids (", f, ctx, table, ids.cpu(), out)
    refused(ops, bad, "out overlaps itself", f, ctx, table, ids, out[:1].expand(6, 16))
    refused(ops, bad, "out overlaps table", f, ctx, table, ids, table[2:8])
    refused(ops, bad, "scale must be finite", f, ctx, table, ids, out, scale=float("inf"))
    refused(ops, bad, "scale must be finite", f, ctx, table, ids, out, scale=1e39)
    refused(ops, bad, "dtable overlaps dout", b, ctx, table[:6], ids, table)
    refused(ops, bad, "dtable overlaps itself", b, ctx, out, ids, table[:1].expand(10, 16))
    d = ops.sdp_embed_desc(1 << 28, 10, 16, ops.SDP_TYPE_F32, ops.SDP_TYPE_F32, ops.SDP_TYPE_I64, ids.data_ptr(), 1.0)
    t, o = ops.sdp_rows(table.data_ptr(), 16), ops.sdp_rows(out.data_ptr(), 16)
    call = lambda: sdp._check(sdp._lib.sdp_embed(ctx, ctypes.byref(d), ctypes.byref(t), ctypes.byref(o), None))
    refused(ops, mem, "overrun", call)
    d.tokens = 1 << 31
    refused(ops, bad, "out of range", call)
    d.tokens, o.stride = 6, -16
    refused(ops, bad, "stride", call)
    o.stride, d.hidden = 16, (1 << 30) + 1
    refused(ops, bad, "hidden out of range", call)
    d.hidden, o.data = 16, out.data_ptr() + 2
    refused(ops, align, "aligned", call)
    d.row_type = 3
    refused(ops, bad, "type", call)
    assert (out == 7).all()
    f(ctx, table, ids, out)
    assert torch.equal(out, table[:6])


def test_block_norm(lib):
    sdp, ops, ctx = lib
    bad, mem = sdp.SDP_ERR_INVALID_ARGUMENT, sdp.SDP_ERR_NOT_DEVICE_MEMORY
    h, y = torch.randn(6, 16, device="cuda"), torch.randn(6, 16, device="cuda")
    ho, no, w = seven(6, 16), seven(6, 16), torch.ones(16, device="cuda")
    f, b = ops.sdp_block_norm, ops.sdp_block_norm_backward
    refused(ops, mem, "h (", f, ctx, h.cpu(), y, ho, no)
    refused(ops, mem, "pre_weight (", f, ctx, h, y, ho, no, pre_weight=w.cpu())
    refused(ops, mem, "gate (", f, ctx, h, y, ho, no, gate=w.cpu())
    refused(ops, bad, "both outputs", f, ctx, h, y, None, None)
    refused(ops, bad, "h_out without y", f, ctx, h, None, ho, no)
    refused(ops, bad, "eps", f, ctx, h, y, ho, no, eps=-1.0)
    refused(ops, bad, "finite", f, ctx, h, y, ho, no, scale=float("nan"))
    refused(ops, bad, "finite", f, ctx, h, y, ho, no, weight_offset=-1e39)
    refused(ops, bad, "h_out overlaps n_out", f, ctx, h, y, ho, ho)
    refused(ops, bad, "n_out overlaps h", f, ctx, h, y, ho, h)
    refused(ops, bad, "h_out overlaps y", f, ctx, h, y, y, no)
    room = torch.randn(7, 16, device="cuda")
    refused(ops, bad, "h_out overlaps h", f, ctx, room[:6], y, room[1:], no)
    refused(ops, bad, "n_out overlaps itself", f, ctx, h, y, ho, no[:1].expand(6, 16))
    refused(ops, bad, "n_out overlaps pre_weight", f, ctx, h, y, ho, no, pre_weight=no[2])
    dh, dy, dw = seven(6, 16), seven(6, 16), seven(16)
    refused(ops, bad, "dh_out and dn are NULL", b, ctx, h, y, None, None, dh, dy)
    refused(ops, bad, "h_out is NULL with dn", b, ctx, None, y, None, no, dh, dy)
    refused(ops, bad, "y is NULL", b, ctx, h, None, ho, no, dh, dy, post_norm=True)
    refused(ops, bad, "y is NULL", b, ctx, h, None, ho, no, dh, dy, gate=w, dgate=dw)
    refused(ops, bad, "dpost_weight without", b, ctx, h, y, ho, no, dh, dy, dpost_weight=dw)
    refused(ops, bad, "dpre_weight without", b, ctx, h, y, ho, None, dh, dy, dpre_weight=dw)
    refused(ops, bad, "dh overlaps dy", b, ctx, h, y, ho, no, dh, dh)
    refused(ops, bad, "dh overlaps h_out", b, ctx, h, y, ho, no, h, dy)
    refused(ops, bad, "dy overlaps dh_out", b, ctx, h, y, ho, no, dh, ho)
    refused(ops, bad, "dpre_weight", b, ctx, h, y, ho, no, dh, dy, post_norm=True, dpost_weight=dw, dpre_weight=dw)
    refused(ops, bad, "overlaps gate", b, ctx, h, y, ho, no, dh, dy, gate=w, dgate=w)
    d = ops.sdp_block_norm_desc(6, 16, 0, 0, 0, 0, ops.SDP_GATE_NONE, 0, 1.0, 1e-6, 0.0)
    r = lambda t: ctypes.pointer(ops.sdp_rows(t.data_ptr(), 16))
    grads = ops.sdp_block_norm_grads(r(dh), r(dy), dw.data_ptr(), 0, None, None)
    refused(ops, bad, "dgate without a gate", lambda: sdp._check(sdp._lib.sdp_block_norm_backward(
        ctx, ctypes.byref(d), r(h), r(y), r(ho), r(no), ctypes.byref(grads), None)))
    for tokens, hidden in ((1 << 31, 16), (6, (1 << 30) + 1)):
        d.tokens, d.hidden = tokens, hidden
        refused(ops, bad, "out of range", lambda: sdp._check(sdp._lib.sdp_block_norm(
            ctx, ctypes.byref(d), r(h), r(y), r(ho), r(no), None)))
    d.tokens, d.hidden, d.gate_form = 6, 16, 9
    refused(ops, bad, "gate_form", lambda: sdp._check(sdp._lib.sdp_block_norm(
        ctx, ctypes.byref(d), r(h), r(y), r(ho), r(no), None)))
    assert all((t == 7).all() for t in (ho, no, dh, dy, dw))
    f(ctx, h, y, ho, no)
    assert torch.allclose(ho, h + y) and torch.allclose(no, ho * (ho.square().mean(1, keepdim=True) + 1e-6).rsqrt(), rtol=1e-5)


def test_route(lib):
    sdp, ops, ctx = lib
    bad, mem = sdp.SDP_ERR_INVALID_ARGUMENT, sdp.SDP_ERR_NOT_DEVICE_MEMORY
    z, index, w = torch.randn(6, 16, device="cuda"), seven(6, 4, dtype=I32), seven(6, 4)
    f, b = ops.sdp_route, ops.sdp_route_backward
    refused(ops, mem, "logits (", f, ctx, z.cpu(), index, w)
    refused(ops, mem, "bias (", f, ctx, z, index, w, bias=torch.zeros(16))
    refused(ops, bad, "top must be", f, ctx, z[:, :3], index, w)
    refused(ops, bad, "top must be", f, ctx, torch.randn(2, 200, device="cuda"), seven(2, 65, dtype=I32), seven(2, 65))
    refused(ops, bad, "top must be", f, ctx, z, index[:, :0].contiguous(), w[:, :0].contiguous())
    refused(ops, bad, "experts", f, ctx, torch.randn(2, 2049, device="cuda"), index[:2], w[:2])
    for groups in (0, -1, 3, 32):
        refused(ops, bad, "groups must divide", f, ctx, z, index, w, groups=groups)
    refused(ops, bad, "groups must divide", f, ctx, torch.randn(2, 128, device="cuda"), index[:2], w[:2], groups=128)
    for more in (dict(top_groups=0), dict(top_groups=5), dict(group_best=0), dict(group_best=3)):
        refused(ops, bad, "top_groups must be", f, ctx, z, index, w, groups=4, **more)
    refused(ops, bad, "scale", f, ctx, z, index, w, scale=float("nan"))
    refused(ops, bad, "weights overlaps", f, ctx, z, index, z.view(-1)[:24].view(6, 4))
    dz = seven(6, 16)
    refused(ops, bad, "dlogits overlaps logits", b, ctx, z[:5], index[:5], w[:5], z[1:])
    refused(ops, bad, "dlogits overlaps itself", b, ctx, z, index, w, dz[:1].expand(6, 16))
    assert (index == 7).all() and (w == 7).all() and (dz == 7).all()
    f(ctx, z, index, w)
    assert torch.equal(index.long(), z.topk(4, dim=1).indices)


def test_experts(lib):
    sdp, ops, ctx = lib
    bad, mem = sdp.SDP_ERR_INVALID_ARGUMENT, sdp.SDP_ERR_NOT_DEVICE_MEMORY
    index, ends, place = torch.zeros((6, 2), dtype=I32, device="cuda"), seven(4, dtype=I32), seven(6, 2, dtype=I32)
    o = ops.sdp_expert_order
    refused(ops, mem, "index (", o, ctx, index.cpu(), ends, place)
    refused(ops, bad, "place overlaps", o, ctx, index, ends, index)
    refused(ops, bad, "experts must be", o, ctx, index, torch.zeros(2049, dtype=I32, device="cuda"), place)
    refused(ops, bad, "overlaps place", o, ctx, index, place.view(-1)[:4], place)
    refused(ops, bad, "place overlaps order", o, ctx, index, ends, place, place.view(-1))
    x, rows, out, w = torch.randn(6, 16, device="cuda"), seven(12, 16), seven(6, 16), torch.ones(6, 2, device="cuda")
    own = torch.arange(12, dtype=I32, device="cuda").view(6, 2)
    refused(ops, mem, "place (", ops.sdp_expert_gather, ctx, x, own.cpu(), rows)
    refused(ops, bad, "rows overlaps x", ops.sdp_expert_gather, ctx, rows[:6], own, rows)
    refused(ops, bad, "rows overlaps itself", ops.sdp_expert_gather, ctx, x, own, rows[:1].expand(12, 16))
    refused(ops, bad, "dx overlaps drows", ops.sdp_expert_gather_backward, ctx, rows, own, rows[:6])
    refused(ops, bad, "out overlaps rows", ops.sdp_expert_combine, ctx, rows, own, w, rows[:6])
    room = torch.randn(7, 16, device="cuda")
    refused(ops, bad, "out overlaps", ops.sdp_expert_combine, ctx, rows, own, w, room[1:], residual=room[:6])
    refused(ops, bad, "drows overlaps dout", ops.sdp_expert_combine_backward, ctx, rows, own, w, rows[:6], rows, None)
    refused(ops, bad, "dweights overlaps weights", ops.sdp_expert_combine_backward, ctx, x.repeat(2, 1), own, w, x, rows, w)
    d = ops.sdp_expert_desc(1 << 20, 1 << 12, 16, 0, 0, 0, own.data_ptr())
    r = lambda t: ctypes.pointer(ops.sdp_rows(t.data_ptr(), 16))
    refused(ops, bad, "out of range", lambda: sdp._check(sdp._lib.sdp_expert_gather(ctx, ctypes.byref(d), r(x), r(rows), None)))
    d.tokens, d.top, d.hidden = 6, 2, (1 << 30) + 1
    refused(ops, bad, "out of range", lambda: sdp._check(sdp._lib.sdp_expert_gather(ctx, ctypes.byref(d), r(x), r(rows), None)))
    d.hidden = 16
    refused(ops, bad, "weights is NULL", lambda: sdp._check(sdp._lib.sdp_expert_combine(
        ctx, ctypes.byref(d), r(rows), None, None, r(out), None)))
    assert (ends == 7).all() and (place == 7).all() and (rows == 7).all() and (out == 7).all()
    ops.sdp_expert_gather(ctx, x, own, rows)
    assert torch.equal(rows, x.repeat_interleave(2, 0))


def test_empty_sizes(lib):
    sdp, ops, ctx = lib
    e = lambda *s, dtype=F32: torch.empty(s, dtype=dtype, device="cuda")
    ops.sdp_embed(ctx, e(4, 8), e(0, dtype=I32), e(0, 8))
    ops.sdp_embed(ctx, e(4, 0), e(3, dtype=I32), e(3, 0))
    out = seven(3, 8)
    ids = torch.tensor([0, -1, 5], dtype=I32, device="cuda")
    ops.sdp_embed(ctx, e(0, 8), ids, out)  # no vocabulary: padding is still padding
    assert torch.isnan(out[0]).all() and (out[1] == 0).all() and torch.isnan(out[2]).all()
    dtable = seven(4, 8)
    ops.sdp_embed_backward(ctx, e(0, 8), e(0, dtype=I32), dtable, accumulate=True)
    assert (dtable == 7).all()
    ops.sdp_embed_backward(ctx, e(0, 8), e(0, dtype=I32), dtable)
    assert (dtable == 0).all()
    ops.sdp_embed_backward(ctx, e(3, 8), ids, e(0, 8))
    ops.sdp_block_norm(ctx, e(0, 8), e(0, 8), e(0, 8), e(0, 8))
    ops.sdp_block_norm(ctx, e(3, 0), e(3, 0), e(3, 0), e(3, 0))
    dpost, dpre, dgate = seven(8), seven(8), seven(8)
    ops.sdp_block_norm_backward(ctx, e(0, 8), e(0, 8), e(0, 8), e(0, 8), e(0, 8), e(0, 8), gate=e(8), dgate=dgate,
                                post_norm=True, dpost_weight=dpost, dpre_weight=dpre)
    assert (dpost == 0).all() and (dpre == 0).all() and (dgate == 0).all()
    ops.sdp_route(ctx, e(0, 8), e(0, 2, dtype=I32), e(0, 2))
    ends = seven(4, dtype=I32)
    ops.sdp_expert_order(ctx, e(0, 2, dtype=I32), ends, e(0, 2, dtype=I32))
    assert (ends == 0).all()
    ops.sdp_expert_gather(ctx, e(0, 8), e(0, 2, dtype=I32), e(0, 8))
    torch.cuda.synchronize()
