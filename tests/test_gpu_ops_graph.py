"""The training operators under HIP graph capture: calls without a workspace replay
with their eager results; calls that use the context's are refused, and both the
capture and the context go on."""
import pytest

import gpu_util

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def lib():
    sdp = gpu_util.need_gpu()
    from paper_2609_34162_amd import ops
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield sdp, ops, c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


def new(*shape, dtype=BF16, sigma=1.0):
    return (torch.randn(shape, device="cuda") * sigma).to(dtype)


def norm_rope(ops, ctx, back):
    q, k, cos, sin = new(2, 50, 4, 64), new(2, 50, 2, 64), new(50, 32, dtype=F32), new(50, 32, dtype=F32)
    out = torch.empty_like(q), torch.empty_like(k)
    if not back:
        return (q, k), out, lambda s: ops.sdp_qk_norm_rope(ctx, q, k, *out, cos, sin, stream=s)
    dq, dk = new(2, 50, 4, 64), new(2, 50, 2, 64)
    return (q, k, dq, dk), out, lambda s: ops.sdp_qk_norm_rope_backward(ctx, q, k, dq, dk, *out, cos, sin, stream=s)


def distill(ops, ctx, back):
    rows, vocab = 300, 5000
    z, loss, lse, dz = new(rows, vocab), torch.empty(rows, device="cuda"), new(rows, 2, dtype=F32), new(rows, vocab)
    g, labels = torch.ones(rows, device="cuda"), torch.randint(0, vocab, (rows,), device="cuda")
    more = dict(labels=labels, distill_weight=0.0, label_weight=1.0)
    if back:
        return (z, lse), (dz,), lambda s: ops.sdp_distill_loss_backward(ctx, z, lse, g, dz, stream=s, **more)
    return (z,), (loss, lse, dz), lambda s: ops.sdp_distill_loss(ctx, z, loss, lse, row_grad=g, dlogits=dz, stream=s, **more)


def grouped(ops, ctx, back):
    x, w, dy = new(700, 256), new(4, 512, 256), new(700, 512)
    ends = torch.tensor([100, 100, 433, 690], dtype=torch.int32, device="cuda")
    if not back:
        y = new(700, 512)
        return (x, w), (y,), lambda s: ops.sdp_grouped_matmul(ctx, x, w, ends, y, stream=s)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    return (x, w, dy), (dx, dw), lambda s: ops.sdp_grouped_matmul_backward(ctx, x, w, ends, dy, dx, dw, stream=s)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("make", [norm_rope, distill, grouped])
def test_replays_give_the_eager_results(lib, make, back):
    sdp, ops, ctx = lib
    inputs, outputs, call = make(ops, ctx, back)
    call(None)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        call(stream)
    for again in range(4):
        for t in inputs:
            t.copy_(torch.randn(t.shape, device="cuda"))
        for t in outputs:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outputs]
        for t in outputs:
            t.fill_(-7.0)
        call(None)
        torch.cuda.synchronize()
        for a, b in zip(got, outputs):
            assert torch.equal(a, b), again


def with_weight_gradients(ops, ctx):
    q, dw = new(2, 50, 4, 64), torch.empty(64, device="cuda")
    dq, dk = torch.empty_like(q), torch.empty_like(q)
    return dw, lambda s: ops.sdp_qk_norm_rope_backward(ctx, q, q, q, q, dq, dk, dq_weight=dw, stream=s)


def loss_alone(ops, ctx):
    z, loss, labels = new(5, 5000), torch.empty(5, device="cuda"), torch.zeros(5, dtype=torch.int64, device="cuda")
    return loss, lambda s: ops.sdp_distill_loss(ctx, z, loss, labels=labels, label_weight=1.0, stream=s)


def few_weights(ops, ctx):
    x, w, dy, ends = new(5000, 136), new(1, 72, 136), new(5000, 72), torch.tensor([5000], device="cuda")
    dw = torch.empty((1, 72, 136), device="cuda")
    return dw, lambda s: ops.sdp_grouped_matmul_backward(ctx, x, w, ends, dy, None, dw, stream=s)


def copied(ops, ctx):
    x, w, ends = new(8200, 1021), new(2, 1033, 1021), torch.tensor([4000, 8200], device="cuda")
    y = new(8200, 1033)
    return y, lambda s: ops.sdp_grouped_matmul(ctx, x, w, ends, y, stream=s)


@pytest.mark.parametrize("make", [with_weight_gradients, loss_alone, few_weights, copied])
def test_a_call_with_workspace_is_refused_while_its_stream_captures(lib, make):
    sdp, ops, _ = lib
    ctx = sdp.sdp_ctx_create(0, 0, 1, 0)  # no workspace yet
    out, call = make(ops, ctx)
    _, kept, fine = norm_rope(ops, ctx, False)
    fine(None)
    out.fill_(7.0)
    torch.cuda.synchronize()
    want = [t.clone() for t in kept]
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        with pytest.raises(ops.SdpError, match="cannot be captured") as e:
            call(stream)
        fine(stream)
    assert e.value.status == sdp.SDP_ERR_INVALID_ARGUMENT
    for t in kept:
        t.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert (out == 7.0).all() and all(torch.equal(a, b) for a, b in zip(kept, want))
    call(stream)  # no longer capturing
    stream.synchronize()
    first = out.clone()
    call(None)
    torch.cuda.synchronize()
    assert torch.equal(first, out) and not (out == 7.0).all()
    sdp.sdp_ctx_destroy(ctx)
