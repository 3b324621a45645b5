"""The training operators around the experts' products under HIP graph capture: calls
without a workspace replay with their eager results; calls that use the context's are
refused, and both the capture and the context go on."""
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


def new(*shape, dtype=BF16):
    return torch.randn(shape, device="cuda").to(dtype)


def ints(n, high, low=0):
    return lambda: torch.randint(low, high, n, device="cuda")


# each: inputs with what refills them, outputs, the call on a stream
def embed(ops, ctx):
    table, out, ids = new(50, 200), new(90, 200), torch.zeros(90, dtype=I32, device="cuda")
    return [(table, None), (ids, ints((90,), 50, -1))], [out], lambda s: ops.sdp_embed(ctx, table, ids, out, stream=s)


def norm(ops, ctx):
    h, y, w, g = new(70, 1003), new(70, 1003), new(1003), new(1003)
    out = [new(70, 1003), new(70, 1003)]
    return [(t, None) for t in (h, y, w, g)], out, lambda s: ops.sdp_block_norm(
        ctx, h, y, *out, gate=g, post_norm=True, post_weight=w, pre_weight=w, stream=s)


def norm_back(ops, ctx):
    h, y, dh_out, dn, g, w = new(70, 1003), new(70, 1003), new(70, 1003), new(70, 1003), new(70, 1), new(1003)
    out = [new(70, 1003), new(70, 1003), new(70, 1)]
    return [(t, None) for t in (h, y, dh_out, dn, g, w)], out, lambda s: ops.sdp_block_norm_backward(
        ctx, h, y, dh_out, dn, out[0], out[1], gate=g, dgate=out[2], gate_sigmoid=True, post_norm=True, post_weight=w,
        pre_weight=w, stream=s)


def route(ops, ctx):
    z, bias = new(300, 64), new(64, dtype=F32)
    index, w = torch.zeros((300, 4), dtype=I32, device="cuda"), new(300, 4, dtype=F32)
    return [(z, None), (bias, None)], [index, w], lambda s: ops.sdp_route(
        ctx, z, index, w, bias=bias, sigmoid=True, groups=8, top_groups=3, group_best=2, renormalize=True, stream=s)


def route_back(ops, ctx):
    z, dw, dz = new(300, 64), new(300, 4, dtype=F32), new(300, 64)
    index = torch.zeros((300, 4), dtype=I32, device="cuda")
    return [(z, None), (dw, None), (index, ints((300, 4), 64, -1))], [dz], lambda s: ops.sdp_route_backward(
        ctx, z, index, dw, dz, stream=s)


def experts(ops, ctx, n=2000):
    """order, gather, combine and both gradients in one graph, as a layer runs them."""
    k, e, h = 4, 24, 136
    index = torch.zeros((n, k), dtype=I32, device="cuda")
    x, w, dout = new(n, h), new(n, k, dtype=F32), new(n, h)
    ends, place = torch.zeros(e, dtype=I32, device="cuda"), torch.zeros((n, k), dtype=I32, device="cuda")
    rows, out, drows, dx = new(n * k, h), new(n, h), new(n * k, h), new(n, h)
    dw = torch.zeros_like(w)

    def call(s):
        ops.sdp_expert_order(ctx, index, ends, place, stream=s)
        ops.sdp_expert_gather(ctx, x, place, rows, stream=s)
        ops.sdp_expert_combine(ctx, rows, place, w, out, residual=x, stream=s)
        ops.sdp_expert_combine_backward(ctx, rows, place, w, dout, drows, dw, stream=s)
        ops.sdp_expert_gather_backward(ctx, drows, place, dx, stream=s)
    return [(index, ints((n, k), e, -1)), (x, None), (w, None), (dout, None)], [ends, place, rows, out, drows, dw, dx], call


def few_experts(ops, ctx):
    return experts(ops, ctx, 30)


@pytest.mark.parametrize("make", [embed, norm, norm_back, route, route_back, experts, few_experts])
def test_replays_give_the_eager_results(lib, make):
    sdp, ops, ctx = lib
    inputs, outputs, call = make(ops, ctx)
    call(None)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        call(stream)
    for again in range(4):
        for t, fill in inputs:
            t.copy_(fill() if fill else torch.randn(t.shape, device="cuda"))
        for t in outputs:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outputs]
        for t in outputs:
            t.fill_(-7)
        call(None)
        torch.cuda.synchronize()
        for a, b in zip(got, outputs):
            assert torch.equal(a, b), again


def embed_back(ops, ctx):
    dout, ids, dtable = new(90, 200), torch.randint(0, 50, (90,), device="cuda"), torch.empty((50, 200), device="cuda")
    return dtable, lambda s: ops.sdp_embed_backward(ctx, dout, ids, dtable, stream=s)


def weight_gradient(ops, ctx):
    h, dn, dw = new(70, 1003), new(70, 1003), torch.empty(1003, device="cuda")
    return dw, lambda s: ops.sdp_block_norm_backward(ctx, h, None, None, dn, None, None, dpre_weight=dw, stream=s)


def gate_gradient(ops, ctx):
    h, y, g, dg = new(70, 1003), new(70, 1003), new(1003), torch.empty(1003, dtype=BF16, device="cuda")
    return dg, lambda s: ops.sdp_block_norm_backward(ctx, None, y, h, None, None, None, gate=g, dgate=dg, stream=s)


@pytest.mark.parametrize("make", [embed_back, weight_gradient, gate_gradient])
def test_a_call_with_workspace_is_refused_while_its_stream_captures(lib, make):
    sdp, ops, _ = lib
    ctx = sdp.sdp_ctx_create(0, 0, 1, 0)  # no workspace yet
    out, call = make(ops, ctx)
    _, kept, fine = norm(ops, ctx)
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


def test_calls_on_several_streams_share_the_workspace(lib):
    """Calls of one context on different streams, one after the other, each with its own result."""
    sdp, ops, ctx = lib
    streams = [torch.cuda.Stream() for _ in range(3)]
    cases = []
    for k in range(12):
        n = 500 + 300 * k
        dout, ids = new(n, 256), torch.randint(-1, 40, (n,), device="cuda")
        cases.append((dout, ids, torch.empty((40, 256), device="cuda"), torch.empty((40, 256), device="cuda")))
    torch.cuda.synchronize()
    for k, (dout, ids, got, _) in enumerate(cases):
        ops.sdp_embed_backward(ctx, dout, ids, got, stream=streams[k % 3])
    torch.cuda.synchronize()
    for dout, ids, got, want in cases:
        ops.sdp_embed_backward(ctx, dout, ids, want)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
