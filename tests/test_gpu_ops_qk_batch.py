"""sdp_qk_norm_rope and its backward on batches: each wave walks several runs of heads,
and the largest go past the last-level cache.  Some tokens' rows are checked against
the 64-bit definition, and the weights' gradients over all of them."""
import pytest

import gpu_util
import ops_ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    sdp = gpu_util.need_gpu()
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)
    torch.cuda.empty_cache()


def heads(gen, b, s, hq, hk, d, dtype, layout):
    """q's and k's heads: of a fused projection, of [b, h, s, d], or of rows at odd offsets."""
    new = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=F32).to(dtype)
    if layout == "heads":
        return new(b, hq, s, d).transpose(1, 2), new(b, hk, s, d).transpose(1, 2)
    if layout == "odd":
        x = new(1 + b * s * ((hq + hk) * d + 3))[1:].view(b, s, (hq + hk) * d + 3)[:, :, :(hq + hk) * d]
        x = x.unflatten(2, (hq + hk, d))
    else:
        x = new(b, s, hq + 2 * hk, d)
    return x[:, :, :hq], x[:, :, hq:hq + hk]


def weight_gradient(x, dy, cos, sin, positions, rotary, interleaved):
    """As ops_ref.norm_rope_back's, a sequence (or many short ones) at a time on the GPU.  A lane adds up to some 50
    rows, then come 6 additions over lanes, 2 over waves, 2 over blocks and 22 more: 256 roundings are more than any
    term goes through, d / 2 of its row's squares and 64 beside them."""
    d = x.shape[-1]
    dw = size = torch.zeros(d, dtype=torch.float64, device="cuda")
    step = max(1, 8192 // x.shape[1])
    for a in range(0, x.shape[0], step):
        xx, yy, at = (t[a:a + step] for t in (x, dy, positions.long()))
        xx, yy, c, s = xx.double(), yy.double(), cos.double()[at], sin.double()[at]
        unit = xx / (xx.square().mean(-1, keepdim=True) + EPS).sqrt()
        dn = ops_ref.rotate(yy, c, s, rotary, interleaved, back=True)
        big = yy.abs()
        lo, hi = ops_ref.pair_index(rotary, interleaved)
        both = yy[..., lo].abs() + yy[..., hi].abs()
        big[..., lo], big[..., hi] = both, both
        dw = dw + (dn * unit).sum((0, 1, 2))
        size = size + (big * unit.abs()).sum((0, 1, 2))
    return dw.cpu(), ops_ref.rounded(dw.cpu(), F32, (256 + d / 2 + 64) * ops_ref.U32 * size.cpu())


@pytest.mark.parametrize("b,s,hq,hk,d,rotary,interleaved,dtype,layout", [
    (4, 8192, 40, 8, 128, 128, False, BF16, "fused"),      # past the cache; runs of 40 and of 8 heads
    (3, 8191, 12, 4, 96, 64, True, F32, "heads"),
    (300001, 1, 2, 1, 64, 64, False, BF16, "fused"),       # several tokens to a wave
    (7, 2071, 9, 0, 128, 64, False, BF16, "fused"),        # three runs to a token, which the waves do not divide by
    (5, 9001, 5, 3, 80, 40, False, BF16, "heads"),         # half pieces as partners
    (2, 9001, 5, 1, 20, 20, False, BF16, "odd"),           # row by row
    (1, 20011, 3, 1, 36, 12, True, F32, "odd"),
])
def test_batches(ctx, b, s, hq, hk, d, rotary, interleaved, dtype, layout):
    from paper_2609_34162_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(d + hq)
    q, k = heads(gen, b, s, hq, hk, d, dtype, layout)
    dq_out, dk_out = heads(gen, b, s, hq, hk, d, dtype, layout)
    angle = torch.randn((777, rotary // 2), generator=gen, device="cuda") * 3
    cos, sin = angle.cos(), angle.sin()
    positions = torch.randint(0, 777, (b, s), generator=gen, device="cuda", dtype=torch.int32)
    w = [1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2)]
    out, dx = ([torch.full(t.shape, 7.0, dtype=dtype, device="cuda") for t in (q, k)] for _ in range(2))
    dw = [torch.full((d,), 7.0, device="cuda") for _ in range(2)]
    more = dict(q_weight=w[0], k_weight=w[1], positions=positions, eps=EPS, interleaved=interleaved)
    ops.sdp_qk_norm_rope(ctx, q, k, *out, cos, sin, **more)
    ops.sdp_qk_norm_rope_backward(ctx, q, k, dq_out, dk_out, *dx, cos, sin, dq_weight=dw[0], dk_weight=dw[1], **more)
    # the first and last tokens, and a prime step through all of them
    some = torch.cat((torch.arange(0, b * s, max(1, b * s // 400) | 1), torch.arange(b * s - 40, b * s))).unique().cuda()
    at = some // s, some % s
    for x, wt, dy, o, g, gw in ((q, w[0], dq_out, out[0], dx[0], dw[0]), (k, w[1], dk_out, out[1], dx[1], dw[1])):
        part = lambda t: t[at][None]
        common = (cos, sin, positions[at][None], rotary, interleaved, EPS)
        ops_ref.check(part(o), *ops_ref.norm_rope(part(x), wt, *common, dtype), "out")
        ops_ref.check(part(g), *ops_ref.norm_rope_back(part(x), wt, part(dy), *common, dtype, F32)[0], "dx")
        ops_ref.check(gw, *weight_gradient(x, dy, cos, sin, positions, rotary, interleaved), "dw")
        # every row was written
        assert not (o == 7.0).all(-1).any() and not (g == 7.0).all(-1).any()
    # the outputs as their own gradients: every row adds to dw with one sign, so that none can be missing
    ops.sdp_qk_norm_rope_backward(ctx, q, k, *out, *dx, cos, sin, dq_weight=dw[0], dk_weight=dw[1], **more)
    for x, o, gw in ((q, out[0], dw[0]), (k, out[1], dw[1])):
        ops_ref.check(gw, *weight_gradient(x, o, cos, sin, positions, rotary, interleaved), "dw of the outputs")
        assert x.shape[2] == 0 or (gw > 0).all()
