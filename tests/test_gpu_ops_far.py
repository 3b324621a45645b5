"""The training operators where offsets pass 32 bits: rows, sequences, weights
and logits more than 2^31 elements from their tensor's first one."""
import pytest

import gpu_util
import ops_ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    sdp = gpu_util.need_gpu()
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)
    torch.cuda.empty_cache()


def far(gen, shape, strides, dtype, fill=True):
    """A tensor of any strides in memory of its own, which is not filled between its elements."""
    size = 1 + sum((n - 1) * s for n, s in zip(shape, strides))
    assert size > 1 << 31
    t = torch.empty(size, dtype=dtype, device="cuda").as_strided(shape, strides)
    if fill:
        t.copy_(torch.randn(shape, generator=gen))
    return t


# a stride that the tiles take, and one that only the element-wise loads do
@pytest.mark.parametrize("stride", [(1 << 21) - 8, (1 << 21) + 3])
def test_grouped_rows(ctx, stride):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(1)
    rows, n_in, n_out = 1100, 64, 72
    ends = torch.tensor([500, 1090], dtype=torch.int32).cuda()
    x, dy = far(gen, (rows, n_in), (stride, 1), BF16), far(gen, (rows, n_out), (stride, 1), BF16)
    y = far(gen, (rows, n_out), (stride, 1), BF16, fill=False)
    dx = far(gen, (rows, n_in), (stride, 1), BF16, fill=False)
    w = torch.randn((2, n_out, n_in), generator=gen).to(BF16).cuda()
    dw = torch.empty((2, n_out, n_in), dtype=F32, device="cuda")
    ops.sdp_grouped_matmul(ctx, x, w, ends, y)
    ops.sdp_grouped_matmul_backward(ctx, x, w, ends, dy, dx, dw)
    near_x, near_dy = x.contiguous(), dy.contiguous()
    ops_ref.check(y.contiguous(), *ops_ref.grouped(near_x, w, ends, BF16), "y")
    (rx, bx), (rw, bw) = ops_ref.grouped_back(near_x, w, ends, near_dy, F32)
    ops_ref.check(dx.contiguous(), rx, bx, "dx")
    ops_ref.check(dw, rw, bw, "dw")


# whole pieces in every row, or (1,025 wide) not
@pytest.mark.parametrize("n_in,n_out", [(1032, 1048), (1025, 1049)])
def test_grouped_weights(ctx, n_in, n_out):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(2)
    groups, used, rows = 2000, 3, 100
    assert groups * n_in * n_out > 1 << 31
    # all rows go to the last three groups
    last = torch.tensor([40, 41, 100], dtype=torch.int64)
    ends = torch.cat((torch.zeros(groups - used, dtype=torch.int64), last)).cuda()
    x, dy = (torch.randn((rows, n), generator=gen).to(BF16).cuda() for n in (n_in, n_out))
    w = torch.empty((groups, n_out, n_in), dtype=BF16, device="cuda")
    w[:-used] = float("nan")
    w[-used:] = torch.randn((used, n_out, n_in), generator=gen)
    y, dx = torch.empty_like(dy), torch.empty_like(x)
    dw = torch.full((groups, n_out, n_in), 7.0, dtype=BF16, device="cuda")
    ops.sdp_grouped_matmul(ctx, x, w, ends, y)
    ops.sdp_grouped_matmul_backward(ctx, x, w, ends, dy, dx, dw)
    near_w, near_ends = w[-used:].contiguous(), last.cuda()
    ops_ref.check(y, *ops_ref.grouped(x, near_w, near_ends, BF16), "y")
    (rx, bx), (rw, bw) = ops_ref.grouped_back(x, near_w, near_ends, dy, BF16)
    ops_ref.check(dx, rx, bx, "dx")
    ops_ref.check(dw[-used:], rw, bw, "dw")
    assert not dw[:-used].any()  # groups without rows


# heads apart and tokens together, or sequences apart; even and odd strides
@pytest.mark.parametrize("strides", [((1 << 31) + 64, 1024, 128, 1), (128, 1024, (1 << 30) + 8, 1),
                                     ((1 << 31) + 3, 1031, 129, 1)])
def test_qk(ctx, strides):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(3)
    b, s, h, d = 2, 5, 4, 128
    if strides[0] == 128:
        b = 1
        strides = (5 * 1024,) + strides[1:]
    q, dy = far(gen, (b, s, h, d), strides, BF16), far(gen, (b, s, h, d), strides, BF16)
    out, dq = far(gen, (b, s, h, d), strides, BF16, fill=False), far(gen, (b, s, h, d), strides, BF16, fill=False)
    k = torch.empty((b, s, 0, d), dtype=BF16, device="cuda")
    angle = torch.randn((16, d // 2), generator=gen)
    cos, sin = angle.cos().cuda(), angle.sin().cuda()
    w = (1 + 0.2 * torch.randn(d, generator=gen)).cuda()
    dw = torch.empty_like(w)
    ops.sdp_qk_norm_rope(ctx, q, k, out, k, cos, sin, q_weight=w, k_weight=w, eps=1e-6)
    ops.sdp_qk_norm_rope_backward(ctx, q, k, dy, k, dq, k, cos, sin, q_weight=w, k_weight=w, dq_weight=dw, eps=1e-6)
    common = (cos, sin, torch.arange(s).expand(b, s), d, False, 1e-6)
    near, near_dy = q.contiguous(), dy.contiguous()
    ops_ref.check(out.contiguous(), *ops_ref.norm_rope(near, w, *common, BF16), "out")
    (rx, bx), (rw, bw) = ops_ref.norm_rope_back(near, w, near_dy, *common, BF16, F32)
    ops_ref.check(dq.contiguous(), rx, bx, "dq")
    ops_ref.check(dw, rw, bw, "dw")


# many rows (held in registers) and few rows far apart (shared by blocks)
@pytest.mark.parametrize("rows,vocab,stride", [(70000, 32000, 32000), (4, 32003, (1 << 30) + 5)])
def test_distill(ctx, rows, vocab, stride):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(4)
    last, k = 3, 16
    z = far(gen, (rows, vocab), (stride, 1), BF16, fill=False)
    dz = far(gen, (rows, vocab), (stride, 1), BF16, fill=False)
    z[:-last] = 0
    z[-last:] = torch.randn((last, vocab), generator=gen).to(BF16).cuda() * 3
    index = torch.randint(0, vocab, (rows, 1), generator=gen) // k + torch.arange(k)
    index = index.clamp(max=vocab - 1).cuda()
    index[:, 1:][index[:, 1:] == index[:, :-1]] = -1
    teacher = torch.randn((rows, k), generator=gen).cuda()
    labels = torch.randint(0, vocab, (rows,), generator=gen).cuda()
    loss, lse = torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")
    g = torch.ones(rows, device="cuda")
    more = dict(teacher_logits=teacher, teacher_index=index, labels=labels, temperature=2.0, distill_weight=1.0,
                label_weight=0.5)
    ops.sdp_distill_loss(ctx, z, loss, lse, row_grad=g, dlogits=dz, **more)
    (rl, bl), (rs, bs), (rg, bg) = ops_ref.distill(z[-last:].contiguous(), teacher[-last:], index[-last:],
                                                   labels[-last:], 2.0, 1.0, 0.5, g[-last:], BF16)
    for again in (False, True):
        ops_ref.check(loss[-last:], rl, bl, "loss")
        ops_ref.check(lse[-last:], rs, bs, "lse")
        ops_ref.check(dz[-last:].contiguous(), rg, bg, "dlogits")
        if not again:
            dz[-last:] = 7.0
            ops.sdp_distill_loss_backward(ctx, z, lse, g, dz, **more)
