"""sdp_distill_loss where the logits lie far from zero: a row's loss and gradient
depend on the differences of its logits alone, and those of its teacher's, so the
64-bit values and the bounds are those of the row moved to a largest value of 0.
(The differences of these inputs have no rounding: both sides are multiples of one
power of two, no more than 2^24 of them apart, or one is too far to count.)"""
import pytest

import gpu_util
import ops_ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SOME = [0, 1, 2, 3, 4, 190, 255, 256, 299]


@pytest.fixture(scope="module")
def ctx():
    sdp = gpu_util.need_gpu()
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


def make(rows, vocab, k, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((rows, vocab), generator=gen, device="cuda") * 3
    index = (torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda") + 7 * torch.arange(k, device="cuda")) % vocab
    index[torch.rand(index.shape, generator=gen, device="cuda") < 0.1] = -1
    index[:, 0] = 3
    teacher = torch.randn((rows, k), generator=gen, device="cuda") * 2
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    return z.to(dtype), index, teacher, labels, torch.rand(rows, generator=gen, device="cuda") + 0.5


def check(ctx, z, index, teacher, labels, g, tau, a=0.6, b=0.4):
    from paper_2609_34162_amd import ops
    rows, vocab = z.shape
    more = dict(teacher_logits=teacher, teacher_index=index, labels=labels, temperature=tau, distill_weight=a,
                label_weight=b)
    alone, loss, lse = (torch.full(s, 7.0, device="cuda") for s in ((rows,), (rows,), (rows, 2)))
    d = torch.full_like(z, 7.0)
    ops.sdp_distill_loss(ctx, z, alone, None, **more)
    ops.sdp_distill_loss(ctx, z, loss, lse, row_grad=g, dlogits=d, **more)
    some = [r for r in SOME if r < rows]
    part = lambda t: t[some].cpu()
    zs = part(z).double()
    zs = zs - zs.max(1, keepdim=True).values
    there, ts = part(index) >= 0, part(teacher).double()
    ts = ts - torch.where(there, ts, -float("inf")).max(1, keepdim=True).values
    (rl, bl), _, (rg, bg) = ops_ref.distill(zs, ts, part(index), part(labels), tau, a, b, part(g), z.dtype)
    ops_ref.check(alone[some], rl, bl, "loss alone")
    ops_ref.check(loss[some], rl, bl, "loss")
    ops_ref.check(d[some], rg, bg, "dlogits")


@pytest.mark.parametrize("rows,vocab", [(3, 1000), (5, 40003), (300, 2003), (300, 40003)])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0, 3.5])
@pytest.mark.parametrize("shift", [-1e5, 1e5])
def test_logits_moved_by_a_constant(ctx, rows, vocab, tau, shift):
    z, index, teacher, labels, g = make(rows, vocab, 16, F32, vocab)
    check(ctx, z + shift, index, teacher, labels, g, tau)
    check(ctx, z, index, teacher + shift, labels, g, tau)
    check(ctx, (z.to(BF16).float() + shift).to(BF16), index, teacher.to(BF16), labels, g, tau)


@pytest.mark.parametrize("rows,vocab", [(3, 1000), (5, 40003), (300, 2003), (300, 40003)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
def test_rows_of_the_lowest_value(ctx, rows, vocab, dtype, tau):
    """All alike: an even distribution over the vocabulary, or over the teacher's entries."""
    z, index, teacher, labels, g = make(rows, vocab, 16, dtype, 5)
    z[0] = z[rows - 1] = torch.finfo(dtype).min
    z[1, 3] = torch.finfo(dtype).max  # and all that there is at the other end
    labels[1] = 3
    index[1] = -1
    index[1, 0] = 3
    teacher[0] = teacher[2] = torch.finfo(BF16).min  # (that of 32 bits would be rounded to minus infinity)
    check(ctx, z, index, teacher, labels, g, tau)
    check(ctx, z, index, teacher.to(BF16), labels, g, tau)
