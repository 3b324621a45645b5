"""sdp_qk_norm_rope and its backward on the GPU against 64-bit definitions."""
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


def heads(gen, b, s, h, d, dtype, layout, extra=0):
    """A [b, s, h, d] view: of rows with `extra` elements more ("tight": 0),
    of [b, h, s, d] ("heads"), or every element of an odd offset ("odd")."""
    if layout == "heads":
        return torch.randn((b, h, s, d), generator=gen).to(dtype).cuda().transpose(1, 2)
    if layout == "odd":
        flat = torch.randn(1 + b * s * (h * d + 3), generator=gen).to(dtype).cuda()
        return flat[1:].view(b, s, h * d + 3)[:, :, :h * d].unflatten(2, (h, d))
    return torch.randn((b, s, h, d + extra), generator=gen).to(dtype).cuda()[..., :d]


def make(b, s, hq, hk, d, rotary, dtype, wdtype, layout="tight", pos=torch.int64, table=64, seed=0, extra=0,
         weights=True, positions=True):
    gen = torch.Generator().manual_seed(seed)
    st = dict(q=heads(gen, b, s, hq, d, dtype, layout, extra), k=heads(gen, b, s, hk, d, dtype, layout, extra))
    angle = torch.randn((table, rotary // 2), generator=gen) * 3
    st["cos"], st["sin"] = (angle.cos().cuda(), angle.sin().cuda()) if rotary else (None, None)
    st["positions"] = torch.randint(0, table, (b, s), generator=gen).to(pos).cuda() if positions else None
    for n in ("q_weight", "k_weight"):
        st[n] = (1 + 0.2 * torch.randn(d, generator=gen)).to(wdtype).cuda() if weights else None
    st["dq_out"], st["dk_out"] = (heads(gen, b, s, h, d, dtype, layout, extra) for h in (hq, hk))
    return st


def at_of(st, b, s):
    return st["positions"] if st["positions"] is not None else torch.arange(s).expand(b, s)


def check_both(ctx, st, rotary, interleaved, out_layout=None, eps=EPS):
    from paper_2609_34162_amd import ops
    q, k = st["q"], st["k"]
    b, s = q.shape[:2]
    more = dict(q_weight=st["q_weight"], k_weight=st["k_weight"], positions=st["positions"], eps=eps,
                interleaved=interleaved)
    new = lambda t: torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda") if out_layout is None else \
        torch.full((t.shape[0], t.shape[2], t.shape[1], t.shape[3] + 8), 7.0, dtype=t.dtype,
                   device="cuda").transpose(1, 2)[..., :t.shape[3]]
    outs = new(q), new(k)
    ops.sdp_qk_norm_rope(ctx, q, k, *outs, st["cos"], st["sin"], **more)
    grads = new(q), new(k)
    wd = st["q_weight"].dtype if st["q_weight"] is not None else F32
    dws = [torch.full((q.shape[3],), 7.0, dtype=wd, device="cuda") for _ in range(2)]
    ops.sdp_qk_norm_rope_backward(ctx, q, k, st["dq_out"], st["dk_out"], *grads, st["cos"], st["sin"],
                                  dq_weight=dws[0], dk_weight=dws[1], **more)
    for x, w, dy, out, dx, dw, n in ((q, st["q_weight"], st["dq_out"], outs[0], grads[0], dws[0], "q"),
                                     (k, st["k_weight"], st["dk_out"], outs[1], grads[1], dws[1], "k")):
        common = (st["cos"], st["sin"], at_of(st, b, s), rotary, interleaved, eps)
        ops_ref.check(out, *ops_ref.norm_rope(x, w, *common, x.dtype), n + "_out")
        (rx, bx), (rw, bw) = ops_ref.norm_rope_back(x, w, dy, *common, x.dtype, wd)
        ops_ref.check(dx, rx, bx, "d" + n)
        ops_ref.check(dw, rw, bw, f"d{n}_weight")


@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 64), (64, 64), (96, 96), (80, 32), (256, 256), (512, 128),
                                      (40, 20), (20, 20), (7, 6), (2, 2), (1024, 1024), (3, 0), (128, 0), (1, 0)])
def test_head_sizes(ctx, d, rotary, interleaved, dtype, wdtype):
    check_both(ctx, make(2, 5, 3, 2, d, rotary, dtype, wdtype, seed=d), rotary, interleaved)


@pytest.mark.parametrize("layout", ["tight", "heads", "odd"])
@pytest.mark.parametrize("b,s,hq,hk", [(1, 1, 1, 1), (1, 1, 40, 8), (3, 17, 5, 1), (2, 1, 64, 64), (1, 333, 4, 0),
                                       (5, 2, 0, 3), (0, 4, 2, 2), (2, 0, 2, 2), (17, 1, 1, 1), (1, 4097, 2, 1)])
def test_shapes_and_strides(ctx, b, s, hq, hk, layout):
    check_both(ctx, make(b, s, hq, hk, 64, 64, BF16, BF16, layout, seed=b + s), 64, False, out_layout="heads")
    check_both(ctx, make(b, s, hq, hk, 32, 16, F32, F32, layout, torch.int32, extra=4, seed=s), 16, True)


def test_no_weights_no_positions(ctx):
    check_both(ctx, make(2, 9, 2, 1, 64, 64, BF16, F32, weights=False, positions=False), 64, False)


def test_rows_of_zeros_and_large_values(ctx):
    st = make(1, 6, 2, 2, 64, 64, F32, F32)
    st["q"][:, 0] = 0.0
    st["k"][:, 1] = 1e15
    st["q"][:, 2] = 1e-15
    check_both(ctx, st, 64, False)
    check_both(ctx, st, 64, False, eps=1e-3)


def test_positions_outside_the_table_give_nan(ctx):
    from paper_2609_34162_amd import ops
    for d in (128, 20):
        st = make(1, 8, 2, 1, d, d // 2, BF16, F32, table=16)
        st["positions"][0, 2], st["positions"][0, 5] = 16, -1
        outs = torch.empty_like(st["q"]), torch.empty_like(st["k"])
        ops.sdp_qk_norm_rope(ctx, st["q"], st["k"], *outs, st["cos"], st["sin"], positions=st["positions"], eps=EPS)
        for x, o in zip((st["q"], st["k"]), outs):
            want = ops_ref.norm_rope(x, None, st["cos"], st["sin"], st["positions"], d // 2, False, EPS, BF16)
            assert torch.isnan(want[0][0, 2]).all() and torch.isnan(want[0][0, 5]).all()
            ops_ref.check(o, *want, "out")


@pytest.mark.parametrize("d", [128, 36])
def test_in_place_and_fused(ctx, d):
    """In place over heads of one fused tensor: the bits of the call with outputs of its own."""
    from paper_2609_34162_amd import ops
    st = make(2, 33, 1, 1, d, d, BF16, BF16, seed=3)
    fused = torch.randn((2, 33, 10, d), device="cuda").to(BF16)
    grad = torch.randn((2, 33, 10, d), device="cuda").to(BF16)
    q, k, dq, dk = fused[:, :, :6], fused[:, :, 6:8], grad[:, :, :6], grad[:, :, 6:8]
    kept = fused[:, :, 8:].clone(), grad[:, :, 8:].clone()
    more = dict(q_weight=st["q_weight"], k_weight=st["k_weight"], positions=st["positions"], eps=EPS)
    dws = [[torch.empty(d, dtype=BF16, device="cuda") for _ in range(2)] for _ in range(2)]
    out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k)
    ops.sdp_qk_norm_rope(ctx, q, k, *out[:2], st["cos"], st["sin"], **more)
    ops.sdp_qk_norm_rope_backward(ctx, q, k, dq, dk, *out[2:], st["cos"], st["sin"], dq_weight=dws[0][0],
                                  dk_weight=dws[0][1], **more)
    ops.sdp_qk_norm_rope_backward(ctx, q, k, dq, dk, dq, dk, st["cos"], st["sin"], dq_weight=dws[1][0],
                                  dk_weight=dws[1][1], **more)
    ops.sdp_qk_norm_rope(ctx, q, k, q, k, st["cos"], st["sin"], **more)
    for a, b in zip(out + tuple(dws[0]), (q, k, dq, dk) + tuple(dws[1])):
        assert torch.equal(a, b)
    assert torch.equal(kept[0], fused[:, :, 8:]) and torch.equal(kept[1], grad[:, :, 8:])


def test_broadcast_gradient(ctx):
    st = make(2, 9, 4, 2, 64, 64, BF16, F32)
    st["dq_out"] = torch.randn((1, 1, 1, 64), device="cuda").to(BF16).expand(2, 9, 4, 64)
    check_both(ctx, st, 64, False)


def test_gradient_against_differences(ctx):
    """<dx, v> and <dw, v> against central differences of <y, dy> in 64 bits."""
    from paper_2609_34162_amd import ops
    st = make(1, 7, 3, 2, 64, 32, F32, F32, seed=11)
    dx = torch.empty_like(st["q"]), torch.empty_like(st["k"])
    dw = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    ops.sdp_qk_norm_rope_backward(ctx, st["q"], st["k"], st["dq_out"], st["dk_out"], *dx, st["cos"], st["sin"],
                                  q_weight=st["q_weight"], k_weight=st["k_weight"], dq_weight=dw[0], dk_weight=dw[1],
                                  positions=st["positions"], eps=EPS)
    x, w, dy = st["q"].cpu().double(), st["q_weight"].cpu().double(), st["dq_out"].cpu().double()
    value = lambda x, w: (ops_ref.norm_rope(x, w, st["cos"], st["sin"], st["positions"], 32, False, EPS, F32)[0] * dy).sum()
    gen = torch.Generator().manual_seed(5)
    h = 1e-5
    for _ in range(4):
        v = torch.randn(x.shape, generator=gen).double()
        want = (value(x + h * v, w) - value(x - h * v, w)) / (2 * h)
        got = (dx[0].cpu().double() * v).sum()
        # differences: h^2 of third derivatives (about 1) and 1e-16 / h of rounding, over 1,344 elements; 32 bits of dx
        assert abs(want - got) <= 1e-5 * (dx[0].cpu().double() * v).abs().sum(), (want, got)
        u = torch.randn(64, generator=gen).double()
        want = (value(x, w + h * u) - value(x, w - h * u)) / (2 * h)
        assert abs(want - (dw[0].cpu().double() * u).sum()) <= 1e-5 * (dy.abs().sum((0, 1, 2)) * 3 * u.abs()).sum()


def test_same_bits_again_and_on_another_stream(ctx):
    from paper_2609_34162_amd import ops
    st = make(4, 512, 8, 2, 128, 128, BF16, F32, seed=9, table=512)
    got = []
    streams = [None, torch.cuda.Stream(), torch.cuda.Stream(), None]
    torch.cuda.synchronize()
    for s in streams:
        out = [torch.empty_like(t) for t in (st["q"], st["k"])]
        dw = [torch.empty(128, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        ops.sdp_qk_norm_rope_backward(ctx, st["q"], st["k"], st["dq_out"], st["dk_out"], *out, st["cos"], st["sin"],
                                      q_weight=st["q_weight"], k_weight=st["k_weight"], dq_weight=dw[0],
                                      dk_weight=dw[1], positions=st["positions"], stream=s)
        got.append(out + dw)
    torch.cuda.synchronize()
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)
