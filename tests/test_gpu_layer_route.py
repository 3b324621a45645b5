"""sdp_route and its backward on the GPU against 64-bit definitions."""
import itertools

import pytest

import gpu_util
import layer_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
I32, I64 = torch.int32, torch.int64
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    sdp = gpu_util.need_gpu()
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


def logits(t, e, dtype, seed=0, pad=0, sigma=1.5):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn((t, e + pad), generator=gen) * sigma).to(dtype).cuda()[:, :e]


def check(ctx, z, top, bias=None, sigmoid=False, groups=1, top_groups=1, group_best=1, renormalize=False, scale=1.0,
          itype=I32, wtype=F32, seed=0):
    from paper_2609_34162_amd import ops
    t, e = z.shape
    index, w = torch.full((t, top), 77, dtype=itype, device="cuda"), torch.full((t, top), 7.0, dtype=wtype, device="cuda")
    ops.sdp_route(ctx, z, index, w, bias=bias, sigmoid=sigmoid, groups=groups, top_groups=top_groups,
                  group_best=group_best, renormalize=renormalize, scale=scale)
    want_i, want_w = ref.route(z, bias, top, sigmoid, groups, top_groups, group_best, renormalize, scale, wtype)
    assert torch.equal(index.cpu().long(), want_i), (index.cpu()[(index.cpu() != want_i).any(1)][:3],
                                                     want_i[(index.cpu() != want_i).any(1)][:3])
    ref.check(w, *want_w, "weights")
    gen = torch.Generator().manual_seed(seed)
    dw = torch.randn((t, top), generator=gen).to(wtype).cuda()
    dz = torch.full(z.shape, 7.0, dtype=z.dtype, device="cuda")
    ops.sdp_route_backward(ctx, z, index, dw, dz, sigmoid=sigmoid, renormalize=renormalize, scale=scale)
    ref.check(dz, *ref.route_back(z, index, dw, sigmoid, renormalize, scale, z.dtype), "dlogits")
    return index, w, dw, dz


@pytest.mark.parametrize("sigmoid,renormalize", list(itertools.product([False, True], [False, True])))
@pytest.mark.parametrize("e,top", [(1, 1), (2, 1), (2, 2), (4, 2), (8, 8), (16, 4), (60, 4), (63, 6), (64, 8), (65, 8),
                                   (96, 6), (128, 8), (160, 6), (256, 8), (257, 5), (384, 8), (512, 10), (1000, 64),
                                   (2048, 8)])
def test_sizes(ctx, e, top, sigmoid, renormalize):
    t = 77 if e < 600 else 21
    gen = torch.Generator().manual_seed(e)
    bias = (0.1 * torch.randn(e, generator=gen)).cuda()
    check(ctx, logits(t, e, F32, e), top, None, sigmoid, renormalize=renormalize, scale=2.5)
    check(ctx, logits(t, e, BF16, e + 1, pad=3), top, bias, sigmoid, renormalize=renormalize, itype=I64, wtype=BF16)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("e,groups,top_groups,best,top", [(256, 8, 4, 2, 8), (64, 8, 3, 2, 6), (160, 8, 3, 1, 6),
                                                          (16, 4, 1, 1, 4), (16, 16, 5, 1, 5), (16, 16, 5, 2, 8),
                                                          (128, 64, 7, 2, 8), (12, 3, 3, 2, 7), (2048, 8, 2, 2, 8),
                                                          (96, 6, 2, 2, 4), (24, 2, 1, 2, 12), (512, 32, 5, 2, 16)])
def test_groups(ctx, e, groups, top_groups, best, top, sigmoid):
    gen = torch.Generator().manual_seed(e + groups)
    bias = (0.1 * torch.randn(e, generator=gen)).cuda()
    for dtype, b in ((F32, bias), (BF16, bias), (BF16, None)):
        check(ctx, logits(55, e, dtype, e), top, b, sigmoid, groups, top_groups, best, renormalize=True, scale=2.5)


@pytest.mark.parametrize("t", [0, 1, 2, 5, 63, 64, 65, 1001, 5000])
def test_token_counts(ctx, t):
    check(ctx, logits(t, 128, F32, t), 8, renormalize=True)
    check(ctx, logits(t, 32, BF16, t), 2, torch.zeros(32, device="cuda"), True)
    check(ctx, logits(t, 8, F32, t), 2)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("e,groups", [(64, 1), (64, 8), (10, 1), (300, 1), (256, 4)])
def test_ties_go_to_the_lowest_index(ctx, e, groups, sigmoid):
    gen = torch.Generator().manual_seed(e)
    z = torch.randint(-2, 3, (99, e), generator=gen).float().cuda()
    z[0], z[1] = 0.0, -3.0
    z[2, ::2] = -0.0
    z[2, 1::2] = 0.0
    zero = torch.zeros(e, device="cuda")
    more = dict(groups=groups, top_groups=max(1, groups // 2), group_best=2, renormalize=True)
    check(ctx, z, 6, None, sigmoid, **more)
    check(ctx, z, 6, zero, sigmoid, **more)
    check(ctx, z.to(BF16), 6, torch.randint(-1, 2, (e,), generator=gen).float().cuda(), sigmoid, **more)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_close_scores(ctx, sigmoid):
    """Neighbouring 32-bit logits: their scores differ in 64 bits alone."""
    gen = torch.Generator().manual_seed(8)
    step = 2.0 ** -23
    z = (1.0 + step * torch.randint(0, 40, (200, 64), generator=gen)).float().cuda()
    bias = (1e-7 * torch.randn(64, generator=gen)).cuda()
    check(ctx, z, 8, None, sigmoid, renormalize=True)
    check(ctx, z, 8, bias, sigmoid, renormalize=True)
    check(ctx, z, 8, bias, sigmoid, 8, 3, 2, renormalize=True)


@pytest.mark.parametrize("above", [0, 5, 7, 8])
@pytest.mark.parametrize("size", [2, 9, 10, 15, 17, 40])
def test_clusters_of_close_scores(ctx, size, above):
    """The choice ends before, in or behind a cluster, whose experts follow each other or lie apart."""
    gen = torch.Generator().manual_seed(size)
    e, t = 256, 60
    z = -3.0 + torch.rand((t, e), generator=gen)
    for i in range(t):
        start = int(torch.randint(0, e - size, (1,), generator=gen))
        at = torch.arange(start, start + size) if i % 2 else torch.randperm(e, generator=gen)[:size]
        z[i, at] = 1.0 + 2.0 ** -23 * torch.randperm(size, generator=gen)
        z[i, (at[-1] + 1 + 7 * torch.arange(above)) % e] = 2.0 + 0.1 * torch.arange(above)
    z, bias = z.cuda(), (1e-7 * torch.randn(e, generator=gen)).cuda()
    for sigmoid in (False, True):
        check(ctx, z, 8, None, sigmoid)
        check(ctx, z, 8, bias, sigmoid, renormalize=True)
        check(ctx, z, 8, bias, sigmoid, 8, 4, 2)


@pytest.mark.parametrize("sigmoid,renormalize", list(itertools.product([False, True], [False, True])))
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_experts(ctx, sigmoid, renormalize, dtype):
    """Minus infinity, in some, all but a few, or all places of a row; rows of the type's lowest value."""
    e = 48
    z = logits(40, e, dtype, 3)
    gen = torch.Generator().manual_seed(1)
    z[torch.rand((40, e), generator=gen).cuda() < 0.5] = -INF
    z[3] = -INF
    z[4], z[4, 47] = -INF, 0.5
    z[5], z[5, 40:43] = -INF, torch.tensor([1.0, -2.0, 1.0]).to(dtype).cuda()
    z[6] = torch.finfo(dtype).min
    z[7, :5] = torch.finfo(dtype).min
    for bias in (None, torch.randn(e, generator=gen).cuda()):
        check(ctx, z, 6, bias, sigmoid, renormalize=renormalize)
        check(ctx, z, 6, bias, sigmoid, 8, 3, 2, renormalize=renormalize)
    bias = torch.zeros(e, device="cuda")
    bias[::3] = -INF
    check(ctx, z, 6, bias, sigmoid, renormalize=renormalize)
    check(ctx, z, 6, bias, sigmoid, 16, 4, 2, renormalize=renormalize)
    check(ctx, z, 6, torch.full((e,), -INF, device="cuda"), sigmoid, renormalize=renormalize)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_scores_below_any_number(ctx, sigmoid):
    """Chosen by their bias, with scores that 32 bits do not hold: the ratios are still right."""
    z = torch.full((4, 32), -200.0, device="cuda")
    z[:, 3:7] = torch.tensor([-140.0, -141.0, -140.5, -143.0], device="cuda")
    z[1] -= 600.0
    if not sigmoid:
        z[:, 20] = 90.0
    bias = torch.zeros(32, device="cuda")
    bias[3:7] = 5.0
    check(ctx, z, 4, bias, sigmoid, renormalize=True)
    check(ctx, z, 4, bias, sigmoid)


def test_nan_counts_as_the_largest(ctx):
    from paper_2609_34162_amd import ops
    for sigmoid, groups in ((False, 1), (True, 1), (True, 4)):
        z = logits(6, 32, F32, 2)
        clean = z.clone()
        z[2, 9] = float("nan")
        index, w = torch.empty((6, 4), dtype=I32, device="cuda"), torch.empty((6, 4), device="cuda")
        ops.sdp_route(ctx, z, index, w, sigmoid=sigmoid, groups=groups, top_groups=2 if groups > 1 else 1, renormalize=True)
        assert torch.isnan(w).any(1).cpu().tolist() == [i == 2 for i in range(6)]
        assert (index[2] == 9).any() or groups == 1 and not sigmoid
        assert len(set(index[2].tolist())) == 4 and 0 <= int(index.min()) and int(index.max()) < 32
        again = torch.empty_like(index)
        ops.sdp_route(ctx, clean, again, w, sigmoid=sigmoid, groups=groups, top_groups=2 if groups > 1 else 1,
                      renormalize=True)
        keep = [i for i in range(6) if i != 2]
        assert torch.equal(again[keep], index[keep])
    index = torch.empty((1, 1), dtype=I32, device="cuda")
    z = logits(1, 32, F32, 2)
    z[0, 30] = float("nan")
    ops.sdp_route(ctx, z, index, torch.empty((1, 1), device="cuda"))
    assert int(index) == 30


def test_infinite_logits(ctx):
    """A sigmoid of infinity is 1; a softmax over it has no value, and its indexes are still experts."""
    from paper_2609_34162_amd import ops
    z = logits(5, 16, F32, 2)
    z[1, 7] = INF
    check(ctx, z, 3, None, True, renormalize=True)
    index, w = torch.empty((5, 3), dtype=I32, device="cuda"), torch.empty((5, 3), device="cuda")
    ops.sdp_route(ctx, z, index, w)
    assert torch.isnan(w[1, 0]) and int(index[1, 0]) == 7 and not torch.isnan(w[[0, 2, 3, 4]]).any()
    assert ((index >= 0) & (index < 16)).all()


def test_indexes_out_of_range_backward(ctx):
    from paper_2609_34162_amd import ops
    z = logits(6, 20, F32, 4)
    index = torch.tensor([[0, 1], [20, 3], [-1, 4], [5, 1 << 40], [-1, -7], [19, 18]]).cuda()
    dw = torch.randn((6, 2), device="cuda")
    for sigmoid, renormalize in itertools.product([False, True], [False, True]):
        dz = torch.empty_like(z)
        ops.sdp_route_backward(ctx, z, index, dw, dz, sigmoid=sigmoid, renormalize=renormalize)
        ref.check(dz, *ref.route_back(z, index, dw, sigmoid, renormalize, 1.0, F32), "dlogits")


def test_an_index_twice_counts_twice(ctx):
    from paper_2609_34162_amd import ops
    z = logits(3, 70, F32, 4)
    index = torch.tensor([[5, 5, 5], [69, 1, 69], [0, -1, 0]], dtype=I32).cuda()
    dw = torch.randn((3, 3), device="cuda")
    for sigmoid, renormalize in itertools.product([False, True], [False, True]):
        dz = torch.empty_like(z)
        ops.sdp_route_backward(ctx, z, index, dw, dz, sigmoid=sigmoid, renormalize=renormalize, scale=0.5)
        ref.check(dz, *ref.route_back(z, index, dw, sigmoid, renormalize, 0.5, F32), "dlogits")


@pytest.mark.parametrize("e", [8, 60, 128, 500])
def test_gradient_in_place(ctx, e):
    from paper_2609_34162_amd import ops
    for sigmoid, renormalize in itertools.product([False, True], [False, True]):
        z = logits(90, e, BF16, e, pad=5)
        index, w, dw, dz = check(ctx, z, 4, None, sigmoid, renormalize=renormalize)
        ops.sdp_route_backward(ctx, z, index, dw, z, sigmoid=sigmoid, renormalize=renormalize)
        assert torch.equal(z, dz)


def test_broadcast_logits(ctx):
    check(ctx, logits(1, 64, F32, 9).expand(30, 64), 8, renormalize=True)


def test_gradient_against_differences(ctx):
    """<dlogits, v> against central differences of <weights, dw> in 64 bits, the choice held."""
    for sigmoid, renormalize in itertools.product([False, True], [False, True]):
        z = logits(7, 40, F32, 6)
        index, w, dw, dz = check(ctx, z, 5, None, sigmoid, renormalize=renormalize, scale=1.5)

        def value(x):
            p = ref.scores(x, sigmoid).gather(1, index.cpu().long())
            return (1.5 * (p / p.sum(1, keepdim=True) if renormalize else p) * ref.f64(dw)).sum()
        gen = torch.Generator().manual_seed(5)
        v, step = torch.randn((7, 40), generator=gen).double(), 1e-5
        want = (value(ref.f64(z) + step * v) - value(ref.f64(z) - step * v)) / (2 * step)
        # step^2 of third derivatives (below 1), 1e-16 / step of rounding; 32 bits of dlogits
        assert abs(want - (ref.f64(dz) * v).sum()) <= 1e-5 * (ref.f64(dz) * v).abs().sum() + 1e-9


def test_same_bits_again_and_on_another_stream(ctx):
    from paper_2609_34162_amd import ops
    z, bias = logits(6000, 256, BF16, 1), torch.randn(256, device="cuda") * 0.1
    got = []
    for s in (None, torch.cuda.Stream(), None):
        index, w = torch.empty((6000, 8), dtype=I64, device="cuda"), torch.empty((6000, 8), device="cuda")
        dz = torch.empty_like(z)
        torch.cuda.synchronize()
        ops.sdp_route(ctx, z, index, w, bias=bias, sigmoid=True, groups=8, top_groups=4, group_best=2, renormalize=True,
                      stream=s)
        ops.sdp_route_backward(ctx, z, index, w, dz, sigmoid=True, renormalize=True, stream=s)
        got.append((index, w, dz))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))
