"""sdp_expert_order, sdp_expert_gather, sdp_expert_combine and their backward on the
GPU against their definitions, and with sdp_grouped_matmul between them."""
import pytest

import gpu_util
import layer_ref as ref
import ops_ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
I32, I64 = torch.int32, torch.int64


@pytest.fixture(scope="module")
def ctx():
    sdp = gpu_util.need_gpu()
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


def choice(t, k, experts, absent=0.1, seed=0, skew=0.0):
    gen = torch.Generator().manual_seed(seed)
    index = (torch.rand((t, k), generator=gen) ** (1 + skew) * experts).long().clamp(max=max(0, experts - 1))
    gone = torch.rand((t, k), generator=gen) < (1.0 if experts == 0 else absent)
    return torch.where(gone, torch.randint(-5, 0, (t, k), generator=gen), index)


def sort(ctx, index, experts, etype=I32, with_order=True):
    from paper_2609_34162_amd import ops
    ends = torch.full((experts,), 77, dtype=etype, device="cuda")
    place = torch.full(index.shape, 77, dtype=I32, device="cuda")
    order = torch.full((index.numel(),), 77, dtype=I32, device="cuda") if with_order else None
    ops.sdp_expert_order(ctx, index, ends, place, order)
    return ends, place, order


def check_order(ctx, index, experts, itype=I32, etype=I32):
    ends, place, order = sort(ctx, index.to(itype).cuda(), experts, etype)
    want = ref.order(index, experts)
    for got, w, name in zip((ends, place, order), want, ("ends", "place", "order")):
        assert torch.equal(got.cpu().long(), w), name
    alone = sort(ctx, index.to(itype).cuda(), experts, etype, with_order=False)
    assert torch.equal(alone[0], ends) and torch.equal(alone[1], place)


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 511, 2047, 2048, 2049, 4095, 4096, 4097, 6143, 6144, 10000, 50001])
@pytest.mark.parametrize("experts", [1, 2, 3, 8, 60, 128])
def test_order_of_counts(ctx, n, experts):
    check_order(ctx, choice(n, 1, experts, seed=n), experts, I64 if n % 2 else I32, I32 if n % 2 else I64)


@pytest.mark.parametrize("experts", [0, 1, 5, 64, 127, 255, 256, 257, 1000, 2047, 2048])
def test_order_of_experts(ctx, experts):
    for n in (30, 5000, 20000):
        check_order(ctx, choice(n, 1, experts, seed=experts), experts)


@pytest.mark.parametrize("n", [1024, 1025, 40960, 40961, 131072, 131073])
@pytest.mark.parametrize("experts", [128, 511, 512, 1024, 2048])
def test_order_around_its_ways(ctx, n, experts):
    """One block, one launch and three launches; few digits and many."""
    check_order(ctx, choice(n, 1, experts, seed=n + experts), experts)


def test_order_of_skewed_choices(ctx):
    for index in (torch.zeros(9000, 1), torch.full((9000, 1), 15), torch.full((9000, 1), -1),
                  torch.arange(9000)[:, None] % 16, 15 - torch.arange(9000)[:, None] * 16 // 9000):
        check_order(ctx, index.long(), 16)
    check_order(ctx, choice(40000, 2, 100, 0.3, seed=5, skew=6.0), 100)


def test_order_of_indexes_out_of_range(ctx):
    index = torch.tensor([[0, 1 << 40], [3, -(1 << 40)], [4, 1], [(1 << 32) + 1, 2], [1 << 31, 3]])
    check_order(ctx, index, 4, I64)


def test_order_of_many_entries(ctx):
    """More than 1,024 blocks of entries: several steps to a block."""
    n, experts = (1 << 21) * 2 + 4321, 37
    gen = torch.Generator().manual_seed(2)
    index = torch.randint(-1, experts, (n,), generator=gen).to(I32)
    ends, place, order = sort(ctx, index.cuda(), experts)
    key = torch.where(index < 0, experts, index)
    want = torch.sort(key, stable=True).indices
    routed = int((index >= 0).sum())
    assert torch.equal(order.cpu()[:routed].long(), want[:routed]) and (order[routed:] == -1).all()
    at = torch.empty(n, dtype=I64)
    at[want] = torch.arange(n)
    assert torch.equal(place.cpu().long(), torch.where(index < 0, -1 - at, at))
    assert torch.equal(ends.cpu().long(), torch.bincount(key, minlength=experts + 1).cumsum(0)[:experts])


def rows(gen, n, h, dtype, pad=0, first=0):
    flat = torch.randn(first + n * (h + pad), generator=gen).to(dtype).cuda()
    return flat[first:].view(n, h + pad)[:, :h]


def check_rows(ctx, t, k, experts, h, dtype=BF16, stream=BF16, wtype=F32, pad=0, first=0, absent=0.1, seed=0):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(seed)
    index = choice(t, k, experts, absent, seed).cuda()
    _, place, _ = sort(ctx, index, experts)
    n = t * k
    make = lambda count, kind: rows(gen, count, h, kind, pad, first)
    x, out = make(t, dtype), make(n, dtype)
    ops.sdp_expert_gather(ctx, x, place, out)
    assert torch.equal(out.cpu(), ref.gather(x, place)), "rows"
    drows, dx = make(n, dtype), make(t, dtype)
    ops.sdp_expert_gather_backward(ctx, drows, place, dx)
    ref.check(dx, *ref.combine(drows, place, None, None, dtype), "dx")
    w = torch.rand((t, k), generator=gen).to(wtype).cuda()
    y, residual, total = make(n, dtype), make(t, stream), make(t, stream)
    for res in (residual, None):
        ops.sdp_expert_combine(ctx, y, place, w, total, residual=res)
        ref.check(total, *ref.combine(y, place, w, res, stream), "out")
    dout, dy, dw = make(t, stream), make(n, dtype), torch.full((t, k), 7.0, dtype=wtype, device="cuda")
    ops.sdp_expert_combine_backward(ctx, y, place, w, dout, dy, dw)
    want_y, want_w = ref.combine_back(y, place, w, dout, dtype, wtype)
    ref.check(dy, *want_y, "drows")
    ref.check(dw, *want_w, "dweights")
    # each alone
    alone_y, alone_w = make(n, dtype), torch.full_like(dw, 7.0)
    ops.sdp_expert_combine_backward(ctx, None, place, w, dout, alone_y, None)
    ops.sdp_expert_combine_backward(ctx, y, place, None, dout, None, alone_w)
    assert torch.equal(alone_y, dy) and torch.equal(alone_w, dw)
    # in place
    into = residual.clone()
    ops.sdp_expert_combine(ctx, y, place, w, total, residual=residual)
    ops.sdp_expert_combine(ctx, y, place, w, into, residual=into)
    assert torch.equal(into, total)
    over = y.clone()
    own = torch.empty_like(dw)
    ops.sdp_expert_combine_backward(ctx, over, place, w, dout, over, own)
    assert torch.equal(over, dy) and torch.equal(own, dw)


@pytest.mark.parametrize("dtype,stream,wtype", [(BF16, BF16, F32), (F32, F32, F32), (BF16, F32, BF16), (F32, BF16, F32)])
@pytest.mark.parametrize("h", [1, 7, 8, 9, 100, 120, 128, 129, 208, 256, 257, 512, 513, 550, 1000, 1024, 2048, 5000])
def test_hidden_sizes_and_types(ctx, h, dtype, stream, wtype):
    check_rows(ctx, 37, 3, 5, h, dtype, stream, wtype, seed=h)


@pytest.mark.parametrize("t", [0, 1, 2, 8, 64, 333])
@pytest.mark.parametrize("k", [1, 2, 6, 8, 9, 33])
def test_token_counts(ctx, t, k):
    check_rows(ctx, t, k, 64, 136, seed=t + k)


@pytest.mark.parametrize("pad,first", [(1, 0), (0, 1), (3, 5), (8, 0)])
def test_strides_and_alignment(ctx, pad, first):
    for h in (136, 1003):
        check_rows(ctx, 50, 4, 9, h, BF16, BF16, F32, pad, first, seed=pad)
        check_rows(ctx, 50, 4, 9, h, F32, BF16, BF16, pad, first, seed=pad)


@pytest.mark.parametrize("absent", [0.0, 1.0])
def test_all_or_no_entries(ctx, absent):
    check_rows(ctx, 70, 2, 6, 200, absent=absent)


def test_no_entries_to_a_token(ctx):
    """top = 0: nothing is chosen; outputs of tokens are the residual, or zeros."""
    from paper_2609_34162_amd import ops
    place, none = torch.empty((5, 0), dtype=I32, device="cuda"), torch.empty((0, 40), device="cuda")
    w, residual = torch.empty((5, 0), device="cuda"), torch.randn((5, 40), device="cuda")
    out = torch.full((5, 40), 7.0, device="cuda")
    ops.sdp_expert_combine(ctx, none, place, w, out, residual=residual)
    assert torch.equal(out, residual)
    ops.sdp_expert_combine(ctx, none, place, w, out)
    assert (out == 0).all()
    out.fill_(7.0)
    ops.sdp_expert_gather_backward(ctx, none, place, out)
    assert (out == 0).all()
    ops.sdp_expert_gather(ctx, residual, place, none)


def test_no_columns(ctx):
    from paper_2609_34162_amd import ops
    place = torch.tensor([[0, 1], [2, -4]], dtype=I32).cuda()
    none = lambda n: torch.empty((n, 0), device="cuda")
    dw = torch.full((2, 2), 7.0, device="cuda")
    ops.sdp_expert_combine_backward(ctx, none(4), place, dw.clone(), none(2), none(4), dw)
    assert (dw == 0).all()
    ops.sdp_expert_combine(ctx, none(4), place, dw, none(2))
    ops.sdp_expert_gather(ctx, none(2), place, none(4))


@pytest.mark.parametrize("h", [64, 1003])
def test_places_that_name_no_row(ctx, h):
    """Never an address: sums over them are NaN, nothing is written for them."""
    from paper_2609_34162_amd import ops
    place = torch.tensor([[0, 5], [6, 1], [-7, 2], [2 ** 31 - 1, -2 ** 31]], dtype=I32).cuda()
    place[0, 1] = 4
    t, k, n = 4, 2, 8
    place[1, 0] = 8
    place[2, 0] = -9
    x = torch.randn((t, h), device="cuda")
    out = torch.full((n, h), 7.0, device="cuda")
    ops.sdp_expert_gather(ctx, x, place, out)
    named = {0: 0, 4: 0, 1: 1, 2: 2}
    for p in range(n):
        assert torch.equal(out[p], x[named[p]]) if p in named else (out[p] == 7.0).all()
    y, w = torch.randn((n, h), device="cuda"), torch.rand((t, k), device="cuda")
    total = torch.empty((t, h), device="cuda")
    ops.sdp_expert_combine(ctx, y, place, w, total)
    ref.check(total, *ref.combine(y, place, w, None, F32), "out")
    assert torch.isnan(total).any(1).cpu().tolist() == [False, True, False, True]
    dy, dw = torch.full((n, h), 7.0, device="cuda"), torch.empty((t, k), device="cuda")
    ops.sdp_expert_combine_backward(ctx, y, place, w, x, dy, dw)
    assert torch.isnan(dw).cpu().tolist() == [[False, False], [True, False], [False, False], [True, False]]
    for p in (3, 5, 6, 7):
        assert (dy[p] == 7.0).all()


def test_rows_without_an_entry_do_not_matter(ctx):
    """NaN in the rows past the last end reach no output, whatever their weight."""
    from paper_2609_34162_amd import ops
    index = torch.tensor([[1, -1], [0, 2], [-1, -1]]).cuda()
    _, place, _ = sort(ctx, index, 3)
    y, w = torch.randn((6, 72), device="cuda"), torch.rand((3, 2), device="cuda")
    y[3:] = float("nan")
    w[2, 1] = float("nan")
    out, dw, dy = torch.empty((3, 72), device="cuda"), torch.empty((3, 2), device="cuda"), torch.empty_like(y)
    ops.sdp_expert_combine(ctx, y, place, w, out)
    ops.sdp_expert_combine_backward(ctx, y, place, w, torch.ones((3, 72), device="cuda"), dy, dw)
    assert not torch.isnan(out).any() and (out[2] == 0).all()
    assert not torch.isnan(dw).any() and (dw[2] == 0).all() and dw[0, 1] == 0
    assert (dy[3:] == 0).all()


def test_bits_are_moved_as_they_are(ctx):
    """Gathering copies NaN payloads, infinities and -0 bit by bit."""
    from paper_2609_34162_amd import ops
    bits = torch.tensor([0x7f81, 0xffc3, 0x7f80, 0xff80, 0x8000, 0x0001, 0x7fff, 0x8001] * 9, dtype=torch.int32)
    x = bits.to(torch.int16).view(1, 72).repeat(3, 1).cuda().view(BF16)
    place = torch.tensor([[2], [0], [1]], dtype=I32).cuda()
    out = torch.empty_like(x)
    ops.sdp_expert_gather(ctx, x, place, out)
    assert torch.equal(out.view(torch.int16), x.view(torch.int16))


def test_with_the_grouped_products(ctx):
    """order, gather, sdp_grouped_matmul, combine and back, against each token's own experts in 64 bits."""
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(3)
    t, k, experts, h = 150, 3, 10, 96
    index = choice(t, k, experts, 0.1, 7).to(I32).cuda()
    ends, place, _ = sort(ctx, index, experts)
    x, wexp = rows(gen, t, h, BF16), (torch.randn((experts, h, h), generator=gen) * 0.1).to(BF16).cuda()
    gathered, y = torch.empty((t * k, h), dtype=BF16, device="cuda"), torch.empty((t * k, h), device="cuda")
    weights, out = torch.rand((t, k), generator=gen).cuda(), torch.empty((t, h), device="cuda")
    ops.sdp_expert_gather(ctx, x, place, gathered)
    ops.sdp_grouped_matmul(ctx, gathered, wexp, ends, y)
    ops.sdp_expert_combine(ctx, y, place, weights, out)
    want, size = torch.zeros((t, h), dtype=torch.float64), torch.zeros((t, h), dtype=torch.float64)
    x64, w64 = ref.f64(x), ref.f64(wexp)
    for i in range(t):
        for j in range(k):
            e = int(index[i, j])
            if e >= 0:
                want[i] += float(weights[i, j]) * (w64[e] @ x64[i])
                size[i] += float(weights[i, j]) * (w64[e].abs() @ x64[i].abs())
    ref.check(out, want, ref.rounded(want, F32, (2 * h + k + 8) * ref.U32 * size), "out")


def test_same_bits_again_and_on_another_stream(ctx):
    from paper_2609_34162_amd import ops
    index = choice(5000, 8, 64, 0.05, 1).to(I32).cuda()
    gen = torch.Generator().manual_seed(1)
    y, w, dout = rows(gen, 40000, 256, BF16), torch.rand((5000, 8), generator=gen).cuda(), rows(gen, 5000, 256, BF16)
    got = []
    for s in (None, torch.cuda.Stream(), None):
        ends, place = torch.empty(64, dtype=I32, device="cuda"), torch.empty((5000, 8), dtype=I32, device="cuda")
        out, dy, dw = torch.empty_like(dout), torch.empty_like(y), torch.empty_like(w)
        torch.cuda.synchronize()
        ops.sdp_expert_order(ctx, index, ends, place, stream=s)
        ops.sdp_expert_combine(ctx, y, place, w, out, stream=s)
        ops.sdp_expert_combine_backward(ctx, y, place, w, dout, dy, dw, stream=s)
        got.append((ends, place, out, dy, dw))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))


def test_gradients_against_differences(ctx):
    """<gradient, direction> against differences of <output, its gradient> in 64 bits; each output
    is linear in each input, so they are exact."""
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(6)
    t, k, experts, h = 40, 3, 7, 70
    _, place, _ = sort(ctx, choice(t, k, experts, 0.2, 2).to(I32).cuda(), experts)
    make = lambda *shape: torch.randn(shape, generator=gen).cuda()
    y, w, dout, drows = make(t * k, h), make(t, k), make(t, h), make(t * k, h)
    dy, dw, dx = torch.empty_like(y), torch.empty_like(w), torch.empty_like(dout)
    ops.sdp_expert_combine_backward(ctx, y, place, w, dout, dy, dw)
    ops.sdp_expert_gather_backward(ctx, drows, place, dx)

    def combined(rows64, weights64):
        return (ref.combine(rows64, place, weights64, None, F32)[0] * ref.f64(dout)).sum()

    def gathered(x64):
        return (ref.f64(ref.gather(x64, place)) * ref.f64(drows)).sum()
    vy, vw, vx = (torch.randn(s.shape, generator=gen).double() for s in (y, w, dout))
    y64, w64, x64 = ref.f64(y), ref.f64(w), torch.zeros((t, h), dtype=torch.float64)
    # each gradient: a rounded product, a sum of 70 of them, or of three rows
    dw_size = ref.combine_back(y.abs(), place, w, dout.abs(), F32, F32)[1][0]
    dx_size = ref.combine(drows.abs(), place, None, None, F32)[0]
    for got, v, want, size, count in (
            (dy, vy, combined(y64 + vy, w64) - combined(y64, w64), dy, 2),
            (dw, vw, combined(y64, w64 + vw) - combined(y64, w64), dw_size, h + 2),
            (dx, vx, gathered(x64 + vx) - gathered(x64), dx_size, k + 1)):
        assert abs((ref.f64(got) * v).sum() - want) <= (count * ref.U32 + 1e-12) * (ref.f64(size).abs() * v.abs()).sum()
