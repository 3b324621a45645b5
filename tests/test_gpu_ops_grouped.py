"""sdp_grouped_matmul and its backward on the GPU against 64-bit products."""
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


def strided(gen, rows, cols, pad, dtype=BF16, offset=0):
    """[rows, cols], rows cols + pad apart, the first element `offset` past an aligned one; NaN between the rows."""
    flat = torch.full((offset + rows * (cols + pad) + 8,), float("nan"), dtype=dtype)
    t = flat.cuda()[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn((rows, cols), generator=gen))
    return t


def check_all(ctx, counts, n_in, n_out, unused=0, out=BF16, ends=torch.int32, pad=0, offset=0, seed=0, want_ends=None):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(seed)
    rows, groups = sum(counts) + unused, len(counts)
    e = torch.tensor(counts, dtype=torch.int64).cumsum(0).to(ends).cuda() if want_ends is None else \
        torch.tensor(want_ends, dtype=ends).cuda()
    x, dy = strided(gen, rows, n_in, pad, offset=offset), strided(gen, rows, n_out, pad, offset=offset)
    if unused:
        # what lies in rows of no group is not used
        x[rows - unused:] = float("inf")
        dy[rows - unused:] = float("nan")
    w = strided(gen, groups * n_out, n_in, 0, offset=offset).view(groups, n_out, n_in)
    y = torch.full((rows, n_out + pad), 7.0, dtype=out, device="cuda")[:, :n_out]
    dx = torch.full((rows, n_in + pad), 7.0, dtype=BF16, device="cuda")[:, :n_in]
    dw = torch.full((groups, n_out, n_in), 7.0, dtype=out, device="cuda")
    ops.sdp_grouped_matmul(ctx, x, w, e, y)
    ops.sdp_grouped_matmul_backward(ctx, x, w, e, dy, dx, dw)
    ops_ref.check(y, *ops_ref.grouped(x, w, e, out), "y")
    (rx, bx), (rw, bw) = ops_ref.grouped_back(x, w, e, dy, out)
    ops_ref.check(dx, rx, bx, "dx")
    ops_ref.check(dw, rw, bw, "dw")
    if pad:
        assert (y.as_strided((rows, pad), (n_out + pad, 1), y.storage_offset() + n_out) == 7).all()
        assert (dx.as_strided((rows, pad), (n_in + pad, 1), dx.storage_offset() + n_in) == 7).all()
    return x, w, e, dy, y, dx, dw


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (128, 256), (8, 8), (1, 1), (7, 130), (129, 33), (200, 72),
                                        (264, 520), (1000, 24), (32, 1000)])
def test_sizes(ctx, n_in, n_out, out):
    check_all(ctx, [5, 0, 70, 1, 129, 0], n_in, n_out, out=out, seed=n_in)


@pytest.mark.parametrize("counts,unused", [([1], 0), ([0], 1), ([0, 0, 0], 3), ([300], 0), ([16] * 9, 5),
                                           ([0, 0, 17, 0, 64, 65, 63, 0], 2), ([1] * 200, 0), ([0] * 130 + [40], 7),
                                           ([2, 3] * 64, 1), ([511, 1, 513], 255), ([], 4), ([0], 0)])
@pytest.mark.parametrize("n_in,n_out", [(96, 136), (75, 50)])
def test_groups(ctx, counts, unused, n_in, n_out):
    check_all(ctx, counts, n_in, n_out, unused, ends=torch.int64, seed=len(counts))


@pytest.mark.parametrize("pad,offset", [(8, 0), (8, 8), (3, 0), (0, 1), (2, 2), (4, 4)])
def test_strides_and_alignment(ctx, pad, offset):
    check_all(ctx, [40, 9, 0, 100], 160, 72, 3, pad=pad, offset=offset, seed=pad)


def test_ends_out_of_order_or_range(ctx):
    """An end below the one before it makes an empty group; one past the rows is the rows."""
    for e in ([10, 4, 30, 12], [-3, 5, 1000, 7], [1 << 30, 2, 3, 4], [-1, -2, -3, -4]):
        check_all(ctx, [10, 0, 20, 5], 72, 40, want_ends=e)


@pytest.mark.parametrize("n_in,n_out", [(512, 768), (515, 770)])
def test_long_contractions(ctx, n_in, n_out):
    check_all(ctx, [700, 1500, 333], n_in, n_out, out=F32, seed=1)


MANY = [0, 1, 63, 64, 65, 0, 127, 128, 129, 256, 257, 300, 0, 5, 17, 40, 511, 2, 0, 9]


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("n_in,n_out,unused", [(72, 8200, 0), (8200, 72, 300), (264, 9000, 1), (128, 8192, 77),
                                               (9000, 24, 0), (4104, 520, 13)])
def test_many_tiles(ctx, n_in, n_out, unused, out):
    """Enough tiles that each block walks several, of groups with few rows and many."""
    check_all(ctx, MANY, n_in, n_out, unused, out=out, seed=n_in)


def test_many_tiles_strides_and_ends(ctx):
    check_all(ctx, MANY, 80, 8192, 5, pad=8, offset=8)
    check_all(ctx, MANY, 8192, 80, 5, pad=16)
    e = torch.tensor(MANY).cumsum(0).tolist()
    e[3], e[7], e[12] = -5, 1 << 30, 3
    check_all(ctx, MANY, 8200, 40, want_ends=e)


@pytest.mark.parametrize("counts,n_in,n_out,unused", [([64], 2048, 264, 0), ([1], 1024, 2048, 0), ([3, 0, 9], 4104, 72, 5),
                                                      ([6000, 2500], 136, 200, 9), ([5000], 129, 75, 1), ([2], 4099, 33, 0),
                                                      ([1, 2, 0, 700], 3000, 8, 0)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_few_tiles_with_long_contractions(ctx, counts, n_in, n_out, unused, out):
    """Products whose contraction is done in parts and joined."""
    check_all(ctx, counts, n_in, n_out, unused, out=out)
    check_all(ctx, counts, n_in, n_out, unused, out=out, pad=3)


@pytest.mark.parametrize("n_in,n_out", [(3, 5), (9, 131), (127, 2), (135, 71), (33, 4097)])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 1), (3, 6)])
def test_ends_of_rows(ctx, n_in, n_out, offset, pad):
    """Rows shorter than a piece, and last pieces of every length, at the ends of the tensors' memory."""
    check_all(ctx, [31, 0, 150, 2, 33], n_in, n_out, 1, pad=pad, offset=offset)


def test_middling_tiles(ctx):
    """Tiles of 128 and 256 in blocks of their own, whole pieces and not."""
    for n_in, n_out in ((1024, 2048), (2000, 1040), (1030, 2045)):
        check_all(ctx, [300, 0, 1000, 77], n_in, n_out, 3)
    check_all(ctx, [2300], 2560, 2304, 0)
    check_all(ctx, [700, 20, 130, 400], 648, 712, 10, out=F32)


def test_many_groups(ctx):
    """More groups than are sorted by size, and than a wave looks at at once."""
    gen = torch.Generator().manual_seed(1)
    counts = torch.randint(0, 4, (700,), generator=gen).tolist()
    check_all(ctx, counts, 64, 264, 3)
    check_all(ctx, counts, 264, 64, 3, ends=torch.int64)


def test_one_gradient_at_a_time(ctx):
    from paper_2609_34162_amd import ops
    x, w, e, dy, _, dx, dw = check_all(ctx, [33, 0, 90], 64, 128)
    a, b = torch.empty_like(dx), torch.empty_like(dw)
    ops.sdp_grouped_matmul_backward(ctx, None, w, e, dy, a, None)
    ops.sdp_grouped_matmul_backward(ctx, x, w, e, dy, None, b)
    assert torch.equal(a, dx) and torch.equal(b, dw)


def test_gradient_against_differences(ctx):
    """y is linear in x and in w: <dx, v> = <y(x + v) - y(x), dy> without a remainder, in 64 bits."""
    x, w, e, dy, _, dx, dw = check_all(ctx, [33, 0, 90], 64, 128, out=F32)
    gen = torch.Generator().manual_seed(2)
    value = lambda x, w: (ops_ref.grouped(x, w, e, F32)[0] * dy.cpu().double()).sum()
    xd, wd = x.cpu().double(), w.cpu().double()
    v, u = torch.randn(x.shape, generator=gen).double(), torch.randn(w.shape, generator=gen).double()
    # dx is rounded to BF16 (2^-9 of each element); dw is in 32 bits over 90 rows
    got = (dx.cpu().double() * v).sum()
    assert abs(value(xd + v, wd) - value(xd, wd) - got) <= 2.0 ** -8 * (dx.cpu().double() * v).abs().sum()
    got = (dw.cpu().double() * u).sum()
    assert abs(value(xd, wd + u) - value(xd, wd) - got) <= 1e-4 * (dw.cpu().double() * u).abs().sum()


def test_same_bits_again(ctx):
    a = check_all(ctx, [100, 300, 0, 29], 256, 192, seed=4)
    b = check_all(ctx, [100, 300, 0, 29], 256, 192, seed=4)
    for x, y in zip(a[4:], b[4:]):
        assert torch.equal(x, y)


def test_infinity_and_nan_stay_in_their_rows_and_groups(ctx):
    """What one row of x or dy holds reaches its own row of y or dx and its own group of dw only."""
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(8)
    for n_in, n_out in ((64, 128), (65, 31)):
        counts = [20, 45, 17]
        e = torch.tensor(counts).cumsum(0).cuda()
        x, dy = strided(gen, 82, n_in, 0), strided(gen, 82, n_out, 0)
        w = torch.randn((3, n_out, n_in), generator=gen).to(BF16).cuda()
        x[25], dy[70] = float("nan"), float("inf")
        y, dx = torch.empty((82, n_out), dtype=BF16, device="cuda"), torch.empty((82, n_in), dtype=BF16, device="cuda")
        dw = torch.empty((3, n_out, n_in), device="cuda")
        ops.sdp_grouped_matmul(ctx, x, w, e, y)
        ops.sdp_grouped_matmul_backward(ctx, x, w, e, dy, dx, dw)
        rows = torch.arange(82)
        assert torch.equal(torch.isfinite(y.cpu()).all(1), rows != 25)
        assert torch.equal(torch.isfinite(dx.cpu()).all(1), rows != 70)
        assert torch.isfinite(dw[0]).all() and torch.isnan(dw[1]).all() and not torch.isfinite(dw[2]).any()


# large enough for copies in whole pieces: every tensor without them, one side only,
# strides or addresses alone; empty groups and rows of no group among them
@pytest.mark.parametrize("counts,n_in,n_out,unused,pad,offset", [([3000, 0, 5190], 1021, 1033, 11, 0, 0),
                                                                 ([1, 9000], 1024, 1027, 0, 0, 0),
                                                                 ([9000], 1001, 1024, 200, 3, 1),
                                                                 ([5000, 5001], 1024, 1024, 3, 5, 0),
                                                                 ([4096, 4099], 1024, 1040, 0, 0, 3)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_copies_in_whole_pieces(ctx, counts, n_in, n_out, unused, pad, offset, out):
    check_all(ctx, counts, n_in, n_out, unused=unused, out=out, pad=pad, offset=offset, seed=11)


def test_copies_on_two_streams(ctx):
    """Two calls that share the workspace, on streams of their own, with nothing between them."""
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(12)
    ends = torch.tensor([4000, 8200], dtype=torch.int32).cuda()
    x = [torch.randn((8200, 1021), generator=gen).to(BF16).cuda() for _ in range(2)]
    w = torch.randn((2, 1033, 1021), generator=gen).to(BF16).cuda()
    y = [torch.empty((8200, 1033), dtype=BF16, device="cuda") for _ in range(4)]
    for i in range(2):
        ops.sdp_grouped_matmul(ctx, x[i], w, ends, y[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, s in enumerate(streams):
        ops.sdp_grouped_matmul(ctx, x[i], w, ends, y[2 + i], stream=s)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(y[i].view(torch.int16), y[2 + i].view(torch.int16))
