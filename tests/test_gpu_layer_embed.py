"""sdp_embed and its backward on the GPU against 64-bit definitions."""
import pytest

import gpu_util
import layer_ref as ref

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


def rows(gen, n, h, dtype, pad=0, first=0):
    """[n, h] rows `pad` elements apart, `first` elements into their memory."""
    flat = torch.randn(first + n * (h + pad), generator=gen).to(dtype).cuda()
    return flat[first:].view(n, h + pad)[:, :h]


def check(ctx, ids, vocab, h, table_type=BF16, row_type=BF16, scale=1.0, pad=0, first=0, seed=0):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(seed)
    ids = ids.cuda()
    n = len(ids)
    table = rows(gen, vocab, h, table_type, pad, first)
    out = rows(gen, n, h, row_type, pad, first)
    ops.sdp_embed(ctx, table, ids, out, scale=scale)
    ref.check(out, *ref.embed(table, ids, scale, row_type), "out")
    dout = rows(gen, n, h, row_type, pad, first)
    dtable = rows(gen, vocab, h, table_type, pad, first)
    ops.sdp_embed_backward(ctx, dout, ids, dtable, scale=scale)
    ref.check(dtable, *ref.embed_back(dout, ids, vocab, scale, table_type), "dtable")
    held = rows(gen, vocab, h, table_type, pad, first)
    base = held.clone()
    ops.sdp_embed_backward(ctx, dout, ids, held, scale=scale, accumulate=True)
    ref.check(held, *ref.embed_back(dout, ids, vocab, scale, table_type, base), "dtable added to")


@pytest.mark.parametrize("table_type,row_type", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("h", [1, 7, 8, 64, 513, 1000, 1024])
def test_sizes_and_types(ctx, h, table_type, row_type):
    gen = torch.Generator().manual_seed(h)
    ids = torch.randint(-1, 101, (333,), generator=gen)
    check(ctx, ids.int() if h % 2 else ids, 101, h, table_type, row_type, scale=1.0 if h < 64 else h ** 0.5, seed=h)


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 128, 500, 2047, 2048, 2049, 4100, 9000])
@pytest.mark.parametrize("vocab", [1, 5, 70, 3000])
def test_token_counts(ctx, n, vocab):
    gen = torch.Generator().manual_seed(n + vocab)
    check(ctx, torch.randint(0, vocab, (n,), generator=gen), vocab, 24, F32, BF16, seed=n)


@pytest.mark.parametrize("ids", [[3] * 1000, [-1] * 200, [0] * 63 + [4] * 130 + [1] * 64, list(range(5)) * 100,
                                 [4] * 64 + [-1] * 64 + [4] * 64])
def test_runs_of_one_id(ctx, ids):
    check(ctx, torch.tensor(ids), 5, 40)


@pytest.mark.parametrize("longest", [3, 20, 40, 130, 300])
@pytest.mark.parametrize("row_type", [BF16, F32])
def test_runs_across_waves_and_pieces(ctx, longest, row_type):
    """Runs of every length, beginning and ending anywhere in a wave's places and a block's."""
    gen = torch.Generator().manual_seed(longest)
    lengths = torch.randint(1, longest + 1, (40,), generator=gen)
    ids = torch.repeat_interleave(torch.arange(40) * 2, lengths)[torch.randperm(int(lengths.sum()), generator=gen)]
    check(ctx, ids, 81, 520, row_type=row_type, seed=longest)


@pytest.mark.parametrize("n", [30000, 131071, 133120, 300000])
def test_many_tokens(ctx, n):
    """The sort's ways for many entries, one pass and two."""
    gen = torch.Generator().manual_seed(n)
    for vocab in (900, 9000):
        check(ctx, torch.randint(-1, vocab, (n,), generator=gen), vocab, 3, F32, F32)


@pytest.mark.parametrize("vocab", [2047, 2048, 2049, 5000, 70000])
def test_digits_of_ids(ctx, vocab):
    gen = torch.Generator().manual_seed(vocab)
    ids = torch.cat((torch.randint(0, vocab, (3000,), generator=gen), torch.tensor([0, vocab - 1, vocab // 2])))
    check(ctx, ids, vocab, 8)


def test_three_digits_of_ids(ctx):
    vocab = (1 << 22) + 5
    ids = torch.tensor([vocab - 1, 0, 1 << 21, vocab - 1, 1 << 11, 2047, 1 << 22, -1, 0])
    check(ctx, ids.int(), vocab, 1)


@pytest.mark.parametrize("pad,first", [(1, 0), (0, 1), (3, 5), (8, 0)])
def test_strides_and_alignment(ctx, pad, first):
    gen = torch.Generator().manual_seed(pad)
    ids = torch.randint(-1, 40, (300,), generator=gen)
    for table_type, row_type in ((BF16, BF16), (F32, F32)):
        check(ctx, ids, 40, 136, table_type, row_type, pad=pad, first=first)


def test_ids_out_of_range(ctx):
    """Past the vocabulary: NaN forward, no part backward; never an address."""
    ids = torch.tensor([0, 7, 6, -1, -(1 << 40), 1 << 40, (1 << 32) + 2, 3, 1 << 31])
    check(ctx, ids, 7, 16)
    check(ctx, torch.tensor([2, 7, 1 << 30, -(1 << 31), 6], dtype=torch.int32), 7, 16, F32, F32)


def test_broadcast_gradient(ctx):
    from paper_2609_34162_amd import ops
    ids = torch.tensor([1, 1, 0, 3, 1]).cuda()
    dout = torch.randn((1, 72), device="cuda").expand(5, 72)
    dtable = torch.empty((4, 72), device="cuda")
    ops.sdp_embed_backward(ctx, dout, ids, dtable, scale=-2.5)
    ref.check(dtable, *ref.embed_back(dout, ids, 4, -2.5, F32), "dtable")


def test_infinities_and_nan_stay_in_their_rows(ctx):
    from paper_2609_34162_amd import ops
    ids = torch.tensor([2, 0, 2, 1, 3]).cuda()
    dout = torch.ones((5, 16), device="cuda")
    dout[0, 3], dout[3, 5], dout[4, 0] = float("nan"), float("inf"), -1e38
    dtable = torch.empty((5, 16), device="cuda")
    ops.sdp_embed_backward(ctx, dout, ids, dtable)
    ref.check(dtable, *ref.embed_back(dout, ids, 5, 1.0, F32), "dtable")


def test_same_bits_again_and_on_another_stream(ctx):
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(3)
    ids = (torch.rand(20000, generator=gen) ** 6 * 500).long().cuda()
    dout = torch.randn((20000, 256), generator=gen).to(BF16).cuda()
    got = []
    for s in (None, torch.cuda.Stream(), torch.cuda.Stream(), None):
        dtable = torch.empty((500, 256), dtype=BF16, device="cuda")
        torch.cuda.synchronize()
        ops.sdp_embed_backward(ctx, dout, ids, dtable, stream=s)
        got.append(dtable)
    torch.cuda.synchronize()
    assert all(torch.equal(got[0], g) for g in got[1:])
    ref.check(got[0], *ref.embed_back(dout, ids, 500, 1.0, BF16), "dtable")


def test_gradient_against_differences(ctx):
    """<dtable, v> against differences of <out, dout>; the lookup is linear, so they are exact."""
    from paper_2609_34162_amd import ops
    gen = torch.Generator().manual_seed(4)
    ids = torch.randint(-1, 12, (50,), generator=gen).cuda()
    dout = torch.randn((50, 20), generator=gen).cuda()
    dtable = torch.empty((12, 20), device="cuda")
    ops.sdp_embed_backward(ctx, dout, ids, dtable, scale=3.0)
    table, v = (torch.randn((12, 20), generator=gen) for _ in range(2))
    value = lambda t: (ref.embed(t, ids, 3.0, F32)[0] * ref.f64(dout)).sum()
    want = value(table.double() + v.double()) - value(table.double())
    got = (ref.f64(dtable) * v.double()).sum()
    # each of 240 elements: up to 12 sums of 32 bits
    assert abs(want - got) <= 16 * 2.0 ** -24 * (ref.embed_back(dout.abs(), ids, 12, 3.0, F32)[0] * v.abs()).sum()
