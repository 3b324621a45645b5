"""sdp_distill_loss and its backward at temperatures of 3 and 4, where one exponential
serves both terms, on few rows (shared by blocks)."""
import pytest

import gpu_util

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_ops_distill import BF16, F32, check_all, make  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    sdp = gpu_util.need_gpu()
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [3.0, 4.0])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 7, 2), (5, 1000, 64), (2, 32003, 20), (33, 257, 256),
                                          (1, 151936, 64), (2, 40000, 0)])
def test_sizes(ctx, rows, vocab, k, tau, dtype):
    check_all(ctx, make(rows, vocab, k, dtype, seed=vocab), tau)
    check_all(ctx, make(rows, vocab, k, dtype, seed=vocab + 1, labels=False), tau)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [3.0, 4.0])
@pytest.mark.parametrize("vocab", [500, 20000])
def test_rows_with_one_term_or_none(ctx, vocab, tau, dtype):
    st = make(8, vocab, 8, dtype, seed=2)
    st["index"][0], st["labels"][0] = -1, 3
    st["index"][1], st["labels"][1] = torch.arange(8).cuda(), -100
    st["index"][2], st["labels"][2] = -1, -100
    st["z"][3, vocab // 2:] = float("-inf")
    st["index"][3], st["labels"][3] = torch.arange(8).cuda(), 1
    st["z"][4, 9:] = torch.finfo(dtype).min
    st["index"][4], st["labels"][4] = torch.arange(8).cuda(), 8
    st["row_grad"][5], st["row_grad"][6] = 0.0, -3.0
    check_all(ctx, st, tau, 0.7, 0.3)
