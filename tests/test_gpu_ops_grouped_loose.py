"""sdp_grouped_matmul_backward of sizes without whole pieces, where the rows of dw are
split between blocks in tiles of 128."""
import pytest

import gpu_util

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_ops_grouped import BF16, F32, check_all  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    sdp = gpu_util.need_gpu()
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


# 216 and 288 tiles of 128; more than 2,048 rows a group on average, an empty one and one of few rows among them
@pytest.mark.parametrize("counts,n_in,n_out", [([2100, 0, 5000, 2600, 2500, 2049, 2300, 2600], 1025, 261),
                                               ([40, 8400, 0, 4000], 1030, 1029)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_rows_of_dw_split(ctx, counts, n_in, n_out, out):
    check_all(ctx, counts, n_in, n_out, unused=3, out=out, seed=9)
