"""What the training operators' binding refuses, without a GPU."""
import pytest

torch = pytest.importorskip("torch")


def test_positions_have_the_tokens_order():
    """[tokens, batch] has as many elements as [batch, tokens], and another meaning."""
    from paper_2609_34162_amd import ops
    q, k, cos = torch.zeros(3, 4, 2, 8), torch.zeros(3, 4, 1, 8), torch.zeros(4, 4)
    call = lambda q, k, at: ops.sdp_qk_norm_rope(None, q, k, q, k, cos, cos, positions=at)
    for shape in ((4, 3), (12, 1), (3, 4, 1), (2, 6), (11,)):
        with pytest.raises(ValueError, match="positions must be"):
            call(q, k, torch.zeros(shape, dtype=torch.int32))
    with pytest.raises(ValueError, match="positions must be"):
        call(q, k, torch.zeros((4, 3), dtype=torch.int32).t())
    # these reach the library, which has no context to run them in
    for a, b, shape in ((q, k, (3, 4)), (q, k, (12,)), (q[0], k[0], (4,)), (q[0], k[0], (1, 4)), (q[:1], k[:1], (4,))):
        with pytest.raises(ops.SdpError, match="context"):
            call(a, b, torch.zeros(shape, dtype=torch.int32))
