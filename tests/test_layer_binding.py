"""What the binding of include/sdp_layer.h refuses of its plain numbers, without a GPU."""
import pytest

torch = pytest.importorskip("torch")


def test_numbers_that_a_description_does_not_hold():
    from paper_2609_34162_amd import ops
    z, h = torch.zeros(6, 8), torch.zeros(6, 8)
    index, w = torch.zeros((6, 2), dtype=torch.int32), torch.zeros(6, 2)
    ids, table, out = torch.zeros(6, dtype=torch.int32), torch.zeros(9, 8), torch.zeros(6, 8)
    for name in ("groups", "top_groups", "group_best"):
        for value in (1 << 31, -(1 << 31) - 1, 1 << 80, 2.0, "2", None):
            with pytest.raises(ValueError, match=f"^{name}"):
                ops.sdp_route(None, z, index, w, **{name: value})
    for value in ("1", None, 10 ** 400, [1.0]):
        with pytest.raises(ValueError, match="^scale"):
            ops.sdp_route(None, z, index, w, scale=value)
        with pytest.raises(ValueError, match="^scale"):
            ops.sdp_route_backward(None, z, index, w, z, scale=value)
        with pytest.raises(ValueError, match="^scale"):
            ops.sdp_embed(None, table, ids, out, scale=value)
        with pytest.raises(ValueError, match="^scale"):
            ops.sdp_embed_backward(None, out, ids, table, scale=value)
        for name in ("scale", "eps", "weight_offset"):
            with pytest.raises(ValueError, match=f"^{name}"):
                ops.sdp_block_norm(None, h, h, h, h, **{name: value})
            with pytest.raises(ValueError, match=f"^{name}"):
                ops.sdp_block_norm_backward(None, h, h, h, h, h, h, **{name: value})
    # these reach the library, which has no context to run them in
    for more in (dict(groups=(1 << 31) - 1), dict(scale=1), dict(scale=torch.tensor(2.5)), dict(top_groups=True)):
        with pytest.raises(ops.SdpError, match="context"):
            ops.sdp_route(None, z, index, w, **more)
