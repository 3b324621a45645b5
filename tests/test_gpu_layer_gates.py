"""sdp_block_norm_backward on the GPU where a gate is NaN: its gradients are NaN, with and
without a gradient of the norm."""
import pytest

import layer_ref as ref
from test_gpu_layer_norm import BF16, EPS, F32, ctx, make  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.mark.parametrize("gate", ["channel", "token", "element"])
@pytest.mark.parametrize("h", [72, 1003, 9001])
@pytest.mark.parametrize("sigmoid,post", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("with_n", [False, True])
def test_nan_gates(ctx, gate, h, sigmoid, post, with_n):  # noqa: F811
    from paper_2609_34162_amd import ops
    st = make(6, h, F32, F32, F32, gate, seed=h)
    if gate == "channel":
        st["gate"][5], st["gate"][h - 1] = NAN, NAN
    elif gate == "token":
        st["gate"][2, 0] = NAN
    else:
        st["gate"][2, 5], st["gate"][4, h - 1] = NAN, NAN
    wp, wn = (st["post_weight"] if post else None), st["pre_weight"]
    dn = st["dn"] if with_n else None
    dh, dy, dgate = torch.empty_like(st["h"]), torch.empty_like(st["y"]), torch.full_like(st["gate"], 7.0)
    dpost = torch.empty(h, device="cuda") if post else None
    ops.sdp_block_norm_backward(ctx, st["h"], st["y"], st["dh_out"], dn, dh, dy, gate=st["gate"], dgate=dgate,
                                gate_sigmoid=sigmoid, post_norm=post, post_weight=wp, dpost_weight=dpost,
                                pre_weight=wn, scale=0.5, eps=EPS)
    wants = ref.norm_back(st["h"], st["y"], st["dh_out"], dn, st["gate"], sigmoid, post, wp, wn, 0.5, EPS, 0.0, F32, F32,
                          F32)
    if sigmoid:
        assert torch.isnan(wants[2][0]).sum() == torch.isnan(st["gate"]).sum()
    for got, want, name in zip((dh, dy, dgate, dpost), wants, ("dh", "dy", "dgate", "dpost")):
        if got is not None:
            ref.check(got, *want, name)
