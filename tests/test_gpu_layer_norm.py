"""sdp_block_norm and its backward on the GPU against 64-bit definitions."""
import itertools

import pytest

import gpu_util
import layer_ref as ref

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


def rows(gen, n, h, dtype, pad=0, first=0, sigma=1.0):
    flat = (torch.randn(first + n * (h + pad), generator=gen) * sigma).to(dtype).cuda()
    return flat[first:].view(n, h + pad)[:, :h]


def like(t, pad, first):
    """A tensor of t's shape and type, filled with 7, laid out like rows()."""
    if t is None:
        return None
    n, h = t.shape
    return torch.full((first + n * (h + pad),), 7.0, dtype=t.dtype, device="cuda")[first:].view(n, h + pad)[:, :h]


def make(t, h, stream=BF16, dtype=BF16, wdtype=BF16, gate="none", weights=True, pad=0, first=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    st = dict(h=rows(gen, t, h, stream, pad, first, 2.0), y=rows(gen, t, h, dtype, pad, first, 1.5),
              dh_out=rows(gen, t, h, stream, pad, first), dn=rows(gen, t, h, dtype, pad, first), gate=None)
    st["gate"] = {"none": lambda: None, "channel": lambda: torch.randn(h, generator=gen).to(dtype).cuda(),
                  "token": lambda: rows(gen, t, 1, dtype, pad, first),
                  "element": lambda: rows(gen, t, h, dtype, pad, first)}[gate]()
    for n in ("post_weight", "pre_weight"):
        st[n] = (1 + 0.2 * torch.randn(h, generator=gen)).to(wdtype).cuda() if weights else None
    return st


def check_both(ctx, st, post=True, sigmoid=False, scale=1.0, eps=EPS, offset=0.0, pad=0, first=0, wdtype=None,
               with_h=True, with_n=True):
    from paper_2609_34162_amd import ops
    h, y, gate, wp, wn = (st[n] for n in ("h", "y", "gate", "post_weight", "pre_weight"))
    stream, dtype = h.dtype, y.dtype
    wdtype = wdtype or (F32 if wn is None else wn.dtype)
    more = dict(gate=gate, gate_sigmoid=sigmoid, post_norm=post, post_weight=wp if post else None, pre_weight=wn,
                scale=scale, eps=eps, weight_offset=offset)
    h_out, n_out = like(h, pad, first) if with_h else None, like(y, pad, first) if with_n else None
    ops.sdp_block_norm(ctx, h, y, h_out, n_out, **more)
    want_h, want_n = ref.norm(h, y, gate, sigmoid, post, wp, wn, scale, eps, offset, stream, dtype)
    if with_h:
        ref.check(h_out, *want_h, "h_out")
    if with_n:
        ref.check(n_out, *want_n, "n_out")
    # backward, from a stream of its own (what h holds)
    dn, dh_out = st["dn"] if with_n else None, st["dh_out"] if with_h else None
    dh, dy = like(h, pad, first), like(y, pad, first)
    dgate = None if gate is None else (like(gate, pad, first) if gate.dim() == 2 else torch.full_like(gate, 7.0))
    new = lambda: torch.full((h.shape[1],), 7.0, dtype=wdtype, device="cuda")
    dpost, dpre = new() if post else None, new() if with_n else None
    ops.sdp_block_norm_backward(ctx, h, y, dh_out, dn, dh, dy, dgate=dgate, dpost_weight=dpost, dpre_weight=dpre, **more)
    wants = ref.norm_back(h, y, dh_out, dn, gate, sigmoid, post, wp, wn, scale, eps, offset, stream, dtype, wdtype)
    for got, want, name in zip((dh, dy, dgate, dpost, dpre), wants, ("dh", "dy", "dgate", "dpost", "dpre")):
        assert (got is None) == (want is None), name
        if got is not None:
            ref.check(got, *want, name)
    return more, (h_out, n_out), (dh, dy, dgate, dpost, dpre)


TYPES = [(BF16, BF16, BF16), (F32, F32, F32), (F32, BF16, F32), (BF16, F32, BF16)]


@pytest.mark.parametrize("stream,dtype,wdtype", TYPES)
@pytest.mark.parametrize("gate", ["none", "channel", "token", "element"])
@pytest.mark.parametrize("post,sigmoid", [(True, False), (False, True)])
def test_forms_and_types(ctx, gate, post, sigmoid, stream, dtype, wdtype):
    st = make(19, 72, stream, dtype, wdtype, gate, seed=1)
    check_both(ctx, st, post, sigmoid, scale=0.7, offset=1.0 if post else 0.0)


# one row to a few lanes, to a wave, to some waves, to 1,024 threads, and past what registers hold
@pytest.mark.parametrize("h", [1, 2, 7, 8, 9, 64, 100, 128, 255, 256, 264, 512, 520, 1000, 1024, 1500, 2048, 2560,
                               4096, 5120, 8000, 8192, 8200, 10000, 16384, 17001, 33000])
@pytest.mark.parametrize("gate,post", [("channel", True), ("token", False)])
def test_hidden_sizes(ctx, h, gate, post):
    st = make(5, h, BF16, BF16, F32, gate, seed=h)
    check_both(ctx, st, post, gate == "token", scale=0.5)
    check_both(ctx, make(3, h, F32, F32, BF16, gate, seed=h + 1), post)


@pytest.mark.parametrize("t", [0, 1, 2, 3, 63, 64, 65, 1000, 3001])
@pytest.mark.parametrize("h", [40, 1003])
def test_token_counts(ctx, t, h):
    for gate in ("none", "channel", "token", "element"):
        check_both(ctx, make(t, h, BF16, BF16, BF16, gate, seed=t), True, False, scale=0.3)


@pytest.mark.parametrize("pad,first", [(1, 0), (0, 1), (3, 5), (8, 0), (5, 8)])
@pytest.mark.parametrize("h", [136, 1003])
def test_strides_and_alignment(ctx, h, pad, first):
    for stream, dtype, wdtype in TYPES[:3]:
        for gate in ("token", "element"):
            st = make(9, h, stream, dtype, wdtype, gate, pad=pad, first=first, seed=pad)
            check_both(ctx, st, True, True, pad=pad, first=first)


@pytest.mark.parametrize("with_h,with_n", [(True, False), (False, True)])
@pytest.mark.parametrize("post", [False, True])
def test_one_output(ctx, with_h, with_n, post):
    check_both(ctx, make(33, 200, F32, BF16, F32, "channel"), post, with_h=with_h, with_n=with_n)


def test_no_weights(ctx):
    check_both(ctx, make(9, 64, F32, F32, weights=False), True, offset=3.0)


def test_the_norm_alone(ctx):
    from paper_2609_34162_amd import ops
    for h in (64, 1003):
        st = make(21, h, F32, BF16, BF16)
        n_out = torch.empty_like(st["y"])
        ops.sdp_block_norm(ctx, st["h"], None, None, n_out, pre_weight=st["pre_weight"], eps=EPS)
        x, w = ref.f64(st["h"]), ref.f64(st["pre_weight"])
        want = x * w / ref.rms(x, EPS)
        ref.check(n_out, want, ref.rounded(want, BF16, (h / 2 + 16) * ref.U32 * want.abs()), "n_out")
        dh, dpre = torch.empty_like(st["h"]), torch.empty_like(st["pre_weight"])
        ops.sdp_block_norm_backward(ctx, st["h"], None, st["dh_out"], st["dn"], dh, None, pre_weight=st["pre_weight"],
                                    dpre_weight=dpre, eps=EPS)
        wants = ref.norm_back(st["h"], None, st["dh_out"], st["dn"], None, False, False, None, st["pre_weight"], 1.0, EPS,
                              0.0, F32, BF16, BF16)
        ref.check(dh, *wants[0], "dh")
        ref.check(dpre, *wants[4], "dpre")


def test_each_gradient_alone(ctx):
    """What is asked for alone has the bits that it has beside the others."""
    from paper_2609_34162_amd import ops
    for gate, h in itertools.product(("channel", "token", "element"), (88, 1003)):
        st = make(37, h, BF16, BF16, F32, gate, seed=h)
        more, _, whole = check_both(ctx, st, True, True, scale=0.5)
        names = ("dh", "dy", "dgate", "dpost_weight", "dpre_weight")
        for k, name in enumerate(names):
            kw = dict(dh=None, dy=None)
            kw[name] = torch.full_like(whole[k], 7.0)
            got = kw[name]
            y = st["y"] if k in (1, 2, 3) else None
            dh, dy = kw.pop("dh"), kw.pop("dy")
            ops.sdp_block_norm_backward(ctx, st["h"], y, st["dh_out"], st["dn"], dh, dy, **kw, **more)
            assert torch.equal(got, whole[k]), (gate, h, name)


def test_rows_of_zeros_and_large_values(ctx):
    st = make(6, 64, F32, F32, F32)
    st["h"][0] = 0.0
    st["y"][0] = 0.0
    st["h"][1] = 1e15
    st["y"][2] = 1e-15
    st["y"][3] = -1e15
    check_both(ctx, st, True)
    check_both(ctx, st, True, eps=1e-3)
    check_both(ctx, st, False)


def test_gates_far_out(ctx):
    """Sigmoids of large and infinite gates: 0 and 1, slopes of 0."""
    st = make(8, 64, F32, F32, F32, "token")
    st["gate"][:, 0] = torch.tensor([90.0, -90.0, 1e4, -1e4, float("inf"), float("-inf"), 0.0, -0.0]).cuda()
    check_both(ctx, st, True, True)


def test_nan_stays_in_its_row(ctx):
    st = make(7, 300, BF16, BF16, F32, "token")
    st["h"][2, 5], st["y"][4, 7] = float("nan"), float("nan")
    from paper_2609_34162_amd import ops
    h_out, n_out = torch.empty_like(st["h"]), torch.empty_like(st["y"])
    ops.sdp_block_norm(ctx, st["h"], st["y"], h_out, n_out, gate=st["gate"], post_norm=True, pre_weight=st["pre_weight"])
    bad = torch.isnan(n_out).any(1).cpu().tolist()
    assert bad == [i in (2, 4) for i in range(7)]


@pytest.mark.parametrize("h", [128, 1003, 5120, 17001])
def test_in_place(ctx, h):
    from paper_2609_34162_amd import ops
    st = make(17, h, BF16, BF16, BF16, "channel", seed=h)
    more, (h_out, n_out), (dh, dy, dgate, dpost, dpre) = check_both(ctx, st, True, scale=0.5)
    hi, yi = st["h"].clone(), st["y"].clone()
    ops.sdp_block_norm(ctx, hi, yi, hi, yi, **more)
    assert torch.equal(hi, h_out) and torch.equal(yi, n_out)
    for into in ("dn", "y"):
        a = {n: st[n].clone() for n in ("y", "dh_out", "dn")}
        ops.sdp_block_norm_backward(ctx, st["h"], a["y"], a["dh_out"], a["dn"], a["dh_out"], a[into], **more)
        assert torch.equal(a["dh_out"], dh) and torch.equal(a[into], dy), into


def test_broadcast_inputs(ctx):
    st = make(9, 72, F32, F32, F32, "element")
    for n in ("y", "dn", "dh_out", "gate"):
        st[n] = st[n][:1].expand(9, 72)
    from paper_2609_34162_amd import ops
    dh, dy, dgate = (torch.empty((9, 72), device="cuda") for _ in range(3))
    more = dict(gate=st["gate"], post_norm=True, post_weight=st["post_weight"], pre_weight=st["pre_weight"])
    ops.sdp_block_norm_backward(ctx, st["h"], st["y"], st["dh_out"], st["dn"], dh, dy, dgate=dgate, **more)
    wants = ref.norm_back(st["h"], st["y"], st["dh_out"], st["dn"], st["gate"], False, True, st["post_weight"],
                          st["pre_weight"], 1.0, EPS, 0.0, F32, F32, F32)
    for got, want, name in zip((dh, dy, dgate), wants, ("dh", "dy", "dgate")):
        ref.check(got, *want, name)


def test_gradients_against_differences(ctx):
    """<gradient, direction> against central differences of <outputs, their gradients> in 64 bits."""
    from paper_2609_34162_amd import ops
    t, h = 6, 40
    for gate, sigmoid in (("channel", False), ("token", True), ("element", True)):
        st = make(t, h, F32, F32, F32, gate, seed=11)
        h0, y, g, wp, wn = (ref.f64(st[n]) for n in ("h", "y", "gate", "post_weight", "pre_weight"))
        out = ref.block_norm(h0, y, g, sigmoid, True, wp, wn, 0.6, EPS, 0.5)[0]
        dh, dy = torch.empty_like(st["h"]), torch.empty_like(st["y"])
        dgate, dpost, dpre = torch.empty_like(st["gate"]), torch.empty(h, device="cuda"), torch.empty(h, device="cuda")
        ops.sdp_block_norm_backward(ctx, out.float().cuda(), st["y"], st["dh_out"], st["dn"], dh, dy, gate=st["gate"],
                                    dgate=dgate, gate_sigmoid=sigmoid, post_norm=True, post_weight=st["post_weight"],
                                    dpost_weight=dpost, pre_weight=st["pre_weight"], dpre_weight=dpre, scale=0.6, eps=EPS,
                                    weight_offset=0.5)
        vh, vn = ref.f64(st["dh_out"]), ref.f64(st["dn"])

        def value(*args):
            a, b, _ = ref.block_norm(args[0], args[1], args[2], sigmoid, True, args[3], args[4], 0.6, EPS, 0.5)
            return (a * vh).sum() + (b * vn).sum()
        gen = torch.Generator().manual_seed(5)
        at, step = [h0, y, g, wp, wn], 1e-5
        for k, grad in enumerate((dh, dy, dgate, dpost, dpre)):
            v = torch.randn(at[k].shape, generator=gen).double()
            up, down = list(at), list(at)
            up[k], down[k] = at[k] + step * v, at[k] - step * v
            want = (value(*up) - value(*down)) / (2 * step)
            got = (ref.f64(grad) * v).sum()
            # differences: step^2 of third derivatives and 1e-16 / step of rounding over 240 elements; the stream's
            # rounding to 32 bits and the gradients' own
            assert abs(want - got) <= 2e-5 * (ref.f64(grad) * v).abs().sum() + 1e-6, (gate, k, want, got)


def test_same_bits_again_and_on_another_stream(ctx):
    from paper_2609_34162_amd import ops
    st = make(4097, 512, BF16, BF16, F32, "channel", seed=9)
    got = []
    for s in (None, torch.cuda.Stream(), torch.cuda.Stream(), None):
        dh, dy, dgate = torch.empty_like(st["h"]), torch.empty_like(st["y"]), torch.empty_like(st["gate"])
        dw = [torch.empty(512, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        ops.sdp_block_norm_backward(ctx, st["h"], st["y"], st["dh_out"], st["dn"], dh, dy, gate=st["gate"], dgate=dgate,
                                    post_norm=True, post_weight=st["post_weight"], dpost_weight=dw[0],
                                    pre_weight=st["pre_weight"], dpre_weight=dw[1], stream=s)
        got.append([dh, dy, dgate] + dw)
    torch.cuda.synchronize()
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
