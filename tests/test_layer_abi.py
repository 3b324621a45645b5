"""The ABI of the training operators around the experts' products without a GPU:
include/sdp_layer.h against the library and the binding, and what the binding
refuses before any call."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sdp_layer.h")


@pytest.fixture(scope="module")
def ops():
    from paper_2609_34162_amd import ops as mod
    return mod


def test_every_declared_call_is_exported_and_bound(ops):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = re.findall(r"^SDP_API int (sdp_\w+)\s*\(", text, flags=re.M)
    assert len(names) == 11, names
    lib = ctypes.CDLL(ops._sdp.LIB_PATH)
    assert all(hasattr(lib, n) and hasattr(ops, n) for n in names)


def test_constants_match(ops):
    found = re.findall(r"^#define\s+(SDP_\w+)\s+(\d+)", open(HEADER).read(), flags=re.M)
    assert len(found) == 7
    for name, value in found:
        assert getattr(ops, name) == int(value), name


def test_c_program(ops, tmp_path):
    exe = tmp_path / "layer_from_c"
    libdir = os.path.dirname(ops._sdp.LIB_PATH)
    extra = ["-Wl,--allow-shlib-undefined"] if os.environ.get("SDP_LIB") else []
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I",
                           os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "c", "layer_from_c.c"), "-o",
                           str(exe), "-L", libdir, "-lsdp", f"-Wl,-rpath,{libdir}", *extra])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stderr)
    got = {ln.split()[0]: [int(x) for x in ln.split()[1:]] for ln in r.stdout.splitlines()}
    for name, fields in (("sdp_rows", ("stride",)), ("sdp_embed_desc", ("ids", "scale")),
                         ("sdp_block_norm_desc", ("scale", "pre_weight")),
                         ("sdp_block_norm_grads", ("dgate", "dpre_weight")),
                         ("sdp_route_desc", ("scale", "logit_stride")), ("sdp_order_desc", ("ends_type",)),
                         ("sdp_expert_desc", ("place",))):
        struct = getattr(ops, name)
        assert got[name] == [ctypes.sizeof(struct)] + [getattr(struct, f).offset for f in fields], name


def test_binding_refuses_tensors_that_do_not_belong_together(ops):
    torch = pytest.importorskip("torch")
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
    bf, i32 = torch.bfloat16, torch.int32
    ids, table, out = z(5, dtype=i32), z(9, 8), z(5, 8)

    def refuses(text, call, *args, **kw):
        with pytest.raises(ValueError, match=text):
            call(None, *args, **kw)
    refuses("out has shape", ops.sdp_embed, table, ids, z(4, 8))
    refuses("tokens must be 1-D", ops.sdp_embed, table, z(5, 1, dtype=i32), out)
    refuses("table must be 2-D", ops.sdp_embed, z(9), ids, out)
    refuses("dtable has type", ops.sdp_embed_backward, out, ids, table.double())
    refuses("last dimension", ops.sdp_embed, z(8, 9).t(), ids, out)
    h, y = z(6, 8), z(6, 8, dtype=bf)
    norm = ops.sdp_block_norm
    refuses("y has shape", norm, h, z(6, 7, dtype=bf), h, None)
    refuses("h_out has another type", norm, h, y, y, None)
    refuses("n_out has another type", norm, h, y, h, h)
    refuses("gate has another type", norm, h, y, h, y, gate=z(6, 8))
    for shape in ((6,), (1,), (1, 1), (6, 2), (2, 8), (1, 6, 8)):
        refuses("gate has shape", norm, h, y, h, y, gate=z(*shape, dtype=bf))
    refuses("gate: the last dimension", norm, h, y, h, y, gate=z(8, 6, dtype=bf).t())
    refuses("pre_weight has shape", norm, h, y, h, y, pre_weight=z(7))
    refuses("a weight has another type", norm, h, y, h, y, pre_weight=z(8), post_weight=z(8, dtype=bf))
    back = ops.sdp_block_norm_backward
    refuses("all None", back, None, y, None, y, None, y)
    refuses("dy has another type", back, h, y, h, y, h, h)
    refuses("dgate has another form", back, h, y, h, y, h, y, gate=z(6, 1, dtype=bf), dgate=z(8, dtype=bf))
    refuses("a weight has another type", back, h, y, h, y, h, y, pre_weight=z(8), dpre_weight=z(8, dtype=bf))
    refuses("dpost_weight has shape", back, h, y, h, y, h, y, post_norm=True, dpost_weight=z(6))
    logits, index, w = z(6, 8), z(6, 2, dtype=i32), z(6, 2)
    refuses("index has 5 rows", ops.sdp_route, logits, z(5, 2, dtype=i32), w)
    refuses("weights has shape", ops.sdp_route, logits, index, z(6, 3))
    refuses("bias has shape", ops.sdp_route, logits, index, w, bias=z(7))
    refuses("bias has another type", ops.sdp_route, logits, index, w, bias=z(8, dtype=bf))
    refuses("index must be contiguous", ops.sdp_route, logits, z(2, 6, dtype=i32).t(), w)
    refuses("dlogits has another type", ops.sdp_route_backward, logits, index, w, logits.to(bf))
    refuses("dlogits has shape", ops.sdp_route_backward, logits, index, w, z(6, 9))
    order = ops.sdp_expert_order
    refuses("place has shape", order, index, z(8, dtype=i32), z(6, 3, dtype=i32))
    refuses("place has another type", order, index, z(8, dtype=i32), z(6, 2, dtype=torch.int64))
    refuses("order has shape", order, index, z(8, dtype=i32), index, z(6, 2, dtype=i32))
    refuses("ends must be 1-D", order, index, z(2, 4, dtype=i32), index)
    x, rows = z(6, 8), z(12, 8)
    refuses("rows has shape", ops.sdp_expert_gather, x, index, z(11, 8))
    refuses("x has shape", ops.sdp_expert_gather, z(5, 8), index, rows)
    refuses("place has another type", ops.sdp_expert_gather, x, index.long(), rows)
    refuses("dx has another type", ops.sdp_expert_gather_backward, rows, index, x.to(bf))
    refuses("weights has shape", ops.sdp_expert_combine, rows, index, z(12), x)
    refuses("residual has another type", ops.sdp_expert_combine, rows, index, w, x, residual=x.to(bf))
    refuses("drows has another type", ops.sdp_expert_combine_backward, rows, index, w, x, rows.to(bf), w)
    refuses("dweights has another type", ops.sdp_expert_combine_backward, rows, index, w, x, rows, w.to(bf))


def test_calls_without_a_context_are_refused(ops):
    torch = pytest.importorskip("torch")
    x, i = torch.zeros(3, 4), torch.zeros((3, 2), dtype=torch.int32)
    calls = [lambda: ops.sdp_embed(None, x, i[:, 0].contiguous(), x), lambda: ops.sdp_block_norm(None, x, x, x, x),
             lambda: ops.sdp_route(None, x, i, x[:, :2].contiguous()),
             lambda: ops.sdp_expert_order(None, i, torch.zeros(4, dtype=torch.int32), i),
             lambda: ops.sdp_expert_gather(None, x, i, torch.zeros(6, 4))]
    for call in calls:
        with pytest.raises(ops.SdpError) as e:
            call()
        assert e.value.status == ops._sdp.SDP_ERR_INVALID_ARGUMENT and "context" in e.value.detail


def test_binding_refuses_what_32_bits_do_not_hold(ops):
    torch = pytest.importorskip("torch")
    n = (1 << 32) + 8
    far = lambda *shape, dtype=torch.bfloat16: torch.zeros(1, dtype=dtype).expand(*shape)
    one, ids = torch.zeros((1, 1), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="table: a dimension"):
        ops.sdp_embed(None, far(2, n), ids, far(1, n))
    with pytest.raises(ValueError, match="the stream: a dimension"):
        ops.sdp_block_norm(None, far(1, n), None, None, far(1, n))
    with pytest.raises(ValueError, match="logits and index: a dimension"):
        ops.sdp_route(None, far(1, n), one, torch.zeros(1, 1))
    with pytest.raises(ValueError, match="place and the rows: a dimension"):
        ops.sdp_expert_gather(None, far(1, n), one, far(1, n))


def test_descriptions_are_packed_as_the_structures_lie(ops):
    for kind in (ops.sdp_rows, ops.sdp_embed_desc, ops.sdp_block_norm_desc, ops.sdp_block_norm_grads, ops.sdp_route_desc,
                 ops.sdp_order_desc, ops.sdp_expert_desc):
        values = [1.5 + k if t is ctypes.c_double else 3 + k for k, (_, t) in enumerate(kind._fields_)]
        one = kind()
        for (name, t), v in zip(kind._fields_, values):
            setattr(one, name, ctypes.cast(v, t) if t not in (ctypes.c_int32, ctypes.c_int64, ctypes.c_double,
                                                              ctypes.c_void_p) else v)
        assert ops._packer(kind)(*values) == bytes(one), kind
