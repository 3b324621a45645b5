"""The training operators' ABI without a GPU: include/sdp_ops.h against the
library and the binding, the host code's decisions (sdp_ops_plan.h), and what
the binding refuses before any call."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sdp_ops.h")


@pytest.fixture(scope="module")
def ops():
    from paper_2609_34162_amd import ops as mod
    return mod


def test_every_declared_call_is_exported_and_bound(ops):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = re.findall(r"^SDP_API int (sdp_\w+)\s*\(", text, flags=re.M)
    assert len(names) == 6, names
    lib = ctypes.CDLL(ops._sdp.LIB_PATH)
    assert all(hasattr(lib, n) and hasattr(ops, n) for n in names)


def test_constants_match(ops):
    found = re.findall(r"^#define\s+(SDP_\w+)\s+(\d+)", open(HEADER).read(), flags=re.M)
    assert len(found) >= 9
    for name, value in found:
        assert getattr(ops, name) == int(value), name


def test_c_program(ops, tmp_path):
    exe = tmp_path / "ops_from_c"
    libdir = os.path.dirname(ops._sdp.LIB_PATH)
    extra = ["-Wl,--allow-shlib-undefined"] if os.environ.get("SDP_LIB") else []
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I",
                           os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "c", "ops_from_c.c"), "-o",
                           str(exe), "-L", libdir, "-lsdp", f"-Wl,-rpath,{libdir}", *extra])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stderr)
    got = {ln.split()[0]: [int(x) for x in ln.split()[1:]] for ln in r.stdout.splitlines()}
    for name, fields in (("sdp_heads", ("head_stride",)), ("sdp_qk_norm_rope_desc", ("eps", "k_weight")),
                         ("sdp_grouped_desc", ("ends", "dx_stride")),
                         ("sdp_distill_desc", ("teacher_logits", "label_weight"))):
        struct = getattr(ops, name)
        assert got[name] == [ctypes.sizeof(struct)] + [getattr(struct, f).offset for f in fields], name


def test_host_decisions(tmp_path):
    exe = tmp_path / "ops_plan_check"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I",
                           os.path.join(ROOT, "paper_2609_34162_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", "ops_plan_check.cpp"), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout


def test_binding_refuses_shapes_that_do_not_belong_together(ops):
    torch = pytest.importorskip("torch")
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
    bf = torch.bfloat16
    q, k, cos = z(1, 4, 2, 8), z(1, 4, 1, 8), z(4, 4)
    with pytest.raises(ValueError, match="differ"):
        ops.sdp_qk_norm_rope(None, q, z(1, 5, 1, 8), q, z(1, 5, 1, 8), cos, cos)
    with pytest.raises(ValueError, match="q_out has shape"):
        ops.sdp_qk_norm_rope(None, q, k, k, k, cos, cos)
    with pytest.raises(ValueError, match="contiguous"):
        ops.sdp_qk_norm_rope(None, q.transpose(2, 3).contiguous().transpose(2, 3), k, q, k, cos, cos)
    with pytest.raises(ValueError, match="k has another type"):
        ops.sdp_qk_norm_rope(None, q, k.to(bf), q, k, cos, cos)
    with pytest.raises(ValueError, match="has type"):
        ops.sdp_qk_norm_rope(None, q.half(), k.half(), q, k, cos, cos)
    with pytest.raises(ValueError, match="positions"):
        ops.sdp_qk_norm_rope(None, q, k, q, k, cos, cos, positions=z(5, dtype=torch.int32))
    with pytest.raises(ValueError, match="q_weight has shape"):
        ops.sdp_qk_norm_rope(None, q, k, q, k, cos, cos, q_weight=z(7))
    x, w, ends = z(5, 8, dtype=bf), z(3, 4, 8, dtype=bf), z(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="x has shape"):
        ops.sdp_grouped_matmul(None, z(5, 7, dtype=bf), w, ends, z(5, 4))
    with pytest.raises(ValueError, match="y has shape"):
        ops.sdp_grouped_matmul(None, x, w, ends, z(5, 5))
    with pytest.raises(ValueError, match="ends has shape"):
        ops.sdp_grouped_matmul(None, x, w, z(4, dtype=torch.int32), z(5, 4))
    with pytest.raises(ValueError, match="dw has shape"):
        ops.sdp_grouped_matmul_backward(None, x, w, ends, z(5, 4, dtype=bf), None, z(3, 8, 4))
    with pytest.raises(ValueError, match="another type"):
        ops.sdp_grouped_matmul(None, x.float(), w, ends, z(5, 4))
    logits, loss = z(6, 100), z(6)
    with pytest.raises(ValueError, match="go together"):
        ops.sdp_distill_loss(None, logits, loss, teacher_logits=z(6, 4))
    with pytest.raises(ValueError, match="teacher_index has shape"):
        ops.sdp_distill_loss(None, logits, loss, teacher_logits=z(6, 4), teacher_index=z(6, 5, dtype=torch.int64))
    with pytest.raises(ValueError, match="loss has shape"):
        ops.sdp_distill_loss(None, logits, z(5), labels=z(6, dtype=torch.int64))
    with pytest.raises(ValueError, match="dlogits has another type"):
        ops.sdp_distill_loss(None, logits, loss, labels=z(6, dtype=torch.int64), row_grad=loss,
                             dlogits=z(6, 100, dtype=bf))


def test_calls_without_a_context_are_refused(ops):
    torch = pytest.importorskip("torch")
    q, cos = torch.zeros(1, 4, 2, 8), torch.zeros(4, 4)
    with pytest.raises(ops.SdpError) as e:
        ops.sdp_qk_norm_rope(None, q, q, q, q, cos, cos)
    assert e.value.status == ops._sdp.SDP_ERR_INVALID_ARGUMENT and "context" in e.value.detail


def test_binding_refuses_what_32_bits_do_not_hold():
    from paper_2609_34162_amd import ops
    torch = pytest.importorskip("torch")
    n = (1 << 32) + 8
    far = lambda *shape: torch.zeros(1, dtype=torch.bfloat16).expand(*shape)
    logits, one, ends = far(1, n), torch.zeros(1), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="logits: a dimension"):
        ops.sdp_distill_loss(None, logits, one, labels=torch.zeros(1, dtype=torch.int64))
    w = torch.empty((1, 0, n), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="w: a dimension"):
        ops.sdp_grouped_matmul(None, far(1, n), w, ends, torch.zeros(1, 0))
    with pytest.raises(ValueError, match="q and k: a dimension"):
        ops.sdp_qk_norm_rope(None, far(1, n, 1, 8), far(1, n, 1, 8), far(1, n, 1, 8), far(1, n, 1, 8))
