"""ctypes binding of the training operators (include/sdp_ops.h): argument
marshalling only.

Every function here has the name of the C entry point it calls; it takes torch
tensors, checks that their shapes belong together and passes their addresses
and strides on.  Outputs are tensors of the caller's.  The library checks the
rest (types, ranges, overlaps) and a negative status becomes an exception.
`stream` is a torch stream or a raw handle; None is the null stream.
"""
import ctypes
from typing import Optional

from . import sdp as _sdp
from .sdp import SdpError, _check, _lib, _stream  # noqa: F401  (SdpError: what the calls raise)

SDP_TYPE_F32 = 0
SDP_TYPE_BF16 = 1
SDP_TYPE_I32 = 2
SDP_TYPE_I64 = 3
SDP_QK_MAX_HEAD_DIM = 1024
SDP_QK_MAX_HEADS = 16384
SDP_DISTILL_MAX_K = 1024
SDP_DISTILL_MAX_ROWS = 4000000
SDP_GROUPED_MAX_GROUPS = 2048


class sdp_heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class sdp_qk_norm_rope_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("type", "weight_type", "batch", "tokens", "q_heads", "k_heads",
                                              "head_dim", "rotary_dim", "interleaved", "position_type")] + \
               [("eps", ctypes.c_double), ("table_rows", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("cos", "sin", "positions", "q_weight", "k_weight")]


class sdp_grouped_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("groups", "in_features", "out_features", "out_type", "ends_type")] + \
               [("ends", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("x_stride", "y_stride", "dx_stride")]


class sdp_distill_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("vocab", ctypes.c_int32), ("logit_type", ctypes.c_int32),
                ("logits", ctypes.c_void_p), ("logit_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("teacher_k", "teacher_type", "index_type")] + \
               [(n, ctypes.c_void_p) for n in ("teacher_logits", "teacher_index", "labels")] + \
               [(n, ctypes.c_double) for n in ("temperature", "distill_weight", "label_weight")]


def _bind():
    vp, i64, P = ctypes.c_void_p, ctypes.c_int64, ctypes.POINTER
    h, qk, gm, ds = P(sdp_heads), P(sdp_qk_norm_rope_desc), P(sdp_grouped_desc), P(sdp_distill_desc)
    for name, args in {
        "sdp_qk_norm_rope": [vp, qk, h, h, h, h, vp],
        "sdp_qk_norm_rope_backward": [vp, qk, h, h, h, h, h, h, vp, vp, vp],
        "sdp_grouped_matmul": [vp, gm, vp, vp, vp, vp],
        "sdp_grouped_matmul_backward": [vp, gm, vp, vp, vp, vp, vp, vp],
        "sdp_distill_loss": [vp, ds, vp, vp, vp, vp, i64, vp],
        "sdp_distill_loss_backward": [vp, ds, vp, vp, vp, i64, vp],
    }.items():
        f = getattr(_lib, name)
        f.restype = ctypes.c_int
        f.argtypes = args


_bind()


# ---- marshalling -----------------------------------------------------------

def _types():
    import torch
    return {torch.float32: SDP_TYPE_F32, torch.bfloat16: SDP_TYPE_BF16, torch.int32: SDP_TYPE_I32,
            torch.int64: SDP_TYPE_I64}


_TYPE_OF = {}


def _type(t, what: str) -> int:
    code = _TYPE_OF.get(t.dtype)
    if code is None:
        _TYPE_OF.update(_types())
        code = _TYPE_OF.get(t.dtype)
        if code is None:
            raise ValueError(f"{what} has type {t.dtype}")
    return code


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _want(ok: bool, text: str) -> None:
    if not ok:
        raise ValueError(text)


def _count(n: int, what: str) -> None:
    # a larger one would lose its upper bits on the way into the descriptor
    if n > 0x7fffffff:
        raise ValueError(f"{what}: a dimension of {n} is too large")


def _has_shape(t, shape, what: str) -> None:
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _dense(t, shape, what: str) -> Optional[int]:
    """The address of a contiguous tensor of this shape (None passes)."""
    if t is None:
        return None
    _has_shape(t, shape, what)
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _same_type(t, code: int, what: str) -> None:
    if t is not None and _TYPE_OF.get(t.dtype) != code and _type(t, what) != code:
        raise ValueError(f"{what} has another type than expected")


def _row_stride(t, shape, what: str) -> int:
    _has_shape(t, shape, what)
    strides = t.stride()
    if strides[1] != 1 and shape[1] > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return strides[0]


def _heads(t, shape, what: str) -> sdp_heads:
    """[batch, tokens, heads, head_dim], or [tokens, heads, head_dim] of one sequence."""
    strides = t.stride()
    if len(strides) == 3:
        t = t.unsqueeze(0)
        strides = t.stride()
    if t.shape != shape:
        _has_shape(t, shape, what)
    if strides[3] != 1 and shape[3] > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return sdp_heads(t.data_ptr(), strides[0], strides[1], strides[2])


def _heads_shape(t):
    shape = t.shape
    if len(shape) == 4:
        return shape
    _want(len(shape) == 3, "q and k must be [batch, tokens, heads, head_dim]")
    return (1, *shape)


def _qk_desc(q, k, cos, sin, q_weight, k_weight, positions, eps, interleaved):
    qs, ks = _heads_shape(q), _heads_shape(k)
    batch, tokens, q_heads, dim = qs
    k_batch, k_tokens, k_heads, k_dim = ks
    if batch != k_batch or tokens != k_tokens or dim != k_dim:
        raise ValueError(f"q {tuple(qs)} and k {tuple(ks)} differ in batch, tokens or head_dim")
    _count(max(batch, tokens, q_heads, k_heads, dim), "q and k")
    code = _type(q, "q")
    _same_type(k, code, "k")
    some = k_weight if q_weight is None else q_weight
    weight_type = SDP_TYPE_F32 if some is None else _type(some, "a weight")
    _same_type(k_weight, weight_type, "a weight")
    shape = (dim,)
    rows = rotary = 0
    if cos is not None:
        table = cos.shape
        _want(len(table) == 2 and sin is not None, "cos and sin must be [table_rows, rotary_dim / 2]")
        _same_type(cos, SDP_TYPE_F32, "cos")
        _same_type(sin, SDP_TYPE_F32, "sin")
        rows, rotary = table[0], 2 * table[1]
        _count(rotary, "cos")
        cos, sin = _dense(cos, table, "cos"), _dense(sin, table, "sin")
    else:
        sin = None
    at, position_type = None, SDP_TYPE_I32
    if positions is not None:
        position_type = _type(positions, "positions")
        given = positions.shape
        if given != (batch, tokens) and given != (batch * tokens,) or not positions.is_contiguous():
            raise ValueError(f"positions must be [{batch}, {tokens}] (or in one dimension), contiguous")
        at = positions.data_ptr()
    # in the fields' order: several times as fast as setting them one by one
    d = sdp_qk_norm_rope_desc(code, weight_type, batch, tokens, q_heads, k_heads, dim, rotary, 1 if interleaved else 0,
                              position_type, eps, rows, cos, sin, at, _dense(q_weight, shape, "q_weight"),
                              _dense(k_weight, shape, "k_weight"))
    return d, qs, ks


# ---- entry points ----------------------------------------------------------

def sdp_qk_norm_rope(ctx, q, k, q_out, k_out, cos=None, sin=None, *, q_weight=None, k_weight=None, positions=None,
                     eps: float = 1e-6, interleaved: bool = False, stream=None) -> None:
    d, qs, ks = _qk_desc(q, k, cos, sin, q_weight, k_weight, positions, eps, interleaved)
    code = d.type
    _same_type(q_out, code, "q_out")
    _same_type(k_out, code, "k_out")
    # (a structure passed for a pointer to one goes by reference)
    _check(_lib.sdp_qk_norm_rope(ctx, d, _heads(q, qs, "q"), _heads(k, ks, "k"), _heads(q_out, qs, "q_out"),
                                 _heads(k_out, ks, "k_out"), _stream(stream)))


def sdp_qk_norm_rope_backward(ctx, q, k, dq_out, dk_out, dq, dk, cos=None, sin=None, *, q_weight=None, k_weight=None,
                              dq_weight=None, dk_weight=None, positions=None, eps: float = 1e-6,
                              interleaved: bool = False, stream=None) -> None:
    d, qs, ks = _qk_desc(q, k, cos, sin, q_weight, k_weight, positions, eps, interleaved)
    code = d.type
    _same_type(dq_out, code, "dq_out")
    _same_type(dk_out, code, "dk_out")
    _same_type(dq, code, "dq")
    _same_type(dk, code, "dk")
    some = dk_weight if dq_weight is None else dq_weight
    if some is not None:
        if q_weight is None and k_weight is None:
            d.weight_type = _type(some, "a weight gradient")
        _same_type(some, d.weight_type, "a weight gradient")
        _same_type(dk_weight, d.weight_type, "a weight gradient")
    shape = (qs[3],)
    _check(_lib.sdp_qk_norm_rope_backward(
        ctx, d, _heads(q, qs, "q"), _heads(k, ks, "k"), _heads(dq_out, qs, "dq_out"), _heads(dk_out, ks, "dk_out"),
        _heads(dq, qs, "dq"), _heads(dk, ks, "dk"), _dense(dq_weight, shape, "dq_weight"),
        _dense(dk_weight, shape, "dk_weight"), _stream(stream)))


def _grouped_desc(rows, w, ends, out, strides, what: str):
    """strides: of x, of y (or dy) and of dx."""
    shape, count = w.shape, ends.shape
    if rows.dim() != 2 or len(shape) != 3 or len(count) != 1:
        raise ValueError(f"{what}: rows must be 2-D, w [groups, out, in] and ends [groups]")
    _want(w.is_contiguous(), "w must be contiguous")
    groups, n_out, n_in = shape
    _count(max(shape), "w")
    n = rows.shape[0]
    _same_type(w, SDP_TYPE_BF16, "w")
    x, y, dx = strides
    _same_type(x, SDP_TYPE_BF16, "x")
    _same_type(dx, SDP_TYPE_BF16, "dx")
    return sdp_grouped_desc(n, groups, n_in, n_out, SDP_TYPE_BF16 if out is None else _type(out, "an output"),
                            _type(ends, "ends"), _dense(ends, (groups,), "ends"),
                            0 if x is None else _row_stride(x, (n, n_in), "x"), _row_stride(y, (n, n_out), "y"),
                            0 if dx is None else _row_stride(dx, (n, n_in), "dx"))


def sdp_grouped_matmul(ctx, x, w, ends, y, *, stream=None) -> None:
    d = _grouped_desc(x, w, ends, y, (x, y, None), "sdp_grouped_matmul")
    _check(_lib.sdp_grouped_matmul(ctx, d, x.data_ptr(), w.data_ptr(), y.data_ptr(), _stream(stream)))


def sdp_grouped_matmul_backward(ctx, x, w, ends, dy, dx=None, dw=None, *, stream=None) -> None:
    """x may be None without dw; w is always given (its shape names the products)."""
    _same_type(dy, SDP_TYPE_BF16, "dy")
    d = _grouped_desc(dy, w, ends, dw, (x, dy, dx), "sdp_grouped_matmul_backward")
    _check(_lib.sdp_grouped_matmul_backward(ctx, d, _ptr(x), w.data_ptr(), dy.data_ptr(), _ptr(dx),
                                            _dense(dw, w.shape, "dw"), _stream(stream)))


def _distill_desc(logits, teacher_logits, teacher_index, labels, temperature, distill_weight, label_weight):
    shape = logits.shape
    _want(len(shape) == 2, "logits must be [rows, vocab]")
    rows, vocab = shape
    _count(vocab, "logits")
    k, teacher_type, index_type = 0, SDP_TYPE_F32, SDP_TYPE_I64
    teacher = index = label = None
    _want((teacher_logits is None) == (teacher_index is None), "teacher_logits and teacher_index go together")
    if teacher_logits is not None:
        given = teacher_logits.shape
        _want(len(given) == 2, "teacher_logits must be [rows, k]")
        k = given[1]
        _count(k, "teacher_logits")
        teacher_type, index_type = _type(teacher_logits, "teacher_logits"), _type(teacher_index, "teacher_index")
        teacher = _dense(teacher_logits, (rows, k), "teacher_logits")
        index = _dense(teacher_index, (rows, k), "teacher_index")
    if labels is not None:
        if teacher_index is not None:
            _same_type(labels, index_type, "labels")
        index_type = _type(labels, "labels")
        label = _dense(labels, (rows,), "labels")
    return sdp_distill_desc(rows, vocab, _type(logits, "logits"), logits.data_ptr(),
                            _row_stride(logits, shape, "logits"), k, teacher_type, index_type, teacher, index, label,
                            temperature, distill_weight, label_weight)


def _dlogits(d, shape, dlogits):
    if dlogits is None:
        return None, 0
    _same_type(dlogits, d.logit_type, "dlogits")
    return dlogits.data_ptr(), _row_stride(dlogits, shape, "dlogits")


def _f32(t, shape, what: str) -> Optional[int]:
    _same_type(t, SDP_TYPE_F32, what)
    return _dense(t, shape, what)


def sdp_distill_loss(ctx, logits, loss, lse=None, *, teacher_logits=None, teacher_index=None, labels=None,
                     temperature: float = 1.0, distill_weight: float = 1.0, label_weight: float = 0.0, row_grad=None,
                     dlogits=None, stream=None) -> None:
    d = _distill_desc(logits, teacher_logits, teacher_index, labels, temperature, distill_weight, label_weight)
    shape = logits.shape
    at, stride = _dlogits(d, shape, dlogits)
    rows = (shape[0],)
    _check(_lib.sdp_distill_loss(ctx, d, _f32(loss, rows, "loss"), _f32(lse, (shape[0], 2), "lse"),
                                 _f32(row_grad, rows, "row_grad"), at, stride, _stream(stream)))


def sdp_distill_loss_backward(ctx, logits, lse, row_grad, dlogits, *, teacher_logits=None, teacher_index=None,
                              labels=None, temperature: float = 1.0, distill_weight: float = 1.0,
                              label_weight: float = 0.0, stream=None) -> None:
    d = _distill_desc(logits, teacher_logits, teacher_index, labels, temperature, distill_weight, label_weight)
    shape = logits.shape
    at, stride = _dlogits(d, shape, dlogits)
    _check(_lib.sdp_distill_loss_backward(ctx, d, _f32(lse, (shape[0], 2), "lse"),
                                          _f32(row_grad, (shape[0],), "row_grad"), at, stride, _stream(stream)))
