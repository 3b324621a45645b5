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
    if not _TYPE_OF:
        _TYPE_OF.update(_types())
    try:
        return _TYPE_OF[t.dtype]
    except KeyError:
        raise ValueError(f"{what} has type {t.dtype}") from None


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _want(ok: bool, text: str) -> None:
    if not ok:
        raise ValueError(text)


def _has_shape(t, shape, what: str) -> None:
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _last_contiguous(t, what: str) -> None:
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")


def _dense(t, shape, what: str) -> Optional[int]:
    """The address of a contiguous tensor of this shape (None passes)."""
    if t is None:
        return None
    _has_shape(t, shape, what)
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _same_type(t, code: int, what: str) -> None:
    if t is not None and _type(t, what) != code:
        raise ValueError(f"{what} has another type than expected")


def _row_stride(t, shape, what: str) -> int:
    _has_shape(t, shape, what)
    _last_contiguous(t, what)
    return t.stride(0)


def _heads(t, shape, what: str) -> sdp_heads:
    """[batch, tokens, heads, head_dim], or [tokens, heads, head_dim] of one sequence."""
    if t.dim() == 3:
        t = t.unsqueeze(0)
    _has_shape(t, shape, what)
    _last_contiguous(t, what)
    return sdp_heads(t.data_ptr(), *t.stride()[:3])


def _qk_desc(q, k, cos, sin, q_weight, k_weight, positions, eps, interleaved):
    def shape(t):
        _want(t.dim() in (3, 4), "q and k must be [batch, tokens, heads, head_dim]")
        return (1, *t.shape) if t.dim() == 3 else tuple(t.shape)
    qs, ks = shape(q), shape(k)
    if qs[:2] != ks[:2] or qs[3] != ks[3]:
        raise ValueError(f"q {qs} and k {ks} differ in batch, tokens or head_dim")
    code = _type(q, "q")
    _same_type(k, code, "k")
    d = sdp_qk_norm_rope_desc()
    d.type, d.batch, d.tokens, d.q_heads, d.k_heads, d.head_dim = code, qs[0], qs[1], qs[2], ks[2], qs[3]
    weights = [w for w in (q_weight, k_weight) if w is not None]
    d.weight_type = _type(weights[0], "a weight") if weights else SDP_TYPE_F32
    for w in weights:
        _same_type(w, d.weight_type, "a weight")
    d.q_weight, d.k_weight = _dense(q_weight, (qs[3],), "q_weight"), _dense(k_weight, (qs[3],), "k_weight")
    d.eps, d.interleaved = eps, int(bool(interleaved))
    if cos is not None:
        _want(cos.dim() == 2 and sin is not None, "cos and sin must be [table_rows, rotary_dim / 2]")
        _same_type(cos, SDP_TYPE_F32, "cos")
        _same_type(sin, SDP_TYPE_F32, "sin")
        d.table_rows, d.rotary_dim = cos.shape[0], 2 * cos.shape[1]
        d.cos, d.sin = _dense(cos, cos.shape, "cos"), _dense(sin, cos.shape, "sin")
    d.position_type = SDP_TYPE_I32
    if positions is not None:
        d.position_type = _type(positions, "positions")
        _want(positions.numel() == qs[0] * qs[1] and positions.is_contiguous(),
              "positions must be [batch, tokens], contiguous")
        d.positions = positions.data_ptr()
    return d, qs, ks


# ---- entry points ----------------------------------------------------------

def sdp_qk_norm_rope(ctx, q, k, q_out, k_out, cos=None, sin=None, *, q_weight=None, k_weight=None, positions=None,
                     eps: float = 1e-6, interleaved: bool = False, stream=None) -> None:
    d, qs, ks = _qk_desc(q, k, cos, sin, q_weight, k_weight, positions, eps, interleaved)
    for t, n in ((q_out, "q_out"), (k_out, "k_out")):
        _same_type(t, d.type, n)
    _check(_lib.sdp_qk_norm_rope(ctx, ctypes.byref(d), ctypes.byref(_heads(q, qs, "q")),
                                 ctypes.byref(_heads(k, ks, "k")), ctypes.byref(_heads(q_out, qs, "q_out")),
                                 ctypes.byref(_heads(k_out, ks, "k_out")), _stream(stream)))


def sdp_qk_norm_rope_backward(ctx, q, k, dq_out, dk_out, dq, dk, cos=None, sin=None, *, q_weight=None, k_weight=None,
                              dq_weight=None, dk_weight=None, positions=None, eps: float = 1e-6,
                              interleaved: bool = False, stream=None) -> None:
    d, qs, ks = _qk_desc(q, k, cos, sin, q_weight, k_weight, positions, eps, interleaved)
    for t, n in ((dq_out, "dq_out"), (dk_out, "dk_out"), (dq, "dq"), (dk, "dk")):
        _same_type(t, d.type, n)
    grads = [w for w in (dq_weight, dk_weight) if w is not None]
    if grads and q_weight is None and k_weight is None:
        d.weight_type = _type(grads[0], "a weight gradient")
    for w in grads:
        _same_type(w, d.weight_type, "a weight gradient")
    _check(_lib.sdp_qk_norm_rope_backward(
        ctx, ctypes.byref(d), ctypes.byref(_heads(q, qs, "q")), ctypes.byref(_heads(k, ks, "k")),
        ctypes.byref(_heads(dq_out, qs, "dq_out")), ctypes.byref(_heads(dk_out, ks, "dk_out")),
        ctypes.byref(_heads(dq, qs, "dq")), ctypes.byref(_heads(dk, ks, "dk")),
        _dense(dq_weight, (qs[3],), "dq_weight"), _dense(dk_weight, (qs[3],), "dk_weight"), _stream(stream)))


def _grouped_desc(x, w, ends, what: str):
    if x.dim() != 2 or w.dim() != 3 or ends.dim() != 1:
        raise ValueError(f"{what}: rows must be 2-D, w [groups, out, in] and ends [groups]")
    _want(w.is_contiguous(), "w must be contiguous")
    d = sdp_grouped_desc()
    d.rows, d.groups, d.out_features, d.in_features = x.shape[0], w.shape[0], w.shape[1], w.shape[2]
    d.ends, d.ends_type = _dense(ends, (w.shape[0],), "ends"), _type(ends, "ends")
    d.out_type = SDP_TYPE_BF16
    _same_type(w, SDP_TYPE_BF16, "w")
    return d


def sdp_grouped_matmul(ctx, x, w, ends, y, *, stream=None) -> None:
    d = _grouped_desc(x, w, ends, "sdp_grouped_matmul")
    _same_type(x, SDP_TYPE_BF16, "x")
    d.x_stride = _row_stride(x, (d.rows, d.in_features), "x")
    d.y_stride = _row_stride(y, (d.rows, d.out_features), "y")
    d.out_type = _type(y, "y")
    _check(_lib.sdp_grouped_matmul(ctx, ctypes.byref(d), x.data_ptr(), w.data_ptr(), y.data_ptr(), _stream(stream)))


def sdp_grouped_matmul_backward(ctx, x, w, ends, dy, dx=None, dw=None, *, stream=None) -> None:
    """x may be None without dw; w is always given (its shape names the products)."""
    d = _grouped_desc(dy, w, ends, "sdp_grouped_matmul_backward")
    _same_type(dy, SDP_TYPE_BF16, "dy")
    d.y_stride = _row_stride(dy, (d.rows, d.out_features), "dy")
    if x is not None:
        _same_type(x, SDP_TYPE_BF16, "x")
        d.x_stride = _row_stride(x, (d.rows, d.in_features), "x")
    if dx is not None:
        _same_type(dx, SDP_TYPE_BF16, "dx")
        d.dx_stride = _row_stride(dx, (d.rows, d.in_features), "dx")
    if dw is not None:
        d.out_type = _type(dw, "dw")
        _dense(dw, w.shape, "dw")
    _check(_lib.sdp_grouped_matmul_backward(ctx, ctypes.byref(d), _ptr(x), w.data_ptr(), dy.data_ptr(), _ptr(dx),
                                            _ptr(dw), _stream(stream)))


def _distill_desc(logits, teacher_logits, teacher_index, labels, temperature, distill_weight, label_weight):
    _want(logits.dim() == 2, "logits must be [rows, vocab]")
    d = sdp_distill_desc()
    d.rows, d.vocab = logits.shape
    d.logit_type, d.logits = _type(logits, "logits"), logits.data_ptr()
    d.logit_stride = _row_stride(logits, logits.shape, "logits")
    d.teacher_type, d.index_type = SDP_TYPE_F32, SDP_TYPE_I64
    _want((teacher_logits is None) == (teacher_index is None), "teacher_logits and teacher_index go together")
    if teacher_logits is not None:
        _want(teacher_logits.dim() == 2, "teacher_logits must be [rows, k]")
        shape = (d.rows, teacher_logits.shape[1])
        d.teacher_k = shape[1]
        d.teacher_type, d.index_type = _type(teacher_logits, "teacher_logits"), _type(teacher_index, "teacher_index")
        d.teacher_logits = _dense(teacher_logits, shape, "teacher_logits")
        d.teacher_index = _dense(teacher_index, shape, "teacher_index")
    if labels is not None:
        if teacher_index is not None:
            _same_type(labels, d.index_type, "labels")
        d.index_type = _type(labels, "labels")
        d.labels = _dense(labels, (d.rows,), "labels")
    d.temperature, d.distill_weight, d.label_weight = temperature, distill_weight, label_weight
    return d


def _dlogits(d, dlogits):
    if dlogits is None:
        return None, 0
    _same_type(dlogits, d.logit_type, "dlogits")
    return dlogits.data_ptr(), _row_stride(dlogits, (d.rows, d.vocab), "dlogits")


def _f32(t, shape, what: str) -> Optional[int]:
    _same_type(t, SDP_TYPE_F32, what)
    return _dense(t, shape, what)


def sdp_distill_loss(ctx, logits, loss, lse=None, *, teacher_logits=None, teacher_index=None, labels=None,
                     temperature: float = 1.0, distill_weight: float = 1.0, label_weight: float = 0.0, row_grad=None,
                     dlogits=None, stream=None) -> None:
    d = _distill_desc(logits, teacher_logits, teacher_index, labels, temperature, distill_weight, label_weight)
    at, stride = _dlogits(d, dlogits)
    _check(_lib.sdp_distill_loss(ctx, ctypes.byref(d), _f32(loss, (d.rows,), "loss"), _f32(lse, (d.rows, 2), "lse"),
                                 _f32(row_grad, (d.rows,), "row_grad"), at, stride, _stream(stream)))


def sdp_distill_loss_backward(ctx, logits, lse, row_grad, dlogits, *, teacher_logits=None, teacher_index=None,
                              labels=None, temperature: float = 1.0, distill_weight: float = 1.0,
                              label_weight: float = 0.0, stream=None) -> None:
    d = _distill_desc(logits, teacher_logits, teacher_index, labels, temperature, distill_weight, label_weight)
    at, stride = _dlogits(d, dlogits)
    _check(_lib.sdp_distill_loss_backward(ctx, ctypes.byref(d), _f32(lse, (d.rows, 2), "lse"),
                                          _f32(row_grad, (d.rows,), "row_grad"), at, stride, _stream(stream)))
