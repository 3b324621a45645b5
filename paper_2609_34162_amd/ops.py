"""ctypes binding of the training operators (include/sdp_ops.h and
include/sdp_layer.h): argument marshalling only.

Every function here has the name of the C entry point it calls; it takes torch
tensors, checks that their shapes belong together and passes their addresses
and strides on.  Outputs are tensors of the caller's.  The library checks the
rest (types, ranges, overlaps) and a negative status becomes an exception.
`stream` is a torch stream or a raw handle; None is the null stream.
"""
import ctypes
import struct
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
SDP_ROUTE_MAX_EXPERTS = 2048
SDP_ROUTE_MAX_TOP = 64
SDP_ROUTE_MAX_GROUPS = 64
SDP_GATE_NONE = 0
SDP_GATE_CHANNEL = 1
SDP_GATE_TOKEN = 2
SDP_GATE_ELEMENT = 3


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


class sdp_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


class sdp_embed_desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("vocab", "hidden", "table_type", "row_type", "id_type")] + \
               [("ids", ctypes.c_void_p), ("scale", ctypes.c_double)]


class sdp_block_norm_desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("hidden", "stream_type", "type", "weight_type", "post_norm", "gate_form",
                                              "gate_sigmoid")] + \
               [(n, ctypes.c_double) for n in ("scale", "eps", "weight_offset")] + \
               [("gate", ctypes.c_void_p), ("gate_stride", ctypes.c_int64), ("post_weight", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p)]


class sdp_block_norm_grads(ctypes.Structure):
    _fields_ = [("dh", ctypes.POINTER(sdp_rows)), ("dy", ctypes.POINTER(sdp_rows)), ("dgate", ctypes.c_void_p),
                ("dgate_stride", ctypes.c_int64), ("dpost_weight", ctypes.c_void_p),
                ("dpre_weight", ctypes.c_void_p)]


class sdp_route_desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("experts", "top", "logit_type", "index_type", "weight_type", "sigmoid",
                                              "renormalize", "groups", "top_groups", "group_best")] + \
               [("scale", ctypes.c_double), ("logit_stride", ctypes.c_int64)]


class sdp_order_desc(ctypes.Structure):
    _fields_ = [("entries", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("experts", "index_type", "ends_type")]


class sdp_expert_desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("top", "hidden", "row_type", "stream_type", "weight_type")] + \
               [("place", ctypes.c_void_p)]


def _codes(kind) -> list:
    codes = {ctypes.c_int32: "i", ctypes.c_int64: "q", ctypes.c_double: "d", ctypes.c_void_p: "P"}
    return [codes.get(t, "P") for _, t in kind._fields_]


def _packer(kind):
    """A function of a structure's fields, in their order, to its bytes: several times as fast as the
    structure itself, and taken like it where a pointer to one is wanted.  Pointers are numbers."""
    return struct.Struct("@" + "".join(_codes(kind)) + "0q").pack


def _refusing_packer(kind):
    """The same where fields are the caller's numbers, one of which may be none that the field holds."""
    whole = _packer(kind)

    def pack(*values):
        try:
            return whole(*values)
        except (struct.error, OverflowError):
            for (name, _), code, v in zip(kind._fields_, _codes(kind), values):
                try:
                    struct.pack(code, v)
                except (struct.error, OverflowError) as e:
                    raise ValueError(f"{name}: {e}") from None
            raise
    return pack


_rows_bytes, _grads_bytes, _order_bytes, _expert_bytes = map(
    _packer, (sdp_rows, sdp_block_norm_grads, sdp_order_desc, sdp_expert_desc))
_embed_bytes, _norm_bytes, _route_bytes = map(
    _refusing_packer, (sdp_embed_desc, sdp_block_norm_desc, sdp_route_desc))


def _bind():
    vp, i32, i64, P = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.POINTER
    h, qk, gm, ds = P(sdp_heads), P(sdp_qk_norm_rope_desc), P(sdp_grouped_desc), P(sdp_distill_desc)
    for name, args in {
        # (descriptions and rows are bytes, or structures by reference)
        "sdp_embed": [vp, vp, vp, vp, vp],
        "sdp_embed_backward": [vp, vp, vp, vp, i32, vp],
        "sdp_block_norm": [vp, vp, vp, vp, vp, vp, vp],
        "sdp_block_norm_backward": [vp, vp, vp, vp, vp, vp, vp, vp],
        "sdp_route": [vp, vp, vp, vp, vp, vp, vp],
        "sdp_route_backward": [vp, vp, vp, vp, vp, vp, i64, vp],
        "sdp_expert_order": [vp, vp, vp, vp, vp, vp, vp],
        "sdp_expert_gather": [vp, vp, vp, vp, vp],
        "sdp_expert_gather_backward": [vp, vp, vp, vp, vp],
        "sdp_expert_combine": [vp, vp, vp, vp, vp, vp, vp],
        "sdp_expert_combine_backward": [vp, vp, vp, vp, vp, vp, vp, vp],
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


_TYPE_OF = {}  # filled by the first call


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


# ---- around the experts' products (include/sdp_layer.h) ------------------------
# What they refuse is found by one comparison of several things at a time, and named after.

def _refuse_rows(t, shape, code: int, what: str) -> None:
    _same_type(t, code, what)
    _row_stride(t, shape, what)


def _at(t, shape, code: int, what: str):
    """Address and row stride of a 2-D tensor of this shape and type."""
    strides = t.stride()
    if t.shape != shape or _TYPE_OF.get(t.dtype) != code or (strides[1] != 1 and shape[1] > 1):
        _refuse_rows(t, shape, code, what)
    return t.data_ptr(), strides[0]


def _rows(t, shape, code: int, what: str) -> Optional[bytes]:
    """The sdp_rows of such a tensor (None passes)."""
    if t is None:
        return None
    strides = t.stride()
    if t.shape != shape or _TYPE_OF.get(t.dtype) != code or (strides[1] != 1 and shape[1] > 1):
        _refuse_rows(t, shape, code, what)
    return _rows_bytes(t.data_ptr(), strides[0])


def _flat(t, shape, code: int, what: str) -> int:
    """The address of a contiguous tensor of this shape and type (0 for None)."""
    if t is None:
        return 0
    if t.shape != shape or _TYPE_OF.get(t.dtype) != code or not t.is_contiguous():
        _same_type(t, code, what)
        _dense(t, shape, what)
    return t.data_ptr()


def _two(t, what: str):
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{what} must be 2-D")
    return shape


def _embed(call, ctx, table, rows, tokens, scale, table_name, rows_name, stream, *more) -> None:
    shape, count = _two(table, table_name), tokens.shape
    vocab, hidden = shape
    if vocab > 0x7fffffff or hidden > 0x7fffffff:
        _count(max(vocab, hidden), table_name)
    if len(count) != 1:
        raise ValueError("tokens must be 1-D")
    n = count[0]
    table_type, row_type, id_type = _type(table, table_name), _type(rows, rows_name), _type(tokens, "tokens")
    d = _embed_bytes(n, vocab, hidden, table_type, row_type, id_type, _flat(tokens, count, id_type, "tokens"), scale)
    t, r = _rows(table, shape, table_type, table_name), _rows(rows, (n, hidden), row_type, rows_name)
    _check(call(ctx, d, r, t, *more, _stream(stream)) if more else call(ctx, d, t, r, _stream(stream)))


def sdp_embed(ctx, table, tokens, out, *, scale: float = 1.0, stream=None) -> None:
    _embed(_lib.sdp_embed, ctx, table, out, tokens, scale, "table", "out", stream)


def sdp_embed_backward(ctx, dout, tokens, dtable, *, scale: float = 1.0, accumulate: bool = False,
                       stream=None) -> None:
    _embed(_lib.sdp_embed_backward, ctx, dtable, dout, tokens, scale, "dtable", "dout", stream, 1 if accumulate else 0)


def _gate(t, tokens: int, hidden: int, code: int, what: str):
    """Form, address and stride of a gate [hidden] or [1, hidden], [tokens, 1] or
    [tokens, hidden]; of one token or one channel the form of the most elements."""
    if t is None:
        return SDP_GATE_NONE, 0, 0
    shape = t.shape
    if shape == (hidden,) or (shape == (1, hidden) and tokens != 1):
        return SDP_GATE_CHANNEL, _flat(t, shape, code, what), 0
    if shape == (tokens, hidden) or shape == (tokens, 1):
        return (SDP_GATE_ELEMENT if shape[1] == hidden else SDP_GATE_TOKEN, *_at(t, shape, code, what))
    raise ValueError(f"{what} has shape {tuple(shape)}, expected [{hidden}], [{tokens}, 1] or [{tokens}, {hidden}]")


def _norm_desc(stream_t, some, weight, gate, sigmoid, post_norm, post_weight, pre_weight, scale, eps, offset):
    """stream_t: a tensor of the stream; some: one of y's type, or None; weight: a weight or its gradient, or None."""
    shape = _two(stream_t, "the stream")
    tokens, hidden = shape
    if hidden > 0x7fffffff:
        _count(hidden, "the stream")
    stream_type = _type(stream_t, "the stream")
    if some is None:
        some = gate
    code = stream_type if some is None else _type(some, "y")
    weight_type = SDP_TYPE_F32 if weight is None else _type(weight, "a weight")
    if weight is not None:
        _same_type(post_weight, weight_type, "a weight")
        _same_type(pre_weight, weight_type, "a weight")
    form, at, stride = _gate(gate, tokens, hidden, code, "gate")
    wide = (hidden,)
    d = _norm_bytes(tokens, hidden, stream_type, code, weight_type, 1 if post_norm else 0, form, 1 if sigmoid else 0,
                    scale, eps, offset, at, stride, _flat(post_weight, wide, weight_type, "post_weight"),
                    _flat(pre_weight, wide, weight_type, "pre_weight"))
    return d, shape, stream_type, code, weight_type, form


def sdp_block_norm(ctx, h, y, h_out, n_out, *, gate=None, gate_sigmoid: bool = False, post_norm: bool = False,
                   post_weight=None, pre_weight=None, scale: float = 1.0, eps: float = 1e-6,
                   weight_offset: float = 0.0, stream=None) -> None:
    """y and h_out may be None (the norm alone), or n_out."""
    d, shape, s, c, _, _ = _norm_desc(h, n_out if y is None else y, post_weight if pre_weight is None else pre_weight,
                                      gate, gate_sigmoid, post_norm, post_weight, pre_weight, scale, eps, weight_offset)
    _check(_lib.sdp_block_norm(ctx, d, _rows(h, shape, s, "h"), _rows(y, shape, c, "y"), _rows(h_out, shape, s, "h_out"),
                               _rows(n_out, shape, c, "n_out"), _stream(stream)))


def _first(*tensors):
    return next((t for t in tensors if t is not None), None)


def sdp_block_norm_backward(ctx, h_out, y, dh_out, dn, dh, dy, *, gate=None, dgate=None, gate_sigmoid: bool = False,
                            post_norm: bool = False, post_weight=None, dpost_weight=None, pre_weight=None,
                            dpre_weight=None, scale: float = 1.0, eps: float = 1e-6, weight_offset: float = 0.0,
                            stream=None) -> None:
    """h_out is the stream after the addition; any tensor that the call does not need may be None."""
    some = _first(h_out, dh_out, dh)
    _want(some is not None, "h_out, dh_out and dh are all None")
    d, shape, s, c, w, form = _norm_desc(some, _first(y, dn, dy),
                                         _first(post_weight, pre_weight, dpost_weight, dpre_weight), gate, gate_sigmoid,
                                         post_norm, post_weight, pre_weight, scale, eps, weight_offset)
    gate_form, at, stride = _gate(dgate, shape[0], shape[1], c, "dgate")
    if dgate is not None and gate_form != form:
        raise ValueError("dgate has another form than gate")
    _same_type(dpost_weight, w, "a weight")
    _same_type(dpre_weight, w, "a weight")
    wide = (shape[1],)
    out_h = None if dh is None else sdp_rows(*_at(dh, shape, s, "dh"))
    out_y = None if dy is None else sdp_rows(*_at(dy, shape, c, "dy"))
    where = ctypes.addressof
    grads = _grads_bytes(0 if out_h is None else where(out_h), 0 if out_y is None else where(out_y), at, stride,
                         _flat(dpost_weight, wide, w, "dpost_weight"), _flat(dpre_weight, wide, w, "dpre_weight"))
    _check(_lib.sdp_block_norm_backward(ctx, d, _rows(h_out, shape, s, "h_out"), _rows(y, shape, c, "y"),
                                        _rows(dh_out, shape, s, "dh_out"), _rows(dn, shape, c, "dn"), grads,
                                        _stream(stream)))


def _route_desc(logits, index, weights, sigmoid, groups, top_groups, group_best, renormalize, scale, name):
    """Description, and the addresses of logits, index and weights."""
    shape, chosen = _two(logits, "logits"), _two(index, "index")
    tokens, experts = shape
    top = chosen[1]
    if experts > 0x7fffffff or top > 0x7fffffff:
        _count(max(experts, top), "logits and index")
    if chosen[0] != tokens:
        raise ValueError(f"index has {chosen[0]} rows, expected {tokens}")
    code, index_type, weight_type = _type(logits, "logits"), _type(index, "index"), _type(weights, name)
    z, stride = _at(logits, shape, code, "logits")
    i, w = _flat(index, chosen, index_type, "index"), _flat(weights, chosen, weight_type, name)
    d = _route_bytes(tokens, experts, top, code, index_type, weight_type, 1 if sigmoid else 0, 1 if renormalize else 0,
                     groups, top_groups, group_best, scale, stride)
    return d, z, i, w, shape, code


def sdp_route(ctx, logits, index, weights, *, bias=None, sigmoid: bool = False, groups: int = 1, top_groups: int = 1,
              group_best: int = 1, renormalize: bool = False, scale: float = 1.0, stream=None) -> None:
    d, z, i, w, shape, _ = _route_desc(logits, index, weights, sigmoid, groups, top_groups, group_best, renormalize,
                                       scale, "weights")
    b = None if bias is None else _flat(bias, (shape[1],), SDP_TYPE_F32, "bias")
    _check(_lib.sdp_route(ctx, d, z, b, i, w, _stream(stream)))


def sdp_route_backward(ctx, logits, index, dweights, dlogits, *, sigmoid: bool = False, renormalize: bool = False,
                       scale: float = 1.0, stream=None) -> None:
    d, z, i, w, shape, code = _route_desc(logits, index, dweights, sigmoid, 1, 1, 1, renormalize, scale, "dweights")
    _check(_lib.sdp_route_backward(ctx, d, z, i, w, *_at(dlogits, shape, code, "dlogits"), _stream(stream)))


def sdp_expert_order(ctx, index, ends, place, order=None, *, stream=None) -> None:
    """index, place: [tokens, top] or [entries]; order: [entries], or None."""
    shape, experts = index.shape, ends.shape
    if len(experts) != 1:
        raise ValueError("ends must be 1-D")
    _count(experts[0], "ends")
    n = index.numel()
    index_type, ends_type = _type(index, "index"), _type(ends, "ends")
    d = _order_bytes(n, experts[0], index_type, ends_type)
    _check(_lib.sdp_expert_order(ctx, d, _flat(index, shape, index_type, "index"), _flat(ends, experts, ends_type, "ends"),
                                 _flat(place, shape, SDP_TYPE_I32, "place"), _flat(order, (n,), SDP_TYPE_I32, "order"),
                                 _stream(stream)))


def _expert_desc(place, hidden: int, row_type: int, stream_type: int, weight_type: int):
    """Description, and the shapes of place, of the tokens' tensors and of the sorted rows."""
    shape = _two(place, "place")
    tokens, top = shape
    if tokens > 0x7fffffff or top > 0x7fffffff or hidden > 0x7fffffff:
        _count(max(tokens, top, hidden), "place and the rows")
    return _expert_bytes(tokens, top, hidden, row_type, stream_type, weight_type,
                         _flat(place, shape, SDP_TYPE_I32, "place")), shape, (tokens, hidden), (tokens * top, hidden)


def sdp_expert_gather(ctx, x, place, rows, *, stream=None) -> None:
    code = _type(x, "x")
    d, _, side, sorted_rows = _expert_desc(place, _two(x, "x")[1], code, code, SDP_TYPE_F32)
    _check(_lib.sdp_expert_gather(ctx, d, _rows(x, side, code, "x"), _rows(rows, sorted_rows, code, "rows"),
                                  _stream(stream)))


def sdp_expert_gather_backward(ctx, drows, place, dx, *, stream=None) -> None:
    code = _type(drows, "drows")
    d, _, side, sorted_rows = _expert_desc(place, _two(drows, "drows")[1], code, code, SDP_TYPE_F32)
    _check(_lib.sdp_expert_gather_backward(ctx, d, _rows(drows, sorted_rows, code, "drows"),
                                           _rows(dx, side, code, "dx"), _stream(stream)))


def sdp_expert_combine(ctx, rows, place, weights, out, *, residual=None, stream=None) -> None:
    code, to, w = _type(rows, "rows"), _type(out, "out"), _type(weights, "weights")
    d, shape, side, sorted_rows = _expert_desc(place, _two(rows, "rows")[1], code, to, w)
    _check(_lib.sdp_expert_combine(ctx, d, _rows(rows, sorted_rows, code, "rows"), _flat(weights, shape, w, "weights"),
                                   _rows(residual, side, to, "residual"), _rows(out, side, to, "out"),
                                   _stream(stream)))


def sdp_expert_combine_backward(ctx, rows, place, weights, dout, drows=None, dweights=None, *, stream=None) -> None:
    """drows or dweights may be None; rows without dweights, weights without drows."""
    some, some_w = _first(rows, drows), _first(weights, dweights)
    to = _type(dout, "dout")
    code, w = to if some is None else _type(some, "rows"), SDP_TYPE_F32 if some_w is None else _type(some_w, "weights")
    d, shape, side, sorted_rows = _expert_desc(place, _two(dout, "dout")[1], code, to, w)
    _check(_lib.sdp_expert_combine_backward(
        ctx, d, _rows(rows, sorted_rows, code, "rows"), _flat(weights, shape, w, "weights"),
        _rows(dout, side, to, "dout"), _rows(drows, sorted_rows, code, "drows"),
        _flat(dweights, shape, w, "dweights"), _stream(stream)))
