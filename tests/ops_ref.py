"""The training operators from their definitions in 64 bits, on the CPU, and
the error that 32-bit arithmetic may make, for the tests.

A bound is returned beside each value: half a unit of the output's type (its
one rounding) plus a count of 32-bit roundings times the size of what they
round.
"""
import torch

U32 = 2.0 ** -24
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # 24 and 8 significant bits
TINY = 1e-37  # below the normal range of both types a rounding is absolute


def check(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(got), bad), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities differ"
    fine = ~bad & ~inf
    off = ((got - want).abs() - bound - TINY)[fine]
    if off.numel():
        worst = off.max().item()
        assert worst <= 0.0, f"{what}: past its bound by {worst:.3e} ({int((off > 0).sum())} of {off.numel()})"


def rounded(want, dtype, more):
    """The bound of a value rounded once to dtype after an error of `more`."""
    return HALF_UNIT[dtype] * (want.abs() + more) * (1 + 2.0 ** -8) + more


# ---- norms and rotation -------------------------------------------------------

def pair_index(rotary, interleaved):
    i = torch.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def rotate(n, cos, sin, rotary, interleaved, back=False):
    """n [batch, tokens, heads, dim] with each pair turned by its angle (back: the transpose)."""
    if rotary == 0:
        return n.clone()
    lo, hi = pair_index(rotary, interleaved)
    c, s = cos[:, :, None], sin[:, :, None] * (-1 if back else 1)
    y = n.clone()
    y[..., lo], y[..., hi] = n[..., lo] * c - n[..., hi] * s, n[..., hi] * c + n[..., lo] * s
    return y


def angles(cos, sin, positions):
    """The tables' rows of each token in 64 bits; NaN for a position outside the table."""
    if cos is None:
        return None, None
    at = positions.cpu().long()
    ok = (at >= 0) & (at < cos.shape[0])
    rows = [t.cpu().double()[at.clamp(0, max(0, cos.shape[0] - 1))] for t in (cos, sin)]
    return tuple(torch.where(ok[..., None], r, float("nan")) for r in rows)


def norm_rope(x, w, cos, sin, positions, rotary, interleaved, eps, dtype):
    x = x.cpu().double()
    d = x.shape[-1]
    w = torch.ones(d, dtype=torch.float64) if w is None else w.cpu().double()
    n = x * w / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    c, s = angles(cos, sin, positions)
    y = rotate(n, c, s, rotary, interleaved)
    out_of_table = torch.isnan(c[..., :1]).any(-1)[:, :, None, None] if rotary else None
    size = n.abs()
    if rotary:
        lo, hi = pair_index(rotary, interleaved)
        both = n[..., lo].abs() + n[..., hi].abs()
        size[..., lo], size[..., hi] = both, both
        y = torch.where(out_of_table, float("nan"), y)
    # the sum of d squares, its root and reciprocal, two products, the rotation's three roundings
    return y, rounded(y, dtype, (d / 2 + 16) * U32 * size)


def norm_rope_back(x, w, dy, cos, sin, positions, rotary, interleaved, eps, dtype, wdtype):
    x, dy = x.cpu().double(), dy.cpu().double()
    d = x.shape[-1]
    w = torch.ones(d, dtype=torch.float64) if w is None else w.cpu().double()
    r = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    unit = x * r
    c, s = angles(cos, sin, positions)
    dn = rotate(dy, c, s, rotary, interleaved, back=True)
    size = dy.abs()
    if rotary:
        dn = torch.where(torch.isnan(c[..., :1]).any(-1)[:, :, None, None], float("nan"), dn)
        lo, hi = pair_index(rotary, interleaved)
        both = dy[..., lo].abs() + dy[..., hi].abs()
        size[..., lo], size[..., hi] = both, both
    dw = (dn * unit).sum((0, 1, 2))
    u = dn * w
    dx = r * (u - unit * (u * unit).mean(-1, keepdim=True))
    big = (size * w.abs())
    dx_size = r * (big + unit.abs() * (big * unit.abs()).mean(-1, keepdim=True))
    rows = x[..., 0].numel()
    dw_size = (size * unit.abs()).sum((0, 1, 2))
    return (dx, rounded(dx, dtype, (d + 32) * U32 * dx_size)), \
           (dw, rounded(dw, wdtype, (rows / 2 + d / 2 + 64) * U32 * dw_size))


# ---- grouped products ------------------------------------------------------------

def group_bounds(ends, rows):
    """Each group's rows: ends that fall back or pass the rows are taken as the one before, or as rows."""
    out, at = [], 0
    for e in ends.cpu().tolist():
        end = max(at, min(max(e, 0), rows))
        out.append((at, end))
        at = end
    return out


def product(a, b, dtype):
    """a @ b in 64 bits and its bound: every product and sum rounded (or cut) to 32 bits."""
    a, b = a.cpu().double(), b.cpu().double()
    want = a @ b
    return want, rounded(want, dtype, 2 * (a.shape[1] + 2) * U32 * (a.abs() @ b.abs()))


def grouped(x, w, ends, dtype):
    rows, out = x.shape[0], w.shape[1]
    want, bound = torch.zeros((rows, out), dtype=torch.float64), torch.zeros((rows, out), dtype=torch.float64)
    for e, (a, b) in enumerate(group_bounds(ends, rows)):
        if b > a:
            want[a:b], bound[a:b] = product(x[a:b], w[e].t(), dtype)
    return want, bound


def grouped_back(x, w, ends, dy, dtype):
    rows, n_in = x.shape[0], w.shape[2]
    dx, dx_b = torch.zeros((rows, n_in), dtype=torch.float64), torch.zeros((rows, n_in), dtype=torch.float64)
    dw, dw_b = torch.zeros(w.shape, dtype=torch.float64), torch.zeros(w.shape, dtype=torch.float64)
    for e, (a, b) in enumerate(group_bounds(ends, rows)):
        if b > a:
            dx[a:b], dx_b[a:b] = product(dy[a:b], w[e], torch.bfloat16)
            dw[e], dw_b[e] = product(dy[a:b].t(), x[a:b], dtype)
    return (dx, dx_b), (dw, dw_b)


# ---- distillation -----------------------------------------------------------------

def distill_loss(z, teacher, index, labels, tau, a, b):
    """Per-row loss, L_tau, L_1 and the teacher's q, in 64 bits; differentiable in z."""
    rows, vocab = z.shape
    l_tau, l_one = torch.logsumexp(z / tau, 1), torch.logsumexp(z, 1)
    loss = torch.zeros(rows, dtype=torch.float64)
    q = torch.zeros((rows, 0 if index is None else index.shape[1]), dtype=torch.float64)
    has_t = torch.zeros(rows, dtype=torch.bool)
    if index is not None and index.shape[1]:
        there = index >= 0
        t = torch.where(there, teacher / tau, float("-inf"))
        has_t = ~torch.isneginf(t).all(1)
        q = torch.where(has_t[:, None], torch.softmax(torch.where(has_t[:, None], t, 0.0), 1), 0.0)
        zi = z.gather(1, index.clamp(0, vocab - 1))
        log_q = torch.where(q > 0, q, 1.0).log()
        term = torch.where(q > 0, q * (log_q - zi / tau + l_tau[:, None]), 0.0)
        term = torch.where(torch.isnan(q), float("nan"), term)
        if a:
            loss = loss + torch.where(has_t, a * tau * tau * term.sum(1), 0.0)
    has_l = torch.zeros(rows, dtype=torch.bool)
    if labels is not None and b:
        has_l = labels >= 0
        zl = z.gather(1, labels.clamp(0, vocab - 1)[:, None])[:, 0]
        loss = loss + torch.where(has_l, b * (l_one - zl), 0.0)
    bad = torch.zeros(rows, dtype=torch.bool)
    if index is not None and index.shape[1]:
        bad |= (index >= vocab).any(1)
    if labels is not None and b:
        bad |= labels >= vocab
    if not a:
        has_t = torch.zeros_like(has_t)
    return loss, l_tau, l_one, q, has_t, has_l, bad


def distill(z, teacher, index, labels, tau, a, b, row_grad, dtype):
    """Loss, lse and the gradient with their bounds."""
    z = z.cpu().double()
    rows, vocab = z.shape
    index = None if index is None else index.cpu().long()
    teacher = None if teacher is None else teacher.cpu().double()
    labels = None if labels is None else labels.cpu().long()
    loss, l_tau, l_one, q, has_t, has_l, bad = distill_loss(z, teacher, index, labels, tau, a, b)
    loss = torch.where(bad, float("nan"), loss)
    lse = torch.stack((l_tau, l_one), 1)
    # the sums' roundings (256 or more lanes share a row), the exponentials'
    # argument (as large as the logits' distance from the top that still counts)
    # and the logarithm
    finite = lambda t: torch.where(torch.isfinite(t), t.abs(), 0.0)
    e_lse = (min(vocab, vocab / 256 + 64) + 64) * U32 + 4 * U32 * (finite(lse) + finite(z.max(1).values)[:, None] / min(tau, 1.0))
    k = q.shape[1]
    size = torch.zeros(rows, dtype=torch.float64)
    if k:
        zi = finite(z.gather(1, index.clamp(0, vocab - 1))) / tau
        ti = torch.where(index >= 0, finite(teacher), 0.0).max(1).values / tau
        size += a * tau * tau * ((q * (zi + 4 * ti[:, None])).sum(1) + 4 * ti + finite(l_tau) + 8 + k / 8) * 8
    zl = finite(z.gather(1, labels.clamp(0, vocab - 1)[:, None])[:, 0]) if labels is not None else 0.0
    size += b * (finite(l_one) + zl) * 4
    e_loss = abs(a) * tau * tau * e_lse[:, 0] + abs(b) * e_lse[:, 1] + U32 * size
    out = [(loss, e_loss), (lse, e_lse + U32 * finite(lse))]
    if row_grad is None:
        return out
    g = row_grad.cpu().double()
    c_t, c_l = (torch.where(m, g * w, 0.0)[:, None] for m, w in ((has_t, a * tau), (has_l, b)))
    p_t = torch.where(c_t != 0, (z / tau - l_tau[:, None]).exp(), 0.0)
    p_l = torch.where(c_l != 0, (z - l_one[:, None]).exp(), 0.0)
    d = torch.where(c_t != 0, c_t * p_t, 0.0) + torch.where(c_l != 0, c_l * p_l, 0.0)
    # an exponent's rounding grows with its size; where that is past 40, the value is below any bound
    rel = 8 * U32 * (8 + torch.minimum(finite(z) / min(tau, 1.0) + finite(lse).max(1).values[:, None], torch.tensor(1e4))) \
        + 2 * e_lse.max(1).values[:, None]
    err = (c_t.abs() * p_t + c_l.abs() * p_l) * rel
    if k:
        hit = torch.zeros_like(d).scatter_add_(1, index.clamp(0, vocab - 1), torch.where(index >= 0, q, 0.0))
        d = d - torch.where(c_t != 0, c_t * hit, 0.0)
        qe = U32 * (8 * ti[:, None] + 32 + k)
        err = err + c_t.abs() * hit * qe
    if labels is not None:
        at = torch.zeros_like(d).scatter_(1, labels.clamp(0, vocab - 1)[:, None], 1.0)
        d = d - torch.where(c_l != 0, c_l * at, 0.0)
        err = err + c_l.abs() * at * 4 * U32
    d = torch.where((bad & (g != 0))[:, None], float("nan"), d)
    out.append((d, rounded(d, dtype, err)))
    return out
