"""The training operators around the experts' products from their definitions in
64 bits, on the CPU, and the error that 32-bit arithmetic may make, for the tests.

A bound is returned beside each value, as in ops_ref.py: half a unit of the
output's type (its one rounding) plus a count of 32-bit roundings times the size
of what they round.  A sum of n terms in any order is off by at most n roundings
of the sum of their sizes; an exponential, a reciprocal or a root by a few.
"""
import torch

from ops_ref import U32, check, rounded  # noqa: F401  (check: what the tests compare with)

INF = float("inf")


def f64(t):
    return None if t is None else t.detach().cpu().double()


# ---- embeddings ---------------------------------------------------------------

def embed(table, ids, scale, dtype):
    table, ids = f64(table), ids.cpu().long()
    vocab = table.shape[0]
    out = table[ids.clamp(0, vocab - 1)] * scale if vocab else torch.zeros((len(ids), table.shape[1]), dtype=torch.float64)
    out = torch.where((ids < 0)[:, None], 0.0, torch.where((ids >= vocab)[:, None], float("nan"), out))
    return out, rounded(out, dtype, 3 * U32 * out.abs())


def embed_back(dout, ids, vocab, scale, dtype, base=None):
    dout, ids = f64(dout), ids.cpu().long()
    on = (ids >= 0) & (ids < vocab)
    total, size = (torch.zeros((vocab, dout.shape[1]), dtype=torch.float64) for _ in range(2))
    total.index_add_(0, ids[on], dout[on])
    size.index_add_(0, ids[on], dout[on].abs())
    count = torch.bincount(ids[on], minlength=vocab).double()[:, None]
    total, size = total * scale, size * abs(scale)
    if base is not None:
        total, size = total + f64(base), size + f64(base).abs()
    bound = rounded(total, dtype, (count + 4) * U32 * size)
    if base is not None:
        bound = torch.where(count > 0, bound, 0.0)  # left as it was
    return total, bound


# ---- norms around a block -------------------------------------------------------

def gate_of(gate, sigmoid, shape):
    """The gate spread over the tokens and channels, and its slope."""
    if gate is None:
        return torch.ones(shape, dtype=torch.float64), None
    z = f64(gate).expand(shape)
    if not sigmoid:
        return z, torch.ones_like(z)
    return torch.sigmoid(z), torch.sigmoid(z) * torch.sigmoid(-z)


def weight_of(w, offset, n):
    return torch.ones(n, dtype=torch.float64) if w is None else f64(w) + offset


def rms(x, eps):
    return (x.square().mean(-1, keepdim=True) + eps).sqrt()


def block_norm(h, y, gate, sigmoid, post, w_post, w_pre, scale, eps, offset):
    """h_out, n_out and the sizes that their bounds are made of; differentiable in what it is given in 64 bits."""
    n = h.shape[1]
    if y is None:
        return h, h * weight_of(w_pre, offset, n) / rms(h, eps), torch.zeros_like(h)
    u = y * weight_of(w_post, offset, n) / rms(y, eps) if post else y
    a, _ = gate_of(gate, sigmoid, h.shape)
    h_out = h + scale * a * u
    return h_out, h_out * weight_of(w_pre, offset, n) / rms(h_out, eps), scale * a * u


def norm(h, y, gate, sigmoid, post, w_post, w_pre, scale, eps, offset, stream, dtype):
    h_out, n_out, added = block_norm(f64(h), f64(y), gate, sigmoid, post, w_post, w_pre, scale, eps, offset)
    d = h.shape[1]
    # the root of a mean of d squares, the gate's exponential, a few products; the addition
    e_h = (d / 2 + 24) * U32 * added.abs() + 3 * U32 * h_out.abs()
    r = 1.0 / rms(h_out, eps)
    # errors of the summands turn up in the root as their mean share of it
    share = (h_out.abs() * e_h).mean(-1, keepdim=True) * r * r
    w = weight_of(w_pre, offset, d).abs()
    e_n = w * r * e_h + n_out.abs() * (share + (d / 2 + 16) * U32) + 2 * U32 * abs(offset) * r * h_out.abs()
    return (h_out, rounded(h_out, stream, e_h)), (n_out, rounded(n_out, dtype, e_n))


def norm_back(h, y, dh_out, dn, gate, sigmoid, post, w_post, w_pre, scale, eps, offset, stream, dtype, wdtype):
    """dh, dy, dgate, dpost, dpre with their bounds (None where an input lacks)."""
    some = next(t for t in (h, dh_out, y) if t is not None)
    t, d = some.shape
    zero = torch.zeros((t, d), dtype=torch.float64)
    h, y, dh_out, dn = f64(h), f64(y), f64(dh_out), f64(dn)
    g, size = (zero, zero) if dh_out is None else (dh_out, dh_out.abs())
    dpre = None
    if dn is not None:
        r = 1.0 / rms(h, eps)
        v = dn * weight_of(w_pre, offset, d)
        g = g + r * (v - h * r * r * (v * h).mean(-1, keepdim=True))
        size = size + r * (v.abs() + h.abs() * r * r * (v * h).abs().mean(-1, keepdim=True))
        dpre = ((dn * h * r).sum(0), rounded((dn * h * r).sum(0), wdtype, (t + d + 32) * U32 * (dn * h * r).abs().sum(0)))
    dh = g, rounded(g, stream, (2 * d + 32) * U32 * size)
    a, slope = gate_of(gate, sigmoid, (t, d))
    du, du_size = scale * a * g, abs(scale) * a.abs() * size
    w = weight_of(w_post, offset, d) if post else torch.ones(d, dtype=torch.float64)
    ry = 1.0 / rms(y, eps) if post and y is not None else torch.ones((t, 1), dtype=torch.float64)
    dgate = dpost = dy = None
    if y is not None and gate is not None:
        u = y * ry * w
        each, each_size = scale * u * g * slope, abs(scale) * u.abs() * size * slope
        if gate.dim() == 1 or gate.shape[0] == 1 != t:
            dims, count = (0,), t
        elif gate.shape[1] == 1 != d:
            dims, count = (1,), d
        else:
            dims, count = (), 0
        if dims:
            each, each_size = each.sum(dims).view(gate.shape), each_size.sum(dims).view(gate.shape)
        dgate = each, rounded(each, dtype, (3 * d + count + 64) * U32 * each_size)
    if post and y is not None:
        dpost = (du * y * ry).sum(0)
        dpost = dpost, rounded(dpost, wdtype, (3 * d + t + 64) * U32 * (du_size * y.abs() * ry).sum(0))
        x = du * w
        dy = ry * (x - y * ry * ry * (x * y).mean(-1, keepdim=True))
        s = du_size * w.abs()
        dy = dy, rounded(dy, dtype, (4 * d + 64) * U32 * ry * (s + y.abs() * ry * ry * (s * y.abs()).mean(-1, keepdim=True)))
    elif not post:
        dy = du, rounded(du, dtype, (2 * d + 48) * U32 * du_size)
    return dh, dy, dgate, dpost, dpre


# ---- routing -----------------------------------------------------------------------

def scores(z, sigmoid):
    if sigmoid:
        return torch.sigmoid(z)
    top = z.max(1, keepdim=True).values
    e = (z - torch.where(top == -INF, 0.0, top)).exp()
    return e / e.sum(1, keepdim=True)


def best(values, k):
    """Places and values of the k largest of a list that are not minus infinity, the lowest first among
    equals, a NaN as the largest."""
    nan = lambda x: x != x
    order = sorted((i for i, v in enumerate(values) if nan(v) or v != -INF),
                   key=lambda i: (not nan(values[i]), 0.0 if nan(values[i]) else -values[i], i))
    return order[:k]


def route(z, bias, top, sigmoid, groups, top_groups, group_best, renormalize, scale, wdtype):
    z = f64(z)
    t, e = z.shape
    p = scores(z, sigmoid)
    key = z if bias is None and groups == 1 else p if bias is None else p + f64(bias)
    gone = z == -INF
    if bias is not None:
        gone = gone | (f64(bias) == -INF)
    key = torch.where(gone, -INF, key)
    index = torch.full((t, top), -1, dtype=torch.int64)
    size = e // groups
    for i, row in enumerate(key.tolist()):
        if groups > 1:
            worth = []
            for g in range(groups):
                part = row[g * size:(g + 1) * size]
                firsts = best(part, group_best)
                worth.append(sum(part[j] for j in firsts) if firsts else -INF)
            keep = best(worth, top_groups)
            row = [v if j // size in keep else -INF for j, v in enumerate(row)]
        at = best(row, top)
        index[i, :len(at)] = torch.tensor(at, dtype=torch.int64)
    has = index >= 0
    w = torch.where(has, p.gather(1, index.clamp(min=0)), 0.0)
    if renormalize:
        # by the logarithms, as the scores' sum may be below any number
        log = torch.nn.functional.logsigmoid(z) if sigmoid else z
        log = torch.where(has, log.gather(1, index.clamp(min=0)), -INF)
        most = log.max(1, keepdim=True).values
        ex = (log - torch.where(most == -INF, 0.0, most)).exp()
        total = ex.sum(1, keepdim=True)
        w = torch.where(has, ex / torch.where(total == 0, 1.0, total), 0.0)
    far = spread(z, index)
    return index, (w * scale, rounded(w * scale, wdtype, (e + top + 64 + 4 * far) * U32 * (w * scale).abs() + 1e-36))


def spread(z, index):
    """How far exponents reach: the distance of a chosen logit from the row's largest one."""
    fine = torch.where(torch.isfinite(z), z, 0.0)
    return (fine.max(1, keepdim=True).values - fine.gather(1, index.clamp(min=0))).abs().clamp(max=200)


def route_back(z, index, dw, sigmoid, renormalize, scale, dtype):
    z, index, dw = f64(z), index.cpu().long(), f64(dw)
    t, e = z.shape
    bad = (index >= e).any(1, keepdim=True)
    has = (index >= 0) & (index < e)
    at = index.clamp(0, e - 1)
    p_all = scores(z, sigmoid)
    p = torch.where(has, p_all.gather(1, at), 0.0)
    g = torch.where(has, dw * scale, 0.0)
    rel = (e + 96 + 8 * spread(z, torch.where(has, index, 0)).max(1, keepdim=True).values) * U32
    rest = torch.sigmoid(-z).gather(1, at) if sigmoid else torch.ones_like(p)
    if renormalize:
        log = torch.where(has, (torch.nn.functional.logsigmoid(z) if sigmoid else z).gather(1, at), -INF)
        most = log.max(1, keepdim=True).values
        ex = (log - torch.where(most == -INF, 0.0, most)).exp()
        total = ex.sum(1, keepdim=True)
        q = torch.where(has, ex / torch.where(total == 0, 1.0, total), 0.0)
        term = q * (g - (g * q).sum(1, keepdim=True)) * rest
        size = q * (g.abs() + (g * q).abs().sum(1, keepdim=True)) * rest
    elif sigmoid:
        term, size = g * p * rest, (g * p * rest).abs()
    else:
        term, size = g * p, (g * p).abs()
    dz, dz_size = (torch.zeros_like(z).scatter_add_(1, at, torch.where(has, x, 0.0)) for x in (term, size))
    if not renormalize and not sigmoid:
        all_ = (g * p).sum(1, keepdim=True)
        dz = dz - torch.where(all_ != 0, p_all * all_, 0.0)
        far = (8 * U32) * torch.where(torch.isfinite(z), (z.max(1, keepdim=True).values - z).abs(), 0.0).clamp(max=200)
        dz_size = dz_size + torch.nan_to_num(p_all) * (g * p).abs().sum(1, keepdim=True) * (1 + far / rel)
    dz = torch.where(bad, float("nan"), dz)
    return dz, rounded(dz, dtype, rel * dz_size + 1e-36)


# ---- rows to the experts and back ----------------------------------------------------

def order(index, experts):
    """ends, place and order, entry by entry."""
    flat = index.cpu().long().flatten().tolist()
    buckets = [[] for _ in range(experts + 1)]
    for e, x in enumerate(flat):
        buckets[x if 0 <= x < experts else experts].append(e)
    at, place, ends = 0, [0] * len(flat), []
    line = [-1] * len(flat)
    for x, entries in enumerate(buckets):
        for e in entries:
            place[e] = at if x < experts else -1 - at
            line[at] = e if x < experts else -1
            at += 1
        ends.append(at)
    return torch.tensor(ends[:-1], dtype=torch.int64), torch.tensor(place, dtype=torch.int64).view(index.shape), \
        torch.tensor(line, dtype=torch.int64)


def gather(x, place):
    t, k = place.shape
    place = place.cpu().long().flatten()
    rows = torch.zeros((t * k, x.shape[1]), dtype=x.dtype)
    on = (place >= 0) & (place < t * k)
    rows[place[on]] = x.cpu()[torch.arange(t * k)[on] // k]
    return rows


def combine(rows, place, weights, residual, dtype):
    rows, place, w = f64(rows), place.cpu().long(), f64(weights)
    t, k = place.shape
    n, h = t * k, rows.shape[1]
    total = torch.zeros((t, h), dtype=torch.float64) if residual is None else f64(residual).clone()
    size = total.abs()
    for j in range(k):
        on, lost = (place[:, j] >= 0) & (place[:, j] < n), place[:, j] >= n
        x = (w[on, j:j + 1] if w is not None else 1.0) * rows[place[on, j]]
        total[on] += x
        size[on] += x.abs()
        total[lost] = float("nan")
    return total, rounded(total, dtype, (k + 4) * U32 * size)


def combine_back(rows, place, weights, dout, dtype, wdtype):
    rows, place, w, dout = f64(rows), place.cpu().long(), f64(weights), f64(dout)
    t, k = place.shape
    n, h = t * k, dout.shape[1]
    drows, dw, dw_size = torch.zeros((n, h), dtype=torch.float64), torch.zeros((t, k), dtype=torch.float64), \
        torch.zeros((t, k), dtype=torch.float64)
    for j in range(k):
        on = (place[:, j] >= 0) & (place[:, j] < n)
        drows[place[on, j]] = w[on, j:j + 1] * dout[on]
        dw[on, j] = (rows[place[on, j]] * dout[on]).sum(1)
        dw_size[on, j] = (rows[place[on, j]] * dout[on]).abs().sum(1)
        dw[place[:, j] >= n, j] = float("nan")
    return (drows, rounded(drows, dtype, 2 * U32 * drows.abs())), (dw, rounded(dw, wdtype, (h + 4) * U32 * dw_size))
