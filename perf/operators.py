"""The training operators beside the update, for timing and comparison.

The update takes BF16 gradients; these operators are where a training step
makes them: the head's distillation loss with its gradient, the norms of
queries and keys with the position rotation, and the experts' products.  The
listed cases are their calls over the sizes that a training program (or the
evaluation and generation beside it) makes, from one token to a whole batch.

A case is a dict of plain values.  Its "kind" is one of
  "qk"        sdp_qk_norm_rope: RMS norm of each query and key head, then the rotation
  "qk_back"   sdp_qk_norm_rope_backward: gradients of q, k and both norm weights
  "distill"   sdp_distill_loss: loss of each row against a teacher's top logits and
              a label, with the gradient of the logits in the same call where "grad"
  "distill_back"  sdp_distill_loss_backward: the gradient from the forward's statistics
  "experts"   sdp_grouped_matmul: rows sorted by expert times that expert's weight
  "experts_back"  sdp_grouped_matmul_backward: gradients of the rows and of the weights
and the other keys are sizes, types and options, explained where the inputs
are made.
"""
import weakref

import torch

own = False

DEV = "cuda:0"
VOCAB = 151936
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INTS = {"i32": torch.int32, "i64": torch.int64}
PLAIN_ROWS = 1024   # rows of logits that the plain form takes at a time


def qk(kind, batch, tokens, q_heads, k_heads, dim, rotary=None, interleaved=False, dtype="bf16", layout="fused",
       weight="bf16", positions="i64", table=0, name=None):
    c = dict(kind=kind, batch=batch, tokens=tokens, q_heads=q_heads, k_heads=k_heads, dim=dim, rotary=rotary or dim,
             interleaved=interleaved, dtype=dtype, layout=layout, weight=weight, positions=positions,
             table=max(table, tokens))
    return dict(c, name=name) if name else c


def distill(kind, rows, vocab, k, dtype="bf16", teacher="f32", index="i64", temperature=1.0, labels=0.0, grad=False,
            pad=0, name=None):
    c = dict(kind=kind, rows=rows, vocab=vocab, k=k, dtype=dtype, teacher=teacher, index=index,
             temperature=temperature, labels=labels, grad=grad, pad=pad)
    return dict(c, name=name) if name else c


def experts(kind, rows, groups, n_in, n_out, skew=0.5, unused=0, out="bf16", ends="i32", name=None):
    c = dict(kind=kind, rows=rows, groups=groups, n_in=n_in, n_out=n_out, skew=skew, unused=unused, out=out, ends=ends)
    return dict(c, name=name) if name else c


def listed():
    return [
        # generation beside training: one new token for each of 8 sequences, the
        # heads of a Qwen3-8B layer (hidden 4096, 1024 keys: 32 and 8 heads of 128)
        qk("qk", 8, 1, 32, 8, 128, table=4096, name="qk_one_token_b8"),
        # a training batch through a Qwen3-14B layer (40 and 8 heads), views of the fused projection
        qk("qk", 4, 8192, 40, 8, 128, name="qk_14b_batch_32k"),
        # odd length, heads apart from tokens, partial interleaved rotation, 32 bits
        qk("qk_back", 3, 1367, 12, 4, 96, rotary=64, interleaved=True, dtype="f32", layout="heads", weight="f32",
           positions="i32", name="qk_back_ragged_f32"),
        # the backward of the training batch
        qk("qk_back", 4, 8192, 40, 8, 128, name="qk_back_14b_batch_32k"),
        # evaluation: the loss alone over the Qwen3 vocabulary, a few hundred answer tokens
        distill("distill", 301, VOCAB, 64, temperature=2.0, labels=0.3, name="distill_eval_301"),
        # a training batch: loss and gradient of 8,192 rows in one call
        distill("distill", 8192, VOCAB, 64, temperature=2.0, labels=0.3, grad=True, name="distill_train_8k"),
        # a small odd vocabulary in 32 bits, rows padded apart
        distill("distill_back", 77, 32003, 20, dtype="f32", teacher="bf16", index="i32", pad=5,
                name="distill_back_odd_f32"),
        # the gradient where the loss's weight came later (the autograd order)
        distill("distill_back", 4096, VOCAB, 128, labels=0.3, name="distill_back_4k"),
        # a few tokens' rows over many experts: the weights are what is read
        experts("experts", 96, 64, 2048, 1024, skew=0.3, name="experts_few_rows"),
        # a batch of 8,192 tokens routed to 8 of 128 experts, the gate and up projection
        experts("experts", 65536, 128, 2048, 1536, name="experts_64k"),
        # few experts, sizes that fit no tile, rows past the last expert
        experts("experts_back", 5003, 12, 1000, 712, skew=1.0, unused=37, out="f32", ends="i64",
                name="experts_back_ragged"),
        # the backward of a batch, fewer and larger experts
        experts("experts_back", 65536, 64, 2048, 1536, name="experts_back_64k"),
    ]


def log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["qk", "qk_back", "distill", "distill", "distill_back", "experts", "experts", "experts_back"])
    if kind.startswith("qk"):
        dim = rng.choice([32, 64, 64, 80, 96, 112, 128, 128, 128, 192, 256])
        k_heads = rng.choice([1, 2, 4, 5, 8, 8, 16])
        q_heads = k_heads * rng.choice([1, 2, 3, 4, 5, 8])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = 4 * 8192 * 48 * 128 // (2 if dtype == "f32" else 1) // ((q_heads + k_heads) * dim)
        total = log_uniform(rng, 1, max(2, most))
        batch = min(total, rng.choice([1, 1, 2, 3, 4, 8]))
        return qk(kind, batch, max(1, total // batch), q_heads, k_heads, dim,
                  rotary=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.3, dtype=dtype,
                  layout=rng.choice(["fused", "fused", "heads"]), weight=rng.choice(["bf16", "f32"]),
                  positions=rng.choice(["i32", "i64"]), table=rng.choice([0, 4096]))
    if kind.startswith("distill"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        vocab = rng.choice([VOCAB, VOCAB, log_uniform(rng, 1000, VOCAB)])
        rows = log_uniform(rng, 1, max(2, 8192 * VOCAB // vocab // (2 if dtype == "f32" else 1)))
        return distill(kind, min(rows, 65536), vocab, min(log_uniform(rng, 1, 256), vocab // 4), dtype=dtype,
                       teacher=rng.choice(["f32", "bf16"]), index=rng.choice(["i32", "i64"]),
                       temperature=rng.choice([1.0, 1.0, 2.0, 3.5]), labels=rng.choice([0.0, 0.3, 0.5]),
                       grad=kind == "distill" and rng.random() < 0.6, pad=rng.choice([0, 0, 0, 3, 8]))
    sizes = [0, 0]
    for i in range(2):
        sizes[i] = 8 * log_uniform(rng, 16, 512)
        if rng.random() < 0.15:
            sizes[i] -= rng.randint(1, 7)
        if sizes[i] == 3072:
            sizes[i] += 8
    n_in, n_out = sizes
    rows = log_uniform(rng, 1, max(2, min(65536, 65536 * 2048 * 1536 // (n_in * n_out))))
    groups = log_uniform(rng, 1, 128)
    return experts(kind, rows, groups, n_in, n_out, skew=rng.choice([0.0, 0.5, 1.0]),
                   unused=rng.choice([0, 0, min(rows - 1, 19)]), out=rng.choice(["bf16", "bf16", "f32"]),
                   ends=rng.choice(["i32", "i64"]))


# ---- inputs ----------------------------------------------------------------

def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return gen


def normal(gen, shape, sigma, dtype):
    """N(0, sigma) made in pieces, so that 32-bit temporaries stay small."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - a)
        flat[a:a + n] = torch.randn(n, generator=gen, device=DEV).mul_(sigma)
    return out


def head_views(case, gen, sigma):
    """q and k as [batch, tokens, heads, dim] views: cut out of a fused
    projection whose rows hold q, k and v beside each other ("fused"), or of
    tensors that keep each head's tokens together ("heads")."""
    b, s, hq, hk, d = (case[n] for n in ("batch", "tokens", "q_heads", "k_heads", "dim"))
    dtype = TYPES[case["dtype"]]
    if case["layout"] == "heads":
        return tuple(normal(gen, (b, h, s, d), sigma, dtype).transpose(1, 2) for h in (hq, hk))
    x = normal(gen, (b, s, hq + 2 * hk, d), sigma, dtype)
    return x[:, :, :hq], x[:, :, hq:hq + hk]


def qk_inputs(case, seed):
    gen = generator(seed)
    b, s, d, rot, table = (case[n] for n in ("batch", "tokens", "dim", "rotary", "table"))
    st = {}
    st["q"], st["k"] = head_views(case, gen, 1.5)
    for n in ("q_weight", "k_weight"):
        st[n] = (1.0 + 0.1 * torch.randn(d, generator=gen, device=DEV)).to(TYPES[case["weight"]])
    # tables of angles position / 10000^(2i / rotary), as a program keeps them
    angle = torch.arange(table, device=DEV, dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
    # each sequence starts somewhere of its own; where packed documents meet, positions start again
    first = torch.randint(0, table - s + 1, (b, 1), generator=gen, device=DEV)
    at = torch.arange(s, device=DEV)[None, :]
    cut = torch.randint(0, s, (b, 1), generator=gen, device=DEV)
    st["positions"] = torch.where(at < cut, first + at, at - cut).to(INTS[case["positions"]]).contiguous()
    if case["kind"] == "qk_back":
        st["dq_out"], st["dk_out"] = head_views(case, gen, 1e-3)
    return st


def distill_inputs(case, seed):
    gen = generator(seed)
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    st = {}
    # logits of a half-trained student; the last few vocabulary entries are padding and masked
    z = normal(gen, (rows, vocab + case["pad"]), 2.0, TYPES[case["dtype"]])
    st["logits"] = z[:, :vocab]
    st["logits"][:, vocab - min(7, vocab // 16):] = float("-inf")
    live = vocab - min(7, vocab // 16)
    # the teacher's top logits, largest first, at distinct places of the vocabulary
    step = torch.randint(1, max(2, live // k), (rows, 1), generator=gen, device=DEV)
    first = torch.randint(0, live, (rows, 1), generator=gen, device=DEV)
    index = (first + step * torch.arange(k, device=DEV)) % live
    t = (torch.randn((rows, k), generator=gen, device=DEV) * 2.5).sort(dim=1, descending=True).values + 12.0
    # the student follows the teacher part of the way
    st["logits"].scatter_(1, index, (0.5 * t + torch.randn((rows, k), generator=gen, device=DEV)).to(z.dtype))
    # some rows have fewer entries; some are a prompt's or padding and have none
    have = torch.randint(1, k + 1, (rows, 1), generator=gen, device=DEV)
    have = torch.where(torch.rand((rows, 1), generator=gen, device=DEV) < 0.8, torch.full_like(have, k), have)
    masked = torch.rand((rows, 1), generator=gen, device=DEV) < 0.1
    keep = (torch.arange(k, device=DEV) < have) & ~masked
    st["labels"] = None
    if case["labels"]:
        label = torch.where(torch.rand(rows, generator=gen, device=DEV) < 0.7, index[:, 0], first[:, 0])
        st["labels"] = torch.where(masked[:, 0], torch.full_like(label, -100), label).to(INTS[case["index"]])
    st["teacher_index"] = torch.where(keep, index, torch.full_like(index, -1)).to(INTS[case["index"]])
    st["teacher_logits"] = t.to(TYPES[case["teacher"]])
    # each row's share of the batch's mean loss
    st["row_grad"] = torch.full((rows,), 1.0 / max(1, int((~masked).sum())), device=DEV)
    st["row_grad"] *= torch.rand(rows, generator=gen, device=DEV).mul_(0.5).add_(0.75)
    if case["kind"] == "distill_back":
        st["lse"] = torch.empty((rows, 2), device=DEV)
        for a in range(0, rows, PLAIN_ROWS):
            x = st["logits"][a:a + PLAIN_ROWS].float()
            st["lse"][a:a + PLAIN_ROWS, 0] = log_sum_exp(x / case["temperature"])
            st["lse"][a:a + PLAIN_ROWS, 1] = log_sum_exp(x)
    return st


def experts_inputs(case, seed):
    gen = generator(seed)
    rows, groups, n_in, n_out = (case[n] for n in ("rows", "groups", "n_in", "n_out"))
    st = {}
    # a router's counts, uneven by "skew"; the rows past the last expert are padding
    share = (case["skew"] * torch.randn(groups, generator=gen, device=DEV)).exp()
    used = rows - case["unused"]
    to = torch.multinomial(share, used, replacement=True, generator=gen)
    ends = torch.bincount(to, minlength=groups).cumsum(0)
    st["ends"] = ends.to(INTS[case["ends"]])
    st["ends_host"] = ends.tolist()
    st["x"] = normal(gen, (rows, n_in), 1.0, torch.bfloat16)
    st["w"] = normal(gen, (groups, n_out, n_in), 0.02, torch.bfloat16)
    if case["kind"] == "experts_back":
        st["dy"] = normal(gen, (rows, n_out), 1e-3, torch.bfloat16)
    return st


def inputs(case, seed):
    kind = case["kind"]
    return (qk_inputs if kind.startswith("qk") else distill_inputs if kind.startswith("distill")
            else experts_inputs)(case, seed)


class Context:
    """An sdp context that is destroyed with the state that holds it."""

    def __init__(self):
        from paper_2609_34162_amd import sdp
        self.handle = sdp.sdp_ctx_create(0, 0, 1, 0)
        weakref.finalize(self, sdp.sdp_ctx_destroy, self.handle)


def buffers(case, st):
    """What the program keeps for the operator to write: activations of the
    next operator, gradient buffers of the update."""
    kind = case["kind"]
    if kind == "qk":
        st["q_out"], st["k_out"] = (torch.empty(t.shape, dtype=t.dtype, device=DEV) for t in (st["q"], st["k"]))
    elif kind == "qk_back":
        # the fused projection's gradient has the projection's layout
        b, s, hq, hk, d = (case[n] for n in ("batch", "tokens", "q_heads", "k_heads", "dim"))
        dx = torch.empty((b, s, hq + 2 * hk, d), dtype=TYPES[case["dtype"]], device=DEV)
        st["dq"], st["dk"] = dx[:, :, :hq], dx[:, :, hq:hq + hk]
        st["dq_weight"], st["dk_weight"] = (torch.empty(d, dtype=TYPES[case["weight"]], device=DEV) for _ in range(2))
    elif kind.startswith("distill"):
        st["loss"] = torch.empty(case["rows"], device=DEV)
        if kind == "distill":
            st["lse"] = torch.empty((case["rows"], 2), device=DEV)
        if kind == "distill_back" or case["grad"]:
            st["dlogits"] = torch.empty((case["rows"], case["vocab"]), dtype=TYPES[case["dtype"]], device=DEV)
    elif kind == "experts":
        st["y"] = torch.empty((case["rows"], case["n_out"]), dtype=TYPES[case["out"]], device=DEV)
    else:
        st["dx"] = torch.empty((case["rows"], case["n_in"]), dtype=torch.bfloat16, device=DEV)
        st["dw"] = torch.empty(st["w"].shape, dtype=TYPES[case["out"]], device=DEV)


def prepare(case, seed):
    st = inputs(case, seed)
    st["case"] = case
    if own:
        st["ctx"] = Context()
        buffers(case, st)
    return st


# ---- one pass --------------------------------------------------------------

def run(st):
    kind = st["case"]["kind"]
    if own:
        return run_own(st["case"], st)
    plain = {"qk": plain_qk, "qk_back": plain_qk_back, "distill": plain_distill, "distill_back": plain_distill,
             "experts": plain_experts, "experts_back": plain_experts_back}
    return plain[kind](st["case"], st)


def run_own(case, st):
    from paper_2609_34162_amd import ops
    kind, ctx = case["kind"], st["ctx"].handle
    stream = torch.cuda.current_stream()
    if kind.startswith("qk"):
        more = dict(q_weight=st["q_weight"], k_weight=st["k_weight"], positions=st["positions"], eps=EPS,
                    interleaved=case["interleaved"], stream=stream)
        if kind == "qk":
            ops.sdp_qk_norm_rope(ctx, st["q"], st["k"], st["q_out"], st["k_out"], st["cos"], st["sin"], **more)
            return st["q_out"], st["k_out"]
        ops.sdp_qk_norm_rope_backward(ctx, st["q"], st["k"], st["dq_out"], st["dk_out"], st["dq"], st["dk"],
                                      st["cos"], st["sin"], dq_weight=st["dq_weight"], dk_weight=st["dk_weight"],
                                      **more)
        return st["dq"], st["dk"], st["dq_weight"], st["dk_weight"]
    if kind.startswith("distill"):
        more = dict(teacher_logits=st["teacher_logits"], teacher_index=st["teacher_index"], labels=st["labels"],
                    temperature=case["temperature"], distill_weight=1.0 - case["labels"],
                    label_weight=case["labels"], stream=stream)
        if kind == "distill_back":
            ops.sdp_distill_loss_backward(ctx, st["logits"], st["lse"], st["row_grad"], st["dlogits"], **more)
            return st["dlogits"]
        if case["grad"]:
            ops.sdp_distill_loss(ctx, st["logits"], st["loss"], st["lse"], row_grad=st["row_grad"],
                                 dlogits=st["dlogits"], **more)
            return st["loss"], st["lse"], st["dlogits"]
        ops.sdp_distill_loss(ctx, st["logits"], st["loss"], st["lse"], **more)
        return st["loss"], st["lse"]
    if kind == "experts":
        ops.sdp_grouped_matmul(ctx, st["x"], st["w"], st["ends"], st["y"], stream=stream)
        return st["y"]
    ops.sdp_grouped_matmul_backward(ctx, st["x"], st["w"], st["ends"], st["dy"], st["dx"], st["dw"], stream=stream)
    return st["dx"], st["dw"]


def pairs(x, case):
    """The two halves of each rotated pair, and what is not rotated."""
    rot = case["rotary"]
    if case["interleaved"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def joined(a, b, rest, case):
    if case["interleaved"]:
        return torch.cat((torch.stack((a, b), -1).flatten(-2), rest), -1)
    return torch.cat((a, b, rest), -1)


def plain_qk(case, st):
    at = st["positions"].long()
    cos, sin = st["cos"][at][:, :, None], st["sin"][at][:, :, None]
    out = []
    for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])):
        x32 = x.float()
        n = x32 * (x32.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float()
        a, b, rest = pairs(n, case)
        out.append(joined(a * cos - b * sin, b * cos + a * sin, rest, case).to(x.dtype))
    return tuple(out)


def plain_qk_back(case, st):
    at = st["positions"].long()
    cos, sin = st["cos"][at][:, :, None], st["sin"][at][:, :, None]
    dx, dw = [], []
    for x, w, dy in ((st["q"], st["q_weight"], st["dq_out"]), (st["k"], st["k_weight"], st["dk_out"])):
        x32 = x.float()
        r = (x32.square().mean(-1, keepdim=True) + EPS).rsqrt()
        xn = x32 * r
        a, b, rest = pairs(dy.float(), case)
        dn = joined(a * cos + b * sin, b * cos - a * sin, rest, case)
        dw.append((dn * xn).sum((0, 1, 2)).to(w.dtype))
        dn = dn * w.float()
        dx.append((r * (dn - xn * (dn * xn).mean(-1, keepdim=True))).to(x.dtype))
    return (*dx, *dw)


def log_sum_exp(x):
    top = x.max(-1, keepdim=True).values
    return (x - top).exp().sum(-1).log() + top[:, 0]


def plain_distill(case, st):
    rows, tau = case["rows"], case["temperature"]
    w_label = case["labels"]
    w_distill = 1.0 - w_label
    z, labels = st["logits"], st["labels"]
    back = case["kind"] == "distill_back"
    loss, lse = torch.empty(rows, device=DEV), torch.empty((rows, 2), device=DEV)
    grad = torch.empty(z.shape, dtype=z.dtype, device=DEV) if back or case["grad"] else None
    for a in range(0, rows, PLAIN_ROWS):
        part = slice(a, min(rows, a + PLAIN_ROWS))
        x = z[part].float()
        if back:
            l_tau, l_one = st["lse"][part, 0], st["lse"][part, 1]
        else:
            l_tau, l_one = log_sum_exp(x / tau), log_sum_exp(x)
            lse[part, 0], lse[part, 1] = l_tau, l_one
        index = st["teacher_index"][part].long()
        t = st["teacher_logits"][part].float() / tau
        t = t.masked_fill(index < 0, float("-inf"))
        has = (index >= 0).any(1)
        at = index.clamp(min=0)
        log_q = t - log_sum_exp(t)[:, None]
        q = torch.where(index >= 0, log_q.exp(), 0.0)
        if not back:
            log_p = x.gather(1, at) / tau - l_tau[:, None]
            per_row = torch.where(q > 0, q * (log_q - log_p), 0.0).sum(1) * (w_distill * tau * tau)
            total = torch.where(has, per_row, 0.0)
            if labels is not None:
                y = labels[part].long()
                total += torch.where(y >= 0, w_label * (l_one - x.gather(1, y.clamp(min=0)[:, None])[:, 0]), 0.0)
            loss[part] = total
        if grad is None:
            continue
        g = st["row_grad"][part][:, None]
        c = torch.where(has[:, None], g * (w_distill * tau), 0.0)
        d = (x / tau - l_tau[:, None]).exp() * c
        d.scatter_add_(1, at, torch.where(has[:, None], -q * c, 0.0))
        if labels is not None:
            y = labels[part].long()[:, None]
            c = torch.where(y >= 0, g * w_label, 0.0)
            d += (x - l_one[:, None]).exp() * c
            d.scatter_add_(1, y.clamp(min=0), -c)
        grad[part] = d
    if back:
        return grad
    return (loss, lse) if grad is None else (loss, lse, grad)


def groups_of(st):
    first = 0
    for e, end in enumerate(st["ends_host"]):
        if end > first:
            yield e, slice(first, end)
        first = end


def plain_experts(case, st):
    y = torch.zeros((case["rows"], case["n_out"]), dtype=TYPES[case["out"]], device=DEV)
    for e, part in groups_of(st):
        y[part] = st["x"][part].float() @ st["w"][e].float().t()
    return y


def plain_experts_back(case, st):
    dx = torch.zeros((case["rows"], case["n_in"]), dtype=torch.bfloat16, device=DEV)
    dw = torch.zeros(st["w"].shape, dtype=TYPES[case["out"]], device=DEV)
    for e, part in groups_of(st):
        dy = st["dy"][part].float()
        dx[part] = dy @ st["w"][e].float()
        dw[e] = dy.t() @ st["x"][part].float()
    return dx, dw


# ---- work and the definitions in 64 bits -----------------------------------

def work(case):
    """Each input read once and each output written once; about 10 operations
    for each element of a head forward and 20 backward, 4 to 8 for each logit,
    and the products' multiplications and additions."""
    kind = case["kind"]
    if kind.startswith("qk"):
        size = 2 if case["dtype"] == "bf16" else 4
        tokens = case["batch"] * case["tokens"]
        n = tokens * (case["q_heads"] + case["k_heads"]) * case["dim"]
        side = tokens * (4 if case["positions"] == "i32" else 8) + min(tokens, case["table"]) * case["rotary"] * 4
        w = 2 * case["dim"] * (2 if case["weight"] == "bf16" else 4)
        return {"bytes": n * size * (2 if kind == "qk" else 3) + side + w * (1 if kind == "qk" else 2),
                "flops": n * (10 if kind == "qk" else 20)}
    if kind.startswith("distill"):
        size = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["vocab"]
        entry = (2 if case["teacher"] == "bf16" else 4) + (4 if case["index"] == "i32" else 8)
        label = (4 if case["index"] == "i32" else 8) if case["labels"] else 0
        out = n * size if kind == "distill_back" or case["grad"] else 0
        return {"bytes": n * size + out + case["rows"] * (case["k"] * entry + label + 12), "flops": n * (8 if out else 4)}
    rows = case["rows"] - case["unused"]
    k, n, groups = case["n_in"], case["n_out"], case["groups"]
    used = round(groups * (1.0 - (1.0 - 1.0 / groups) ** rows))  # experts that get a row, if all are as likely
    out = 2 if case["out"] == "bf16" else 4
    if kind == "experts":
        return {"bytes": 2 * rows * k + 2 * used * n * k + out * case["rows"] * n, "flops": 2 * rows * k * n}
    return {"bytes": 2 * rows * (k + n) + 2 * used * n * k + 2 * case["rows"] * k + out * groups * n * k,
            "flops": 4 * rows * k * n}


def exact(case, seed):
    st = inputs(case, seed)
    kind = case["kind"]
    if kind.startswith("qk"):
        return exact_qk(case, st)
    if kind.startswith("distill"):
        return exact_distill(case, st)
    x, w = st["x"], st["w"]
    starts = [0] + st["ends_host"]
    if kind == "experts":
        y = torch.zeros((case["rows"], case["n_out"]), dtype=torch.float64, device=DEV)
        for e in range(case["groups"]):
            rows = range(starts[e], starts[e + 1])
            y[rows.start:rows.stop] = torch.mm(x[rows.start:rows.stop].double(), w[e].double().t().contiguous())
        return y
    dy = st["dy"]
    dx = torch.zeros((case["rows"], case["n_in"]), dtype=torch.float64, device=DEV)
    dw = torch.zeros(w.shape, dtype=torch.float64, device=DEV)
    for e in range(case["groups"]):
        a, b = starts[e], starts[e + 1]
        dx[a:b] = torch.mm(dy[a:b].double(), w[e].double())
        dw[e] = torch.mm(dy[a:b].double().t().contiguous(), x[a:b].double())
    return dx, dw


def exact_qk(case, st):
    """The operator written as a matrix: y = R (w * x / rms(x)), with R the
    rotation of each pair; one sequence at a time."""
    rot, d = case["rotary"], case["dim"]
    i = torch.arange(rot // 2, device=DEV)
    lo, hi = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
    back = case["kind"] == "qk_back"
    outs = [torch.empty(st[n].shape, dtype=torch.float64, device=DEV) for n in ("q", "k")]
    dws = [torch.zeros(d, dtype=torch.float64, device=DEV) for _ in range(2)]
    for b in range(case["batch"]):
        at = st["positions"][b].long()
        cos, sin = st["cos"].double()[at][:, None, :], st["sin"].double()[at][:, None, :]
        for j, n in enumerate(("q", "k")):
            x, w = st[n][b].double(), st[n + "_weight"].double()
            ms = (x * x).sum(-1, keepdim=True) / d + EPS
            unit = x / ms.sqrt()
            if not back:
                y = unit * w
                first, second = y[..., lo].clone(), y[..., hi].clone()
                y[..., lo], y[..., hi] = first * cos - second * sin, first * sin + second * cos
                outs[j][b] = y
                continue
            g = st["d%s_out" % n][b].double()
            first, second = g[..., lo].clone(), g[..., hi].clone()
            g[..., lo], g[..., hi] = first * cos + second * sin, second * cos - first * sin
            dws[j] += (g * unit).sum((0, 1))
            g = g * w
            outs[j][b] = (g - unit * ((g * unit).sum(-1, keepdim=True) / d)) / ms.sqrt()
    return (*outs, *dws) if back else tuple(outs)


def exact_distill(case, st):
    """Row by row from the definition, a few hundred rows at a time:
    loss = a tau^2 sum_j q_j (log q_j - log p_j) + b (-log p'_label), with p
    the softmax of z / tau over the vocabulary, q the teacher's over its own
    entries and p' the softmax of z."""
    rows, tau = case["rows"], case["temperature"]
    b_ = case["labels"]
    a_ = 1.0 - b_
    back = case["kind"] == "distill_back"
    loss = torch.zeros(rows, dtype=torch.float64, device=DEV)
    lse = torch.zeros((rows, 2), dtype=torch.float64, device=DEV)
    want = back or case["grad"]
    grad = torch.zeros((rows, case["vocab"]), dtype=torch.float64, device=DEV) if want else None
    for at in range(0, rows, 512):
        sl = slice(at, min(rows, at + 512))
        z = st["logits"][sl].double()
        lse[sl, 0], lse[sl, 1] = torch.logsumexp(z / tau, 1), torch.logsumexp(z, 1)
        idx, t = st["teacher_index"][sl].long(), st["teacher_logits"][sl].double()
        there = idx >= 0
        some = there.any(1, keepdim=True)
        t = torch.where(there, t / tau, float("-inf"))
        q = torch.softmax(torch.where(some, t, 0.0), 1) * (there & some)
        zi = z.gather(1, idx.clamp(min=0))
        kl = torch.where(q > 0, q * (q.clamp(min=1e-300).log() - zi / tau + lse[sl, 0:1]), 0.0).sum(1)
        loss[sl] = a_ * tau * tau * kl
        on = some.double()
        if want:
            g = st["row_grad"][sl].double()[:, None]
            d = a_ * tau * on * torch.exp(z / tau - lse[sl, 0:1])
            d.scatter_add_(1, idx.clamp(min=0), -a_ * tau * q)
        if st["labels"] is not None:
            y = st["labels"][sl].long()[:, None]
            on = (y >= 0).double()
            zy = z.gather(1, y.clamp(min=0))
            loss[sl] += b_ * torch.where(y >= 0, lse[sl, 1:2] - zy, 0.0)[:, 0]
            if want:
                d += b_ * on * torch.exp(z - lse[sl, 1:2])
                d.scatter_add_(1, y.clamp(min=0), -b_ * on)
        if want:
            grad[sl] = d * g
    if back:
        return grad
    return (loss, lse, grad) if want else (loss, lse)
