"""The training operators around the experts' products, for timing and comparison.

Between a token and the experts' grouped products a training program looks up
embeddings, adds each block's output to the residual stream and norms it for
the next block, routes tokens to experts, and takes their rows to the experts
and back.  The listed cases are those calls over the sizes that a training
program (or the evaluation and generation beside it) makes, from a few tokens
to a whole batch.

A case is a dict of plain values.  Its "kind" is one of
  "embed"         sdp_embed: scaled rows of the table at the tokens' ids
  "embed_back"    sdp_embed_backward: the table's gradient
  "norm"          sdp_block_norm: norm after a block, gate, residual scale, residual
                  addition, norm before the next block
  "norm_back"     sdp_block_norm_backward: gradients of the stream, the block's
                  output, the gate and both norm weights
  "route"         sdp_route: the chosen experts of each token and their weights
  "route_back"    sdp_route_backward: the router logits' gradient
  "dispatch"      sdp_expert_order and sdp_expert_gather: rows sorted by expert, and
                  the experts' ends
  "combine"       sdp_expert_combine: the weighted sum of each token's rows, added
                  to the residual stream
  "combine_back"  sdp_expert_combine_backward: gradients of the rows and the weights
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
PIECE = 1 << 25     # elements that the plain forms turn to 32 bits at a time


def embed(kind, tokens, vocab, hidden, dtype="bf16", grad="bf16", ids="i64", scale=1.0, padded=0.0, name=None):
    c = dict(kind=kind, tokens=tokens, vocab=vocab, hidden=hidden, dtype=dtype, grad=grad, ids=ids, scale=scale,
             padded=padded)
    return dict(c, name=name) if name else c


def norm(kind, tokens, hidden, dtype="bf16", stream="bf16", post=True, gate="none", sigmoid=False, scale=1.0,
         offset=0.0, weight="bf16", pad=0, name=None):
    c = dict(kind=kind, tokens=tokens, hidden=hidden, dtype=dtype, stream=stream, post=post, gate=gate,
             sigmoid=sigmoid, scale=scale, offset=offset, weight=weight, pad=pad)
    return dict(c, name=name) if name else c


def route(kind, tokens, experts, top, dtype="f32", sigmoid=False, bias=False, groups=1, top_groups=1, group_best=1,
          renormalize=True, scale=1.0, index="i32", masked=0.0, name=None):
    c = dict(kind=kind, tokens=tokens, experts=experts, top=top, dtype=dtype, sigmoid=sigmoid, bias=bias, groups=groups,
             top_groups=top_groups, group_best=group_best, renormalize=renormalize, scale=scale, index=index,
             masked=masked)
    return dict(c, name=name) if name else c


def rows(kind, tokens, experts, top, hidden, dtype="bf16", stream="bf16", index="i32", ends="i32", skew=0.5,
         masked=0.0, residual=True, name=None):
    c = dict(kind=kind, tokens=tokens, experts=experts, top=top, hidden=hidden, dtype=dtype, stream=stream,
             index=index, ends=ends, skew=skew, masked=masked, residual=residual)
    return dict(c, name=name) if name else c


def listed():
    return [
        # evaluation of odd documents in 32 bits, a small vocabulary, scaled embeddings, some padding
        embed("embed", 1367, 32003, 1000, dtype="f32", ids="i32", scale=31.6227766, padded=0.1,
              name="embed_odd_f32"),
        # a training batch of four sequences: the gradient of a Qwen3-8B table
        embed("embed_back", 32768, VOCAB, 4096, padded=0.05, name="embed_back_32k"),
        # generation beside training: one new token for each of 8 sequences of a Qwen3-8B layer
        norm("norm", 8, 4096, post=False, name="norm_one_token_b8"),
        # a training batch through a Qwen3-14B layer, norms on both sides, a learned scale for each channel
        norm("norm", 32768, 5120, gate="channel", scale=0.5, name="norm_14b_batch_32k"),
        # odd sizes in 32 bits, a sigmoid gate of each token's own, rows padded apart
        norm("norm_back", 3 * 1367, 1003, dtype="f32", stream="f32", gate="element", sigmoid=True, weight="f32",
             offset=1.0, pad=5, name="norm_back_ragged_f32"),
        # the backward of the training batch
        norm("norm_back", 32768, 5120, gate="channel", scale=0.5, name="norm_back_14b_batch_32k"),
        # generation: 8 tokens to 8 of 128 experts
        route("route", 8, 128, 8, name="route_one_token_b8"),
        # a training batch, 256 experts in 8 groups, sigmoid scores with a bias for balance
        route("route", 32768, 256, 8, sigmoid=True, bias=True, groups=8, top_groups=4, group_best=2, scale=2.5,
              masked=0.02, name="route_groups_32k"),
        # the backward of an odd batch, scores over all experts
        route("route_back", 3 * 4099, 60, 4, dtype="bf16", renormalize=False, index="i64", masked=0.02,
              name="route_back_odd"),
        # a batch of 8,192 tokens to 8 of 128 experts: their rows for the grouped products
        rows("dispatch", 8192, 128, 8, 2048, masked=0.02, name="dispatch_8k"),
        # odd sizes in 32 bits
        rows("combine", 1367, 12, 2, 1003, dtype="f32", stream="f32", skew=1.0, name="combine_odd_f32"),
        # the backward of the batch
        rows("combine_back", 8192, 128, 8, 2048, masked=0.02, name="combine_back_8k"),
    ]


def log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def width(rng, lo, hi):
    """Mostly whole pieces of 8, and odd ones among them."""
    n = 8 * log_uniform(rng, lo // 8, hi // 8)
    return n - rng.randint(1, 7) if rng.random() < 0.2 else n


def draw(rng):
    kind = rng.choice(["embed", "embed_back", "norm", "norm", "norm_back", "norm_back", "route", "route", "route_back",
                       "dispatch", "combine", "combine_back"])
    if kind.startswith("embed"):
        hidden, dtype = width(rng, 128, 5120), rng.choice(["bf16", "bf16", "f32"])
        vocab = min(rng.choice([VOCAB, VOCAB, log_uniform(rng, 1000, VOCAB)]), VOCAB * 2048 // hidden)
        most = 32768 * 2048 // hidden
        return embed(kind, log_uniform(rng, 1, min(32768, most)), vocab, hidden, dtype=dtype,
                     grad=rng.choice(["bf16", "bf16", "f32"]), ids=rng.choice(["i32", "i64"]),
                     scale=rng.choice([1.0, float(hidden) ** 0.5]), padded=rng.choice([0.0, 0.0, 0.2]))
    if kind.startswith("norm"):
        hidden, dtype = width(rng, 128, 8192), rng.choice(["bf16", "bf16", "f32"])
        stream = "f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"])
        most = 32768 * 5120 // hidden // (2 if stream == "f32" else 1)
        gate = rng.choice(["none", "none", "channel", "token", "element"])
        if gate == "element":
            most //= 2
        return norm(kind, log_uniform(rng, 1, min(65536, most)), hidden, dtype=dtype, stream=stream,
                    post=rng.random() < 0.5, gate=gate, sigmoid=rng.random() < 0.4, scale=rng.choice([1.0, 0.5, 0.22]),
                    offset=rng.choice([0.0, 0.0, 1.0]), weight=rng.choice(["bf16", "f32"]),
                    pad=rng.choice([0, 0, 0, 3, 8]))
    if kind.startswith("route"):
        experts = rng.choice([4, 8, 16, 60, 64, 64, 96, 128, 128, 160, 256, 256, 384, 512])
        top = min(experts, rng.choice([1, 2, 4, 6, 8, 8]))
        groups = rng.choice([1, 1, 4, 8]) if experts % 8 == 0 and experts >= 64 and kind == "route" else 1
        return route(kind, log_uniform(rng, 1, min(65536, 32768 * 256 // experts)), experts, top,
                     dtype=rng.choice(["f32", "bf16"]), sigmoid=rng.random() < 0.5, bias=rng.random() < 0.5,
                     groups=groups, top_groups=1 if groups == 1 else rng.choice([groups // 2, groups - 1]),
                     group_best=rng.choice([1, 2]), renormalize=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]),
                     index=rng.choice(["i32", "i64"]), masked=rng.choice([0.0, 0.0, 0.1]))
    hidden, dtype = width(rng, 128, 5120), rng.choice(["bf16", "bf16", "f32"])
    experts = rng.choice([4, 8, 12, 16, 60, 64, 128, 128, 256])
    top = min(experts, rng.choice([1, 2, 4, 6, 8]))
    most = 8192 * 8 * 2048 // (top * hidden) // (2 if dtype == "f32" else 1)
    return rows(kind, log_uniform(rng, 1, max(2, min(65536, most))), experts, top, hidden, dtype=dtype,
                stream="f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]) if kind != "dispatch" else dtype,
                index=rng.choice(["i32", "i64"]), ends=rng.choice(["i32", "i64"]), skew=rng.choice([0.0, 0.5, 1.0]),
                masked=rng.choice([0.0, 0.0, 0.1]), residual=rng.random() < 0.7)


# ---- inputs ----------------------------------------------------------------

def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return gen


def normal(gen, shape, sigma, dtype, pad=0):
    """N(0, sigma) made in pieces, so that 32-bit temporaries stay small; each
    row may be followed by `pad` elements that are not the tensor's."""
    whole = torch.empty((shape[0], shape[1] + pad), dtype=dtype, device=DEV)
    flat = whole.view(-1)
    for a in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - a)
        flat[a:a + n] = torch.randn(n, generator=gen, device=DEV).mul_(sigma)
    return whole[:, :shape[1]]


def embed_inputs(case, seed):
    gen = generator(seed)
    n, vocab, hidden = case["tokens"], case["vocab"], case["hidden"]
    st = {}
    # the vocabulary's entries by frequency: the k-th about 1 / k as often as the first
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    ids = ((vocab + 1.0) ** u - 1.0).long().clamp(0, vocab - 1)
    # what pads a batch has no embedding
    ids = torch.where(torch.rand(n, generator=gen, device=DEV) < case["padded"], torch.full_like(ids, -1), ids)
    st["tokens"] = ids.to(INTS[case["ids"]])
    if case["kind"] == "embed":
        st["table"] = normal(gen, (vocab, hidden), 0.02, TYPES[case["dtype"]])
    else:
        st["dout"] = normal(gen, (n, hidden), 1e-3, TYPES[case["dtype"]])
    return st


def norm_inputs(case, seed):
    gen = generator(seed)
    t, h, pad = case["tokens"], case["hidden"], case["pad"]
    dtype, stream, weight = (TYPES[case[n]] for n in ("dtype", "stream", "weight"))
    st = {"y": normal(gen, (t, h), 1.5, dtype, pad), "gate": None}
    st["h"] = normal(gen, (t, h), 2.0, stream, pad)
    for n in ("post_weight", "pre_weight"):
        st[n] = (1.0 - case["offset"] + 0.1 * torch.randn(h, generator=gen, device=DEV)).to(weight)
    if not case["post"]:
        st["post_weight"] = None
    # a gate for each channel, for each token, or for each channel of each token
    if case["gate"] == "channel":
        st["gate"] = (0.3 + 0.1 * torch.randn((1, h), generator=gen, device=DEV)).to(dtype)
    elif case["gate"] == "token":
        st["gate"] = torch.randn((t, 1), generator=gen, device=DEV).to(dtype)
    elif case["gate"] == "element":
        st["gate"] = normal(gen, (t, h), 1.0, dtype, pad)
    if case["kind"] == "norm_back":
        # h is the stream after the addition
        st["dn"], st["dh_out"] = normal(gen, (t, h), 1e-3, dtype, pad), normal(gen, (t, h), 1e-3, stream, pad)
    return st


def route_inputs(case, seed):
    gen = generator(seed)
    t, e, k = case["tokens"], case["experts"], case["top"]
    st = {"bias": None}
    z = 1.2 * torch.randn((t, e), generator=gen, device=DEV) + 0.5 * torch.randn((1, e), generator=gen, device=DEV)
    # tokens that pad the batch are routed nowhere
    empty = torch.rand((t, 1), generator=gen, device=DEV) < case["masked"]
    st["logits"] = z.masked_fill(empty, float("-inf")).to(TYPES[case["dtype"]])
    if case["bias"]:
        st["bias"] = 0.05 * torch.randn(e, generator=gen, device=DEV)
    if case["kind"] == "route_back":
        index = (z + (st["bias"] if case["bias"] else 0.0)).topk(k, dim=1).indices
        st["index"] = torch.where(empty, torch.full_like(index, -1), index).to(INTS[case["index"]])
        st["dweights"] = 1e-3 * torch.randn((t, k), generator=gen, device=DEV)
    return st


def placed(index, experts):
    """Where each entry of a router's choice stands among the rows sorted by
    expert; those without an expert stand behind, and are marked by ~."""
    key = index.long().flatten()
    absent = key < 0
    key = torch.where(absent, torch.full_like(key, experts), key)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=DEV)
    place = torch.where(absent, ~place, place)
    ends = (key[:, None] == torch.arange(experts, device=DEV)).sum(0).cumsum(0)
    return place.view(index.shape).to(torch.int32), ends


def rows_inputs(case, seed):
    gen = generator(seed)
    t, e, k, h = (case[n] for n in ("tokens", "experts", "top", "hidden"))
    dtype, stream = TYPES[case["dtype"]], TYPES[case["stream"]]
    # a router's choice, uneven by "skew"; tokens that pad the batch have none
    like = torch.rand((t, e), generator=gen, device=DEV).log().neg().log().neg()
    index = (like + case["skew"] * torch.randn((1, e), generator=gen, device=DEV)).topk(k, dim=1).indices
    empty = torch.rand((t, 1), generator=gen, device=DEV) < case["masked"]
    index = torch.where(empty, torch.full_like(index, -1), index)
    st = {}
    if case["kind"] == "dispatch":
        st["index"] = index.to(INTS[case["index"]])
        st["x"] = normal(gen, (t, h), 1.0, dtype)
        return st
    st["place"], _ = placed(index, e)
    w = torch.rand((t, k), generator=gen, device=DEV) + 0.1
    st["weights"] = torch.where(empty, torch.zeros_like(w), w / w.sum(1, keepdim=True))
    st["rows"] = normal(gen, (t * k, h), 1.0, dtype)
    if case["kind"] == "combine":
        st["residual"] = normal(gen, (t, h), 2.0, stream) if case["residual"] else None
    else:
        st["dout"] = normal(gen, (t, h), 1e-3, stream)
    return st


def inputs(case, seed):
    kind = case["kind"]
    return (embed_inputs if kind.startswith("embed") else norm_inputs if kind.startswith("norm")
            else route_inputs if kind.startswith("route") else rows_inputs)(case, seed)


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
    new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device=DEV)
    like = lambda t: None if t is None else torch.empty(t.shape, dtype=t.dtype, device=DEV)
    if kind == "embed":
        st["out"] = new(case["tokens"], case["hidden"], dtype=TYPES[case["dtype"]])
    elif kind == "embed_back":
        st["dtable"] = new(case["vocab"], case["hidden"], dtype=TYPES[case["grad"]])
    elif kind == "norm":
        st["h_out"], st["n_out"] = like(st["h"]), like(st["y"])
    elif kind == "norm_back":
        st["dh"], st["dy"], st["dgate"] = like(st["h"]), like(st["y"]), like(st["gate"])
        st["dpost_weight"], st["dpre_weight"] = like(st["post_weight"]), like(st["pre_weight"])
    elif kind == "route":
        st["index"] = new(case["tokens"], case["top"], dtype=INTS[case["index"]])
        st["weights"] = new(case["tokens"], case["top"], dtype=torch.float32)
    elif kind == "route_back":
        st["dlogits"] = like(st["logits"])
    elif kind == "dispatch":
        n = case["tokens"] * case["top"]
        st["place"] = new(case["tokens"], case["top"], dtype=torch.int32)
        st["ends"] = new(case["experts"], dtype=INTS[case["ends"]])
        st["rows"] = new(n, case["hidden"], dtype=TYPES[case["dtype"]])
    elif kind == "combine":
        st["out"] = new(case["tokens"], case["hidden"], dtype=TYPES[case["stream"]])
    else:
        st["drows"], st["dweights"] = like(st["rows"]), like(st["weights"])


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
    plain = {"embed": plain_embed, "embed_back": plain_embed_back, "norm": plain_norm, "norm_back": plain_norm_back,
             "route": plain_route, "route_back": plain_route_back, "dispatch": plain_dispatch,
             "combine": plain_combine, "combine_back": plain_combine_back}
    return plain[kind](st["case"], st)


def given(*outs):
    return tuple(t for t in outs if t is not None)


def run_own(case, st):
    from paper_2609_34162_amd import ops
    kind, ctx = case["kind"], st["ctx"].handle
    stream = torch.cuda.current_stream()
    if kind == "embed":
        ops.sdp_embed(ctx, st["table"], st["tokens"], st["out"], scale=case["scale"], stream=stream)
        return st["out"]
    if kind == "embed_back":
        ops.sdp_embed_backward(ctx, st["dout"], st["tokens"], st["dtable"], scale=case["scale"], stream=stream)
        return st["dtable"]
    if kind.startswith("norm"):
        more = dict(gate=st["gate"], gate_sigmoid=case["sigmoid"], post_norm=case["post"],
                    post_weight=st["post_weight"], pre_weight=st["pre_weight"], scale=case["scale"], eps=EPS,
                    weight_offset=case["offset"], stream=stream)
        if kind == "norm":
            ops.sdp_block_norm(ctx, st["h"], st["y"], st["h_out"], st["n_out"], **more)
            return st["h_out"], st["n_out"]
        ops.sdp_block_norm_backward(ctx, st["h"], st["y"], st["dh_out"], st["dn"], st["dh"], st["dy"],
                                    dgate=st["dgate"], dpost_weight=st["dpost_weight"],
                                    dpre_weight=st["dpre_weight"], **more)
        return given(st["dh"], st["dy"], st["dgate"], st["dpost_weight"], st["dpre_weight"])
    if kind == "route":
        ops.sdp_route(ctx, st["logits"], st["index"], st["weights"], bias=st["bias"], sigmoid=case["sigmoid"],
                      groups=case["groups"], top_groups=case["top_groups"], group_best=case["group_best"],
                      renormalize=case["renormalize"], scale=case["scale"], stream=stream)
        return st["index"], st["weights"]
    if kind == "route_back":
        ops.sdp_route_backward(ctx, st["logits"], st["index"], st["dweights"], st["dlogits"], sigmoid=case["sigmoid"],
                               renormalize=case["renormalize"], scale=case["scale"], stream=stream)
        return st["dlogits"]
    if kind == "dispatch":
        ops.sdp_expert_order(ctx, st["index"], st["ends"], st["place"], stream=stream)
        ops.sdp_expert_gather(ctx, st["x"], st["place"], st["rows"], stream=stream)
        return st["ends"], st["place"], st["rows"]
    if kind == "combine":
        ops.sdp_expert_combine(ctx, st["rows"], st["place"], st["weights"], st["out"], residual=st["residual"],
                               stream=stream)
        return st["out"]
    ops.sdp_expert_combine_backward(ctx, st["rows"], st["place"], st["weights"], st["dout"], st["drows"],
                                    st["dweights"], stream=stream)
    return st["drows"], st["dweights"]


def parts(n, width_):
    """Slices of n rows, of about PIECE elements each."""
    step = max(1, PIECE // max(1, width_))
    return [slice(a, min(n, a + step)) for a in range(0, n, step)]


def plain_embed(case, st):
    ids = st["tokens"].long()
    out = st["table"][ids.clamp(min=0)].float() * case["scale"]
    return torch.where((ids < 0)[:, None], 0.0, out).to(st["table"].dtype)


def plain_embed_back(case, st):
    ids = st["tokens"].long()
    there = ids >= 0
    total = torch.zeros((case["vocab"], case["hidden"]), device=DEV)
    total.index_put_((ids[there],), st["dout"][there].float() * case["scale"], accumulate=True)
    return total.to(TYPES[case["grad"]])


def gate_of(case, st, part):
    """The gate of these rows in 32 bits, and its derivative by the gate's input."""
    if st["gate"] is None:
        return 1.0, None
    z = (st["gate"] if case["gate"] == "channel" else st["gate"][part]).float()
    if not case["sigmoid"]:
        return z, 1.0
    a = 1.0 / (1.0 + (-z).exp())
    return a, a * (1.0 - a)


def weight_of(case, w):
    return 1.0 if w is None else w.float() + case["offset"]


def inverse_rms(x):
    return (x.square().mean(-1, keepdim=True) + EPS).rsqrt()


def plain_norm(case, st):
    h_out, n_out = torch.empty(st["h"].shape, dtype=st["h"].dtype, device=DEV), \
        torch.empty(st["y"].shape, dtype=st["y"].dtype, device=DEV)
    for part in parts(case["tokens"], case["hidden"]):
        u = st["y"][part].float()
        if case["post"]:
            u = u * inverse_rms(u) * weight_of(case, st["post_weight"])
        h = st["h"][part].float() + case["scale"] * gate_of(case, st, part)[0] * u
        h_out[part] = h
        n_out[part] = h * inverse_rms(h) * weight_of(case, st["pre_weight"])
    return h_out, n_out


def norm_gradient(x, r, v):
    """The gradient of x r, r = 1 / rms(x), from that of its value."""
    unit = x * r
    return r * (v - unit * (v * unit).mean(-1, keepdim=True))


def plain_norm_back(case, st):
    new = lambda t: torch.empty(t.shape, dtype=t.dtype, device=DEV)
    dh, dy = new(st["h"]), new(st["y"])
    dgate = None if st["gate"] is None else new(st["gate"])
    sums = {n: 0.0 for n in ("pre", "post", "gate")}
    for part in parts(case["tokens"], case["hidden"]):
        h, y, dn = st["h"][part].float(), st["y"][part].float(), st["dn"][part].float()
        r = inverse_rms(h)
        g = st["dh_out"][part].float() + norm_gradient(h, r, dn * weight_of(case, st["pre_weight"]))
        sums["pre"] = sums["pre"] + (dn * h * r).sum(0)
        dh[part] = g
        a, slope = gate_of(case, st, part)
        u, ry = y, None
        if case["post"]:
            ry = inverse_rms(y)
            u = y * ry * weight_of(case, st["post_weight"])
        if dgate is not None:
            d = case["scale"] * u * g * slope
            if case["gate"] == "channel":
                sums["gate"] = sums["gate"] + d.sum(0, keepdim=True)
            else:
                dgate[part] = d.sum(1, keepdim=True) if case["gate"] == "token" else d
        du = case["scale"] * a * g
        if case["post"]:
            sums["post"] = sums["post"] + (du * y * ry).sum(0)
            du = norm_gradient(y, ry, du * weight_of(case, st["post_weight"]))
        dy[part] = du
    if case["gate"] == "channel":
        dgate.copy_(sums["gate"])
    weight = TYPES[case["weight"]]
    return given(dh, dy, dgate, sums["post"].to(weight) if case["post"] else None, sums["pre"].to(weight))


def scores_of(case, z):
    if case["sigmoid"]:
        return 1.0 / (1.0 + (-z).exp())
    top = z.max(-1, keepdim=True).values
    e = (z - torch.where(top == float("-inf"), torch.zeros_like(top), top)).exp()
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def first_of(x, k):
    """Places of the k largest of each row, the lowest first among equals."""
    return x.sort(dim=-1, descending=True, stable=True).indices[..., :k]


def plain_route(case, st):
    z, k, g = st["logits"], case["top"], case["groups"]
    there = z != float("-inf")
    # close scores are next to a border: the choice is made in 64 bits
    key = z.double()
    if st["bias"] is not None or g > 1:
        key = scores_of(case, key) + (st["bias"].double() if st["bias"] is not None else 0.0)
    key = key.masked_fill(~there, float("-inf"))
    if g > 1:
        best = key.view(key.shape[0], g, -1).sort(dim=-1, descending=True).values[..., :case["group_best"]]
        some = best[..., 0] != float("-inf")
        best = torch.where(some, torch.where(best == float("-inf"), 0.0, best).sum(-1), float("-inf"))
        keep = torch.zeros_like(some).scatter_(1, first_of(best, case["top_groups"]), True)
        key = key.masked_fill(~keep.repeat_interleave(key.shape[1] // g, 1), float("-inf"))
    chosen = first_of(key, k)
    has = key.gather(1, chosen) != float("-inf")
    w = torch.where(has, scores_of(case, z.float()).gather(1, chosen), 0.0)
    if case["renormalize"]:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total == 0, torch.ones_like(total), total)
    return torch.where(has, chosen, -1).to(INTS[case["index"]]), w * case["scale"]


def plain_route_back(case, st):
    z, index = st["logits"].float(), st["index"].long()
    has, at = index >= 0, index.clamp(min=0)
    p = scores_of(case, z)
    w = torch.where(has, p.gather(1, at), 0.0)
    g = torch.where(has, st["dweights"] * case["scale"], 0.0)
    if case["renormalize"]:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total == 0, torch.ones_like(total), total)
        d = w * (g - (g * w).sum(1, keepdim=True))
        if case["sigmoid"]:
            d = d * (1.0 - p.gather(1, at))
    elif case["sigmoid"]:
        d = g * w * (1.0 - w)
    else:
        d = g * w
    dz = torch.zeros_like(z).scatter_add_(1, at, d)
    if not case["renormalize"] and not case["sigmoid"]:
        dz -= p * (g * w).sum(1, keepdim=True)
    return dz.to(st["logits"].dtype)


def plain_dispatch(case, st):
    place, ends = placed(st["index"], case["experts"])
    flat = place.flatten().long()
    there = flat >= 0
    rows_ = torch.zeros((flat.numel(), case["hidden"]), dtype=st["x"].dtype, device=DEV)
    token = torch.arange(flat.numel(), device=DEV) // case["top"]
    rows_[flat[there]] = st["x"][token[there]]
    return ends.to(INTS[case["ends"]]), place, rows_


def plain_combine(case, st):
    out = torch.empty((case["tokens"], case["hidden"]), dtype=TYPES[case["stream"]], device=DEV)
    for part in parts(case["tokens"], case["hidden"] * case["top"]):
        place = st["place"][part].long()
        picked = torch.where((place >= 0)[..., None], st["rows"][place.clamp(min=0)].float(), 0.0)
        total = (picked * st["weights"][part][..., None]).sum(1)
        out[part] = total if st["residual"] is None else st["residual"][part].float() + total
    return out


def plain_combine_back(case, st):
    drows = torch.zeros_like(st["rows"])
    dw = torch.zeros_like(st["weights"])
    for part in parts(case["tokens"], case["hidden"] * case["top"]):
        place = st["place"][part].long()
        there = place >= 0
        d = st["dout"][part].float()
        picked = st["rows"][place.clamp(min=0)].float()
        dw[part] = torch.where(there, (picked * d[:, None]).sum(-1), 0.0)
        drows[place[there]] = (d[:, None] * st["weights"][part][..., None])[there].to(drows.dtype)
    return drows, dw


# ---- work and the definitions in 64 bits -----------------------------------

def size_of(name):
    return {"bf16": 2, "f32": 4, "i32": 4, "i64": 8}[name]


def work(case):
    """Each input read once and each output written once (of a table, the rows
    that the tokens name: about as many as there are tokens, at most all), and
    the operations of the formulas on each element."""
    kind, t = case["kind"], case["tokens"]
    if kind.startswith("embed"):
        v, h = case["vocab"], case["hidden"]
        ids = t * size_of(case["ids"])
        if kind == "embed":
            return {"bytes": ids + (min(t, v) + t) * h * size_of(case["dtype"]), "flops": t * h}
        return {"bytes": ids + t * h * size_of(case["dtype"]) + v * h * size_of(case["grad"]), "flops": 2 * t * h}
    if kind.startswith("norm"):
        h, back = case["hidden"], kind == "norm_back"
        n = t * h
        gate = {"none": 0, "channel": h, "token": t, "element": n}[case["gate"]] * size_of(case["dtype"])
        weights = h * size_of(case["weight"]) * (2 if case["post"] else 1)
        both = n * (size_of(case["dtype"]) + size_of(case["stream"]))
        return {"bytes": both * (3 if back else 2) + (gate + weights) * (2 if back else 1),
                "flops": n * (24 if back else 12)}
    if kind.startswith("route"):
        n, k = t * case["experts"], t * case["top"]
        bias = 4 * case["experts"] if case["bias"] and kind == "route" else 0
        z = n * size_of(case["dtype"]) * (2 if kind == "route_back" else 1)
        return {"bytes": z + bias + k * (size_of(case["index"]) + 4), "flops": n * 10}
    k, h = case["top"], case["hidden"]
    n, row, side = t * k, h * size_of(case["dtype"]), h * size_of(case["stream"])
    if kind == "dispatch":
        return {"bytes": n * (size_of(case["index"]) + 4) + case["experts"] * size_of(case["ends"]) + (n + t) * row,
                "flops": 0}
    if kind == "combine":
        return {"bytes": n * (row + 8) + t * side * (2 if case["residual"] else 1), "flops": 2 * n * h}
    return {"bytes": n * (2 * row + 12) + t * side, "flops": 3 * n * h}


def exact(case, seed):
    st = inputs(case, seed)
    kind = case["kind"]
    if kind.startswith("embed"):
        return exact_embed(case, st)
    if kind.startswith("norm"):
        return exact_norm(case, st)
    if kind.startswith("route"):
        return exact_route(case, st)
    return exact_rows(case, st)


def exact_embed(case, st):
    ids = st["tokens"].long()
    at = torch.nonzero(ids >= 0)[:, 0]
    if case["kind"] == "embed":
        out = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device=DEV)
        out[at] = st["table"].index_select(0, ids[at]).double() * case["scale"]
        return out
    total = torch.zeros((case["vocab"], case["hidden"]), dtype=torch.float64, device=DEV)
    total.index_add_(0, ids[at], st["dout"].index_select(0, at).double())
    return total * case["scale"]


def exact_norm(case, st):
    """From the definition, with each norm's gradient as a derivative of
    w . x / s, s = sqrt(mean(x x) + eps): dx = (w v - x <x, w v> / (H s s)) / s."""
    hid, s_ = case["hidden"], case["scale"]
    back = case["kind"] == "norm_back"
    f64 = dict(dtype=torch.float64, device=DEV)
    outs = [torch.empty((case["tokens"], hid), **f64) for _ in range(2)]
    ones = torch.ones(hid, **f64)
    w_pre = st["pre_weight"].double() + case["offset"]
    w_post = st["post_weight"].double() + case["offset"] if case["post"] else ones
    d_pre, d_post = torch.zeros(hid, **f64), torch.zeros(hid, **f64)
    d_gate = None if st["gate"] is None else torch.zeros(st["gate"].shape, **f64)
    for sl in parts(case["tokens"], hid):
        h, y = st["h"][sl].double(), st["y"][sl].double()
        gate = torch.ones((1, 1), **f64)
        if st["gate"] is not None:
            gate = (st["gate"] if case["gate"] == "channel" else st["gate"][sl]).double()
        act = torch.sigmoid(gate) if case["sigmoid"] and st["gate"] is not None else gate
        s_y = torch.sqrt((y * y).sum(1, keepdim=True) / hid + EPS) if case["post"] else torch.ones((1, 1), **f64)
        u = w_post * y / s_y
        if not back:
            stream = h + s_ * act * u
            outs[0][sl] = stream
            outs[1][sl] = w_pre * stream / torch.sqrt((stream * stream).sum(1, keepdim=True) / hid + EPS)
            continue
        v = st["dn"][sl].double()
        s_h = torch.sqrt((h * h).sum(1, keepdim=True) / hid + EPS)
        d_pre += (v * h / s_h).sum(0)
        g = st["dh_out"][sl].double() + (w_pre * v - h * (h * w_pre * v).sum(1, keepdim=True) / (hid * s_h * s_h)) / s_h
        outs[0][sl] = g
        if d_gate is not None:
            d = s_ * g * u * (act * (1.0 - act) if case["sigmoid"] else 1.0)
            if case["gate"] == "channel":
                d_gate += d.sum(0, keepdim=True)
            else:
                d_gate[sl] = d.sum(1, keepdim=True) if case["gate"] == "token" else d
        du = s_ * act * g
        if case["post"]:
            d_post += (du * y / s_y).sum(0)
            du = (w_post * du - y * (y * w_post * du).sum(1, keepdim=True) / (hid * s_y * s_y)) / s_y
        outs[1][sl] = du
    return given(*outs, d_gate, d_post if case["post"] else None, d_pre) if back else tuple(outs)


def exact_route(case, st):
    """Chosen one at a time: the largest that is left, the first of equals."""
    z = st["logits"].double()
    t, e = z.shape
    k, g = case["top"], case["groups"]
    low = float("-inf")
    p = torch.sigmoid(z) if case["sigmoid"] else torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
    if case["kind"] == "route_back":
        dw, idx = st["dweights"].double() * case["scale"], st["index"].long()
        dz = torch.zeros((t, e), dtype=torch.float64, device=DEV)
        chosen = torch.zeros((t, e), dtype=torch.float64, device=DEV)
        g_at = torch.zeros((t, e), dtype=torch.float64, device=DEV)
        for j in range(k):
            one = (torch.arange(e, device=DEV)[None] == idx[:, j:j + 1]).double()
            chosen += one
            g_at += one * dw[:, j:j + 1]
        q = p * chosen
        if case["renormalize"]:
            total = q.sum(1, keepdim=True)
            q = torch.where(total > 0, q / total.clamp(min=1e-300), 0.0)
            dz = q * (g_at - (g_at * q).sum(1, keepdim=True)) * ((1.0 - p) if case["sigmoid"] else 1.0)
        elif case["sigmoid"]:
            dz = g_at * p * (1.0 - p)
        else:
            dz = p * (g_at - (g_at * p).sum(1, keepdim=True))
        return dz
    key = z.clone()
    if case["bias"] or g > 1:
        key = p.clone()
        if case["bias"]:
            key += st["bias"].double()
    key[z == low] = low

    def take(x, n):
        x, places, values = x.clone(), [], []
        line = torch.arange(x.shape[1], device=DEV)[None]
        for _ in range(n):
            top = x.max(1, keepdim=True).values
            at = torch.where(x == top, line, x.shape[1]).min(1, keepdim=True).values
            places.append(torch.where(top == low, -1, at))
            values.append(top)
            x.scatter_(1, at, low)
        return torch.cat(places, 1), torch.cat(values, 1)

    if g > 1:
        each = key.view(t * g, e // g)
        values = take(each, case["group_best"])[1]
        sums = torch.where(values == low, 0.0, values).sum(1)
        sums[values[:, 0] == low] = low
        which = take(sums.view(t, g), case["top_groups"])[0]
        keep = (which[:, None, :] == torch.arange(g, device=DEV)[None, :, None]).any(2)
        key = torch.where(keep[:, :, None], key.view(t, g, -1), low).view(t, e)
    index = take(key, k)[0]
    w = torch.where(index >= 0, p.gather(1, index.clamp(min=0)), 0.0)
    if case["renormalize"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total.clamp(min=1e-300), 0.0)
    return index.to(INTS[case["index"]]), w * case["scale"]


def exact_rows(case, st):
    t, k, h = case["tokens"], case["top"], case["hidden"]
    f64 = dict(dtype=torch.float64, device=DEV)
    if case["kind"] == "dispatch":
        # an entry's place: the entries of lower experts, and those of its own before it
        idx = st["index"].long().flatten()
        n = idx.numel()
        counts, place, before = [], torch.zeros(n, dtype=torch.int64, device=DEV), 0
        for e in list(range(case["experts"])) + [-1]:
            mine = idx == e
            count = int(mine.sum())
            place[mine] = before + torch.arange(count, device=DEV)
            before += count
            counts.append(before)
        out = torch.zeros((n, h), **f64)
        out[place[idx >= 0]] = st["x"].double().repeat_interleave(k, 0)[idx >= 0]
        ends = torch.tensor(counts[:-1], device=DEV).to(INTS[case["ends"]])
        return ends, torch.where(idx >= 0, place, -1 - place).view(t, k).to(torch.int32), out
    place, w = st["place"].long(), st["weights"].double()
    if case["kind"] == "combine":
        out = torch.zeros((t, h), **f64) if st["residual"] is None else st["residual"].double()
        for j in range(k):
            on = place[:, j] >= 0
            out[on] += w[on, j:j + 1] * st["rows"][place[on, j]].double()
        return out
    drows, dw = torch.zeros((t * k, h), **f64), torch.zeros((t, k), **f64)
    for j in range(k):
        on = place[:, j] >= 0
        d = st["dout"][on].double()
        drows[place[on, j]] = w[on, j:j + 1] * d
        dw[on, j] = (st["rows"][place[on, j]].double() * d).sum(1)
    return drows, dw
