"""A block with routed experts from the operators alone, as they are used: embedding, norm,
routing, the entries' order, rows to experts, their products, rows back, and the norm around
the block with its gate; forward and every gradient against the same block in 64 bits, and
forward for single tokens and small batches from a captured graph."""
import pytest

import gpu_util

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
VOCAB, EXPERTS, TOP, GROUPS, TOP_GROUPS, SCALE, ROUTED = 300, 16, 4, 4, 2, 8.0, 2.5
HOW = dict(sigmoid=True, groups=GROUPS, top_groups=TOP_GROUPS, group_best=2, renormalize=True, scale=ROUTED)


@pytest.fixture(scope="module")
def lib():
    sdp = gpu_util.need_gpu()
    from paper_2609_34162_amd import ops
    c = sdp.sdp_ctx_create(0, 0, 1, 0)
    yield ops, c
    torch.cuda.synchronize()
    sdp.sdp_ctx_destroy(c)


class Block:
    def __init__(self, lib, tokens, hidden, stream, seed=0):
        self.ops, self.ctx = lib
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *shape, dtype=BF16, by=1.0: (torch.randn(shape, generator=gen) * by).to(dtype).cuda()
        self.gen, self.tokens, self.hidden, self.stream = gen, tokens, hidden, stream
        self.table = rand(VOCAB, hidden, by=0.1)
        self.w0, self.post, self.w1, self.gate = (rand(hidden, by=0.3) for _ in range(4))
        self.router = rand(EXPERTS, hidden, dtype=F32, by=hidden ** -0.5)
        self.experts = rand(EXPERTS, hidden, hidden, by=hidden ** -0.5)
        self.bias = rand(EXPERTS, dtype=F32, by=0.1)
        self.bias[3] = float("-inf")  # an expert that takes none
        self.ids = torch.zeros(tokens, dtype=torch.int64, device="cuda")
        self.read()
        new = lambda *shape, dtype=BF16: torch.empty(shape, dtype=dtype, device="cuda")
        n = tokens * TOP
        self.h0, self.h1 = new(tokens, hidden, dtype=stream), new(tokens, hidden, dtype=stream)
        self.n0, self.c, self.n1 = new(tokens, hidden), new(tokens, hidden), new(tokens, hidden)
        self.logits, self.share = new(tokens, EXPERTS, dtype=F32), new(tokens, TOP, dtype=F32)
        self.index, self.place = new(tokens, TOP, dtype=I32), new(tokens, TOP, dtype=I32)
        self.ends = new(EXPERTS, dtype=I32)
        self.rows, self.y = new(n, hidden), new(n, hidden)
        self.dn, self.dh = rand(tokens, hidden), rand(tokens, hidden, dtype=stream)

    def read(self):
        """Other tokens, some of them padding and some the same."""
        ids = torch.randint(0, VOCAB, (self.tokens,), generator=self.gen)
        ids[self.tokens // 2::5] = -1
        self.ids.copy_(ids)

    def around(self):
        return dict(gate=self.gate, gate_sigmoid=True, post_norm=True, post_weight=self.post, pre_weight=self.w1,
                    scale=0.7, weight_offset=1.0)

    def forward(self, s=None):
        o, c = self.ops, self.ctx
        o.sdp_embed(c, self.table, self.ids, self.h0, scale=SCALE, stream=s)
        o.sdp_block_norm(c, self.h0, None, None, self.n0, pre_weight=self.w0, weight_offset=1.0, stream=s)
        with torch.cuda.stream(s):
            torch.mm(self.n0.float(), self.router.t(), out=self.logits)
        o.sdp_route(c, self.logits, self.index, self.share, bias=self.bias, stream=s, **HOW)
        o.sdp_expert_order(c, self.index, self.ends, self.place, stream=s)
        o.sdp_expert_gather(c, self.n0, self.place, self.rows, stream=s)
        o.sdp_grouped_matmul(c, self.rows, self.experts, self.ends, self.y, stream=s)
        o.sdp_expert_combine(c, self.y, self.place, self.share, self.c, stream=s)
        o.sdp_block_norm(c, self.h0, self.c, self.h1, self.n1, stream=s, **self.around())
        return [self.h1, self.n1]

    def backward(self):
        o, c, like = self.ops, self.ctx, torch.empty_like
        how = {k: v for k, v in HOW.items() if k in ("sigmoid", "renormalize", "scale")}
        g = {n: like(getattr(self, n)) for n in ("table", "w0", "post", "w1", "gate", "experts")}
        dh, dc, dn0 = like(self.h0), like(self.c), like(self.n0)
        o.sdp_block_norm_backward(c, self.h1, self.c, self.dh, self.dn, dh, dc, dgate=g["gate"], dpost_weight=g["post"],
                                  dpre_weight=g["w1"], **self.around())
        dy, dshare, drows, dlogits = like(self.y), like(self.share), like(self.rows), like(self.logits)
        o.sdp_expert_combine_backward(c, self.y, self.place, self.share, dc, dy, dshare)
        o.sdp_grouped_matmul_backward(c, self.rows, self.experts, self.ends, dy, drows, g["experts"])
        o.sdp_route_backward(c, self.logits, self.index, dshare, dlogits, **how)
        o.sdp_expert_gather_backward(c, drows, self.place, dn0)
        g["router"] = dlogits.t().contiguous() @ self.n0.float()
        dn0 = (dn0.float() + dlogits @ self.router).to(BF16)
        o.sdp_block_norm_backward(c, self.h0, None, dh, dn0, dh, None, pre_weight=self.w0, dpre_weight=g["w0"],
                                  weight_offset=1.0)
        o.sdp_embed_backward(c, dh, self.ids, g["table"], scale=SCALE)
        return g

    def plain(self):
        """The same in 64 bits on the CPU, for the experts that were chosen: outputs and gradients."""
        w = {n: getattr(self, n).cpu().double().requires_grad_()
             for n in ("table", "w0", "post", "w1", "gate", "experts", "router")}
        ids, index = self.ids.cpu(), self.index.cpu().long()
        norm = lambda x, weight: x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * (1.0 + weight)
        h0 = torch.where((ids >= 0)[:, None], w["table"][ids.clamp(min=0)] * SCALE, 0.0)
        n0 = norm(h0, w["w0"])
        score = torch.sigmoid(n0 @ w["router"].t())
        mine = score.gather(1, index)
        share = mine / mine.sum(-1, keepdim=True) * ROUTED
        c = sum(share[:, k:k + 1] * (w["experts"][index[:, k]] @ n0[:, :, None])[:, :, 0] for k in range(TOP))
        h1 = h0 + 0.7 * torch.sigmoid(w["gate"]) * norm(c, w["post"])
        n1 = norm(h1, w["w1"])
        ((h1 * self.dh.cpu().double()).sum() + (n1 * self.dn.cpu().double()).sum()).backward()
        return h1, n1, {n: t.grad for n, t in w.items()}


# Forward five roundings to BF16 lie between the table and an output (the stream twice,
# the norm, the products, their sum), each at most 2^-8 of a norm, and the block's own norm
# divides by what it is given: 6 x 2^-8 = 0.024 with its own.  Backward as many again lie
# on the way (dc, dy, drows, dn0, dh), through factors that carry forward's: 12 x 2^-8, and
# the share's gradient is the difference of sums that partly cancel, which doubles it.
OUTPUT, GRADIENT = 0.024, 0.094


@pytest.mark.parametrize("stream", [BF16, F32])
@pytest.mark.parametrize("tokens,hidden", [(1, 64), (7, 136), (257, 200), (1500, 512)])
def test_outputs_and_gradients(lib, tokens, hidden, stream):
    block = Block(lib, tokens, hidden, stream, seed=tokens)
    block.forward()
    got = block.backward()
    h1, n1, want = block.plain()
    assert not (block.index == 3).any()
    for name, mine, plain, most in [("h1", block.h1, h1, OUTPUT), ("n1", block.n1, n1, OUTPUT)] + [
            (n, got[n], want[n], GRADIENT) for n in want]:
        off, size = float((mine.cpu().double() - plain).norm()), float(plain.norm())
        assert off <= most * size, (name, off, size)


def test_the_same_bits_again(lib):
    block = Block(lib, 900, 256, BF16)
    first = [t.clone() for t in block.forward()] + list(block.backward().values())
    again = [t.clone() for t in block.forward()] + list(block.backward().values())
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("tokens", [1, 8, 65])
def test_serving_from_a_graph(lib, tokens):
    block = Block(lib, tokens, 192, BF16, seed=tokens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    block.forward(s)  # what libraries set up at their first call
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        block.forward(s)
    for _ in range(4):
        block.read()
        for t in (block.h1, block.n1, block.index):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (block.h1, block.n1, block.index)]
        block.forward(s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (block.h1, block.n1, block.index)))
