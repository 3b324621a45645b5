"""A small training program around the update: a student with normed and rotated
queries and keys and routed experts learns a teacher's top logits.

One decoder layer: attention whose queries and keys go through
sdp_qk_norm_rope, then a mixture of experts whose products are
sdp_grouped_matmul (the tokens sorted by expert), then the head and
sdp_distill_loss, which gives the loss and the logits' gradient in one call.
The backward calls write BF16 gradients straight into the flat gradient buffer
of an sdp_segment -- the experts' as they come from
sdp_grouped_matmul_backward -- and sdp_agg_adam_step clips them, takes the step
on the FP32 master weights and gives back the BF16 weights.  Attention's
scores, the router and the dense products are plain torch.

    python3 examples/train_step.py [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_34162_amd import ops, sdp  # noqa: E402

DEV, BF16 = "cuda", torch.bfloat16
BATCH, TOKENS, HIDDEN, Q_HEADS, K_HEADS, DIM = 4, 128, 256, 8, 2, 32
EXPERTS, TOP, FFN, VOCAB, TEACHER_K = 8, 2, 192, 4000, 16


class Weights:
    """Every weight in one flat segment: FP32 master and moments, BF16 weights
    and BF16 gradients, each weight a view of them."""

    def __init__(self, shapes, sigma, gen):
        sizes = {n: torch.Size(s).numel() for n, s in shapes.items()}
        total = sum((k + 63) // 64 * 64 for k in sizes.values())
        self.master = torch.zeros(total, device=DEV)
        self.m, self.v = torch.zeros_like(self.master), torch.zeros_like(self.master)
        self.bf16, self.grad = (torch.zeros(total, dtype=BF16, device=DEV) for _ in range(2))
        self.w, self.g, at = {}, {}, 0
        for n, shape in shapes.items():
            part = slice(at, at + sizes[n])
            self.master[part] = 1.0 if len(shape) == 1 else torch.randn(sizes[n], generator=gen, device=DEV) * sigma
            self.w[n], self.g[n] = self.bf16[part].view(shape), self.grad[part].view(shape)
            at += (sizes[n] + 63) // 64 * 64
        self.bf16.copy_(self.master)
        self.segments = sdp.segments_from_tensors([(self.master, self.m, self.v, self.bf16, [self.grad])])


class NormRope(torch.autograd.Function):
    """sdp_qk_norm_rope on heads of the fused projection; the norm weights' gradients go to `grads`."""

    @staticmethod
    def forward(ctx, qkv, prog, w, g):
        q, k = qkv[:, :, :Q_HEADS], qkv[:, :, Q_HEADS:Q_HEADS + K_HEADS]
        out = torch.empty(q.shape, dtype=BF16, device=DEV), torch.empty(k.shape, dtype=BF16, device=DEV)
        ops.sdp_qk_norm_rope(prog.ctx, q, k, *out, prog.cos, prog.sin, q_weight=w["q_norm"], k_weight=w["k_norm"],
                             stream=torch.cuda.current_stream())
        ctx.saved = qkv, prog, w, g
        return out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        qkv, prog, w, g = ctx.saved
        dqkv = torch.zeros_like(qkv)  # the values' part is added by their own path
        part = lambda t: (t[:, :, :Q_HEADS], t[:, :, Q_HEADS:Q_HEADS + K_HEADS])
        ops.sdp_qk_norm_rope_backward(prog.ctx, *part(qkv), dq_out.contiguous(), dk_out.contiguous(), *part(dqkv),
                                      prog.cos, prog.sin, q_weight=w["q_norm"], k_weight=w["k_norm"],
                                      dq_weight=g["q_norm"], dk_weight=g["k_norm"],
                                      stream=torch.cuda.current_stream())
        return dqkv, None, None, None


class Experts(torch.autograd.Function):
    """Rows sorted by expert times that expert's weight; its gradient goes to `grad`."""

    @staticmethod
    def forward(ctx, x, prog, w, grad, ends):
        y = torch.empty((x.shape[0], w.shape[1]), dtype=BF16, device=DEV)
        ops.sdp_grouped_matmul(prog.ctx, x, w, ends, y, stream=torch.cuda.current_stream())
        ctx.saved = x, prog, w, grad, ends
        return y

    @staticmethod
    def backward(ctx, dy):
        x, prog, w, grad, ends = ctx.saved
        dx = torch.empty_like(x)
        ops.sdp_grouped_matmul_backward(prog.ctx, x, w, ends, dy.contiguous(), dx, grad,
                                        stream=torch.cuda.current_stream())
        return dx, None, None, None, None


class Program:
    def __init__(self, seed=0):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.ctx = sdp.sdp_ctx_create(torch.cuda.current_device(), 0, 1, 0)
        qkv = (Q_HEADS + 2 * K_HEADS) * DIM
        self.shapes = dict(embed=(VOCAB, HIDDEN), qkv=(qkv, HIDDEN), q_norm=(DIM,), k_norm=(DIM,),
                           o=(HIDDEN, Q_HEADS * DIM), router=(EXPERTS, HIDDEN), up=(EXPERTS, 2 * FFN, HIDDEN),
                           down=(EXPERTS, HIDDEN, FFN), head=(VOCAB, HIDDEN))
        angle = torch.arange(TOKENS, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, DIM, 2, device=DEV) / DIM)
        self.cos, self.sin = angle.cos(), angle.sin()
        self.student, self.teacher = Weights(self.shapes, 0.05, gen), Weights(self.shapes, 0.05, gen)
        self.tokens = torch.randint(0, VOCAB, (BATCH, TOKENS), generator=gen, device=DEV)
        # the first tokens are a prompt: nothing is learned from them
        self.learned = (torch.arange(TOKENS, device=DEV) >= TOKENS // 4).expand(BATCH, TOKENS).reshape(-1)
        logits = self.forward(self.teacher, self.teacher.w, None)
        top = logits.float().topk(TEACHER_K, dim=1)
        self.top_logits = top.values.contiguous()
        self.top_index = torch.where(self.learned[:, None], top.indices, -1).contiguous()
        self.labels = torch.where(self.learned, top.indices[:, 0], -100).contiguous()

    def forward(self, weights, leaf, grads):
        """Logits of every token; `leaf`: the weights that plain torch differentiates."""
        g = grads if grads is not None else {n: torch.empty_like(t) for n, t in weights.w.items()}
        w = weights.w
        x = leaf["embed"][self.tokens]
        qkv = (x.flatten(0, 1) @ leaf["qkv"].t()).view(BATCH, TOKENS, Q_HEADS + 2 * K_HEADS, DIM)
        q, k = NormRope.apply(qkv, self, w, g)
        v = qkv[:, :, Q_HEADS + K_HEADS:]
        rep = Q_HEADS // K_HEADS
        q, k, v = (t.float().transpose(1, 2) for t in (q, k.repeat_interleave(rep, 2), v.repeat_interleave(rep, 2)))
        score = q @ k.transpose(2, 3).contiguous() * DIM ** -0.5
        later = torch.ones(TOKENS, TOKENS, dtype=torch.bool, device=DEV).triu(1)
        a = score.masked_fill(later, float("-inf")).softmax(-1) @ v
        x = x + (a.transpose(1, 2).reshape(BATCH * TOKENS, -1).to(BF16) @ leaf["o"].t()).view_as(x)
        x = x.flatten(0, 1)
        share, chosen = (x @ leaf["router"].t()).float().softmax(-1).topk(TOP, dim=-1)
        order = chosen.flatten().argsort(stable=True)
        ends = torch.bincount(chosen.flatten(), minlength=EXPERTS).cumsum(0)
        rows = x[order // TOP]
        gate, up = Experts.apply(rows, self, w["up"], g["up"], ends).chunk(2, dim=1)
        h = (torch.nn.functional.silu(gate.float()) * up.float()).to(BF16)
        y = Experts.apply(h, self, w["down"], g["down"], ends)
        y = y.float() * share.flatten()[order][:, None]
        x = x + torch.zeros_like(x, dtype=torch.float32).index_add(0, order // TOP, y).to(BF16)
        return x @ leaf["head"].t()

    def step(self, number, lr):
        s = self.student
        mine = ("q_norm", "k_norm", "up", "down")  # whose gradients the operators write
        leaf = {n: t if n in mine else t.detach().requires_grad_() for n, t in s.w.items()}
        logits = self.forward(s, leaf, s.g)
        loss = torch.empty(logits.shape[0], device=DEV)
        row_grad = torch.full_like(loss, 1.0 / int(self.learned.sum()))
        dlogits = torch.empty_like(logits)
        ops.sdp_distill_loss(self.ctx, logits.detach(), loss, teacher_logits=self.top_logits,
                             teacher_index=self.top_index, labels=self.labels, temperature=2.0, distill_weight=0.7,
                             label_weight=0.3, row_grad=row_grad, dlogits=dlogits,
                             stream=torch.cuda.current_stream())
        logits.backward(dlogits)
        for n, t in leaf.items():
            if n not in mine:
                s.g[n].copy_(t.grad)
        hp = sdp.make_params(lr=lr, weight_decay=0.0, max_grad_norm=1.0, step=number)
        norm = sdp.sdp_agg_adam_step(self.ctx, s.segments, hp, 0, torch.cuda.current_stream(), want_norm=True)
        return float((loss * row_grad).sum()), norm

    def close(self):
        torch.cuda.synchronize()
        sdp.sdp_ctx_destroy(self.ctx)


def main(steps):
    program = Program()
    losses = []
    for number in range(1, steps + 1):
        loss, norm = program.step(number, 3e-3)
        losses.append(loss)
        if number == 1 or number % 5 == 0:
            print(f"step {number}: loss {loss:.4f}, gradient norm {norm:.4f}", flush=True)
    program.close()
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=40)
    main(parser.parse_args().steps)
