"""The training operators and the update together, as examples/train_step.py uses
them: every step's loss and the first step's gradients agree with the same model
and the same update in plain 32-bit torch."""
import importlib.util
import os

import pytest

import gpu_util

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    gpu_util.need_gpu()
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def plain_loss(example, p, w):
    """The same layer in 32 bits, the experts one by one, and its loss."""
    x = w["embed"][p.tokens]
    B, S, H, K, D = example.BATCH, example.TOKENS, example.Q_HEADS, example.K_HEADS, example.DIM
    qkv = (x @ w["qkv"].t()).view(B, S, H + 2 * K, D)

    def turned(t, weight):
        t = t * (t.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight
        a, b = t[..., :D // 2], t[..., D // 2:]
        c, sn = p.cos[None, :, None], p.sin[None, :, None]
        return torch.cat((a * c - b * sn, b * c + a * sn), -1)
    q, k, v = turned(qkv[:, :, :H], w["q_norm"]), turned(qkv[:, :, H:H + K], w["k_norm"]), qkv[:, :, H + K:]
    q, k, v = (t.transpose(1, 2) for t in (q, k.repeat_interleave(H // K, 2), v.repeat_interleave(H // K, 2)))
    score = q @ k.transpose(2, 3).contiguous() * D ** -0.5
    later = torch.ones(S, S, dtype=torch.bool, device="cuda").triu(1)
    a = score.masked_fill(later, float("-inf")).softmax(-1) @ v
    x = (x + a.transpose(1, 2).reshape(B, S, -1) @ w["o"].t()).flatten(0, 1)
    share, chosen = (x @ w["router"].t()).softmax(-1).topk(example.TOP, dim=-1)
    out = x
    for e in range(example.EXPERTS):
        at = (chosen == e).nonzero()
        gate, up = (x[at[:, 0]] @ w["up"][e].t()).chunk(2, dim=1)
        y = (torch.nn.functional.silu(gate) * up) @ w["down"][e].t()
        out = out.index_add(0, at[:, 0], y * share[at[:, 0], at[:, 1]][:, None])
    z = out @ w["head"].t()
    there = p.top_index >= 0
    q_t = torch.where(there, torch.softmax(p.top_logits / 2.0, 1), 0.0)
    log_p = torch.log_softmax(z / 2.0, 1).gather(1, p.top_index.clamp(min=0))
    kl = torch.where(there, q_t * (q_t.clamp(min=1e-30).log() - log_p), 0.0).sum(1) * 4.0
    ce = torch.nn.functional.cross_entropy(z, p.labels, reduction="none", ignore_index=-100)
    return ((0.7 * kl + 0.3 * ce) / int(p.learned.sum())).sum()


def start(example, p):
    return {n: t.float().clone().requires_grad_() for n, t in p.student.w.items()}


# Activations and gradients in BF16 carry up to 2^-8 relative each, over about ten
# roundings on the way down and up: a few hundredths in a norm; a router's close
# choice may fall the other way for a token in a hundred.
LOSS, GRADIENT = 0.02, 0.15


def test_the_student_learns_as_plain_torch_does(example):
    p = example.Program()
    w, lr, (b1, b2, eps) = start(example, p), 3e-3, (0.9, 0.999, 1e-8)
    moments = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in w.items()}
    losses = []
    for number in range(1, 26):
        want = plain_loss(example, p, w)
        grads = torch.autograd.grad(want, list(w.values()))
        clip = min(1.0, 1.0 / float(sum(g.square().sum() for g in grads).sqrt()))
        with torch.no_grad():
            for (n, t), g in zip(w.items(), grads):
                m, v = moments[n]
                m.mul_(b1).add_(g * clip, alpha=1 - b1)
                v.mul_(b2).add_((g * clip).square(), alpha=1 - b2)
                t -= lr * (m / (1 - b1 ** number)) / ((v / (1 - b2 ** number)).sqrt() + eps)
        losses.append(p.step(number, lr)[0])
        assert abs(losses[-1] - want.item()) <= LOSS * want.item(), (number, losses[-1], want.item())
    p.close()
    assert losses[-1] < losses[0], losses


def test_gradients_against_plain_torch(example):
    p = example.Program(seed=3)
    w = start(example, p)
    loss, _ = p.step(1, 0.0)
    want = plain_loss(example, p, w)
    want.backward()
    p.close()
    assert abs(loss - want.item()) <= LOSS * abs(want.item())
    for n, t in w.items():
        off = float((p.student.g[n].float() - t.grad).norm() / t.grad.norm())
        assert off <= GRADIENT, (n, off)
