"""One pipeline stage, a transformer block in R replicas, trained with the framework's own calls:

    forward weights of the stage -> linear, qk_norm -> loss -> their gradients in the flat arrays of the step
    -> grad_norm -> Stage.step_scaled (local step, clipped, look-ahead and delayed sparse averaging)

Attention itself is plain PyTorch: it owns no parameters.  The task is synthetic: map random rows to what a fixed random block makes
of them, each replica with rows of its own.

    python examples/train_block.py [--steps 60] [--width 256] [--tokens 512] [--replicas 2]
"""
import argparse
import math
import sys
from pathlib import Path

import torch

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

import paper_2601_22442_amd as am  # noqa: E402


class Block:
    """Where the parameters of a block lie in the stage's flat arrays, and its two passes over all replicas."""

    def __init__(self, width, heads, tokens):
        self.width, self.heads, self.dim, self.tokens = width, heads, width // heads, tokens
        d = width
        shapes = {"qkv": (3 * d, d), "qkv_bias": (3 * d,), "q_gain": (self.dim,), "k_gain": (self.dim,), "out": (d, d), "out_bias": (d,),
                  "up": (4 * d, d), "up_bias": (4 * d,), "down": (d, 4 * d), "down_bias": (d,)}
        self.places, at = {}, 0
        for name, shape in shapes.items():
            self.places[name] = (at, shape)
            at += (math.prod(shape) + 7) // 8 * 8          # whole chunks of 16 bytes: the fast case of the products
        self.n = at
        self.cos, self.sin = am.rotation_table(tokens, self.dim)

    def view(self, flats, name):
        at, shape = self.places[name]
        return [f[at:at + math.prod(shape)].view(shape) for f in flats]

    def first_weights(self, seed):
        g = torch.Generator().manual_seed(seed)
        w = torch.zeros(self.n)
        for name, (at, shape) in self.places.items():
            k = math.prod(shape)
            w[at:at + k] = 1.0 if name.endswith("gain") else 0.0 if name.endswith("bias") else torch.randn(k, generator=g) / math.sqrt(shape[-1])
        return w

    def attention(self, q, k, v):
        """Causal attention of one replica in fp32: [tokens, heads, dim] each."""
        q, k, v = (x.float().transpose(0, 1) for x in (q, k, v))
        scores = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(self.dim)
        mask = torch.ones(self.tokens, self.tokens, dtype=torch.bool, device=q.device).triu(1)
        return torch.matmul(scores.masked_fill(mask, float("-inf")).softmax(-1), v.contiguous()).transpose(0, 1)

    def forward(self, weights, x):
        p = lambda name: self.view(weights, name)                                  # noqa: E731
        d, heads = self.width, (self.heads, self.dim)
        s = {"x": x}
        s["qkv"] = am.linear(x, p("qkv"), p("qkv_bias"))
        q, k, v = ([t[:, i * d:(i + 1) * d].unflatten(1, heads) for t in s["qkv"]] for i in range(3))
        s["q"], s["k"] = q, k
        qn, kn = am.qk_norm(q, k, p("q_gain"), p("k_gain"), self.cos, self.sin)
        s["leaves"] = [[t.detach().requires_grad_(True) for t in leaves] for leaves in zip(qn, kn, v)]
        s["attended"] = [self.attention(*leaves) for leaves in s["leaves"]]
        s["rows"] = [a.detach().to(x[0].dtype).reshape(self.tokens, d) for a in s["attended"]]
        s["h"] = am.linear(s["rows"], p("out"), p("out_bias"), residual=x)
        s["u"], s["pre"] = am.linear(s["h"], p("up"), p("up_bias"), act=am.ACT_GELU, with_pre=True)
        return am.linear(s["u"], p("down"), p("down_bias"), residual=s["h"]), s

    def backward(self, weights, grads, dy, s):
        """Fills the flat gradient arrays."""
        p = lambda name: self.view(weights, name)                                  # noqa: E731
        g = lambda name: self.view(grads, name)                                    # noqa: E731
        du = am.linear_backward(dy, s["u"], p("down"), dw=g("down"), db=g("down_bias"))
        dh = am.linear_backward(du, s["h"], p("up"), act=am.ACT_GELU, pre=s["pre"], dw=g("up"), db=g("up_bias"))
        dh = [a + b for a, b in zip(dh, dy)]
        drows = am.linear_backward(dh, s["rows"], p("out"), dw=g("out"), db=g("out_bias"))
        inner = [torch.autograd.grad(a, leaves, r.view(a.shape).float()) for a, leaves, r in zip(s["attended"], s["leaves"], drows)]
        dq, dk = am.qk_norm_backward([i[0].contiguous() for i in inner], [i[1].contiguous() for i in inner], s["q"], s["k"], p("q_gain"), p("k_gain"),
                                     self.cos, self.sin, dq_gain=g("q_gain"), dk_gain=g("k_gain"))
        dqkv = [torch.cat([a.flatten(1), b.flatten(1), i[2].flatten(1)], 1) for a, b, i in zip(dq, dk, inner)]
        am.linear_backward(dqkv, s["x"], p("qkv"), dw=g("qkv"), db=g("qkv_bias"), need_dx=False)


def train(steps=60, width=256, tokens=512, replicas=2, lr=1e-3, seed=0, report=print):
    """Returns the mean loss over the replicas of every step."""
    block = Block(width, max(1, width // 64), tokens)
    cfg = am.make_config(block.n, replicas, delay=2, fraction=0.05, seed=seed, lookahead=True, gamma=0.5, fwd_dtype=am.BF16, grad_dtype=am.BF16)
    stage = am.init_state(cfg, block.first_weights(seed).cuda())
    for f, w in zip(stage.fwd, stage.w):
        f.copy_(w)                                        # before the first step the forward weights are the weights
    teacher = [block.first_weights(seed + 1).cuda().bfloat16()] * replicas
    grads = [torch.zeros(block.n, dtype=torch.bfloat16, device="cuda") for _ in range(replicas)]
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    losses = []
    for t in range(1, steps + 1):
        x = [torch.randn(tokens, width, generator=g, device="cuda").bfloat16() for _ in range(replicas)]
        want, _ = block.forward(teacher, x)
        got, kept = block.forward(stage.fwd, x)
        error = [a.float() - b.float() for a, b in zip(got, want)]
        losses.append(torch.stack([e.square().mean() for e in error]).mean())
        block.backward(stage.fwd, grads, [(e * (2 / e.numel())).bfloat16() for e in error], kept)
        norm, factor = am.grad_norm([[f] for f in grads], max_norm=1.0)
        stage.step_scaled(t, grads, lr, am.ema_lambda(t, steps), 1.0, factor)
        if report and (t == 1 or t % 10 == 0):
            report(f"step {t}: loss {losses[-1].item():.4f}, gradient norms {[round(v, 4) for v in norm.tolist()]}")
    return [v.item() for v in losses]


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("steps", 60), ("width", 256), ("tokens", 512), ("replicas", 2)):
        parser.add_argument("--" + name, type=int, default=default)
    train(**vars(parser.parse_args()))
