"""examples/train_block.py: the layers, the gradient norm and the stage's step as one training program."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(amlib):
    path = Path(__file__).resolve().parent.parent / "examples" / "train_block.py"
    spec = importlib.util.spec_from_file_location("train_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_loss_falls(example):
    losses = example.train(steps=40, width=128, tokens=256, replicas=3, report=None)
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5]), losses


def test_gradients_of_the_block_against_autograd(example):
    """Every parameter's gradient against PyTorch's own of the same block in fp64.  Activations are rounded to bf16 (2^-8) some ten times on
    the way, each by a random amount: a relative error of a few 2^-8 of the gradient's own root mean square; the bound is 2^-4 of it."""
    T, d = 96, 128
    block = example.Block(d, 2, T)
    gen = torch.Generator().manual_seed(3)
    flat = [block.first_weights(s).cuda().bfloat16() for s in (1, 2)]
    x = [torch.randn(T, d, generator=gen).bfloat16().cuda() for _ in flat]
    dy = [(torch.randn(T, d, generator=gen) / T).bfloat16().cuda() for _ in flat]
    grads = [torch.zeros(block.n, dtype=torch.bfloat16, device="cuda") for _ in flat]
    _, kept = block.forward(flat, x)
    block.backward(flat, grads, dy, kept)
    for i in range(2):
        p = {name: block.view([flat[i]], name)[0].double().requires_grad_(True) for name in block.places}
        X = x[i].double()
        qkv = X @ p["qkv"].t() + p["qkv_bias"]
        q, k, v = (t.unflatten(1, (2, d // 2)) for t in qkv.split(d, 1))
        c, s = block.cos.double()[:, None], block.sin.double()[:, None]
        turned = []
        for t, gain in ((q, p["q_gain"]), (k, p["k_gain"])):
            u = t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain
            a, b = u.chunk(2, -1)
            turned.append(torch.cat([a * c - b * s, b * c + a * s], -1).transpose(0, 1))
        scores = turned[0] @ turned[1].transpose(1, 2) / math.sqrt(d // 2)
        scores = scores.masked_fill(torch.ones(T, T, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        rows = (scores.softmax(-1) @ v.transpose(0, 1)).transpose(0, 1).reshape(T, d)
        h = rows @ p["out"].t() + p["out_bias"] + X
        z = h @ p["up"].t() + p["up_bias"]
        y = (z * (1 + torch.erf(z / math.sqrt(2))) / 2) @ p["down"].t() + p["down_bias"] + h
        y.backward(dy[i].double())
        for name in block.places:
            want, got = p[name].grad, block.view([grads[i]], name)[0].double()
            error, size = (got - want).square().mean().sqrt(), want.square().mean().sqrt()
            assert error <= 2.0 ** -4 * size, (name, float(error / size))
