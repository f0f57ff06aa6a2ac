"""The example that trains an FFN and serves it, at a small size, against the same training in plain torch with autograd in fp32.

Both see the same tokens, so their losses differ by the rounding of gradients to bf16 and of moments to 8 bits, which is noise of
relative size 2^-8 (2^-7) on steps that change the loss by a third in all: 2 % of a loss is several times that."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def plain_training(steps, tokens, width, hidden, bias=-0.5, lr=5e-4, seed=0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    normal = lambda *shape, std=1.0: torch.randn(shape, generator=gen, device=DEV) * std  # noqa: E731
    teacher = [normal(hidden, width, std=width ** -0.5).bfloat16().float() for _ in range(3)]
    masters = [w.clone() for w in teacher] + [torch.full((hidden,), bias, device=DEV)]
    m, v = ([torch.zeros_like(w) for w in masters] for _ in range(2))
    losses = []
    for step in range(1, steps + 1):
        x = normal(tokens, width).bfloat16().float()
        w = [(t.bfloat16().float() if t.dim() == 2 else t.clone()).requires_grad_() for t in masters]
        want = (torch.nn.functional.silu(x @ teacher[0].T) * (x @ teacher[1].T)) @ teacher[2]
        error = (torch.relu(x @ w[0].T + w[3]) * (x @ w[1].T)) @ w[2] - want
        loss = error.square().mean()
        grads = torch.autograd.grad(loss, w)
        clip = min(1.0, 1.0 / (sum(float(g.square().sum()) for g in grads) ** 0.5 + 1e-6))
        rate = lr * min(1.0, 10 * step / steps, 2 * (1 - (step - 1) / steps))
        for i, g in enumerate(grads):
            g = g * clip
            m[i] = 0.9 * m[i] + 0.1 * g
            v[i] = 0.999 * v[i] + 0.001 * g * g
            part = (m[i] / (1 - 0.9 ** step)) / ((v[i] / (1 - 0.999 ** step)).sqrt() + 1e-8)
            masters[i] = masters[i] * (1 - rate * (0.01 if i < 3 else 0.0)) - rate * part
        if step % max(1, steps // 10) == 0 or step == 1:
            losses.append((loss / want.square().mean()).item())
    return losses


@pytest.mark.parametrize("bits", [8, 32])
def test_training_and_serving(bits):
    path = Path(__file__).resolve().parent.parent / "examples" / "train_ffn.py"
    spec = importlib.util.spec_from_file_location("train_ffn", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, fired, worst = example.main(steps=60, bits=bits, tokens=1024, width=256, hidden=1024, quiet=True)
    want = plain_training(60, 1024, 256, 1024)
    assert want[-1] < want[0] and len(losses) == len(want)
    assert all(abs(a - b) <= 0.02 * b for a, b in zip(losses, want)), (losses, want)
    assert 0 < fired < 1
    assert worst < 2 ** -7           # bf16's rounding of h and of y, 2^-8 each at most
