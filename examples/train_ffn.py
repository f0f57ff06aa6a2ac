"""Casts a dense gated FFN to a sparse one and serves it: a SiLU-gated teacher's weights get the activation RELU (and a gate
bias), are trained to give the teacher's outputs again (forward and backward pass, norm of the gradients, AdamW with clipping), and
then run through the sparse decode path as they are.

    python examples/train_ffn.py [--steps 200] [--bits 8] [--tokens 4096] [--width 1024] [--hidden 4096]
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
import paper_2609_31975_b200 as ffn  # noqa: E402


def main(steps=200, bits=8, tokens=4096, width=1024, hidden=4096, bias=-0.5, lr=5e-4, seed=0, device="cuda:0", quiet=False):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    normal = lambda *shape, std=1.0: torch.randn(shape, generator=gen, device=device) * std  # noqa: E731
    teacher = [normal(hidden, width, std=width ** -0.5).bfloat16() for _ in range(3)]
    # bf16 weights with copies in 32 bits that take the steps; the gate bias is in 32 bits itself
    params = [w.clone() for w in teacher] + [torch.full((hidden,), bias, device=device)]
    masters = [w.float() for w in params[:3]] + [None]
    states = [ffn.adamw_state(p, bits) for p in params]
    losses = []
    for step in range(1, steps + 1):
        x = normal(tokens, width).bfloat16()
        want, _, _ = ffn.gated_ffn_forward(x, teacher[0], None, teacher[1], teacher[2], "silu", save=False)
        y, z, u = ffn.gated_ffn_forward(x, params[0], params[3], params[1], params[2], "relu")
        error = y.float() - want.float()
        dy = (error * (2.0 / error.numel())).bfloat16()
        g = ffn.gated_ffn_backward(dy, x, z, u, params[0], params[1], params[2], "relu", need=("dW_g", "dW_up", "dW_down", "db_g"))
        grads = [g["dW_g"], g["dW_up"], g["dW_down"], g["db_g"]]
        norm = ffn.grad_norm(grads)                          # stays on the device: clips the step, or leaves it out
        ffn.adamw_step(params, grads, states, step, lr=lr * min(1.0, 10 * step / steps, 2 * (1 - (step - 1) / steps)),
                       weight_decay=[0.01, 0.01, 0.01, 0.0], masters=masters, grad_norm=norm, max_norm=1.0)
        if step % max(1, steps // 10) == 0 or step == 1:
            losses.append((error.square().mean() / want.float().square().mean()).item())
            if not quiet:
                print(f"step {step:5d}: error {losses[-1]:.4f} of the teacher's energy, gradient norm {norm.item():.2e}")
    assert ffn.training_status(device) == 0
    # decode: one token at a time through the sparse path, which reads the rows of the neurons that fire
    served = ffn.SparseFFN(width, hidden, torch.bfloat16, device=device)
    x = normal(8, width).bfloat16()
    dense, z, _ = ffn.gated_ffn_forward(x, params[0], params[3], params[1], params[2], "relu")
    worst = 0.0
    for t in range(8):
        out = served.sparse_ffn_forward(x[t], {"W_g": params[0]}, params[3], params[1], params[2], "relu")
        worst = max(worst, ((out - dense[t].float()).norm() / dense[t].float().norm()).item())
    fired = (z > 0).float().mean().item()
    if not quiet:
        print(f"served: {100 * fired:.1f} % of the neurons fire; sparse decode within {worst:.1e} of the training forward pass")
    return losses, fired, worst


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--bits", type=int, choices=(8, 32), default=8, help="of the moments")
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--width", type=int, default=1024)
    p.add_argument("--hidden", type=int, default=4096)
    main(**vars(p.parse_args()))
