"""Trains a stack of residual FFN blocks and serves it token by token: norms before and after every block with a gate for every
channel, the blocks' matrices stepped by Muon, their gains, gates and biases by AdamW, decoding through the sparse path.

    python examples/train_block.py [--layers 2] [--steps 100] [--tokens 2048] [--width 512] [--hidden 2048]
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
import paper_2609_31975_b200 as ffn  # noqa: E402

MATRICES, VECTORS = ("W_g", "W_up", "W_down"), ("b_g", "pre_gain", "post_gain", "gate")


def make_model(layers, width, hidden, dtype, gen, bias=-0.3):
    """A list of blocks (dicts of parameters) and the gain of the norm behind the last one."""
    normal = lambda *shape, std=1.0: torch.randn(shape, generator=gen, device=gen.device) * std  # noqa: E731
    blocks = []
    for _ in range(layers):
        block = {k: normal(hidden, width, std=width ** -0.5).to(dtype) for k in MATRICES}
        block.update(b_g=torch.full((hidden,), bias, device=gen.device), pre_gain=1 + normal(width, std=0.1), post_gain=1 + normal(width, std=0.1),
                     gate=0.5 + normal(width, std=0.1))
        blocks.append(block)
    return blocks, torch.ones(width, device=gen.device)


def forward(blocks, last_gain, x, act="relu"):
    """The output for x [T, D] (a norm of the last stream), and what the backward pass needs.  A block's norm after and the next one's norm
    before are one call."""
    h, n, stats = ffn.block_norm_forward(None, x, None, blocks[0]["pre_gain"])
    saved = [dict(h=h, n=n, stats=stats, y=None)]
    for i, b in enumerate(blocks):
        y, z, u = ffn.gated_ffn_forward(n, b["W_g"], b["b_g"], b["W_up"], b["W_down"], act)
        saved[-1].update(z=z, u=u)
        gain = blocks[i + 1]["pre_gain"] if i + 1 < len(blocks) else last_gain
        h, n, stats = ffn.block_norm_forward(y, h, b["post_gain"], gain, b["gate"], scale=1.0)
        saved.append(dict(h=h, n=n, stats=stats, y=y))
    return n, saved


def backward(blocks, last_gain, saved, dn, act="relu"):
    """Gradients of every parameter, as (list of dicts, of the last gain), from that of the output."""
    grads, dh, dlast = [dict() for _ in blocks], None, None
    for i in range(len(blocks), 0, -1):
        b, at, before = blocks[i - 1], saved[i], saved[i - 1]
        gain = blocks[i]["pre_gain"] if i < len(blocks) else last_gain
        g = ffn.block_norm_backward(dh, dn, at["y"], at["h"], at["stats"], b["post_gain"], gain, b["gate"], scale=1.0)
        if i < len(blocks):
            grads[i]["pre_gain"] = g["dpre_gain"]
        else:
            dlast = g["dpre_gain"]
        grads[i - 1].update(post_gain=g["dpost_gain"], gate=g["dgate"])
        dh = g["dresid"]
        f = ffn.gated_ffn_backward(g["dy"], before["n"], before["z"], before["u"], b["W_g"], b["W_up"], b["W_down"], act)
        grads[i - 1].update(W_g=f["dW_g"], W_up=f["dW_up"], W_down=f["dW_down"], b_g=f["db_g"])
        dn = f["dx"]
    first = saved[0]
    grads[0]["pre_gain"] = ffn.block_norm_backward(dh, dn, None, first["h"], first["stats"], None, blocks[0]["pre_gain"], need=("dpre_gain",))["dpre_gain"]
    return grads, dlast


def main(layers=2, steps=100, tokens=2048, width=512, hidden=2048, lr=0.02, seed=0, device="cuda:0", quiet=False):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    teacher, teacher_gain = make_model(layers, width, hidden, torch.bfloat16, gen)
    blocks, last_gain = make_model(layers, width, hidden, torch.bfloat16, gen)
    matrices = [b[k] for b in blocks for k in MATRICES]
    masters = [w.float() for w in matrices]                              # copies in 32 bits that take the steps
    vectors = [b[k] for b in blocks for k in VECTORS] + [last_gain]
    momenta, moments = [ffn.muon_state(w) for w in matrices], [ffn.adamw_state(v) for v in vectors]
    losses = []
    for step in range(1, steps + 1):
        x = torch.randn((tokens, width), generator=gen, device=device).bfloat16()
        want, _ = forward(teacher, teacher_gain, x, "silu")
        out, saved = forward(blocks, last_gain, x)
        error = out.float() - want.float()
        grads, dlast = backward(blocks, last_gain, saved, (error * (2.0 / error.numel())).bfloat16())
        of_matrices = [g[k] for g in grads for k in MATRICES]
        of_vectors = [g[k] for g in grads for k in VECTORS] + [dlast]
        norm = ffn.grad_norm(of_matrices + of_vectors)                   # stays on the device: clips both steps, or leaves them out
        rate = min(1.0, 10 * step / steps, 2 * (1 - (step - 1) / steps))
        ffn.muon_step(matrices, of_matrices, momenta, lr=lr * rate, weight_decay=0.01, masters=masters, grad_norm=norm, max_norm=1.0)
        ffn.adamw_step(vectors, of_vectors, moments, step, lr=0.1 * lr * rate, weight_decay=0.0, grad_norm=norm, max_norm=1.0)
        if step % max(1, steps // 10) == 0 or step == 1:
            losses.append((error.square().mean() / want.float().square().mean()).item())
            if not quiet:
                print(f"step {step:5d}: error {losses[-1]:.4f} of the teacher's energy, gradient norm {norm.item():.2e}")
    assert ffn.training_status(device) == 0
    # decode: one token at a time; the FFN's fp32 output goes onto the bf16 stream
    served = ffn.SparseFFN(width, hidden, torch.bfloat16, device=device)
    x = torch.randn((4, width), generator=gen, device=device).bfloat16()
    dense, _ = forward(blocks, last_gain, x)
    worst = 0.0
    for t in range(4):
        h, n, _ = ffn.block_norm_forward(None, x[t], None, blocks[0]["pre_gain"], save=False)
        for i, b in enumerate(blocks):
            y = served.sparse_ffn_forward(n, {"W_g": b["W_g"]}, b["b_g"], b["W_up"], b["W_down"], "relu")
            gain = blocks[i + 1]["pre_gain"] if i + 1 < layers else last_gain
            h, n, _ = ffn.block_norm_forward(y.view(-1), h, b["post_gain"], gain, b["gate"], scale=1.0, save=False)
        worst = max(worst, ((n.float() - dense[t].float()).norm() / dense[t].float().norm()).item())
    if not quiet:
        print(f"served: decoding within {worst:.1e} of the training forward pass")
    return losses, worst


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--width", type=int, default=512)
    p.add_argument("--hidden", type=int, default=2048)
    main(**vars(p.parse_args()))
