"""The example that trains a stack of residual blocks: its gradients against autograd in 64 bits, that it runs, and that what it serves is
what it trained."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def example():
    path = Path(__file__).resolve().parent.parent / "examples" / "train_block.py"
    spec = importlib.util.spec_from_file_location("train_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(blocks, last_gain, x, act):
    norm = lambda v, g: v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt() * g  # noqa: E731
    h, n = x, norm(x, blocks[0]["pre_gain"])
    for i, b in enumerate(blocks):
        z, u = n @ b["W_g"].T + b["b_g"], n @ b["W_up"].T
        y = ((torch.relu(z) if act == "relu" else torch.nn.functional.silu(z)) * u) @ b["W_down"]
        h = h + b["gate"] * norm(y, b["post_gain"])
        n = norm(h, blocks[i + 1]["pre_gain"] if i + 1 < len(blocks) else last_gain)
    return n


@pytest.mark.parametrize("dtype,room", [
    # fp32: products within 1e-6 of their terms' size, some ten of them one after another; a neuron's gate changes sides for |z| below 1e-6
    (torch.float32, 1e-4),
    # bf16: n, h, y, z, u, h of the neurons and as many gradients are rounded by 2^-8 at most, in each of two blocks: 24 roundings
    (torch.bfloat16, 24 * 2.0 ** -8)])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_gradients(example, dtype, room, act):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    blocks, last = example.make_model(2, 128, 320, dtype, gen)
    x = torch.randn((200, 128), generator=gen, device=DEV).to(dtype)
    up = (torch.randn((200, 128), generator=gen, device=DEV) / 200).to(dtype)
    out, saved = example.forward(blocks, last, x, act)
    grads, dlast = example.backward(blocks, last, saved, up, act)
    leaves = [{k: v.double().requires_grad_() for k, v in b.items()} for b in blocks]
    last64 = last.double().requires_grad_()
    want = plain(leaves, last64, x.double(), act)
    assert (out.double() - want).norm() <= room * want.norm()
    (want * up.double()).sum().backward()
    for got, leaf in zip(grads, leaves):
        assert got.keys() == leaf.keys()
        for k in leaf:
            assert (got[k].double() - leaf[k].grad).norm() <= room * leaf[k].grad.norm(), (k, act)
    assert (dlast.double() - last64.grad).norm() <= room * last64.grad.norm()


def test_runs_and_serves(example):
    """Decoding takes the sparse path, whose y is fp32 where training rounds it: n, h and y of two blocks, 2^-8 each."""
    losses, worst = example.main(steps=5, tokens=300, width=128, hidden=512, quiet=True)
    assert len(losses) >= 5 and all(torch.isfinite(torch.tensor(losses)))
    assert worst < 8 * 2.0 ** -8
