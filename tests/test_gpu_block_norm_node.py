"""The graph node of the norms around a block takes inputs as they lie: parts of something longer, entries apart, one row for all.  Run with
`-m gpu` on a B200."""
import pytest
import torch

from test_gpu_block_norm import BF16, DEV, F32, gen, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu
B, T, D = 3, 7, 64
NAMES = ("y", "resid", "post_gain", "pre_gain", "gate")


def shifted(t):
    """The same values, one entry past an aligned address."""
    room = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
    out = room[1:].view(t.shape)
    out.copy_(t)
    assert out.data_ptr() % 16
    return out


def apart(t):
    """The same values, two entries apart."""
    room = torch.empty((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype, device=DEV)
    out = room[..., ::2]
    out.copy_(t)
    return out


def off(t):
    """The same values in rows that are one entry longer, so that most of them start off 16 bytes."""
    room = torch.empty((*t.shape[:-1], t.shape[-1] + 1), dtype=t.dtype, device=DEV)
    out = room[..., :-1]
    out.copy_(t)
    return out


def swapped(t):
    """The same values, the first two dimensions the other way round in memory."""
    return t.transpose(0, 1).contiguous().transpose(0, 1) if t.dim() == 3 else t


@pytest.mark.parametrize("gate", ["channel", "token", "full"])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("lay", [shifted, apart, off, swapped])
def test_as_they_lie(lib, lay, types, gate):  # noqa: F811
    g = gen(3)
    c = dict(y=rand((B, T, D), types[0], g), resid=rand((B, T, D), types[1], g), post_gain=rand((D,), F32, g), pre_gain=rand((D,), F32, g),
             gate=rand({"channel": (D,), "token": (B, T, 1), "full": (B, T, D)}[gate], types[1] if gate == "full" else F32, g))
    a, b = rand((B, T, D), types[1], g), rand((B, T, D), types[1], g)

    def run(values, a, b):
        leaves = [v.requires_grad_() for v in values]
        h, n = lib.BlockNormFunction.apply(*leaves, 0.7, 1e-5)
        return [h, n, *torch.autograd.grad([h, n], leaves, [a, b])]

    want = run([c[k].clone() for k in NAMES], a, b)
    got = run([lay(c[k]) for k in NAMES], lay(a), lay(b))
    for w, o in zip(want, got):
        assert w.shape == o.shape and torch.equal(w, o)
    for k in range(5):  # one at a time
        got = run([lay(c[n]) if i == k else c[n].clone() for i, n in enumerate(NAMES)], a, b)
        assert all(torch.equal(w, o) for w, o in zip(want, got)), NAMES[k]


def test_one_row_for_all(lib):  # noqa: F811
    """Expanded inputs, and gradients that come expanded, as those of a sum do."""
    g = gen(4)
    y, x, gain = rand((1, 1, D), F32, g), rand((B, T, D), F32, g), rand((D,), F32, g)
    full = rand((1, 1, D), F32, g).expand(B, T, D)

    def run(y, full):
        leaves = [t.requires_grad_() for t in (y, x.clone(), gain.clone(), gain.clone(), full)]
        h, n = lib.BlockNormFunction.apply(*leaves)
        return [h, n, *torch.autograd.grad(h.sum() + n.sum(), leaves)]

    for w, o in zip(run(y.expand(B, T, D).contiguous(), full.contiguous()), run(y.expand(B, T, D).detach(), full.detach())):
        assert torch.equal(w, o)


def test_only_a_norm_of_what_lies_apart(lib):  # noqa: F811
    """Without y, h is a tensor of its own, also where resid had to be copied to be read."""
    x, gain = rand((T, D), F32, gen(5)), rand((D,), F32, gen(6))
    want = lib.BlockNormFunction.apply(None, x, None, gain)
    for lay in (shifted, apart, off, torch.clone):
        r = lay(x)
        h, n = lib.BlockNormFunction.apply(None, r, None, gain)
        assert torch.equal(h, x) and torch.equal(n, want[1]) and h.data_ptr() != r.data_ptr()
        h.zero_()
        assert torch.equal(r, x)


def test_what_it_takes_is_not_copied(lib):  # noqa: F811
    """Rows at a stride of 16 bytes go in as they are: what is saved is the caller's memory, and a change of it is noticed."""
    room = rand((T, D + 8), BF16, gen(7))
    y, x, gain = room[:, :D].requires_grad_(), rand((T, D), BF16, gen(8)), rand((D,), F32, gen(9))
    h, _ = lib.BlockNormFunction.apply(y, x, gain, gain)
    with torch.no_grad():
        y.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        h.float().sum().backward()
