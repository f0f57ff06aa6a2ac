"""How exact the products of the Newton-Schulz steps are: 16 bits against a model of operands of eleven bits, 32 bits where U has a null space or sums
are of one sign.  Run with `-m gpu` on a B200."""
import pytest
import torch

import muon_products as model
import muon_reference as ref
from test_gpu_muon import BF16, DEV, F32, gen, lib, normal  # noqa: F401

pytestmark = pytest.mark.gpu
SHAPES = [(64, 300), (129, 128), (256, 256), (257, 300), (1024, 256), (513, 520), (1000, 640), (640, 1000), (767, 2050), (1300, 1290), (2048, 1024), (4096, 700),
          (3000, 2100), (700, 4096), (4096, 4096)]


def off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_16_bits(lib, shape, dtype):  # noqa: F811
    u = normal(shape, gen(shape[0]), 1e-2, dtype)
    want = ref.orthogonal(u)
    assert off(lib.orthogonalize(u, bits=16), want) <= model.room16(u, want, dtype)


@pytest.mark.parametrize("shape,n", [((256, 64), 7), ((600, 256), 20), ((1024, 512), 6)], ids=str)
def test_16_bits_of_batches(lib, shape, n):  # noqa: F811
    us = [normal(shape, gen(i), 1e-3 * (i + 1)) for i in range(n)]
    for u, o in zip(us, lib.orthogonalize(us, bits=16)):
        want = ref.orthogonal(u)
        assert off(o, want) <= model.room16(u, want, F32)


def test_16_bits_of_a_step(lib):  # noqa: F811
    """fp32 parameters of zero: what the step leaves is O."""
    for shape in ((1024, 256), (767, 2050)):
        u = normal(shape, gen(1), 1e-3)
        p = torch.zeros(shape, device=DEV)
        lib.muon_step([p], [u], [lib.muon_state(p)], lr=1.0, momentum=0.0, weight_decay=0.0, scale=1.0, bits=16)
        want = ref.orthogonal(u)
        assert off(-p, want) <= model.room16(u, want, F32)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_32_bits_of_full_rank(lib, shape):  # noqa: F811
    """What the header says: within 2e-5 in five steps; and bf16 matrices no further off than their own rounding and that."""
    u = normal(shape, gen(shape[1]), 1e-2)
    want = ref.orthogonal(u)
    assert off(lib.orthogonalize(u), want) <= min(2e-5, model.room32(want.norm().item(), 5))
    b = u.bfloat16()
    want = ref.orthogonal(b)
    assert off(lib.orthogonalize(b, bits=32), want) <= off(want.bfloat16(), want) + 2e-5


def low_rank(shape, rank, heavy, seed):
    g = gen(seed)
    left, right = normal((shape[0], rank), g), normal((rank, shape[1]), g)
    return (left * torch.exp(heavy * normal((shape[0], 1), g))) @ right


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("shape", [(4, 19), (33, 70), (600, 300), (1145, 1914), (2230, 2876), (2876, 2230)], ids=str)
def test_32_bits_of_low_rank(lib, shape, steps):  # noqa: F811
    """Ranks of one and two, rows as large as one another and far apart."""
    for rank in (1, 2):
        for heavy in (0.0, 1.0, 2.0, 3.0):
            u = low_rank(shape, rank, heavy, 8 * rank + int(heavy))
            want = ref.orthogonal(u, steps=steps)
            assert off(lib.orthogonalize(u, steps=steps, bits=32), want) <= model.room32(want.norm().item(), steps), (rank, heavy)


@pytest.mark.parametrize("steps", [1, 2, 5, 6])
@pytest.mark.parametrize("shape", [(33, 70), (238, 4), (601, 1976), (1311, 823), (5000, 400), (400, 20000)], ids=str)
def test_32_bits_of_one_sign(lib, shape, steps):  # noqa: F811
    """Sums that only grow: what the accumulators truncate has one sign too."""
    for u in (normal(shape, gen(1)).abs(), torch.ones(shape, device=DEV), low_rank(shape, 1, 2.0, 3).abs(), 1 + 0.1 * normal(shape, gen(2))):
        want = ref.orthogonal(u, steps=steps)
        assert off(lib.orthogonalize(u, steps=steps, bits=32), want) <= model.room32(want.norm().item(), steps)
