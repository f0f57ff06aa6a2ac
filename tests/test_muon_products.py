"""The model that the 16-bit products are held against, on the CPU: it is the formula where nothing is rounded, and the room that it leaves for eleven bits
is too small for ten, and for bf16."""
import pytest
import torch

import muon_products as model
import muon_reference as ref


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def test_without_roundings_it_is_the_formula():
    for shape in ((60, 90), (90, 60)):
        u, want = normal(shape, 1), ref.orthogonal(normal(shape, 1))
        for company in (1, 2):
            assert (model.modelled(u, 50, company=company) - want).norm() < 1e-10 * want.norm()
    x = torch.tensor([1.0, 1 + 2.0 ** -11, 1 + 2.0 ** -10, -3.0, 1e-30, 0.0], dtype=torch.float64)
    assert torch.equal(model.rounded(x, model.FP16)[:4], x.half().double()[:4]) and torch.equal(model.rounded(x, model.BF16), x.bfloat16().double())


@pytest.mark.parametrize("shape", [(64, 300), (129, 128), (256, 256), (1024, 256), (513, 520), (640, 1000)], ids=str)
def test_fewer_bits_do_not_fit(shape):
    u = normal(shape, 1)
    want = ref.orthogonal(u)
    off = lambda bits, company, v=u, w=want: ((model.modelled(v, bits, company=company) - w).norm() / w.norm()).item()  # noqa: E731
    limit = model.room16(u, want, torch.float32)
    ten = [off(model.FP16 - 1, n) for n in (1, 2)]
    assert max(ten) > 1.4 * limit and ten[0] > 1.1 * limit                       # (small matrices take their steps one at a time)
    bf16 = [off(model.BF16, n) for n in (1, 2)]
    assert min(bf16) > 2.5 * limit and min(bf16) > model.room16(u, want, torch.bfloat16)
    v = normal(shape, 2)  # another draw fits the room of this one
    assert max(off(model.FP16, n, v, ref.orthogonal(v)) for n in (1, 2)) < limit
