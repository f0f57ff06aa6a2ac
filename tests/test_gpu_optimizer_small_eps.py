"""AdamW steps with an eps that does not hide the smallest second moments: zero, and up to 1e-8.  Run with `-m gpu` on a B200."""
import pytest
import torch

import training_reference as ref
from test_gpu_optimizer import HYPER, check, copied, tensors

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    return m


@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-25, 1e-20, 1e-15, 1e-12, 1e-8])
@pytest.mark.parametrize("step,betas", [(1, (0.9, 0.999)), (700, (0.9, 0.999)), (3, (0.0, 0.99999))])
@pytest.mark.parametrize("offset,g_dtype", [(0, F32), (1, F32), (0, BF16)])
def test_second_moments_down_to_the_smallest(lib, eps, step, betas, offset, g_dtype):
    """v between 2^-140 and 2^-90, where fp32's normal range ends.  Its roundings are within 4 units, below that range two halves of 2^-149, half of
    that relative to v in the root; the rest is a root, a quotient and a few products (32 units, as in the other tests).  The first
    moment stays in the normal range, and weights are zero, so that the step is all there is."""
    n, lr = 4099, 0.25
    g = torch.Generator(device=DEV)
    g.manual_seed(step + offset)
    exponent = torch.linspace(-140, -90, n, device=DEV).double()
    v = torch.zeros(n + offset, device=DEV)[offset:]
    v.copy_((2.0 ** exponent * (1 + torch.rand(n, generator=g, device=DEV).double())).float())
    grad = torch.zeros(n + offset, device=DEV, dtype=g_dtype)[offset:]
    grad.copy_((torch.randn(n, generator=g, device=DEV).double() * 2.0 ** (exponent / 2)).to(g_dtype))
    grad[::3] = 0
    m = torch.zeros(n + offset, device=DEV)[offset:]
    m.copy_((torch.randn(n, generator=g, device=DEV).double() * 2.0 ** (exponent / 2)).float())
    p = torch.zeros(n + offset, device=DEV)[offset:]
    want, m1, v1 = ref.adamw(p, grad, m, v, step, lr, betas, eps, 0.1)
    em = 8 * ref.U32 * (betas[0] * m.cpu().double().abs() + (1 - betas[0]) * grad.cpu().double().abs())
    ev = 4 * ref.U32 * v1 + 1.01 * 2.0 ** -149
    assert float((ev / v1).max()) < 2 ** -8
    lib.adamw_step([p], [grad], [dict(m=m, v=v)], step, lr=lr, betas=betas, eps=eps, weight_decay=0.1)
    torch.cuda.synchronize()
    root = (v1 / (1 - betas[1] ** step)).sqrt()
    eroot = root * (0.55 * ev / v1)
    part = lr / (1 - betas[0] ** step)
    bound = 1.02 * (part * em / (root + eps) + want.abs() * (eroot / (root + eps) + 32 * ref.U32)) + 1e-44
    off = (p.cpu().double() - want).abs()
    assert torch.isfinite(p).all()
    assert (off <= bound).all(), (float((off / bound).max()), int((off > bound).sum()))


def test_an_entry_of_zeros_without_eps(lib):
    """0 / 0, as in the formula; with any eps nothing moves."""
    for eps, moved in ((0.0, True), (1e-40, False), (1e-8, False)):
        p, zero = torch.ones(300, device=DEV), torch.zeros(300, device=DEV)
        lib.adamw_step([p], [zero], [lib.adamw_state(p)], 1, lr=0.1, eps=eps, weight_decay=0.0)
        assert torch.isnan(p).all() if moved else (p == 1).all(), eps


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype,g_dtype,master", [(F32, F32, False), (F32, BF16, False), (BF16, BF16, False), (BF16, F32, False), (BF16, BF16, True)],
                         ids=["f32", "f32_gbf16", "bf16", "bf16_gf32", "master"])
def test_every_kind_of_storage(lib, bits, p_dtype, g_dtype, master):
    """An eps of 1e-14 takes other roots than one of 1e-8: the step against its formula, and moments that do not depend on eps."""
    hyper = dict(HYPER, eps=1e-14)
    rows = [tensors(lib, n, p_dtype, g_dtype, bits, master, offset, n, zero_groups=n % 2 == 0) for n in (1, 255, 512, 4099, 70000) for offset in (0, 1, 8)]
    before = [(p.clone(), g.clone(), copied(s), None if w is None else w.clone()) for p, g, s, w in rows]
    twin = [(p.clone(), copied(s), None if w is None else w.clone()) for p, g, s, w in rows]
    ps, gs, ss, ws = (list(c) for c in zip(*rows))
    lib.adamw_step(ps, gs, ss, 3, masters=ws, **hyper)
    lib.adamw_step([p for p, _, _ in twin], gs, [s for _, s, _ in twin], 3, masters=[w for *_, w in twin], **HYPER)
    torch.cuda.synchronize()
    for i, b in enumerate(before):
        check(b, (ps[i], ss[i], ws[i]), 3, 1.0, (i, bits), hyper)
        assert all(torch.equal(ss[i][k], twin[i][1][k]) for k in ss[i]), i


def test_refused(lib):
    p = torch.ones(300, device=DEV)
    for eps in (0.0, 8e-16):
        with pytest.raises(lib.SFFNError) as err:
            lib.adamw_step([p, p.clone()], [p, p], [lib.adamw_state(p), lib.adamw_state(p, 8)], 1, lr=0.1, eps=eps)
        assert err.value.code == 2
    assert (p == 1).all()
