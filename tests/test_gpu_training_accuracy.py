"""Errors of the training calls on the tensor cores, norm by norm: fp32 storage keeps fp32's accuracy, and bf16 storage that of its sums in
fp32.  Run with `-m gpu` on a B200."""
import pytest
import torch

import training_reference as ref
import training_terms as tt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    yield m
    assert m.training_status(DEV) == 0


@pytest.mark.parametrize("act,act_up", tt.ACTS)
@pytest.mark.parametrize("T,D,H", tt.SHAPES)
def test_fp32_on_the_tensor_cores(lib, T, D, H, act, act_up):
    t = tt.make(T, D, H, DEV)
    w = [t[k] for k in tt.FORWARD]
    got = dict(zip(("y", "z", "u"), lib.gated_ffn_forward(*w, act, act_up)))
    want = ref.forward(*w, act, act_up)
    off = {k: tt.error(got[k], want[k]) for k in want}
    w = [t[k] for k in tt.BACKWARD]
    got = lib.gated_ffn_backward(*w, act, act_up)
    want = ref.backward(*w, act, act_up)
    off.update({k: tt.error(got[k], want[k]) for k in want})
    assert all(e <= tt.LIMIT for e in off.values()), off


@pytest.mark.parametrize("T,D,H", [(520, 4096, 1032), (300, 2048, 2045)])
def test_the_bias_gradient_of_bf16_tokens(lib, T, D, H):
    """Sums of products that keep fp32 up to the end: dh in runs of 768 k, each truncated by 5e-8 for 64 of them (6e-7 in all; one run of 4096
    would be 3e-6), its additions and dz's own rounding some units of 2^-24."""
    t = {k: v if k == "b_g" else v.bfloat16() for k, v in tt.make(T, D, H, DEV).items()}
    ld = (H + 7) // 8 * 8
    for k in ("z", "u"):
        rows = torch.zeros(T, ld, dtype=torch.bfloat16, device=DEV)[:, :H]
        rows.copy_(t[k])
        t[k] = rows
    w = [t[k] for k in tt.BACKWARD]
    got = lib.gated_ffn_backward(*w, "relu", None, need=["db_g"])
    e = tt.error(got["db_g"], ref.backward(*w, "relu", None)["db_g"])
    assert e <= tt.LIMIT
