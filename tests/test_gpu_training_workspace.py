"""Training calls stay within the workspace that they ask for: what lies behind it keeps its marker, at sizes whose tiles are cut into many
and into few pieces, whole or short of rows.  Run with `-m gpu` on a B200."""
import ctypes

import pytest
import torch

from test_training_abi import Call, Grads

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = [(1, 64, 40), (5, 256, 1024), (33, 128, 4096), (64, 256, 1024), (100, 1024, 300), (130, 512, 2048), (255, 512, 1000), (256, 512, 1000), (257, 512, 1000), (300, 2048, 2045),
          (520, 1032, 4099), (1100, 1024, 2600), (40, 2048, 4097), (1000, 4096, 1024)]


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    return m.load_library()


@pytest.mark.parametrize("code,dtype", [(0, torch.float32), (1, torch.bfloat16)], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D,H", SHAPES)
def test_nothing_behind_the_workspace_is_written(lib, T, D, H, code, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(T + H)
    rnd = lambda r, c, std=1.0: (torch.randn(r, c, generator=g, device=DEV) * std).to(dtype)  # noqa: E731
    ld = (H + 7) // 8 * 8
    x, dy, z, u, W = rnd(T, D), rnd(T, D), rnd(T, ld), rnd(T, ld), [rnd(H, D, D ** -0.5) for _ in range(3)]
    y, dx, dW, db = torch.empty_like(x), torch.empty_like(x), [torch.empty_like(w) for w in W], torch.empty(H, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    for backward in (0, 1):
        need = ctypes.c_size_t(0)
        assert lib.sffn_train_workspace_bytes(T, D, H, code, backward, ctypes.byref(need)) == 0
        ws = torch.full((need.value + (96 << 20),), 0xa5, dtype=torch.uint8, device=DEV)
        c = Call(T, D, H, code, 1, 4, p(x), D, p(W[0]), p(W[1]), p(W[2]), None, p(z), p(u), ld, p(ws), need.value, p(status))
        if backward:
            grads = Grads(p(dx), D, p(dW[0]), p(dW[1]), p(dW[2]), p(db))
            assert lib.gated_ffn_backward(ctypes.byref(c), p(dy), ctypes.c_int64(D), ctypes.byref(grads), stream) == 0
        else:
            assert lib.gated_ffn_forward(ctypes.byref(c), p(y), ctypes.c_int64(D), stream) == 0
        torch.cuda.synchronize()
        assert (ws[need.value:] == 0xa5).all()
    assert status.item() == 0
