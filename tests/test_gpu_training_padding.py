"""What lies past the last column of z and u, between the rows of strided matrices, and in the workspace before a call, is not read into
any result: NaN there changes no bit.  Run with `-m gpu` on a B200."""
import ctypes

import pytest
import torch

from test_training_abi import Call, Grads

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
ACTS = [(0, 3), (1, 4), (2, 0), (4, 3), (4, 2)]   # relu, sqrelu with silu, rsplus with relu, silu, silu with rsplus


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    return m.load_library()


def p(t):
    return ctypes.c_void_p(t.data_ptr())


def rows(values, fill, gap):
    """The values as rows of a matrix whose other columns, to the next 16 bytes and `gap` beyond, are `fill`."""
    T, N = values.shape
    whole = torch.full((T, (N + 7) // 8 * 8 + gap), fill, dtype=values.dtype, device=DEV)
    whole[:, :N] = values
    return whole


def run(lib, fill, T, D, H, dtype, act, act_up, gap):
    g = torch.Generator(device=DEV)
    g.manual_seed(T + D + H)
    rnd = lambda r, c, std=1.0: (torch.randn(r, c, generator=g, device=DEV) * std).to(dtype)  # noqa: E731
    code = 1 if dtype == BF16 else 0
    W = [rnd(H, D, D ** -0.5) for _ in range(3)]
    bias = torch.randn(H, generator=g, device=DEV)
    x, dy, zin, uin = (rows(t, fill, gap) for t in (rnd(T, D), rnd(T, D), rnd(T, H), rnd(T, H)))
    y, dx = (rows(torch.zeros(T, D, dtype=dtype, device=DEV), 5.0, gap) for _ in range(2))
    z, u = (rows(torch.zeros(T, H, dtype=dtype, device=DEV), 5.0, gap) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    dW, db = [torch.zeros(H, D, dtype=dtype, device=DEV) for _ in range(3)], torch.zeros(H, device=DEV)
    need = ctypes.c_size_t(0)

    def workspace(backward):
        assert lib.sffn_train_workspace_bytes(T, D, H, code, backward, ctypes.byref(need)) == 0
        return torch.full((need.value,), 255 if fill != fill else 0, dtype=torch.uint8, device=DEV)   # bytes of NaN, in either type

    ws = workspace(0)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    c = Call(T, D, H, code, act, act_up, p(x), x.stride(0), p(W[0]), p(W[1]), p(W[2]), p(bias), p(z), p(u), z.stride(0), p(ws), need.value, p(status))
    assert lib.gated_ffn_forward(ctypes.byref(c), p(y), ctypes.c_int64(y.stride(0)), stream) == 0
    ws2 = workspace(1)
    c = Call(T, D, H, code, act, act_up, p(x), x.stride(0), p(W[0]), p(W[1]), p(W[2]), None, p(zin), p(uin), zin.stride(0), p(ws2), need.value, p(status))
    grads = Grads(p(dx), dx.stride(0), p(dW[0]), p(dW[1]), p(dW[2]), p(db))
    assert lib.gated_ffn_backward(ctypes.byref(c), p(dy), ctypes.c_int64(dy.stride(0)), ctypes.byref(grads), stream) == 0
    torch.cuda.synchronize()
    assert status.item() == 0
    for t, n in ((y, D), (dx, D), (z, H), (u, H)):
        assert (t[:, n:] == 5.0).all()
    return [y[:, :D], z[:, :H], u[:, :H], dx[:, :D], *dW, db]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D,H", [(1, 64, 7), (1, 256, 1023), (4, 72, 50), (5, 72, 50), (16, 64, 129), (17, 64, 129), (40, 136, 213), (65, 64, 257), (3, 1096, 2057),
                                   (300, 200, 1531), (300, 2048, 2045), (40, 2048, 4097), (700, 328, 901), (520, 1032, 4099), (257, 1024, 1025)])
def test_nan_where_nothing_is_read(lib, T, D, H, dtype):
    act, act_up = ACTS[(T + H) % len(ACTS)]
    for gap in (0, 8):
        clean = run(lib, 0.0, T, D, H, dtype, act, act_up, gap)
        dirty = run(lib, float("nan"), T, D, H, dtype, act, act_up, gap)
        assert all(torch.isfinite(t).all() for t in dirty)
        assert all(torch.equal(a, b) for a, b in zip(clean, dirty))
