"""Training calls whose outputs lie over inputs, where they may, and whose matrices are columns of one.  Run with `-m gpu` on a B200."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = [(3, 64, 40), (5, 128, 128), (40, 128, 128), (300, 520, 520), (700, 1024, 1024)]
DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    yield m
    assert m.training_status(DEV) == 0


def make(T, D, H, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(T + D)
    rnd = lambda r, c, std=1.0: (torch.randn(r, c, generator=g, device=DEV) * std).to(dtype)  # noqa: E731
    return rnd(T, D), [rnd(H, D, D ** -0.5) for _ in range(3)], torch.randn(H, generator=g, device=DEV), rnd(T, D)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D,H", SHAPES)
def test_dx_over_what_it_may_lie_over_and_y_over_x(lib, T, D, H, dtype):
    x, W, b_g, dy = make(T, D, H, dtype)
    y, z, u = lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2], "sqrelu", "silu")
    want = lib.gated_ffn_backward(dy, x, z, u, *W, "sqrelu", "silu")
    for name in ("dy", "x", "z", "u")[:4 if D == H else 2]:
        a = dict(dy=dy.clone(), x=x.clone(), z=z.clone(), u=u.clone())
        got = lib.gated_ffn_backward(*a.values(), *W, "sqrelu", "silu", out=dict(dx=a[name]))
        assert got["dx"] is a[name] or got["dx"].data_ptr() == a[name].data_ptr()
        assert all(torch.equal(got[k], want[k]) for k in want), name
    whole = torch.cat([dy.clone(), dy[:1]])                                     # and over it in part, a row further on
    whole[:T] = dy
    got = lib.gated_ffn_backward(whole[:T], x, z, u, *W, "sqrelu", "silu", out=dict(dx=whole[1:]))
    assert all(torch.equal(got[k], want[k]) for k in want)
    own = x.clone()
    y1, z1, u1 = lib.gated_ffn_forward(own, W[0], b_g, W[1], W[2], "sqrelu", "silu", y=own)
    assert torch.equal(own, y) and torch.equal(z1, z) and torch.equal(u1, u)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_matrices_that_are_columns_of_one(lib, dtype):
    """z beside u, x beside y: rows of one stride that lie between each other's."""
    T, D, H = 70, 64, 40
    x, W, b_g, dy = make(T, D, H, dtype)
    want = lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2])
    grads = lib.gated_ffn_backward(dy, x, want[1], want[2], *W)
    zu, xy = torch.zeros(T, 2 * H, dtype=dtype, device=DEV), torch.zeros(T, 3 * D, dtype=dtype, device=DEV)
    xy[:, :D] = x
    got = lib.gated_ffn_forward(xy[:, :D], W[0], b_g, W[1], W[2], y=xy[:, D:2 * D], z=zu[:, :H], u=zu[:, H:])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(xy[:, :D], x)
    more = lib.gated_ffn_backward(dy, xy[:, :D], zu[:, :H], zu[:, H:], *W, out=dict(dx=xy[:, 2 * D:]))
    assert all(torch.equal(more[k], grads[k]) for k in grads)
    rows = torch.zeros(2 * T, D, dtype=dtype, device=DEV)                        # every other row
    rows[::2] = x
    assert torch.equal(lib.gated_ffn_forward(rows[::2], W[0], b_g, W[1], W[2], y=rows[1::2])[0], want[0])


def test_refused(lib):
    x, W, b_g, dy = make(16, 64, 64, torch.bfloat16)
    y, z, u = lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2])
    for call in (lambda: lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2], z=x), lambda: lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2], z=z, u=z),
                 lambda: lib.gated_ffn_backward(dy, x, z, u, *W, out=dict(dW_g=W[0])), lambda: lib.gated_ffn_backward(dy, x, z, u, *W, out=dict(dW_g=W[1], dW_up=W[1]))):
        with pytest.raises(lib.SFFNError) as err:
            call()
        assert err.value.code == 1
