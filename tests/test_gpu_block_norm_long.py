"""The norms' backward pass where a CTA meets more rows than it holds statistics of, and wide rows, which lie in no ring, where a CTA meets more
than one.  Run with `-m gpu` on a B200."""
import pytest
import torch

from test_gpu_block_norm import BF16, DEV, F32, TYPES, both, gen, inputs, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu
MIXED = (BF16, F32, BF16)


@pytest.mark.parametrize("types", [TYPES[1], MIXED], ids=["bf16", "mixed"])
@pytest.mark.parametrize("D", [64, 264, 520, 1032, 2056])
def test_more_rows_than_statistics_at_once(lib, D, types):  # noqa: F811
    """A row's warps hold statistics of as many rows as they have threads: 512 threads an SM, 75776 rows on 148 SMs."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    T = 512 * sms + 4321
    both(lib, T, D, types, "token", True, True, seed=D)
    if D == 264:
        both(lib, T, D, types, "channel", True, True, seed=D)


def test_more_wide_rows_than_statistics_at_once(lib):  # noqa: F811
    """The same of 1024 threads a row.  Rows have nothing to do with one another: each is as in a call with few of them, bit by bit."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    T, D = 1024 * sms + 99, 8200
    g = gen(1)
    few = 500
    base = {k: rand((few, D), BF16, g) for k in ("y", "h", "dh", "dn")}
    order = torch.randint(0, few, (T,), generator=g, device=DEV)
    order[:few] = torch.arange(few, device=DEV)
    gains = [1 + rand((D,), F32, g, 0.3) for _ in range(2)]
    stats, token = rand((2, few), F32, g).abs(), rand((few, 1), F32, g)
    need = ("dy", "dresid", "dgate")
    one = lib.block_norm_backward(base["dh"], base["dn"], base["y"], base["h"], stats, *gains, token, need=need)
    big = {k: t[order] for k, t in base.items()}
    got = lib.block_norm_backward(big["dh"], big["dn"], big["y"], big["h"], stats[:, order].contiguous(), *gains, token[order].contiguous(), need=need,
                                  out=dict(dresid=big["dh"], dy=torch.empty_like(big["y"])))
    for k in need:
        for i in range(0, T, 20000):
            assert torch.equal(got[k][i:i + 20000], one[k][order[i:i + 20000]]), (k, i)


@pytest.mark.parametrize("gate", ["channel", "token", "full"])
@pytest.mark.parametrize("types", [TYPES[0], TYPES[1], MIXED], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("D", [8200, 16392, 32768])
def test_many_wide_rows(lib, D, types, gate):  # noqa: F811
    T = 400
    both(lib, T, D, types, gate, True, True, seed=D)
    c, dh, dn = inputs(T, D, types, gate, True, True, seed=D)
    h, n, stats = lib.block_norm_forward(**c, n_dtype=types[2])
    args = (dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], c["gate"])
    want = lib.block_norm_backward(dh, *args)
    again = lib.block_norm_backward(dh, *args)
    over = dh.clone()
    got = lib.block_norm_backward(over, *args, out=dict(dresid=over))
    assert got["dresid"].data_ptr() == over.data_ptr()
    for k in want:
        assert torch.equal(want[k], got[k]) and torch.equal(want[k], again[k]), k


@pytest.mark.parametrize("post,pre", [(True, False), (False, True)])
def test_parts_of_many_wide_rows(lib, post, pre):  # noqa: F811
    for D in (8200, 16392):
        both(lib, 400, D, TYPES[1], "none", post, pre, seed=D)
        both(lib, 400, D, TYPES[0], "token", post, pre, seed=D)
