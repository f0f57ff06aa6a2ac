"""CPU-side check of the Python side of the norms around a block: what reaches the compiled calls."""
import pytest
import torch

from paper_2609_31975_b200 import block


class Recorded:
    def __init__(self):
        self.need = None

    def block_backward(self, dh, dn, y, h, stats, post_gain, pre_gain, gate, scale, need, out):
        self.need = need
        return (0, *[torch.zeros(1) if need >> i & 1 else None for i in range(5)])


@pytest.mark.parametrize("kind", [tuple, list, set, iter, dict.fromkeys, lambda names: (n for n in names)])
def test_need_in_any_form(monkeypatch, kind):
    """Gradients asked for by a list, a set or an iterator, which can be gone through once."""
    calls = Recorded()
    monkeypatch.setattr(block, "_calls", lambda: calls)
    t = torch.zeros(2, 8)
    for names in (("dresid",), ("dy", "dpre_gain"), block.BLOCK_GRADS, ()):
        got = block.block_norm_backward(t, t, t, t, torch.zeros(2, 2), need=kind(names))
        assert calls.need == sum(1 << block.BLOCK_GRADS.index(n) for n in names) and set(got) == set(names)
    one = block.block_norm_backward(t[0], t[0], t[0], t[0], torch.zeros(2, 1), need=kind(("dpost_gain", "dgate")))
    assert set(one) == {"dpost_gain", "dgate"}
    with pytest.raises(ValueError):
        block.block_norm_backward(t, t, t, t, None, need=kind(("dy", "dx")))
