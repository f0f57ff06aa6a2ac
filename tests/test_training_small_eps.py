"""An eps too small for moments in 8 bits is refused, before anything reaches a device."""
import ctypes

import pytest

from test_training_abi import A, Config, Step, lib  # noqa: F401


@pytest.mark.parametrize("eps", [0.0, 1e-30, 8.8e-16])
def test_refused(lib, eps):  # noqa: F811
    words = Step(p=A, g=A, m=A, v=A, n=8, p_dtype=1, g_dtype=1, state_bits=32, lr=1e-3, weight_decay=0.1)
    codes = Step(p=A, g=A, m=A, v=A, m_scale=A, v_scale=A, n=8, p_dtype=1, g_dtype=1, state_bits=8, lr=1e-3, weight_decay=0.1)
    config = Config(beta1=0.9, beta2=0.99, eps=eps, step=1)
    assert lib.sffn_adamw_step((Step * 2)(words, codes), 2, ctypes.byref(config), None) == 2
