"""The oracle's activations keep their digits far out, where 1 + tanh z and the like have none left in fp64."""
import decimal

import numpy as np
import pytest

from oracle import blocks as OB


@pytest.mark.parametrize("v", [-9.0, -7.1875, -6.8125, -3.0, -1e-3, 0.0, 2.0, 30.0])
def test_gelu_tanh_and_silu_against_long_decimals(v):
    with decimal.localcontext() as c:
        c.prec = 60
        D = decimal.Decimal
        pi = D("3.14159265358979323846264338327950288419716939937510582097494459")
        z = 2 * (2 / pi).sqrt() * (D(v) + D("0.044715") * D(v) ** 3)
        tanh = float(D(v) / (1 + (-z).exp()))
        silu = float(D(v) / (1 + (-D(v)).exp()))
    assert np.allclose(OB.activation([v], "gelu_tanh"), tanh, rtol=1e-13, atol=0)
    assert np.allclose(OB.activation([v], "silu"), silu, rtol=1e-13, atol=0)
