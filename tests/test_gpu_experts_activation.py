"""The activation of mw_experts over its whole range: silu(gate) * up, gate far below zero, where e^-gate leaves float32 and the product need not.

One row of ones, gate and up set by single weights, so that both are exact; every output is I equal terms with W_down = 1 / I (a power
of two).  Tolerance: a rounding of the activation and one of y to bf16, 2^-9 each, and the exponential's 2 + 1.2 |gate| units in the last place of float32 (2^-16 at
most; below 2^-126 its step is 2^-149: 2^-149 / e^gate more), well within 2^-7 + 2^-20.
"""
import math

import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_experts import forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gate", [-1000.0, -104.0, -100.0, -95.0, -90.0, -88.5, -88.0, -87.5, -87.0, -80.0, -20.0, -3.0, -2.0 ** -20, 0.0, 2.0 ** -20, 3.0, 88.0, 1000.0])
@pytest.mark.parametrize("T", [1, 20])
def test_silu_far_from_zero(gate, T):
    torch = torch_mod()
    H, I, up = 64, 32, 2.0 ** 100 if gate < -50 else 1.0
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    d = dict(T=T, E=1, K=1, H=H, I=I, first=0, count=1, x=torch.ones(T, H, dtype=torch.bfloat16, device="cuda"), wgu=z(1, 2, I, H), wd=z(1, H, I),
             weights=torch.ones(T, 1, device="cuda"), ids=torch.zeros(T, 1, dtype=torch.int32, device="cuda"))
    d["wgu"][0, 0, :, 3], d["wgu"][0, 1, :, 5] = gate, up
    d["wd"][:] = 1.0 / I
    gate = float(d["wgu"][0, 0, 0, 3])
    got, status = forward(d)
    assert status == mw.MW_OK
    e = math.exp(-abs(gate))
    want = gate * (e if gate < 0 else 1.0) / (1 + e) * up
    step = 2.0 ** -149 / e * abs(want) if gate < -87 and e > 0 else 2.0 ** -149 * abs(gate) * up
    assert bool(((got.double() - want).abs() <= (2.0 ** -7 + 2.0 ** -20) * abs(want) + step).all())


def test_silu_of_infinities():
    """silu(-inf) is -inf * 0, which is NaN; silu(inf) is inf."""
    torch = torch_mod()
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for gate, check in ((float("inf"), torch.isposinf), (float("-inf"), torch.isnan)):
        d = dict(T=2, E=1, K=1, H=64, I=16, first=0, count=1, x=torch.ones(2, 64, dtype=torch.bfloat16, device="cuda"), wgu=z(1, 2, 16, 64), wd=z(1, 64, 16),
                 weights=torch.ones(2, 1, device="cuda"), ids=torch.zeros(2, 1, dtype=torch.int32, device="cuda"))
        d["wgu"][0, 0, :, 3], d["wgu"][0, 1, :, 5] = gate, 1.0
        d["wd"][:] = 1.0
        got, _ = forward(d)
        assert bool(check(got.float()).all())
