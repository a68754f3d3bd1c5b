"""The gated block in fp16 at the ends of its range.  h, dg and du are operands of products of 16 bits, rounded once each: beyond 65504 (from 65520 on, which is nearer to
the next step) they are infinite, below 2^-14 they have a step of 2^-24.  What is infinite stays with its token: only that token's row of y or dx, and the gradients of
the weights that sum over it, are not finite."""
import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_gated import backward_formula, handle, make, rounding, run_backward, run_forward, within

pytestmark = pytest.mark.gpu


def one_unit(T, gate, up, dtype="f16"):
    """Width 8, of which unit 0 alone is used: g = x[0], u = x[1], y[c] = h for every c."""
    torch = torch_mod()
    d = make(T, 64, 8, dtype, seed=1)
    for w in (d["w_gate_up"], d["w_down"], d["x"]):
        w.zero_()
    d["w_gate_up"][0, 0, 0] = d["w_gate_up"][1, 0, 1] = 1.0
    d["w_down"][:, 0] = 1.0
    d["x"][:, 0], d["x"][:, 1] = gate, up
    return d, torch


@pytest.mark.parametrize("T", [1, 2, 40, 600])
def test_h_at_the_largest_value(T):
    # silu(256) is 256 in float32 (exp(-256) is nothing beside 1): h = 256 u
    d, torch = one_unit(T, 256.0, 255.75)                       # 65472, which fp16 has
    y, _ = run_forward(d)
    assert bool((y == 65472).all())
    d["x"][T // 2, 1] = 256.0                                   # 65536
    y2, _ = run_forward(d)
    others = torch.arange(T, device="cuda") != T // 2
    assert torch.equal(y2[others], y[others]) and bool(torch.isinf(y2[T // 2]).all())
    b, _ = one_unit(T, 256.0, 256.0, "bf16")                    # bf16 has it
    assert bool((run_forward(b)[0] == 65536).all())


@pytest.mark.parametrize("T", [1, 40, 600])
@pytest.mark.parametrize("kept_as", ["f32", "own"])
def test_gradients_beyond_the_largest_value(T, kept_as):
    """dg = dh u act'(g): 64 channels of dy = 16 make dh 1024, which 128 takes past the end.  Each channel of that token's dx has a product with it, infinite or, where
    the weight is zero, NaN.  (The gradients of the weights in float32: du x[0] is 2^18 for a token.)"""
    d, torch = one_unit(T, 16.0, 0.5)
    d["dy"].fill_(16.0)
    kept = torch.zeros(T, 16, device="cuda")
    kept[:, 0], kept[:, 8] = 16.0, 0.5
    own = lambda: kept if kept_as == "f32" else kept.half()  # noqa: E731
    dx = run_backward(d, own(), want=("dx",))["dx"]
    within(dx, backward_formula(d, kept[:, :8].double(), kept[:, 8:].double())["dx"], "dx")
    kept[T // 2, 8] = 128.0
    got = run_backward(d, own(), dw="f32")
    others = torch.arange(T, device="cuda") != T // 2
    assert torch.equal(got["dx"][others], dx[others])
    assert bool(torch.isinf(got["dx"][T // 2, 0])) and not bool(torch.isfinite(got["dx"][T // 2]).any())
    assert not bool(torch.isfinite(got["dw_gate_up"][0, 0, 0])) and bool(torch.isfinite(got["dw_gate_up"][1]).all()) and bool(torch.isfinite(got["dw_down"]).all())


@pytest.mark.parametrize("T,H,I", [(40, 512, 136), (600, 256, 264)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_small_gradients(T, H, I, dtype):
    """dy of 2^-18: dg and du lie below fp16's smallest normal value and are off by half of its step at most; in bf16 they are as good as any."""
    d = make(T, H, I, dtype, seed=T)
    d["dy"] *= 2.0 ** -18
    _, kept = run_forward(d, keep=True)
    got, want = run_backward(d, kept, dw="f32"), backward_formula(d, kept[:, :I].double(), kept[:, I:].double(), dw=torch_mod().float32)
    for k in got:
        within(got[k], want[k], k)
    if dtype == "bf16":
        assert float((got["dx"].double() - want["dx"][0]).norm()) <= 2 * rounding(d["kind"])[0] * float(want["dx"][0].norm())
    with handle(d, train=True) as h:
        assert h.mw_gated_get_status() == mw.MW_OK
