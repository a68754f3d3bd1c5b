"""mw_project_forward where adapters hold infinities, or low-rank values are near the end of the type's range.

The low-rank values v = scale A x go to B as two terms, hi + lo.  The formula multiplies B by their sum: an infinite element of B gives an
infinity of v's sign (NaN only where v is 0, or where infinities of both signs meet), whatever the two terms are.  Values of B that are not
finite touch their own rows of their own adapter's tokens only: all other outputs keep the bits they have without them.
"""
import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_project import forward, make

pytestmark = pytest.mark.gpu

INF = float("inf")


def expected(d):
    """B v in float64 for every token with an adapter, 0 for the others."""
    torch = torch_mod()
    y = torch.zeros(d["T"], d["O"], dtype=torch.float64, device="cuda")
    for a in range(d["n"]):
        t = torch.nonzero(d["ids"] == a).squeeze(1)
        if t.numel():
            v = d["scale"][a].double() * (d["x"][t].double() @ d["a"][a].double().t())
            y[t] = (v.unsqueeze(1) * d["b"][a].double().unsqueeze(0)).sum(2)
    return y


# plain dot products (T * r <= 4096) and lists; many adapters to sixteen tokens and one; ranks held in registers and beyond; accumulators with
# and without columns for the additions
@pytest.mark.parametrize("T,H,O,n,r,segment", [(1, 64, 40, 1, 8, 1), (40, 128, 200, 5, 16, 1), (48, 128, 130, 2, 72, 48), (300, 64, 150, 6, 24, 1),
                                              (300, 128, 257, 3, 64, 100), (200, 96, 140, 7, 128, 3)])
@pytest.mark.parametrize("integers", [True, False])
def test_infinite_elements_of_b(T, H, O, n, r, segment, integers):
    torch = torch_mod()
    d = make(T, H, O, n, r, seed=T + r, segment=segment, integers=integers)
    clean, status = forward(d, f32=True)
    assert status == mw.MW_OK
    g = torch.Generator("cuda").manual_seed(1)
    odd = torch.rand(n, O, device="cuda", generator=g) < 0.3           # rows with one element that is not finite, some with two
    at = torch.randint(0, r, (n, O), device="cuda", generator=g)
    value = torch.tensor([INF, -INF, float("nan")], device="cuda").bfloat16()[torch.randint(0, 3, (n, O), device="cuda", generator=g)]
    b = d["b"].clone()
    for shift, also in ((0, odd), (1, odd & (torch.rand(n, O, device="cuda", generator=g) < 0.3))):
        k = ((at + shift) % r).unsqueeze(2)
        b.scatter_(2, k, torch.where(also, value, b.gather(2, k).squeeze(2)).unsqueeze(2))
    bad = dict(d, b=b)
    got, _ = forward(bad, f32=True)
    want = expected(bad)
    touched = torch.zeros(T, O, dtype=torch.bool, device="cuda")
    has = d["ids"] >= 0
    touched[has] = odd[d["ids"][has].long()]
    assert bool(touched.any()) or not bool(has.any())
    assert torch.equal(got[~touched], clean[~touched])
    assert torch.equal(torch.isnan(got[touched]), torch.isnan(want[touched]))
    assert torch.equal(got[touched] == INF, want[touched] == INF) and torch.equal(got[touched] == -INF, want[touched] == -INF)


@pytest.mark.parametrize("T,r", [(3, 8), (600, 8)])
def test_values_near_the_end_of_the_range(T, r):
    """v beyond the largest bf16 value (3.3895e38) and below the largest float32: finite, so B v is; v infinite: so is B v."""
    torch = torch_mod()
    d = make(T, 64, 33, 2, r, seed=2, none=0.0)
    d["w"].zero_()
    d["x"].fill_(1.0)
    d["a"].zero_()
    d["a"][:, :, 0] = 1.0
    d["b"].fill_(2.0 ** -20)
    d["scale"] = torch.tensor([3.4e38, INF], device="cuda")
    got, _ = forward(d, f32=True)
    want = r * 2.0 ** -20 * float(d["scale"][0])
    first = got[d["ids"] == 0].double()
    assert first.numel() and bool(((first - want).abs() <= (2.0 ** -16 + (64 + r + 2) * 2.0 ** -23) * want).all())
    assert bool((got[d["ids"] == 1] == INF).all())
