"""The low-rank values of mw_project: sixteen significant bits reach the product with B, and adapters stay apart on every route.

v = scale A x is kept as hi + lo, two bf16: hi is v to 8 bits, lo what that leaves to 8 bits, so |v - hi - lo| <= 2^-9 2^-9 |v|; the header
promises sixteen bits, 2^-16 |v|.  Integers of up to sixteen bits are exact, and so is every sum here (all below 2^24): no tolerance.
  real values, float32 outputs:   dv = (H + 2) 2^-23 |scale| sum |A x| + 2^-16 |v|
                                  dy = (H + 2 r) 2^-23 (sum |W x| + sum |B| (|v| + dv)) + sum |B| dv
Both would fail for values of 8 bits; each test says so of its own inputs.
Routes: plain dot products up to T * r = 4096, lists and a product on the tensor cores above; additions beside the products (T <= 128) or after them.
"""
import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_project import forward, make

pytestmark = pytest.mark.gpu

# T, H, O, adapters, rank, segment
ROUTES = [(1, 64, 40, 1, 8, 1), (40, 128, 200, 5, 16, 1), (32, 96, 130, 2, 128, 16), (120, 128, 150, 7, 40, 1), (128, 64, 257, 2, 64, 64), (300, 128, 200, 7, 40, 11),
          (280, 96, 136, 3, 128, 90), (1000, 64, 100, 30, 8, 1)]


def parts(d):
    """Per adapter: its tokens, v and B in float64."""
    torch = torch_mod()
    for a in range(d["n"]):
        t = torch.nonzero(d["ids"] == a).squeeze(1)
        if t.numel():
            yield t, float(d["scale"][a]), d["a"][a].double(), d["scale"][a].double() * (d["x"][t].double() @ d["a"][a].double().t()), d["b"][a].double()


@pytest.mark.parametrize("T,H,O,n,r,segment", ROUTES)
def test_integers_of_sixteen_bits_are_exact(T, H, O, n, r, segment):
    torch = torch_mod()
    d = make(T, H, O, n, r, seed=H + T, segment=segment, none=0.1 if T > 1 else 0.0, integers=True)
    most = max(float((d["x"].double().abs() @ d["a"][a].double().abs().t()).max()) for a in range(n))
    d["scale"] = torch.full((n,), float(int(65535 // most)), device="cuda") - torch.arange(n, device="cuda")
    y, rounded = d["x"].double() @ d["w"].double().t(), 0
    for t, _, _, v, b in parts(d):
        assert float(v.abs().max()) < 65536 and r * 65536 < 2 ** 24
        rounded += int((v.bfloat16().double() != v).sum())
        y[t] += v @ b.t()
    assert rounded > 0
    got, status = forward(d, f32=True)
    assert status == mw.MW_OK and torch.equal(got.double(), y)


@pytest.mark.parametrize("T,H,O,n,r,segment", ROUTES)
def test_real_values_to_sixteen_bits(T, H, O, n, r, segment):
    torch = torch_mod()
    d = make(T, H, O, n, r, seed=7 * T + r, segment=segment, none=0.1 if T > 1 else 0.0)
    x, w = d["x"].double(), d["w"].double()
    y, mag = x @ w.t(), x.abs() @ w.abs().t()
    dy, coarse = torch.zeros_like(y), torch.zeros_like(y)
    for t, s, a, v, b in parts(d):
        dv = (H + 2) * 2.0 ** -23 * abs(s) * (x[t].abs() @ a.abs().t()) + 2.0 ** -16 * v.abs()
        y[t] += v @ b.t()
        mag[t] += (v.abs() + dv) @ b.abs().t()
        dy[t] += dv @ b.abs().t()
        coarse[t] = (v.bfloat16().double() - v) @ b.t()
    bound = dy + (H + 2 * r) * 2.0 ** -23 * mag
    assert bool((coarse.abs() > bound).any())
    got, status = forward(d, f32=True)
    assert status == mw.MW_OK
    assert bool(((got.double() - y).abs() <= bound).all())


@pytest.mark.parametrize("T,H,O,n,r,segment", [(40, 128, 96, 6, 16, 1), (120, 128, 130, 7, 64, 1), (128, 64, 257, 6, 64, 30), (300, 128, 96, 6, 16, 1),
                                              (300, 128, 200, 9, 72, 40), (600, 64, 140, 40, 128, 3)])
def test_adapters_and_rows_stay_apart(T, H, O, n, r, segment):
    """NaN and infinities in an adapter, in one that nobody names, or in a token's row reach nobody else: all other bits stay."""
    torch = torch_mod()
    d = make(T, H, O, n, r, seed=5, segment=segment, none=0.1)
    d["ids"] = torch.where(d["ids"] == n - 1, 0, d["ids"]).int().contiguous()
    clean, _ = forward(d)
    d["a"][n - 1], d["b"][n - 1] = float("nan"), float("inf")
    got, _ = forward(d)
    assert torch.equal(got, clean)
    for value in (float("nan"), float("inf")):
        for what in ("a", "b"):
            bad = dict(d, **{what: d[what].clone()})
            bad[what][1] = value
            got, _ = forward(bad)
            other = d["ids"] != 1
            assert torch.equal(got[other], clean[other])
            if value != value:
                assert bool(torch.isnan(got[~other].float()).all())
    d["x"][13] = float("inf")
    d["x"][T - 2] = float("nan")
    got, _ = forward(d)
    keep = [t for t in range(T) if t not in (13, T - 2)]
    assert torch.equal(got[keep], clean[keep])
