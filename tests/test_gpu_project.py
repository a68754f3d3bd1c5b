"""mw_project_forward against its formula in float64.

Tolerances, derived: u = 2^-8 (unit roundoff of bf16: 8 significant bits, to nearest), float32 sums of n products within n * 2^-23 of the sum of absolute values.
  low-rank product  v = scale A x:   dv = (H + 2) 2^-23 |scale| sum |A x| + u |v|        (one rounding to bf16)
  output            dy = (H + r) 2^-23 (sum |W x| + sum |B v|) + sum |B| dv + u |y| (bf16 outputs only)
Inputs that are small integers make every step exact: those cases have no tolerance.
"""
import pytest

from gpu_util import Guarded, torch_mod
from paper_2605_22428_b200 import binding as mw

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


def make(T, H, O, n=0, r=0, seed=0, segment=1, none=0.2, integers=False):
    torch = torch_mod()
    g = torch.Generator("cuda").manual_seed(seed)
    if integers:
        draw = lambda *s, std=1.0: torch.randint(-1, 2, s, device="cuda", generator=g).bfloat16()  # noqa: E731
    else:
        draw = lambda *s, std=1.0: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(0, std, generator=g)  # noqa: E731
    d = dict(T=T, H=H, O=O, n=n, r=r, x=draw(T, H), w=draw(O, H, std=H ** -0.5), a=None, b=None, scale=None, ids=None)
    if n:
        d["a"], d["b"] = draw(n, r, H, std=H ** -0.5), draw(n, O, r, std=r ** -0.5)
        d["scale"] = torch.randint(1, 3, (n,), device="cuda", generator=g).float() if integers else 0.5 + torch.rand(n, device="cuda", generator=g)
        req = torch.randint(0, n, (-(-T // segment),), device="cuda", generator=g)
        req = torch.where(torch.rand(len(req), device="cuda", generator=g) < none, -1, req)
        d["ids"] = req.repeat_interleave(segment)[:T].int().contiguous()
    return d


def plain(d, f32):
    torch = torch_mod()
    x, w = d["x"].double(), d["w"].double()
    y, mag = x @ w.t(), x.abs() @ w.abs().t()
    dy = torch.zeros_like(y)
    if d["ids"] is not None:
        for a in range(d["n"]):
            t = torch.nonzero(d["ids"] == a).squeeze(1)
            if not t.numel():
                continue
            s = d["scale"][a].double() if d["scale"] is not None else 1.0
            A, B = d["a"][a].double(), d["b"][a].double()
            v = s * (x[t] @ A.t())
            dv = (d["H"] + 2) * 2.0 ** -23 * abs(s) * (x[t].abs() @ A.abs().t()) + U * v.abs()
            y[t] += v @ B.t()
            mag[t] += (v.abs() + dv) @ B.abs().t()
            dy[t] += dv @ B.abs().t()
    dy = dy + (d["H"] + d["r"]) * 2.0 ** -23 * mag
    return y, dy if f32 else dy + U * (y.abs() + dy)


def forward(d, f32=False, handle=None, flags=0):
    torch = torch_mod()
    T, O = d["T"], d["O"]
    y = Guarded(T * O * (4 if f32 else 2))
    out = y.body.view(torch.float32 if f32 else torch.bfloat16)
    h = handle or mw.Projection(d["H"], O, max(T, 1), d["w"], d["n"], d["r"], d["a"], d["b"], d["scale"], flags=flags)
    h.mw_project_forward(d["x"], d["ids"], T, out)
    torch.cuda.synchronize()
    assert y.guards_intact()
    status = h.mw_project_get_status()
    if handle is None:
        h.close()
    return out.clone().reshape(T, O), status


def check(d, got, f32=False):
    torch = torch_mod()
    y, bound = plain(d, f32)
    err = (got.double() - y).abs()
    assert torch.isfinite(got).all()
    assert bool((err <= bound + 1e-30).all()), float((err - bound).max())
    if not f32 and float(y.norm()) > 0:
        assert float(err.norm() / y.norm()) <= U


SHAPES = [  # T, H, O, adapters, rank, segment
    (1, 8, 1, 1, 8, 1), (1, 1024, 1024, 4, 16, 1), (1, 7168, 257, 3, 64, 1), (2, 72, 128, 2, 8, 1), (5, 200, 63, 5, 24, 1), (16, 512, 129, 16, 16, 1),
    (17, 640, 300, 40, 32, 1), (64, 1024, 512, 32, 16, 1), (64, 256, 130, 64, 128, 1), (77, 1000, 1003, 5, 40, 9), (128, 128, 96, 7, 72, 3),
    (255, 192, 200, 300, 8, 1), (256, 320, 256, 1, 64, 256), (257, 264, 255, 9, 104, 50), (600, 512, 384, 12, 16, 77), (1025, 320, 640, 100, 48, 1),
    (1500, 256, 1000, 6, 128, 400)]


@pytest.mark.parametrize("T,H,O,n,r,segment", SHAPES)
def test_against_the_formula(T, H, O, n, r, segment):
    d = make(T, H, O, n, r, seed=T + O, segment=segment)
    got, status = forward(d)
    assert status == mw.MW_OK
    check(d, got)


@pytest.mark.parametrize("T,H,O,n,r,segment", [(1, 64, 40, 2, 8, 1), (50, 128, 200, 10, 16, 1), (300, 200, 150, 7, 40, 11), (280, 96, 136, 3, 128, 90)])
def test_small_integers_are_exact(T, H, O, n, r, segment):
    torch = torch_mod()
    d = make(T, H, O, n, r, seed=H, segment=segment, integers=True)
    got, _ = forward(d, f32=True)
    y, _ = plain(d, True)
    v = max(float((d["x"].double().abs() @ d["a"][a].double().abs().t()).max()) for a in range(n)) * 2
    assert v <= 256                              # v is exact in bf16
    assert torch.equal(got.double(), y)


@pytest.mark.parametrize("T", [1, 40, 333])
def test_without_adapters(T):
    """No adapter held, none named, or all ids -1: the plain product, the same bits in all three."""
    torch = torch_mod()
    d = make(T, 320, 192, 4, 16, seed=T)
    ids = d["ids"]
    d["ids"] = None
    one, _ = forward(d)
    d["ids"] = torch.full_like(ids, -1)
    two, status = forward(d)
    assert status == mw.MW_OK and torch.equal(one, two)
    bare = dict(d, n=0, r=0, a=None, b=None, scale=None, ids=None)
    three, _ = forward(bare)
    assert torch.equal(one, three)
    check(bare, three)


@pytest.mark.parametrize("T,O", [(3, 64), (64, 256), (300, 65)])
def test_float32_outputs(T, O):
    d = make(T, 1024, O, 6, 16, seed=O)
    got, _ = forward(d, f32=True)
    check(d, got, True)
    d = make(T, 7168, O, seed=O)
    got, _ = forward(d, f32=True)
    check(d, got, True)


def test_no_scale_means_one():
    torch = torch_mod()
    d = make(30, 128, 64, 4, 16, seed=1)
    d["scale"] = None
    one, _ = forward(d)
    d["scale"] = torch.ones(4, device="cuda")
    two, _ = forward(d)
    assert torch.equal(one, two)
    check(d, one)


def test_bad_ids_count_as_none():
    torch = torch_mod()
    d = make(30, 128, 64, 4, 16, seed=3)
    bad = d["ids"].clone()
    bad[2], bad[9], bad[10] = 4, -5, 2 ** 31 - 1
    good = bad.clone()
    good[[2, 9, 10]] = -1
    got, status = forward(dict(d, ids=bad))
    want, fine = forward(dict(d, ids=good))
    assert status == mw.MW_ERR_BAD_INDEX and fine == mw.MW_OK and torch.equal(got, want)


def test_adapters_and_rows_stay_apart():
    """Infinities in one token's row and NaN in an adapter that no token of the batch names reach nobody else."""
    torch = torch_mod()
    d = make(40, 128, 96, 6, 16, seed=5, none=0.0)
    d["ids"] = (d["ids"] % 5).int().contiguous()
    clean, _ = forward(d)
    d["a"][5], d["b"][5] = float("nan"), float("inf")
    got, _ = forward(d)
    assert torch.equal(got, clean)
    d["x"][13] = float("inf")
    got, _ = forward(d)
    keep = [t for t in range(40) if t != 13]
    assert torch.equal(got[keep], clean[keep])
    d["x"][13] = 1.0
    d["b"][2] = float("nan")
    got, _ = forward(d)
    other = (d["ids"] != 2) & (torch.arange(40, device="cuda") != 13)
    assert torch.equal(got[other], clean[other]) and bool(torch.isnan(got[d["ids"] == 2].float()).all())


def test_strides_and_a_long_lived_handle():
    torch = torch_mod()
    big = make(300, 192, 101, 8, 24, seed=12, segment=3)
    with mw.Projection(192, 101, 300, big["w"], 8, 24, big["a"], big["b"], big["scale"]) as h:
        for T in (300, 1, 64, 0, 17, 300):
            d = dict(big, T=T, x=big["x"][:T], ids=big["ids"][:T])
            wide_x = torch.zeros(max(T, 1), 192 + 24, dtype=torch.bfloat16, device="cuda")
            wide_x[:T, 8:200] = d["x"]
            wide_y = torch.full((max(T, 1), 111), 7.0, dtype=torch.bfloat16, device="cuda")
            for _ in range(2):
                h.mw_project_forward(wide_x[:, 8:], d["ids"], T, wide_y[:, 3:], x_stride_bytes=216 * 2, y_stride_bytes=222)
                torch.cuda.synchronize()
            if T:
                got = wide_y[:, 3:104].contiguous()
                check(d, got)
                assert bool((wide_y[:, :3] == 7).all()) and bool((wide_y[:, 104:] == 7).all())
                again, _ = forward(d, handle=h)
                assert torch.equal(got, again)
        big["w"].mul_(0.5)
        big["a"].mul_(2.0)
        big["b"].neg_()
        big["scale"].mul_(0.25)
        got, _ = forward(big, handle=h)
        check(big, got)
        assert h.mw_project_kernel_launches() > 0


def test_side_stream_graph_and_no_overlap():
    torch = torch_mod()
    d = make(24, 512, 128, 8, 16, seed=15)
    want, _ = forward(d)
    plain_launch, _ = forward(d, flags=mw.MW_FLAG_NO_OVERLAP)
    assert torch.equal(want, plain_launch)
    with mw.Projection(512, 128, 24, d["w"], 8, 16, d["a"], d["b"], d["scale"]) as h:
        y = torch.zeros_like(want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        h.mw_project_forward(d["x"], d["ids"], 24, y, stream=side)
        side.synchronize()
        assert torch.equal(y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h.mw_project_forward(d["x"], d["ids"], 24, y, stream=side)
        for seed in (1, 2):
            other = make(24, 512, 128, 8, 16, seed=seed)
            d["x"].copy_(other["x"])
            d["ids"].copy_(other["ids"])
            graph.replay()
            torch.cuda.synchronize()
            check(d, y)


@pytest.mark.parametrize("T,H,O,n,r,segment", [(40, 1024, 700, 9, 16, 1), (300, 512, 1500, 5, 64, 60), (64, 4096, 256, 20, 32, 1)])
def test_many_calls_in_a_row_give_the_same_bits(T, H, O, n, r, segment):
    torch = torch_mod()
    a, b = (make(T, H, O, n, r, seed=s, segment=segment) for s in (1, 2))
    with mw.Projection(H, O, T, a["w"], n, r, a["a"], a["b"], a["scale"]) as ha, mw.Projection(H, O, T, b["w"], n, r, b["a"], b["b"], b["scale"]) as hb:
        want = [forward(d, handle=h)[0] for d, h in ((a, ha), (b, hb))]
        check(a, want[0])
        check(b, want[1])
        ys = [torch.zeros(300, T, O, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for i in range(300):
            for d, h, y in ((a, ha, ys[0]), (b, hb, ys[1])):
                h.mw_project_forward(d["x"], d["ids"], T, y[i])
        torch.cuda.synchronize()
        assert ha.mw_project_get_status() == mw.MW_OK and hb.mw_project_get_status() == mw.MW_OK
        for y, w in zip(ys, want):
            assert bool((y.view(torch.int16) == w.view(torch.int16)).all())


@pytest.mark.parametrize("T,r", [(60, 16), (500, 64)])
def test_one_handle_with_inputs_that_take_turns(T, r):
    """Nothing of one call may reach the next: two batches take turns on one handle, nothing waits between the calls."""
    torch = torch_mod()
    a = make(T, 512, 640, 6, r, seed=1, segment=7)
    b = dict(make(T, 512, 640, 6, r, seed=2, segment=5), w=a["w"], a=a["a"], b=a["b"], scale=a["scale"])
    with mw.Projection(512, 640, T, a["w"], 6, r, a["a"], a["b"], a["scale"]) as h:
        want = [forward(d, handle=h)[0] for d in (a, b)]
        check(b, want[1])
        y = torch.zeros(200, T, 640, dtype=torch.bfloat16, device="cuda")
        for i in range(200):
            d = (a, b)[i & 1]
            h.mw_project_forward(d["x"], d["ids"], T, y[i])
        torch.cuda.synchronize()
        for k in (0, 1):
            assert bool((y[k::2].view(torch.int16) == want[k].view(torch.int16)).all())


@pytest.mark.parametrize("T,r", [(3, 16), (300, 64)])
def test_a_wait_that_gives_up_is_reported_and_recovered_from(T, r):
    torch = torch_mod()
    d = make(T, 256, 200, 4, r, seed=T)
    with mw.Projection(256, 200, T, d["w"], 4, r, d["a"], d["b"], d["scale"], flags=mw.MW_FLAG_SHORT_WAITS) as h:
        want, status = forward(d, handle=h)
        assert status == mw.MW_OK
        check(d, want)
        h.mw_project_test_skew_waits()
        _, status = forward(d, handle=h)
        assert status == mw.MW_ERR_TIMEOUT
        for _ in range(2):
            got, status = forward(d, handle=h)
            assert status == mw.MW_OK and torch.equal(got, want)
    assert mw.lib().mw_project_test_skew_waits(None) == mw.MW_ERR_INVALID_ARG


def test_refusals():
    torch = torch_mod()
    d = make(4, 64, 40, 3, 16)
    ok = dict(H=64, O=40, max_tokens=4, w=d["w"], adapters=3, rank=16, a=d["a"], b=d["b"], scale=d["scale"])
    for bad in (dict(H=60), dict(H=0), dict(O=0), dict(max_tokens=0), dict(adapters=-1), dict(rank=12), dict(rank=0), dict(rank=136), dict(w=None),
                dict(a=None), dict(b=None), dict(adapters=0), dict(device=-1), dict(flags=1 << 30)):
        with pytest.raises(mw.MwError) as err:
            mw.Projection(**{**ok, **bad})
        assert err.value.code == mw.MW_ERR_INVALID_ARG, bad
    for bad in (dict(w=d["w"].data_ptr() + 2), dict(a=d["a"].data_ptr() + 8), dict(b=d["b"].data_ptr() + 4), dict(scale=d["scale"].data_ptr() + 2)):
        with pytest.raises(mw.MwError) as err:
            mw.Projection(**{**ok, **bad})
        assert err.value.code == mw.MW_ERR_ALIGNMENT, bad
    y = torch.zeros(4, 40, dtype=torch.bfloat16, device="cuda")
    L = mw.lib()
    with mw.Projection(**ok) as h:
        def rc(x=d["x"].data_ptr(), ids=d["ids"].data_ptr(), T=4, yy=y.data_ptr(), dt=mw.MW_DTYPE_BF16, xs=0, ys=0):
            return L.mw_project_forward(h._h, x, xs, ids, T, yy, dt, ys, None)
        assert rc() == mw.MW_OK and rc(T=0) == mw.MW_OK
        for bad in (dict(T=5), dict(T=-1), dict(x=None), dict(yy=None), dict(dt=2), dict(xs=112), dict(ys=64), dict(xs=-128)):
            assert rc(**bad) == mw.MW_ERR_INVALID_ARG, bad
        for bad in (dict(x=d["x"].data_ptr() + 2), dict(yy=y.data_ptr() + 1), dict(xs=136), dict(ys=83), dict(ids=d["ids"].data_ptr() + 1)):
            assert rc(**bad) == mw.MW_ERR_ALIGNMENT, bad
        torch.cuda.synchronize()
        assert h.mw_project_get_status() == mw.MW_OK
    assert L.mw_project_forward(None, 16, 0, None, 1, 16, 1, 0, None) == mw.MW_ERR_INVALID_ARG
    assert L.mw_project_get_status(None, None, None) == mw.MW_ERR_INVALID_ARG
    assert L.mw_project_destroy(None) == mw.MW_OK
