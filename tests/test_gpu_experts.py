"""mw_experts_forward against its formula in float64 (weights and rows bf16, exactly representable there).

Tolerances, derived: u = 2^-8 is the unit roundoff of bf16 (8 significant bits, to nearest), e = n * 2^-23 bounds a float32 sum of n products (relative to the sum of
their absolute values; one unit in the last place per addition, rounding or truncating).
  gate, up:    dg = H 2^-23 sum |W_gate x|, du likewise
  activation:  |silu'| <= 1.1:   dh = 1.1 dg |up| + |silu(gate)| du + 1.1 dg du + (u + 2^-20) |h|    (one rounding to bf16)
  output:      dy = sum_k |w| ( sum |W_down| dh + (I + K) 2^-23 sum |W_down| (|h| + dh) ) + u (|y| + ...)
Every value is held to that bound.  It is a worst case; over a whole tensor the roundings are independent, so the relative
2-norm of the error is well below u, and is held to u = 3.9e-3.
"""
import numpy as np
import pytest

from gpu_util import Guarded, torch_mod
from paper_2605_22428_b200 import binding as mw

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


def make(T, E, K, H, I, first=0, count=None, seed=0, ids=None):
    torch = torch_mod()
    count = E - first if count is None else count
    g = torch.Generator("cuda").manual_seed(seed)
    n = lambda *s, std=1.0: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(0, std, generator=g)  # noqa: E731
    d = dict(T=T, E=E, K=K, H=H, I=I, first=first, count=count, x=n(T, H), wgu=n(count, 2, I, H, std=H ** -0.5),
             wd=n(count, H, I, std=I ** -0.5), weights=torch.rand(T, K, device="cuda", generator=g) - 0.2)
    if ids is None:
        ids = torch.rand(T, E, device="cuda", generator=g).argsort(1)[:, :K].int()
    d["ids"] = torch.as_tensor(ids, dtype=torch.int32, device="cuda").contiguous()
    return d


def plain(d):
    """(y, bound) in float64."""
    torch = torch_mod()
    T, K, H, I = d["T"], d["K"], d["H"], d["I"]
    y = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    dy, mag = torch.zeros_like(y), torch.zeros_like(y)
    x = d["x"].double()
    for e in range(d["count"]):
        token, slot = torch.nonzero(d["ids"] == d["first"] + e, as_tuple=True)
        if token.numel() == 0:
            continue
        r, wg, wu, wd = x[token], d["wgu"][e, 0].double(), d["wgu"][e, 1].double(), d["wd"][e].double()
        gate, up = r @ wg.t(), r @ wu.t()
        h = gate * torch.sigmoid(gate) * up
        dg, du = H * 2.0 ** -23 * (r.abs() @ wg.abs().t()), H * 2.0 ** -23 * (r.abs() @ wu.abs().t())
        dh = 1.1 * dg * up.abs() + (gate * torch.sigmoid(gate)).abs() * du + 1.1 * dg * du
        dh = dh + (U + 2.0 ** -20) * (h.abs() + dh)
        w = d["weights"][token, slot].double().unsqueeze(1) if d["weights"] is not None else torch.ones(len(token), 1, device="cuda", dtype=torch.float64)
        m = w.abs() * ((h.abs() + dh) @ wd.abs().t())
        y.index_add_(0, token, w * (h @ wd.t()))
        dy.index_add_(0, token, w.abs() * (dh @ wd.abs().t()) + (I + K) * 2.0 ** -23 * m)
        mag.index_add_(0, token, m)
    return y, dy + U * (y.abs() + dy)


def forward(d, flags=0, handle=None, stream=None):
    torch = torch_mod()
    T, H = d["T"], d["H"]
    y = Guarded(T * H * 2)
    own = handle is None
    h = handle or mw.Experts(d["E"], d["K"], max(T, 1), H, d["I"], d["wgu"], d["wd"], expert_first=d["first"], expert_count=d["count"], flags=flags)
    h.mw_experts_forward(d["x"], d["ids"], d["weights"], T, y.ptr(), stream=stream)
    torch.cuda.synchronize()
    assert y.guards_intact()
    status = h.mw_experts_get_status()
    if own:
        h.close()
    return y.body.clone().view(torch.bfloat16).reshape(T, H), status


def check(d, got):
    torch = torch_mod()
    y, bound = plain(d)
    err = (got.double() - y).abs()
    assert torch.isfinite(got.float()).all()
    assert bool((err <= bound + 1e-30).all()), float((err - bound).max())
    if float(y.norm()) > 0:
        assert float(err.norm() / y.norm()) <= U


SHAPES = [  # T, E, K, H, I
    (1, 1, 1, 8, 16), (1, 8, 2, 64, 64), (1, 32, 4, 1024, 512), (2, 4, 4, 72, 48), (3, 8, 3, 128, 80), (7, 32, 4, 1024, 512), (16, 16, 8, 256, 128),
    (17, 5, 2, 1000, 176), (33, 8, 8, 136, 144), (64, 256, 8, 512, 64), (100, 3, 1, 264, 272), (200, 16, 4, 640, 208), (257, 4, 3, 320, 96),
    (513, 2, 2, 192, 160), (1024, 8, 8, 128, 64)]


@pytest.mark.parametrize("T,E,K,H,I", SHAPES)
def test_against_the_formula(T, E, K, H, I):
    d = make(T, E, K, H, I, seed=T + H)
    got, status = forward(d)
    assert status == mw.MW_OK
    check(d, got)


def test_full_width_expert_rows():
    d = make(5, 16, 8, 7168, 2048, first=4, count=3, seed=3)
    got, status = forward(d)
    assert status == mw.MW_OK
    check(d, got)


@pytest.mark.parametrize("T", [1, 31, 300])
def test_a_rank_takes_its_own_experts_only(T):
    d = make(T, 64, 6, 256, 96, first=24, count=8, seed=T)
    got, status = forward(d)
    assert status == mw.MW_OK
    check(d, got)
    away = ((d["ids"] < 24) | (d["ids"] >= 32)).all(1)
    assert bool((got[away] == 0).all())


def test_every_token_on_one_expert_and_repeated_experts():
    """One expert gets everything (several token tiles), a token names it more than once: it counts as often as it is named."""
    torch = torch_mod()
    ids = torch.full((300, 3), 2, dtype=torch.int32)
    ids[::3, 1] = 1
    ids[::5, 2] = -1
    d = make(300, 4, 3, 192, 112, seed=8, ids=ids)
    got, status = forward(d)
    assert status == mw.MW_OK
    check(d, got)


def test_padding_empty_tokens_and_bad_ids():
    torch = torch_mod()
    ids = torch.randint(0, 12, (40, 4), dtype=torch.int32)
    ids[3] = -1
    ids[10:20] = -1
    ids[5, 2] = 12
    ids[6, 0] = -2
    ids[7, 1] = 2 ** 31 - 1
    ids[8, 3] = -2 ** 31
    d = make(40, 12, 4, 128, 64, seed=4, ids=ids)
    got, status = forward(d)
    assert status == mw.MW_ERR_BAD_INDEX
    check(d, got)
    assert bool((got[3] == 0).all()) and bool((got[10:20] == 0).all())
    d["ids"][:] = -1
    got, status = forward(d)
    assert status == mw.MW_OK and bool((got == 0).all())


def test_without_weights_and_zero_weights():
    d = make(21, 8, 2, 256, 64, seed=2)
    d["weights"] = None
    got, _ = forward(d)
    check(d, got)
    d = make(21, 8, 2, 256, 64, seed=2)
    d["weights"].zero_()
    got, _ = forward(d)
    assert bool((got == 0).all())


def test_one_tokens_infinity_stays_its_own():
    """Tokens of one expert share a tile: a row of infinities or NaN must not reach its neighbours."""
    torch = torch_mod()
    d = make(20, 2, 2, 256, 64, seed=6)
    clean, _ = forward(d)
    d["x"][7] = float("inf")
    d["x"][11] = float("nan")
    got, _ = forward(d)
    keep = [t for t in range(20) if t not in (7, 11)]
    assert torch.equal(got[keep], clean[keep])
    assert bool(torch.isnan(got[11].float()).all())


def test_strides_and_a_long_lived_handle():
    """Rows inside wider rows, several calls of several sizes on one handle, weights rewritten between calls, the same bits each time."""
    torch = torch_mod()
    big = make(130, 16, 4, 320, 80, seed=12)
    with mw.Experts(16, 4, 130, 320, 80, big["wgu"], big["wd"]) as h:
        for T in (130, 1, 64, 0, 17, 130):
            d = dict(big, T=T, x=big["x"][:T], ids=big["ids"][:T], weights=big["weights"][:T])
            wide_x = torch.zeros(max(T, 1), 320 + 24, dtype=torch.bfloat16, device="cuda")
            wide_x[:T, 8:328] = d["x"]
            wide_y = torch.full((max(T, 1), 320 + 40), 7.0, dtype=torch.bfloat16, device="cuda")
            for _ in range(2):
                h.mw_experts_forward(wide_x[:, 8:], d["ids"], d["weights"], T, wide_y[:, 16:], x_stride_bytes=344 * 2, y_stride_bytes=360 * 2)
                torch.cuda.synchronize()
            if T:
                got = wide_y[:, 16:336].contiguous()
                check(d, got)
                assert bool((wide_y[:, :16] == 7).all()) and bool((wide_y[:, 336:] == 7).all())
                again, _ = forward(d, handle=h)
                assert torch.equal(got, again)
        big["wgu"].mul_(0.5)
        big["wd"].mul_(-2.0)
        got, status = forward(big, handle=h)
        assert status == mw.MW_OK
        check(big, got)
        assert h.mw_experts_kernel_launches() > 0


def test_side_stream_graph_and_no_overlap():
    torch = torch_mod()
    d = make(24, 8, 3, 512, 128, seed=15)
    want, _ = forward(d)
    plain_launch, _ = forward(d, flags=mw.MW_FLAG_NO_OVERLAP)
    assert torch.equal(want, plain_launch)
    with mw.Experts(8, 3, 24, 512, 128, d["wgu"], d["wd"]) as h:
        y = torch.zeros_like(want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        h.mw_experts_forward(d["x"], d["ids"], d["weights"], 24, y, stream=side)
        side.synchronize()
        assert torch.equal(y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h.mw_experts_forward(d["x"], d["ids"], d["weights"], 24, y, stream=side)
        for seed in (1, 2):
            other = make(24, 8, 3, 512, 128, seed=seed)
            d["x"].copy_(other["x"])
            d["ids"].copy_(other["ids"])
            graph.replay()
            torch.cuda.synchronize()
            check(d, y)


@pytest.mark.parametrize("T,E,K,H,I,others", [(256, 32, 4, 1024, 688, False), (64, 24, 6, 512, 240, False), (150, 40, 4, 640, 400, True)])
def test_many_calls_in_a_row_give_the_same_bits(T, E, K, H, I, others):
    """Blocks run at different speeds from call to call: tiles that are cut between them, and the hand-over from the first product to the
    second, must not depend on who is early.  Two handles take turns, nothing waits between the calls."""
    torch = torch_mod()
    a, b = (make(T, E, K, H, I, seed=s, first=8 if others else 0, count=16 if others else None) for s in (1, 2))
    with mw.Experts(E, K, T, H, I, a["wgu"], a["wd"], expert_first=a["first"], expert_count=a["count"]) as ha, \
            mw.Experts(E, K, T, H, I, b["wgu"], b["wd"], expert_first=b["first"], expert_count=b["count"]) as hb:
        want = [forward(d, handle=h)[0] for d, h in ((a, ha), (b, hb))]
        check(a, want[0])
        check(b, want[1])
        ys = [torch.zeros(400, T, H, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for i in range(400):
            for d, h, y in ((a, ha, ys[0]), (b, hb, ys[1])):
                h.mw_experts_forward(d["x"], d["ids"], d["weights"], T, y[i])
        torch.cuda.synchronize()
        assert ha.mw_experts_get_status() == mw.MW_OK and hb.mw_experts_get_status() == mw.MW_OK
        for y, w in zip(ys, want):
            assert bool((y.view(torch.int16) == w.view(torch.int16)).all())


def test_handles_on_streams_at_once():
    """The blocks of a call wait for one another; calls of several handles on several streams must not keep each other from finishing."""
    torch = torch_mod()
    ds = [make(100, 32, 4, 1024, 512, seed=s) for s in range(3)]
    hs = [mw.Experts(32, 4, 100, 1024, 512, d["wgu"], d["wd"]) for d in ds]
    want = [forward(d, handle=h)[0] for d, h in zip(ds, hs)]
    streams = [torch.cuda.Stream(priority=p) for p in (0, -1, 0)]
    ys = [torch.zeros(100, 100, 1024, dtype=torch.bfloat16, device="cuda") for _ in ds]
    torch.cuda.synchronize()
    for i in range(100):
        for d, h, st, y in zip(ds, hs, streams, ys):
            h.mw_experts_forward(d["x"], d["ids"], d["weights"], 100, y[i], stream=st)
    torch.cuda.synchronize()
    for h, y, w in zip(hs, ys, want):
        assert h.mw_experts_get_status() == mw.MW_OK
        assert bool((y.view(torch.int16) == w.view(torch.int16)).all())
        h.close()


def test_one_handle_with_inputs_that_take_turns():
    """Nothing of one call may reach the next: two batches take turns on one handle, nothing waits between the calls."""
    torch = torch_mod()
    a = make(90, 20, 4, 512, 256, seed=1)
    b = dict(make(90, 20, 4, 512, 256, seed=2), wgu=a["wgu"], wd=a["wd"])
    with mw.Experts(20, 4, 90, 512, 256, a["wgu"], a["wd"]) as h:
        want = [forward(d, handle=h)[0] for d in (a, b)]
        check(b, want[1])
        y = torch.zeros(200, 90, 512, dtype=torch.bfloat16, device="cuda")
        for i in range(200):
            d = (a, b)[i & 1]
            h.mw_experts_forward(d["x"], d["ids"], d["weights"], 90, y[i])
        torch.cuda.synchronize()
        for k in (0, 1):
            assert bool((y[k::2].view(torch.int16) == want[k].view(torch.int16)).all())


@pytest.mark.parametrize("T", [3, 150])
def test_a_wait_that_gives_up_is_reported_and_recovered_from(T):
    """Every pipeline stage is announced too large, so nothing ever completes: each wait runs out, the status says so, the call
    after mw_experts_get_status is right again."""
    torch = torch_mod()
    d = make(T, 8, 2, 256, 64, seed=T)
    with mw.Experts(8, 2, T, 256, 64, d["wgu"], d["wd"], flags=mw.MW_FLAG_SHORT_WAITS) as h:
        want, status = forward(d, handle=h)
        assert status == mw.MW_OK
        check(d, want)
        h.mw_experts_test_skew_waits()
        _, status = forward(d, handle=h)
        assert status == mw.MW_ERR_TIMEOUT
        for _ in range(2):
            got, status = forward(d, handle=h)
            assert status == mw.MW_OK and torch.equal(got, want)
    assert mw.lib().mw_experts_test_skew_waits(None) == mw.MW_ERR_INVALID_ARG


def test_refusals():
    torch = torch_mod()
    d = make(4, 4, 2, 64, 32)
    ok = dict(E=4, K=2, max_tokens=4, H=64, I=32, w_gate_up=d["wgu"], w_down=d["wd"])
    for bad in (dict(E=0), dict(K=0), dict(K=65), dict(max_tokens=0), dict(max_tokens=1025), dict(H=60), dict(I=24), dict(H=0), dict(I=0),
                dict(expert_first=-1), dict(expert_first=2, expert_count=3), dict(expert_count=0), dict(w_gate_up=None), dict(w_down=None),
                dict(device=-1), dict(flags=1 << 30), dict(K=64, max_tokens=1024), dict(E=2000, expert_count=1025)):
        with pytest.raises(mw.MwError) as err:
            mw.Experts(**{**ok, **bad})
        assert err.value.code == mw.MW_ERR_INVALID_ARG, bad
    with pytest.raises(mw.MwError) as err:
        mw.Experts(**{**ok, "w_down": d["wd"].data_ptr() + 2})
    assert err.value.code == mw.MW_ERR_ALIGNMENT
    y = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    with mw.Experts(**ok) as h:
        def rc(x=d["x"], ids=d["ids"], w=d["weights"], T=4, yy=y, xs=0, ys=0):
            return h.mw_experts_forward(x, ids, w, T, yy, x_stride_bytes=xs, y_stride_bytes=ys, check=False)
        assert rc() == mw.MW_OK and rc(T=0) == mw.MW_OK
        for bad in (dict(T=5), dict(T=-1), dict(x=None), dict(ids=None), dict(yy=None), dict(xs=112), dict(ys=64), dict(xs=-128)):
            assert rc(**bad) == mw.MW_ERR_INVALID_ARG, bad
        for bad in (dict(x=d["x"].data_ptr() + 2), dict(yy=y.data_ptr() + 8), dict(xs=136), dict(ys=130), dict(ids=d["ids"].data_ptr() + 1)):
            assert rc(**bad) == mw.MW_ERR_ALIGNMENT, bad
        torch.cuda.synchronize()
        assert h.mw_experts_get_status() == mw.MW_OK
    assert mw.lib().mw_experts_forward(None, 16, 0, 16, None, 1, 16, 0, None) == mw.MW_ERR_INVALID_ARG
    assert mw.lib().mw_experts_get_status(None, None, None) == mw.MW_ERR_INVALID_ARG
    assert mw.lib().mw_experts_destroy(None) == mw.MW_OK
