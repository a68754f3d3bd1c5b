"""What mw_gated_forward keeps for the backward call, in the rows' own type instead of float32.

The sums are the same, so everything is compared exactly: what is kept is the float32 values rounded once, y does not change, and the gradients are those of
the same rounded values given in float32.  Those in turn are held against the formula (its tolerances in test_gpu_gated.py).
"""
import pytest

from gpu_util import Guarded, torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_gated import CASES, backward_formula, handle, make, run_backward, run_forward, within

pytestmark = pytest.mark.gpu


def forward_kept(d, h=None, stream=None):
    torch = torch_mod()
    T, H, I = d["T"], d["H"], d["I"]
    y, kept = Guarded(T * H * 2), Guarded(T * 2 * I * 2)
    own = h or handle(d)
    own.mw_gated_forward(d["x"], T, y.body.view(d["kind"]), gate_up=kept.body.view(d["kind"]), stream=stream)
    torch.cuda.synchronize()
    assert y.guards_intact() and kept.guards_intact()
    assert own.mw_gated_get_status() == mw.MW_OK
    if not h:
        own.close()
    return y.body.view(d["kind"]).reshape(T, H), kept.body.view(d["kind"]).reshape(T, 2 * I)


@pytest.mark.parametrize("T,H,I,dtype,act", CASES)
def test_forward_rounds_what_it_keeps(T, H, I, dtype, act):
    torch = torch_mod()
    d = make(T, H, I, dtype, act, seed=T + I)
    want_y, want = run_forward(d, keep=True)
    y, kept = forward_kept(d)
    assert torch.equal(y, want_y) and torch.equal(kept, want.to(d["kind"]))


@pytest.mark.parametrize("T,H,I,dtype,act", CASES)
@pytest.mark.parametrize("dw", ["own", "f32"])
def test_backward_goes_by_what_was_kept(T, H, I, dtype, act, dw):
    torch = torch_mod()
    d = make(T, H, I, dtype, act, seed=T + H)
    _, kept = forward_kept(d)
    got, want = run_backward(d, kept, dw=dw), run_backward(d, kept.float(), dw=dw)
    assert all(torch.equal(got[k], want[k]) for k in want)
    formula = backward_formula(d, kept[:, :I].double(), kept[:, I:].double(), dw=torch.float32 if dw == "f32" else None)
    for k in got:
        within(got[k], formula[k], k)


@pytest.mark.parametrize("T", [0, 1, 64, 700])
def test_added_to_captured_and_in_wider_rows(T):
    """A step as a training program has it: rows inside wider arrays, gradients added to what is there, captured and replayed."""
    torch = torch_mod()
    d = make(T, 512, 136, "f16", mw.MW_ACT_GELU, seed=T)
    with handle(d, train=True) as h:
        want_y, kept = forward_kept(d, h)
        before = {k: torch.randn(v.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(2)) for k, v in (("dw_gate_up", d["w_gate_up"]), ("dw_down", d["w_down"]))}
        want = run_backward(d, kept, h, dw="f32", accumulate=before)
        x, dy, y, dx = (torch.full((T, 576), 7.0, dtype=d["kind"], device="cuda") for _ in range(4))
        x[:, :512], dy[:, :512] = d["x"], d["dy"]
        kept2, dw = torch.empty_like(kept), {k: v.clone() for k, v in before.items()}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h.mw_gated_forward(x, T, y, gate_up=kept2, x_stride_bytes=1152, y_stride_bytes=1152)
            h.mw_gated_backward(x, kept2, dy, T, dx=dx, **dw, accumulate=True, x_stride_bytes=1152, dy_stride_bytes=1152, dx_stride_bytes=1152)
        for k in dw:
            dw[k].copy_(before[k])
        graph.replay()
        torch.cuda.synchronize()
        assert h.mw_gated_get_status() == mw.MW_OK
    assert torch.equal(y[:, :512], want_y) and torch.equal(kept2, kept) and torch.equal(dx[:, :512], want["dx"])
    assert bool((y[:, 512:] == 7).all()) and bool((dx[:, 512:] == 7).all())
    assert all(torch.equal(dw[k], want[k]) for k in dw)


def test_types_of_what_is_kept_and_the_calls_without_one():
    torch = torch_mod()
    d = make(8, 64, 40, seed=0)
    y, kept, narrow = torch.empty_like(d["x"]), torch.empty(8, 80, device="cuda"), torch.empty(8, 80, dtype=torch.bfloat16, device="cuda")
    L = mw.lib()
    with handle(d, train=True) as h:
        want_y, want = run_forward(d, h, keep=True)
        x, stream = d["x"].data_ptr(), torch.cuda.current_stream().cuda_stream
        for bad in (mw.MW_DTYPE_F16, mw.MW_DTYPE_I8, -1):
            assert L.mw_gated_forward_keep(h._h, x, 0, 8, y.data_ptr(), 0, narrow.data_ptr(), bad, stream) == mw.MW_ERR_INVALID_ARG
            assert L.mw_gated_backward_kept(h._h, x, 0, narrow.data_ptr(), bad, d["dy"].data_ptr(), 0, 8, y.data_ptr(), 0, None, None, 0, 0, stream) == mw.MW_ERR_INVALID_ARG
        assert L.mw_gated_forward_keep(h._h, x, 0, 8, y.data_ptr(), 0, narrow.data_ptr() + 8, mw.MW_DTYPE_BF16, stream) == mw.MW_ERR_ALIGNMENT
        with pytest.raises(TypeError, match="^gate_up"):
            h.mw_gated_forward(d["x"], 8, y, gate_up=narrow.half())
        with pytest.raises(TypeError, match="^gate_up"):
            h.mw_gated_backward(d["x"], narrow.half(), d["dy"], 8, dx=y)
        with pytest.raises(ValueError, match="^gate_up"):
            h.mw_gated_forward(d["x"], 8, y, gate_up=narrow.t())
        # the entry points without a type keep float32
        assert L.mw_gated_forward(h._h, x, 0, 8, y.data_ptr(), 0, kept.data_ptr(), stream) == mw.MW_OK
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(kept, want)
        grad = run_backward(d, kept, h)["dx"]
        assert L.mw_gated_backward(h._h, x, 0, kept.data_ptr(), d["dy"].data_ptr(), 0, 8, y.data_ptr(), 0, None, None, 0, 0, stream) == mw.MW_OK
        torch.cuda.synchronize()
        assert torch.equal(y, run_backward(d, kept, h, want=("dx",))["dx"]) and grad.shape == y.shape
