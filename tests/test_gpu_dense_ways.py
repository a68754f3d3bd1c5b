"""The dense operators on every kind of tile that large calls have: accumulators of 256, 224, 128 and 64 columns, more tiles than pairs of blocks (so that both buffers of
sums and the waits between tiles are used), tiles of the last round cut in two.  Each case says what it is to reach, and the library says what it did, so that a
changed choice does not move a case away unseen.  Widths end inside a tile, and inside or before the right half of a cut one.  Tolerances are those of test_gpu_gated.py and
test_gpu_int8.py.
"""
import pytest

from gpu_util import Guarded, torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_gated import backward_formula, forward_formula, handle, make, run_backward, run_forward, types, within
from test_gpu_int8 import check, product_formula
from test_gpu_int8 import make as make_integers

pytestmark = pytest.mark.gpu

FORWARD = ("gate", "down")
SILU, GELU = mw.MW_ACT_SILU, mw.MW_ACT_GELU


def kind_of(way):
    """(columns, more tiles than pairs, cut) of pairs, (0, pieces) of clusters."""
    columns, tiles, halves, pieces = way
    pairs = torch_mod().cuda.get_device_properties(0).multi_processor_count // 2
    return (columns, tiles > pairs, halves > 0) if columns else (0, pieces)


# T, H, I, and what the launches of the forward call are to be
@pytest.mark.parametrize("T,H,I,dtype,act,gate,down", [
    (1300, 200, 2808, "bf16", SILU, (256, True, False), None),
    (8192, 1024, 264, "bf16", SILU, (256, True, True), None),           # cut tiles whose right half lies beyond I
    (8192, 1024, 360, "f16", GELU, (256, True, True), None),            # and such whose right half I ends in
    (600, 1024, 2808, "bf16", GELU, (256, False, False), None),
    (777, 200, 4104, "f16", SILU, (224, True, False), None),
    (300, 200, 4104, "bf16", SILU, (224, False, False), None),
    (600, 200, 2808, "f16", GELU, (128, True, False), None),
    (4000, 200, 264, "bf16", SILU, (64, True, False), None),
    (600, 7168, 72, "bf16", SILU, None, (256, True, True)),
    (4000, 2048, 72, "f16", GELU, None, (256, True, False)),
    (777, 7168, 72, "bf16", SILU, None, (224, True, False)),
])
def test_forward(T, H, I, dtype, act, gate, down):
    """y and what is kept, with nothing kept (h rounded before it is turned), float32, and the rows' type."""
    torch = torch_mod()
    d = make(T, H, I, dtype, act, seed=T + I)
    want = forward_formula(d)
    with handle(d) as h:
        def launches():
            ways = h.mw_gated_test_ways()
            assert len(ways) == 2
            for way, expected in zip(ways, (gate, down)):
                assert expected is None or kind_of(way) == expected, ways
            return ways
        y, _ = run_forward(d, h)
        ways = launches()
        within(y, want["y"], "y")
        again, kept = run_forward(d, h, keep=True)
        assert launches() == ways and torch.equal(again, y)
        within(kept[:, :I], want["g"], "g")
        within(kept[:, I:], want["u"], "u")
        rounded = Guarded(T * 2 * I * 2)
        again = torch.empty_like(y)
        h.mw_gated_forward(d["x"], T, again, gate_up=rounded.body.view(d["kind"]))
        torch.cuda.synchronize()
        assert launches() == ways and torch.equal(again, y) and rounded.guards_intact()
        assert torch.equal(rounded.body.view(d["kind"]).reshape(T, 2 * I), kept.to(d["kind"]))


# ... and of the backward call: the gradient of h, then those of x and the weights
@pytest.mark.parametrize("T,H,I,dtype,act,expected", [
    (2000, 200, 4104, "bf16", SILU, [(256, True, False)]),
    (2500, 200, 1992, "f16", GELU, [(256, True, True)]),
    (2600, 136, 2008, "bf16", GELU, [(256, True, True)]),               # cut tiles whose right half I ends in
    (3500, 200, 1992, "bf16", SILU, [(224, True, False)]),
    (6000, 200, 1032, "f16", SILU, [(128, True, False)]),
    (4000, 200, 520, "bf16", GELU, [(64, True, False)]),
    (8192, 1024, 72, "bf16", SILU, [None, (256, True, False), (0, 4)]),
    (5000, 1024, 72, "f16", GELU, [None, (256, True, True)]),
    (4000, 7168, 520, "bf16", SILU, [None, (128, True, False)]),
    (3, 1024, 1992, "bf16", SILU, [None, None, (256, True, True)]),
    (3, 2048, 1032, "f16", GELU, [None, None, (224, True, False)]),
    (600, 7168, 72, "bf16", GELU, [None, (256, True, False)]),
    (3, 7168, 264, "f16", SILU, [None, (256, True, True)]),
])
@pytest.mark.parametrize("kept_as", ["f32", "own"])
def test_backward(T, H, I, dtype, act, expected, kept_as):
    """Gradients of the weights in the operands' type (whose launches are looked at) and, added to something, in float32."""
    torch = torch_mod()
    d = make(T, H, I, dtype, act, seed=T + H)
    x, w = d["x"].float(), d["w_gate_up"].float()
    kept = torch.cat((x @ w[0].t(), x @ w[1].t()), 1).to(torch.float32 if kept_as == "f32" else d["kind"])
    g, u = kept[:, :I].double(), kept[:, I:].double()
    with handle(d, train=True) as h:
        got = run_backward(d, kept, h)
        ways = h.mw_gated_test_ways()
        assert len(ways) >= len(expected)
        for way, e in zip(ways, expected):
            assert e is None or kind_of(way) == e, ways
        want = backward_formula(d, g, u)
        for k in got:
            within(got[k], want[k], k)
        before = {k: torch.randn(v.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(2)) for k, v in (("dw_gate_up", d["w_gate_up"]), ("dw_down", d["w_down"]))}
        alone = run_backward(d, kept, h, dw="f32")
        onto = run_backward(d, kept, h, dw="f32", accumulate=before)
    want = backward_formula(d, g, u, dw=torch.float32)
    for k in ("dw_gate_up", "dw_down"):
        within(alone[k], want[k], k)
        assert torch.equal(onto[k], alone[k] + before[k])


@pytest.mark.parametrize("T,H,O,dtype,expected", [
    (777, 64, 5008, "f32", (256, True, True)), (5000, 64, 5008, "bf16", (256, True, True)), (5000, 64, 1003, "f16", (256, True, True)), (5000, 64, 1003, "f32", (256, True, True)),
    (4000, 64, 2200, "f32", (256, True, False)), (2500, 64, 5008, "bf16", (256, True, False)), (8192, 64, 1003, "bf16", (256, True, False)),
    (777, 64, 7168, "f32", (224, True, False)), (777, 64, 7160, "f16", (224, True, False)), (2500, 64, 1003, "f32", (224, False, False)),
    (777, 256, 5008, "f32", (128, True, False)), (300, 64, 7168, "bf16", (128, True, False)), (5000, 2048, 1003, "bf16", (128, True, False)),
    (4000, 64, 520, "f32", (64, True, False)), (4000, 64, 520, "bf16", (64, True, False)),
])
def test_product_in_8_bits(T, H, O, dtype, expected):
    torch = torch_mod()
    d = make_integers(T, H, O, seed=T + O)
    if dtype == "f16":                          # (its largest is 65504)
        d["x_scale"] *= 1e-4
    y = Guarded(T * O * (4 if dtype == "f32" else 2))
    out = y.body.view(types()[dtype])
    with mw.Int8Projection(H, O, T, d["w"], d["w_scale"]) as h:
        h.mw_int8_forward(d["q"], d["x_scale"], T, out)
        torch.cuda.synchronize()
        assert y.guards_intact() and h.mw_int8_get_status() == mw.MW_OK
        ways = h.mw_int8_test_ways()
    assert len(ways) == 1 and kind_of(ways[0]) == expected, ways
    check(out.reshape(T, O), product_formula(d, dtype))


def test_of_no_call_and_of_no_handle():
    """Nothing before the first call, dot products for one token; refused without a handle."""
    torch = torch_mod()
    d = make(4, 64, 40)
    y = torch.empty_like(d["x"])
    with handle(d) as h:
        assert h.mw_gated_test_ways() == []
        h.mw_gated_forward(d["x"], 1, y)
        assert [kind_of(w) for w in h.mw_gated_test_ways()] == [(0, 0), (0, 0)]
        torch.cuda.synchronize()
    assert mw.lib().mw_gated_test_ways(None, None, None) == mw.lib().mw_int8_test_ways(None, None, None) == mw.MW_ERR_INVALID_ARG
