"""Tensors of the dense operators that lie on another GPU than the handle's (or, where there is no handle, than the current one) are refused before the
library is called.  (No device is needed: the tensors are as much of one as the binding looks at.)"""
import types

import pytest

from paper_2605_22428_b200 import binding as mw


class OnGpu:
    is_cuda = True

    def __init__(self, dtype, index, elements=1 << 20):
        self.dtype, self.index, self.elements = dtype, index, elements

    @property
    def device(self):
        return f"cuda:{self.index}"

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def stride(self, dim):
        return 1

    def numel(self):
        return self.elements

    def data_ptr(self):
        return 4096


@pytest.fixture
def calls(monkeypatch):
    """Names of the library's functions that are reached; the current device is 0."""
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or mw.MW_OK
    monkeypatch.setattr(mw, "lib", lambda: Library())
    monkeypatch.setattr(mw, "_current_device", lambda: 0, raising=False)
    return reached


def block(device):
    import torch
    return mw.Gated(64, 40, 8, OnGpu(torch.bfloat16, device), OnGpu(torch.bfloat16, device), train=True, device=device)


def product(device):
    import torch
    return mw.Int8Projection(64, 40, 8, OnGpu(torch.int8, device), OnGpu(torch.float32, device), device=device)


def test_on_the_handles_device(calls):
    """Whatever the current device is."""
    import torch
    b, f = OnGpu(torch.bfloat16, 1), OnGpu(torch.float32, 1)
    block(1).mw_gated_forward(b, 4, b, gate_up=f, stream=4)
    block(1).mw_gated_backward(b, f, b, 4, dx=b, dw_gate_up=f, dw_down=f, stream=4)
    product(1).mw_int8_forward(b, None, 4, f, stream=4)
    product(1).mw_int8_forward(OnGpu(torch.int8, 1), f, 4, f, x_stride_bytes=64, stream=4)
    assert [c for c in calls if "forward" in c or "backward" in c] == ["mw_gated_forward_keep", "mw_gated_backward_kept", "mw_int8_forward", "mw_int8_forward"]


@pytest.mark.parametrize("off", ["x", "y", "gate_up"])
def test_forward_refuses_another_device(calls, off):
    import torch
    t = {k: OnGpu(torch.float32 if k == "gate_up" else torch.bfloat16, 0 if k == off else 1) for k in ("x", "y", "gate_up")}
    h = block(1)
    with pytest.raises(ValueError, match=f"^{off}: a tensor on cuda:1 expected, got one on cuda:0"):
        h.mw_gated_forward(t["x"], 4, t["y"], gate_up=t["gate_up"], stream=4)
    assert "mw_gated_forward_keep" not in calls


@pytest.mark.parametrize("off", ["x", "gate_up", "dy", "dx", "dw_gate_up", "dw_down"])
def test_backward_refuses_another_device(calls, off):
    import torch
    t = {k: OnGpu(torch.float32 if k == "gate_up" else torch.bfloat16, 1 if k == off else 0) for k in ("x", "gate_up", "dy", "dx", "dw_gate_up", "dw_down")}
    h = block(0)
    with pytest.raises(ValueError, match=f"^{off}: a tensor on cuda:0 expected"):
        h.mw_gated_backward(t["x"], t["gate_up"], t["dy"], 4, dx=t["dx"], dw_gate_up=t["dw_gate_up"], dw_down=t["dw_down"], stream=4)
    assert "mw_gated_backward_kept" not in calls


@pytest.mark.parametrize("off", ["x", "x_scale", "y"])
def test_the_product_refuses_another_device(calls, off):
    import torch
    kinds = dict(x=torch.int8, x_scale=torch.float32, y=torch.float32)
    t = {k: OnGpu(v, 1 if k == off else 0) for k, v in kinds.items()}
    h = product(0)
    with pytest.raises(ValueError, match=f"^{off}: a tensor on cuda:0 expected"):
        h.mw_int8_forward(t["x"], t["x_scale"], 4, t["y"], stream=4)
    assert "mw_int8_forward" not in calls


def test_weights_on_another_device(calls):
    import torch
    with pytest.raises(ValueError, match="^w_down: a tensor on cuda:0 expected"):
        mw.Gated(64, 40, 8, OnGpu(torch.bfloat16, 0), OnGpu(torch.bfloat16, 1))
    with pytest.raises(ValueError, match="^w_scale: a tensor on cuda:1 expected"):
        mw.Int8Projection(64, 40, 8, OnGpu(torch.int8, 1), OnGpu(torch.float32, 0), device=1)
    assert calls == ["mw_gated_create", "mw_int8_create"]          # (the library has looked at the configuration; the handles are closed again)


def test_rows_in_8_bits_are_made_on_the_current_device(calls):
    import torch
    on = lambda x, q, scale: (OnGpu(torch.bfloat16, x), 4, 64, OnGpu(torch.int8, q), OnGpu(torch.float32, scale))  # noqa: E731
    for where, what in (((1, 1, 1), "x"), ((0, 1, 0), "q"), ((0, 0, 1), "scale"), ((1, 0, 0), "x")):
        with pytest.raises(ValueError, match=f"^{what}: a tensor on cuda:0 expected, got one on cuda:1"):
            mw.mw_quantise_rows(*on(*where), stream=4)
    assert not calls
    mw.mw_quantise_rows(*on(0, 0, 0), stream=4)
    assert calls == ["mw_quantise_rows"]
