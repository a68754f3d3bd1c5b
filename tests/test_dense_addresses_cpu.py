"""Gradients of the weights given to the binding as addresses: nothing of them says their type, so the caller does.  (No device is needed: the library's
function is replaced by one that keeps its arguments.)"""
import types

import pytest

from paper_2605_22428_b200 import binding as mw
from test_dense_cpu import without_a_handle


class OnGpu:
    """As much of a tensor on the GPU as the binding looks at."""
    is_cuda = True

    def __init__(self, dtype, address=4096):
        self.dtype, self.address = dtype, address

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.address

    def get_device(self):
        return 0


@pytest.fixture
def call(monkeypatch):
    """The binding's backward call on a handle of bf16; (address, address, type) of the gradients as the library gets them."""
    seen = []
    monkeypatch.setattr(mw, "lib", lambda: types.SimpleNamespace(mw_gated_backward_kept=lambda *a: seen.append((a[10], a[11], a[12])) or (mw.MW_OK if a[12] >= 0 else mw.MW_ERR_INVALID_ARG),
                                                                 mw_gated_destroy=lambda h: mw.MW_OK, mw_strerror=lambda code: b""))

    def backward(**kw):
        without_a_handle(mw.Gated).mw_gated_backward(256, 512, 768, 4, stream=4, **kw)
        return seen[-1]
    return backward


def test_an_address_has_the_type_that_is_said(call):
    import torch
    assert call(dw_gate_up=1024, dw_down=2048, dw_dtype=torch.bfloat16) == (1024, 2048, mw.MW_DTYPE_BF16)
    assert call(dw_down=2048, dw_dtype=torch.float32) == (None, 2048, mw.MW_DTYPE_F32)


def test_an_address_beside_a_tensor_has_its_type(call):
    import torch
    for dtype, code in ((torch.bfloat16, mw.MW_DTYPE_BF16), (torch.float32, mw.MW_DTYPE_F32)):
        assert call(dw_gate_up=1024, dw_down=OnGpu(dtype)) == (1024, 4096, code)
        assert call(dw_gate_up=OnGpu(dtype), dw_down=1024) == (4096, 1024, code)
        assert call(dw_gate_up=OnGpu(dtype), dw_down=OnGpu(dtype, 8192)) == (4096, 8192, code)
        assert call(dw_gate_up=OnGpu(dtype), dw_dtype=dtype) == (4096, None, code)


def test_an_address_of_no_type_is_refused(call):
    for kw in (dict(dw_gate_up=1024), dict(dw_down=1024), dict(dw_gate_up=1024, dw_down=2048)):
        with pytest.raises(mw.MwError) as err:
            call(**kw)
        assert err.value.code == mw.MW_ERR_INVALID_ARG


def test_types_that_do_not_go_together_are_refused(call):
    import torch
    for kw in (dict(dw_gate_up=OnGpu(torch.float32), dw_down=OnGpu(torch.bfloat16)), dict(dw_gate_up=OnGpu(torch.bfloat16), dw_dtype=torch.float32),
               dict(dw_gate_up=1024, dw_down=OnGpu(torch.float16)), dict(dw_down=1024, dw_dtype=torch.float16), dict(dw_down=1024, dw_dtype=torch.float64)):
        with pytest.raises(TypeError, match="gradients of the weights|^dw_down"):
            call(**kw)


def test_without_gradients_of_the_weights_no_type_is_needed(call):
    assert call(dx=1024) == (None, None, mw.MW_DTYPE_F32)
