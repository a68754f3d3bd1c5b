"""The binding of the serving operators, as far as it needs no device: errors of a call surface as MwError with the code."""
import ctypes

import pytest

from paper_2605_22428_b200 import binding as mw
from paper_2605_22428_b200 import build as mwbuild


@pytest.fixture(scope="module", autouse=True)
def library():
    mwbuild.build_library()
    return mw.lib()


def without_a_handle(kind):
    """An object whose create never ran: every call of the library is refused."""
    h = kind.__new__(kind)
    h._h = ctypes.c_void_p()
    return h


@pytest.mark.parametrize("kind,call", [(mw.Experts, "mw_experts_get_status"), (mw.Experts, "mw_experts_test_skew_waits"),
                                       (mw.Projection, "mw_project_get_status"), (mw.Projection, "mw_project_test_skew_waits")])
def test_a_refused_call_raises_with_its_code(kind, call):
    h = without_a_handle(kind)
    args = () if call.endswith("skew_waits") else (4,)          # (a stream, so that none has to be asked for)
    with pytest.raises(mw.MwError) as err:
        getattr(h, call)(*args)
    assert err.value.code == mw.MW_ERR_INVALID_ARG and call in str(err.value)


# ---- tensors that the kernels would read as they lie ----
def tensors():
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)  # noqa: E731
    return torch, z


def forward(x=None, ids=None, weights=None, y=None, **more):
    return without_a_handle(mw.Experts).mw_experts_forward(x, ids, weights, 4, y, stream=4, **more)


def project(x=None, ids=None, y=None, **more):
    return without_a_handle(mw.Projection).mw_project_forward(x, ids, 4, y, stream=4, **more)


def test_types_of_tensors():
    torch, z = tensors()
    for bad, name in ((dict(x=z(4, 64, dtype=torch.float16)), "x"), (dict(ids=z(4, 2, dtype=torch.int64)), "topk_ids"),
                      (dict(weights=z(4, 2)), "weights"), (dict(weights=z(4, 2, dtype=torch.float64)), "weights"), (dict(y=z(4, 64, dtype=torch.float32)), "y")):
        with pytest.raises(TypeError, match=f"^{name}: a tensor of torch"):
            forward(**bad)
    for bad, name in ((dict(x=z(4, 64, dtype=torch.float32), y=z(4, 8)), "x"), (dict(ids=z(4, dtype=torch.int64), y=z(4, 8)), "adapter_ids")):
        with pytest.raises(TypeError, match=f"^{name}: a tensor of torch"):
            project(**bad)
    l, i, w = z(4, 16, dtype=torch.float32), z(4, 2, dtype=torch.int32), z(4, 2, dtype=torch.float32)
    for ids, weights, bias in ((i.long(), 256, None), (256, w.double(), None), (256, 256, z(16))):
        with pytest.raises(TypeError):
            mw.mw_route(l, bias, 4, 16, 2, 0, 1.0, ids, weights, stream=4)
    w8 = z(3, 8, 64, dtype=torch.float32)
    for make in (lambda: mw.Experts(2, 1, 4, 64, 16, w8, 512), lambda: mw.Experts(2, 1, 4, 64, 16, 256, w8), lambda: mw.Projection(64, 8, 4, w8),
                 lambda: mw.Projection(64, 8, 4, 256, 3, 8, w8, 512), lambda: mw.Projection(64, 8, 4, 256, 3, 8, 512, w8),
                 lambda: mw.Projection(64, 8, 4, 256, 3, 8, 512, 768, w8.bfloat16())):
        with pytest.raises(TypeError, match="a tensor of torch"):
            make()


def test_tensors_with_gaps():
    torch, z = tensors()
    wide, turned = z(4, 72), z(64, 4).t()
    for call in (lambda: forward(x=wide[:, :64]), lambda: forward(x=turned), lambda: forward(x=turned, x_stride_bytes=128), lambda: forward(y=wide[:, 8:]),
                 lambda: forward(ids=z(2, 4, dtype=torch.int32).t()), lambda: project(x=wide[:, :64], y=z(4, 8)), lambda: project(x=256, y=turned),
                 lambda: mw.Projection(64, 64, 4, z(64, 64).t()), lambda: mw.Experts(2, 1, 4, 64, 16, 256, z(2, 16, 64).transpose(1, 2))):
        with pytest.raises(ValueError, match="has gaps"):
            call()


def test_tensors_that_are_not_on_the_gpu():
    torch, z = tensors()
    for call in (lambda: forward(x=z(4, 64)), lambda: forward(x=z(4, 72)[:, :64], x_stride_bytes=144), lambda: project(x=256, y=z(4, 8)),
                 lambda: mw.mw_route(z(4, 16), None, 4, 16, 2, 0, 1.0, 256, 256, stream=4), lambda: mw.Projection(64, 64, 4, z(64, 64))):
        with pytest.raises(TypeError, match="on the GPU expected"):
            call()


def test_addresses_are_taken_as_they_are():
    for call in (lambda: forward(256, 256, 256, 256), lambda: forward(256, 256, None, 256)):
        with pytest.raises(mw.MwError) as err:
            call()
        assert err.value.code == mw.MW_ERR_INVALID_ARG          # of the handle that is not there


def test_weights_smaller_than_the_handle_reads():
    """After the library has taken the configuration; the handle is closed again."""
    torch, z = tensors()

    class Handle:
        closed = 0

        def close(self):
            self.closed += 1

    h = Handle()
    mw._holds(h, w=(z(4, 8), 32), a=(None, 0), b=(256, 10 ** 9))       # large enough, not there, an address
    assert h.closed == 0
    with pytest.raises(ValueError, match="^w: 33 elements expected, the tensor has 32"):
        mw._holds(h, w=(z(4, 8), 33))
    assert h.closed == 1


@pytest.mark.gpu
def test_small_weights_are_refused():
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    e = dict(E=4, K=2, max_tokens=4, H=64, I=32, w_gate_up=z(4, 2, 32, 64), w_down=z(4, 64, 32))
    p = dict(H=64, O=40, max_tokens=4, w=z(40, 64), adapters=3, rank=16, a=z(3, 16, 64), b=z(3, 40, 16), scale=z(3, dtype=torch.float32))
    mw.Experts(**e).close()
    mw.Projection(**p).close()
    for kind, good, names in ((mw.Experts, e, ("w_gate_up", "w_down")), (mw.Projection, p, ("w", "a", "b", "scale"))):
        for name in names:
            with pytest.raises(ValueError, match=f"^{name}: .* elements expected"):
                kind(**{**good, name: good[name][:-1]})
