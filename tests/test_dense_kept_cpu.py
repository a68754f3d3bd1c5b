"""The binding of the gated block: the types of what a forward call keeps, as far as no device is needed."""
import pytest

from paper_2605_22428_b200 import binding as mw
from paper_2605_22428_b200 import build as mwbuild
from test_dense_cpu import without_a_handle


@pytest.fixture(scope="module", autouse=True)
def lib():
    mwbuild.build_library()
    return mw.lib()


def test_gate_and_up_may_be_kept_in_the_rows_type():
    """float32 or the handle's type are looked at for their place (on the CPU here), any other type is refused by name."""
    import torch
    g = without_a_handle(mw.Gated)
    for dtype in (torch.float32, torch.bfloat16):
        kept = torch.zeros(4, 80, dtype=dtype)
        with pytest.raises(TypeError, match="^gate_up: .* on the GPU"):
            g.mw_gated_forward(256, 4, 512, gate_up=kept, stream=4)
        with pytest.raises(TypeError, match="^gate_up: .* on the GPU"):
            g.mw_gated_backward(256, kept, 768, 4, dx=1024, stream=4)
    for dtype in (torch.float16, torch.float64):
        with pytest.raises(TypeError, match="^gate_up: a tensor of"):
            g.mw_gated_forward(256, 4, 512, gate_up=torch.zeros(4, 80, dtype=dtype), stream=4)
