"""mw_quantise_rows runs on the current device without a handle that would say which: memory that this device does not reach is refused before anything is launched."""
import ctypes

import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw

pytestmark = pytest.mark.gpu


def test_memory_of_the_host_is_refused():
    torch = torch_mod()
    x, q, scale = torch.randn(4, 64, device="cuda").bfloat16(), torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    host = ctypes.create_string_buffer(4096)
    plain = (ctypes.addressof(host) + 15) & ~15
    good = (x.data_ptr(), q.data_ptr(), scale.data_ptr())
    call = lambda x, q, scale: mw.lib().mw_quantise_rows(x, mw.MW_DTYPE_BF16, 0, 4, 64, 0, q, scale, None)  # noqa: E731
    for at in range(3):
        assert call(*good[:at], plain, *good[at + 1:]) == mw.MW_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert not bool(q.any()) and not bool(scale.any())
    assert call(*good) == mw.MW_OK
    torch.cuda.synchronize()
    assert bool(q.any()) and bool((scale > 0).all())


def test_mapped_host_memory_and_parts_of_allocations():
    """Pinned memory is reached, and so is any place inside an allocation."""
    torch = torch_mod()
    big = torch.randn(100, 64, device="cuda").bfloat16()
    want = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    mw.mw_quantise_rows(big[90:94], 4, 64, *want)
    pinned = big[90:94].cpu().pin_memory()
    got = torch.zeros(4, 64, dtype=torch.int8).pin_memory(), torch.zeros(4).pin_memory()
    stream = torch.cuda.current_stream().cuda_stream or None
    assert mw.lib().mw_quantise_rows(pinned.data_ptr(), mw.MW_DTYPE_BF16, 0, 4, 64, 0, got[0].data_ptr(), got[1].data_ptr(), stream) == mw.MW_OK
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0].cpu()) and torch.equal(got[1], want[1].cpu())
