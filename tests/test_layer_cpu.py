"""CPU-side checks of the serving operators' boundary: struct layouts, and the refusals that need no device (they come before any
CUDA call, so they also hold on a machine without a GPU)."""
import ctypes
import os
import subprocess

import pytest

from paper_2605_22428_b200 import binding as mw
from paper_2605_22428_b200 import build as mwbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    mwbuild.build_library()
    return mw.lib()


def test_struct_layouts_match_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mw.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(mw_experts_config), '
                   'offsetof(mw_experts_config, expert_first), offsetof(mw_experts_config, flags), sizeof(mw_project_config), '
                   'offsetof(mw_project_config, adapters), offsetof(mw_project_config, flags)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    e, p = mw.mw_experts_config, mw.mw_project_config
    assert got == [ctypes.sizeof(e), e.expert_first.offset, e.flags.offset, ctypes.sizeof(p), p.adapters.offset, p.flags.offset]


@pytest.mark.parametrize("change", [dict(E=0), dict(K=0), dict(K=65), dict(max_tokens=0), dict(max_tokens=1025), dict(H=12), dict(H=0), dict(H=65544),
                                    dict(I=40), dict(I=0), dict(expert_first=-1), dict(expert_first=3), dict(expert_count=0), dict(device=-1), dict(flags=2),
                                    dict(K=16, max_tokens=513)])
def test_experts_refuses_bad_configurations(lib, change):
    good = dict(E=4, K=2, max_tokens=8, H=64, I=32, expert_first=0, expert_count=4, device=0, flags=0, reserved=0)
    h = ctypes.c_void_p(1)
    cfg = mw.mw_experts_config(**{**good, **change})
    assert lib.mw_experts_create(ctypes.byref(h), ctypes.byref(cfg), 256, 512) == mw.MW_ERR_INVALID_ARG and not h.value


@pytest.mark.parametrize("change", [dict(H=12), dict(H=0), dict(O=0), dict(max_tokens=0), dict(max_tokens=262145), dict(adapters=-1), dict(rank=12), dict(rank=0),
                                    dict(rank=136), dict(adapters=0), dict(device=-1), dict(flags=2)])
def test_project_refuses_bad_configurations(lib, change):
    good = dict(H=64, O=40, max_tokens=8, adapters=3, rank=16, device=0, flags=0, reserved=0)
    h = ctypes.c_void_p(1)
    cfg = mw.mw_project_config(**{**good, **change})
    assert lib.mw_project_create(ctypes.byref(h), ctypes.byref(cfg), 256, 512, 768, None) == mw.MW_ERR_INVALID_ARG and not h.value


def test_null_and_misaligned_pointers(lib):
    h = ctypes.c_void_p()
    e = mw.mw_experts_config(4, 2, 8, 64, 32, 0, 4, 0, 0, 0)
    p = mw.mw_project_config(64, 40, 8, 3, 16, 0, 0, 0)
    assert lib.mw_experts_create(None, ctypes.byref(e), 256, 512) == mw.MW_ERR_INVALID_ARG
    assert lib.mw_experts_create(ctypes.byref(h), None, 256, 512) == mw.MW_ERR_INVALID_ARG
    assert lib.mw_experts_create(ctypes.byref(h), ctypes.byref(e), None, 512) == mw.MW_ERR_INVALID_ARG
    assert lib.mw_experts_create(ctypes.byref(h), ctypes.byref(e), 256, 520) == mw.MW_ERR_ALIGNMENT
    assert lib.mw_project_create(ctypes.byref(h), ctypes.byref(p), None, 512, 768, None) == mw.MW_ERR_INVALID_ARG
    assert lib.mw_project_create(ctypes.byref(h), ctypes.byref(p), 256, None, 768, None) == mw.MW_ERR_INVALID_ARG
    assert lib.mw_project_create(ctypes.byref(h), ctypes.byref(p), 256, 512, 776, None) == mw.MW_ERR_ALIGNMENT
    assert lib.mw_project_create(ctypes.byref(h), ctypes.byref(p), 256, 512, 768, 2) == mw.MW_ERR_ALIGNMENT
    assert lib.mw_experts_forward(None, 256, 0, 256, None, 1, 256, 0, None) == mw.MW_ERR_INVALID_ARG
    assert lib.mw_project_forward(None, 256, 0, None, 1, 256, 1, 0, None) == mw.MW_ERR_INVALID_ARG
    assert lib.mw_experts_kernel_launches(None) == 0 and lib.mw_project_kernel_launches(None) == 0
    assert lib.mw_experts_destroy(None) == mw.MW_OK and lib.mw_project_destroy(None) == mw.MW_OK


def test_route_refuses_bad_arguments(lib):
    def rc(logits=256, dtype=0, stride=0, bias=None, T=4, E=16, K=4, flags=0, ids=256, w=256):
        return lib.mw_route(logits, dtype, stride, bias, T, E, K, flags, 1.0, ids, w, None)

    assert rc(T=0, logits=None, ids=None, w=None) == mw.MW_OK
    for bad in (dict(T=-1), dict(E=0), dict(E=1025), dict(K=0), dict(K=17), dict(E=128, K=65), dict(dtype=2), dict(flags=4), dict(stride=-4), dict(stride=60),
                dict(logits=None), dict(ids=None), dict(w=None)):
        assert rc(**bad) == mw.MW_ERR_INVALID_ARG, bad
    for bad in (dict(logits=258), dict(stride=66), dict(bias=257), dict(ids=257), dict(w=258), dict(dtype=1, logits=257)):
        assert rc(**bad) == mw.MW_ERR_ALIGNMENT, bad
