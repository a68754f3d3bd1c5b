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
