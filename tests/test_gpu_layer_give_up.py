"""A call whose waits give up leaves nothing behind that could reach the next kernel on its SMs: loads that were under way land before
its blocks end.  Calls that give up (mw_*_test_skew_waits) take turns with calls of another handle, nothing waits in between; the other
handle's bits do not change, and the first handle is right again once its status has been read.
"""
import pytest

import test_gpu_experts as experts
import test_gpu_project as project
from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [3, 120])
def test_experts(T):
    torch = torch_mod()
    a, b = (experts.make(T, 16, 4, 512, 256, seed=s) for s in (1, 2))
    with mw.Experts(16, 4, T, 512, 256, a["wgu"], a["wd"], flags=mw.MW_FLAG_SHORT_WAITS) as ha, mw.Experts(16, 4, T, 512, 256, b["wgu"], b["wd"]) as hb:
        want_a, want_b = experts.forward(a, handle=ha)[0], experts.forward(b, handle=hb)[0]
        experts.check(a, want_a)
        experts.check(b, want_b)
        dropped = torch.zeros(T, 512, dtype=torch.bfloat16, device="cuda")
        y = torch.zeros(20, T, 512, dtype=torch.bfloat16, device="cuda")
        for i in range(20):
            ha.mw_experts_test_skew_waits()
            ha.mw_experts_forward(a["x"], a["ids"], a["weights"], T, dropped)
            hb.mw_experts_forward(b["x"], b["ids"], b["weights"], T, y[i])
        torch.cuda.synchronize()
        assert ha.mw_experts_get_status() == mw.MW_ERR_TIMEOUT and hb.mw_experts_get_status() == mw.MW_OK
        assert bool((y.view(torch.int16) == want_b.view(torch.int16)).all())
        got, status = experts.forward(a, handle=ha)
        assert status == mw.MW_OK and torch.equal(got, want_a)


@pytest.mark.parametrize("T,r", [(5, 16), (200, 64)])
def test_project(T, r):
    torch = torch_mod()
    a, b = (project.make(T, 512, 640, 4, r, seed=s) for s in (1, 2))
    with mw.Projection(512, 640, T, a["w"], 4, r, a["a"], a["b"], a["scale"], flags=mw.MW_FLAG_SHORT_WAITS) as ha, \
            mw.Projection(512, 640, T, b["w"], 4, r, b["a"], b["b"], b["scale"]) as hb:
        want_a, want_b = project.forward(a, handle=ha)[0], project.forward(b, handle=hb)[0]
        project.check(a, want_a)
        project.check(b, want_b)
        dropped = torch.zeros(T, 640, dtype=torch.bfloat16, device="cuda")
        y = torch.zeros(20, T, 640, dtype=torch.bfloat16, device="cuda")
        for i in range(20):
            ha.mw_project_test_skew_waits()
            ha.mw_project_forward(a["x"], a["ids"], T, dropped)
            hb.mw_project_forward(b["x"], b["ids"], T, y[i])
        torch.cuda.synchronize()
        assert ha.mw_project_get_status() == mw.MW_ERR_TIMEOUT and hb.mw_project_get_status() == mw.MW_OK
        assert bool((y.view(torch.int16) == want_b.view(torch.int16)).all())
        got, status = project.forward(a, handle=ha)
        assert status == mw.MW_OK and torch.equal(got, want_a)
