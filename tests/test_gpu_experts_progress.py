"""A call of mw_experts ends, with the same bits, however few of its blocks run at a time: blocks wait only for work that a running
block has begun.  mw_experts_test_few_blocks launches fewer blocks than there are shares, which is what a partition of the device, or calls on
other streams that hold the other SMs, come to for the blocks that do run.

Shapes: tokens gathered where they lie and tokens copied to the list's order (more than sixteen of an expert), tiles cut between shares of both
products, whole rounds of tiles, more shares than work, nothing to do at all.  Bits are compared with the full launch, which is held to the formula.
"""
import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_experts import check, forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,K,H,I,first,count", [(1, 8, 4, 512, 256, 0, 8), (40, 4, 2, 1024, 144, 0, 4), (300, 6, 3, 320, 96, 2, 3), (64, 32, 4, 1024, 512, 0, 32),
                                                   (2, 4, 2, 4096, 64, 0, 4), (5, 16, 1, 64, 16, 12, 4)])
def test_few_blocks_give_the_same_bits(T, E, K, H, I, first, count):
    torch = torch_mod()
    d = make(T, E, K, H, I, first=first, count=count, seed=T)
    with mw.Experts(E, K, T, H, I, d["wgu"], d["wd"], expert_first=first, expert_count=count) as h:
        want, status = forward(d, handle=h)
        assert status == mw.MW_OK
        check(d, want)
        for blocks in (1, 2, 3, 17, 100, 147, 148, 1000):
            h.mw_experts_test_few_blocks(blocks)
            got, status = forward(d, handle=h)
            assert status == mw.MW_OK and torch.equal(got, want), blocks
            got, status = forward(d, handle=h)          # the call after it has all blocks again
            assert status == mw.MW_OK and torch.equal(got, want), blocks


def test_few_blocks_with_nothing_to_do():
    torch = torch_mod()
    d = make(9, 4, 2, 64, 32, seed=1, ids=torch.full((9, 2), -1, dtype=torch.int32))
    with mw.Experts(4, 2, 9, 64, 32, d["wgu"], d["wd"]) as h:
        for blocks in (1, 60):
            h.mw_experts_test_few_blocks(blocks)
            got, status = forward(d, handle=h)
            assert status == mw.MW_OK and bool((got == 0).all())


def test_few_blocks_from_call_to_call():
    """Calls with different numbers of blocks follow one another, nothing waits in between: tickets and counts begin anew with each."""
    torch = torch_mod()
    d = make(120, 16, 4, 512, 128, seed=3)
    with mw.Experts(16, 4, 120, 512, 128, d["wgu"], d["wd"]) as h:
        want, _ = forward(d, handle=h)
        check(d, want)
        y = torch.zeros(60, 120, 512, dtype=torch.bfloat16, device="cuda")
        for i in range(60):
            if i % 3:
                h.mw_experts_test_few_blocks(1 + 23 * i % 148)
            h.mw_experts_forward(d["x"], d["ids"], d["weights"], 120, y[i])
        torch.cuda.synchronize()
        assert h.mw_experts_get_status() == mw.MW_OK
        assert bool((y.view(torch.int16) == want.view(torch.int16)).all())


def test_refusals():
    d = make(2, 2, 1, 64, 16)
    with mw.Experts(2, 1, 2, 64, 16, d["wgu"], d["wd"]) as h:
        for blocks in (0, -1):
            with pytest.raises(mw.MwError) as err:
                h.mw_experts_test_few_blocks(blocks)
            assert err.value.code == mw.MW_ERR_INVALID_ARG
    assert mw.lib().mw_experts_test_few_blocks(None, 1) == mw.MW_ERR_INVALID_ARG
