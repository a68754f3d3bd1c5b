"""The streaming engine's equal pieces: where a round of whole tiles has gone before and sums are long (64 steps of 64 elements or more), the
tiles left over are cut into as many equal pieces as there are shares, so that a piece may end one tile and begin the next, cuts
fall anywhere, and a tile has one to five contributors.  Each case asserts that it is such a one: more than 148 tiles, at least 37 left over,
and enough units of `steps` steps in these for `least` in every piece.

Tolerances are those of test_gpu_experts.py and test_gpu_project.py.
"""
import pytest

import test_gpu_experts as experts
import test_gpu_project as project
from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw

pytestmark = pytest.mark.gpu


def equal_pieces(tiles: int, depth: int, steps: int, least: int) -> bool:
    torch = torch_mod()
    shares = torch.cuda.get_device_properties(0).multi_processor_count
    return tiles > shares and tiles % shares * 4 >= shares and -(-depth // 64) >= 64 and tiles % shares * -(-depth // (64 * steps)) >= shares * least


# gate and up cut (H long), down cut (I long); tokens gathered, copied, in several tiles of an expert
@pytest.mark.parametrize("T,E,K,H,I,product", [(1, 8, 8, 4160, 1600, 0), (20, 8, 8, 4160, 1600, 0), (1, 8, 8, 3200, 4224, 1), (300, 2, 2, 4160, 3008, 0),
                                               (140, 4, 2, 6400, 4112, 1)])
def test_experts(T, E, K, H, I, product):
    torch = torch_mod()
    few = T * K <= min(48 * E, 2048)
    tiles = -(-T // (128 if few else 256)) * E * (-(-H // 128) if product else -(-I // 64))
    assert equal_pieces(tiles, I if product else H, 4 if few else 2, 4 if few else 8)
    d = experts.make(T, E, K, H, I, seed=T)
    with mw.Experts(E, K, T, H, I, d["wgu"], d["wd"]) as h:
        want, status = experts.forward(d, handle=h)
        assert status == mw.MW_OK
        experts.check(d, want)
        for blocks in (0, 0, 147, 60, 5, 1):
            if blocks:
                h.mw_experts_test_few_blocks(blocks)
            got, status = experts.forward(d, handle=h)
            assert status == mw.MW_OK and torch.equal(got, want)
        y = torch.zeros(50, T, H, dtype=torch.bfloat16, device="cuda")
        for i in range(50):
            h.mw_experts_forward(d["x"], d["ids"], d["weights"], T, y[i])
        torch.cuda.synchronize()
        assert h.mw_experts_get_status() == mw.MW_OK and bool((y.view(torch.int16) == want.view(torch.int16)).all())


@pytest.mark.parametrize("T,O,n,r", [(1, 24325, 2, 16), (20, 24325, 0, 0), (50, 25600, 5, 16), (100, 24325, 3, 32), (300, 12160, 4, 16), (300, 12160, 0, 0)])
def test_project(T, O, n, r):
    torch = torch_mod()
    assert equal_pieces(-(-T // 256) * -(-O // 128), 4160, 4 if T <= 32 else 2 if T <= 64 else 1, 2)
    d = project.make(T, 4160, O, n, r, seed=T, segment=3)
    with mw.Projection(4160, O, T, d["w"], n, r, d["a"], d["b"], d["scale"]) as h:
        want, status = project.forward(d, handle=h)
        assert status == mw.MW_OK
        project.check(d, want)
        y = torch.zeros(20, T, O, dtype=torch.bfloat16, device="cuda")
        for i in range(20):
            h.mw_project_forward(d["x"], d["ids"], T, y[i])
        torch.cuda.synchronize()
        assert h.mw_project_get_status() == mw.MW_OK and bool((y.view(torch.int16) == want.view(torch.int16)).all())


def test_low_rank_values_of_many_adapters():
    """The same cuts in the product that makes the low-rank values: 10 tiles of 64 tokens, 19 or 20 adapters of rank 128 in each, one to a tile of rows."""
    torch = torch_mod()
    d = project.make(640, 4160, 256, 20, 128, seed=1, none=0.0)
    groups = sum(len(set(d["ids"][i:i + 64].tolist())) for i in range(0, 640, 64))
    assert equal_pieces(groups, 4160, 2, 4)
    with mw.Projection(4160, 256, 640, d["w"], 20, 128, d["a"], d["b"], d["scale"]) as h:
        want, status = project.forward(d, f32=True, handle=h)
        assert status == mw.MW_OK
        project.check(d, want, f32=True)
        for _ in range(10):
            got, status = project.forward(d, f32=True, handle=h)
            assert status == mw.MW_OK and torch.equal(got, want)
