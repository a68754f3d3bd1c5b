"""mw_route with MW_ROUTE_SCORE_BIAS: the choice goes by score + bias, weights are the scores.

Reference in float64.  The kernel's keys are float32, so two experts whose exact keys lie closer than their errors may change places:
  sigmoid: exp to 2 units in the last place, one sum, one division:                    |d score| <= 4 * 2^-23 score
  softmax: as for weights, n terms, arguments to half a unit of |l - m|:               |d score| <= (n + 16 + 2 max|l - m|) 2^-23 score
  key: one rounding of the sum:                                                        |d key| <= |d score| + 2^-24 |key|
Ids have to be those of the reference wherever neighbours in its order are further apart than the two keys' errors; everywhere the
chosen experts have to be in order, and before all others, up to these errors.  Weights as for the other forms (test_gpu_route.py).
"""
import numpy as np
import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw
from test_gpu_route import run

pytestmark = pytest.mark.gpu

SIG, REN, SB = mw.MW_ROUTE_SIGMOID, mw.MW_ROUTE_RENORMALISE, mw.MW_ROUTE_SCORE_BIAS
EPS = 2.0 ** -23


def reference(logits, bias, flags):
    """Scores, keys (-inf: never chosen) and the keys' error bounds, in float64."""
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    with np.errstate(over="ignore", invalid="ignore"):
        if flags & SIG:
            score = np.where(l >= 0, 1 / (1 + np.exp(-np.abs(l))), np.exp(-np.abs(l)) / (1 + np.exp(-np.abs(l))))
            off = 4 * EPS * score
        else:
            m = l.max(1, keepdims=True)
            p = np.exp(l - m)
            score = p / p.sum(1, keepdims=True)
            spread = np.where(np.isfinite(l), m - l, 0).max(1, keepdims=True)
            off = (l.shape[1] + 16 + 2 * spread) * EPS * score
    key = np.where(np.isfinite(l), score + bias, -np.inf)
    key = np.where(np.isnan(key), -np.inf, key)
    return score, key, off + np.where(np.isfinite(key), np.abs(key), 0) * EPS / 2


def check(logits, bias, K, flags, scale, got):
    ids, w = got
    score, key, off = reference(logits, bias, flags)
    T, E = logits.shape
    clear = 0
    for t in range(T):
        n = min(K, int((key[t] > -np.inf).sum()))
        order = sorted(range(E), key=lambda e: (-key[t, e], e))
        row = ids[t, :n].tolist()
        assert len(set(row)) == n and all(0 <= e < E and key[t, e] > -np.inf for e in row) and (ids[t, n:] == -1).all() and (w[t, n:] == 0).all()
        for j, e in enumerate(row):                  # nobody that comes later, chosen or not, is before it beyond the errors
            rest = [r for r in range(E) if r not in row[:j + 1]]
            if rest:
                assert (key[t, rest] - off[t, rest]).max() <= key[t, e] + off[t, e]
        near = [key[t, order[j]] - key[t, order[j + 1]] <= off[t, order[j]] + off[t, order[j + 1]] for j in range(min(n, E - 1)) if key[t, order[j + 1]] > -np.inf]
        if not any(near):
            assert row == order[:n]
            clear += 1
        s = score[t, row]
        want = scale * (s / s.sum() if flags & REN else s)
        l = logits[t][np.isfinite(logits[t])].astype(np.float64)
        tol = (E + 16 + 2 * (l.max() - l.min() if l.size else 0)) * EPS
        assert np.all(np.abs(w[t, :n] - want) <= tol * np.abs(want) + 1e-37)
    return clear


@pytest.mark.parametrize("T,E,K", [(1, 1, 1), (1, 256, 8), (5, 31, 4), (9, 33, 33), (64, 64, 8), (100, 256, 8), (17, 384, 8), (6, 1000, 40), (3, 1024, 64)])
@pytest.mark.parametrize("flags", [SIG, SIG | REN, 0, REN])
def test_choice_by_biased_scores(T, E, K, flags):
    torch = torch_mod()
    rng = np.random.default_rng(100 * T + E + flags)
    logits = (rng.standard_normal((T, E)) + 0.5 * rng.standard_normal(E)).astype(np.float32)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32) / (1 if flags & SIG else E)
    got = run(torch.from_numpy(logits).cuda(), torch.from_numpy(bias).cuda(), K, flags | SB, 2.5)
    check(logits, bias.astype(np.float64), K, flags, 2.5, got)


def test_it_is_another_choice_than_by_biased_logits():
    torch = torch_mod()
    rng = np.random.default_rng(3)
    logits = rng.standard_normal((200, 256)).astype(np.float32)
    bias = (0.1 * rng.standard_normal(256)).astype(np.float32)
    l, b = torch.from_numpy(logits).cuda(), torch.from_numpy(bias).cuda()
    by_score = run(l, b, 8, SIG | REN | SB, 1.0)
    by_logit = run(l, b, 8, SIG | REN, 1.0)
    assert check(logits, bias.astype(np.float64), 8, SIG | REN, 1.0, by_score) >= 190
    assert (np.sort(by_score[0], 1) != np.sort(by_logit[0], 1)).any(1).mean() > 0.9


@pytest.mark.parametrize("flags", [SIG, REN])
def test_without_a_bias_it_changes_nothing(flags):
    torch = torch_mod()
    l = torch.randn(70, 96, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 30      # sigmoid saturates: the logits' order stays
    one, two = run(l, None, 8, flags, 1.0), run(l, None, 8, flags | SB, 1.0)
    assert np.array_equal(one[0], two[0]) and np.array_equal(one[1], two[1])


@pytest.mark.parametrize("flags", [SIG, SIG | REN, 0, REN])
def test_masked_experts_empty_rows_and_ties(flags):
    """A masked expert's score is 0, not its key: a bias does not bring it back.  Equal keys: the lowest experts."""
    torch = torch_mod()
    rng = np.random.default_rng(9)
    logits = rng.standard_normal((6, 70)).astype(np.float32)
    logits[0] = -np.inf
    logits[1] = np.nan
    logits[2, 3:] = -np.inf
    logits[3, ::2] = np.nan
    logits[4] = 0.25
    bias = np.full(70, 0.5, np.float32)
    bias[69] = -np.inf
    bias[68] = np.nan
    ids, w = run(torch.from_numpy(logits).cuda(), torch.from_numpy(bias).cuda(), 8, flags | SB, 1.0)
    assert (ids[:2] == -1).all() and (w[:2] == 0).all()
    assert sorted(ids[2, :3].tolist()) == [0, 1, 2] and (ids[2, 3:] == -1).all()
    assert (ids[3] % 2 == 1).all() and not np.isin(ids, (68, 69)).any()
    assert ids[4].tolist() == list(range(8))
    rows = [2, 3, 4, 5]
    check(logits[rows], bias.astype(np.float64), 8, flags, 1.0, (ids[rows], w[rows]))


def test_bf16_logits():
    torch = torch_mod()
    rng = np.random.default_rng(4)
    l = torch.from_numpy(rng.standard_normal((50, 160)).astype(np.float32)).cuda().bfloat16()
    bias = (0.1 * rng.standard_normal(160)).astype(np.float32)
    got = run(l, torch.from_numpy(bias).cuda(), 6, SIG | REN | SB, 2.5)
    check(l.float().cpu().numpy(), bias.astype(np.float64), 6, SIG | REN, 2.5, got)
