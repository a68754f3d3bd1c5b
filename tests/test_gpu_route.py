"""mw_route against a plain float64 / exact-integer statement of its definition.

Ids have no tolerance: the choice goes by float32 keys (one exact addition), ties to the lowest expert.  Weights: every
exponential is good to 2 units in the last place of float32 (2^-23 relative), its argument l - m to half a unit of |l - m|, a sum of n
terms to n * 2^-24; so a weight is within (n + 16 + 2 max|l - m|) * 2^-23 relative of the exact one, n = E terms at most.
"""
import numpy as np
import pytest

from gpu_util import Guarded, torch_mod
from paper_2605_22428_b200 import binding as mw

pytestmark = pytest.mark.gpu

SIG, REN = mw.MW_ROUTE_SIGMOID, mw.MW_ROUTE_RENORMALISE


def plain(logits: np.ndarray, bias, K: int, flags: int, scale: float):
    """Definition, token by token, in float64 (keys in float32).  Returns ids, weights."""
    T, E = logits.shape
    ids = np.full((T, K), -1, np.int32)
    w = np.zeros((T, K))
    for t in range(T):
        l32 = logits[t].astype(np.float32)
        key = l32 if bias is None else l32 + bias
        order = sorted((e for e in range(E) if key[e] > -np.inf), key=lambda e: (-key[e], e))[:K]
        l = np.where(np.isnan(l32), -np.inf, l32).astype(np.float64)
        if not order:
            continue
        c = l[order]
        if flags & SIG:
            logp = np.minimum(c, 0) - np.log1p(np.exp(-np.abs(c)))
        elif flags & REN:
            logp = c
        else:
            m = l.max()
            logp = c - m - np.log(np.exp(l - m).sum())
        if flags & REN:
            logp = logp - logp.max()
            logp = logp - np.log(np.exp(logp).sum())
        ids[t, :len(order)] = order
        w[t, :len(order)] = np.exp(logp) * scale
    return ids, w


def run(logits_d, bias_d, K, flags, scale, T=None, E=None, stride=0):
    torch = torch_mod()
    T = logits_d.shape[0] if T is None else T
    E = logits_d.shape[1] if E is None else E
    ids, w = Guarded(T * K * 4), Guarded(T * K * 4)
    mw.mw_route(logits_d, bias_d, T, E, K, flags, scale, ids.ptr(), w.ptr(), logits_stride_bytes=stride)
    torch.cuda.synchronize()
    assert ids.guards_intact() and w.guards_intact()
    return ids.host().view(np.int32).reshape(T, K), w.host().view(np.float32).reshape(T, K)


def check(logits: np.ndarray, bias, K, flags, scale, got):
    ids, w = plain(logits, bias, K, flags, scale)
    assert np.array_equal(got[0], ids)
    finite = logits[np.isfinite(logits)]
    spread = float(finite.max() - finite.min()) if finite.size else 0.0
    tol = (logits.shape[1] + 16 + 2 * spread) * 2.0 ** -23
    assert np.all(np.abs(got[1] - w) <= tol * np.abs(w) + 1e-37)


SHAPES = [(1, 1, 1), (1, 256, 8), (3, 2, 2), (5, 31, 4), (7, 32, 32), (9, 33, 33), (64, 64, 8), (33, 100, 6), (130, 256, 8), (17, 384, 8),
          (4, 1000, 64), (2, 1024, 40), (513, 160, 6)]


@pytest.mark.parametrize("T,E,K", SHAPES)
@pytest.mark.parametrize("flags", [0, SIG, REN, SIG | REN])
def test_choice_and_weights(T, E, K, flags):
    torch = torch_mod()
    rng = np.random.default_rng(1000 * T + E + flags)
    logits = (2 * rng.standard_normal((T, E))).astype(np.float32)
    bias = (0.3 * rng.standard_normal(E)).astype(np.float32) if (T + flags) % 2 else None
    got = run(torch.from_numpy(logits).cuda(), None if bias is None else torch.from_numpy(bias).cuda(), K, flags, 2.5)
    check(logits, bias, K, flags, 2.5, got)


@pytest.mark.parametrize("flags", [0, REN])
def test_bf16_scores_and_ties(flags):
    """Scores on a coarse grid: most tokens have ties at the boundary; the lowest experts win."""
    torch = torch_mod()
    rng = np.random.default_rng(5)
    logits = (rng.integers(-6, 7, (300, 96)) / 4).astype(np.float32)
    logits[0] = 0.0
    logits[1, ::2], logits[1, 1::2] = 0.0, -0.0          # equal as numbers
    got = run(torch.from_numpy(logits).cuda().bfloat16(), None, 8, flags, 1.0)
    check(logits, None, 8, flags, 1.0, got)
    assert got[0][0].tolist() == list(range(8)) and got[0][1].tolist() == list(range(8))


@pytest.mark.parametrize("flags", [0, SIG, REN, SIG | REN])
def test_masked_experts_and_empty_rows(flags):
    """-inf and NaN logits are never chosen; the type's lowest value is an ordinary number; a row may be left with fewer than K, or none."""
    torch = torch_mod()
    rng = np.random.default_rng(9)
    logits = rng.standard_normal((8, 70)).astype(np.float32)
    logits[0] = -np.inf
    logits[1] = np.nan
    logits[2, 3:] = -np.inf
    logits[3, ::2] = np.nan
    logits[4, 5:] = np.finfo(np.float32).min
    logits[5, :64] = -np.inf
    logits[6] = np.finfo(np.float32).min
    T, E = logits.shape
    ids, w = run(torch.from_numpy(logits).cuda(), None, 8, flags, 1.0)
    assert (ids[0] == -1).all() and (w[0] == 0).all() and (ids[1] == -1).all() and (w[1] == 0).all()
    assert (ids[2][3:] == -1).all() and (w[2][3:] == 0).all()
    assert (ids[5][6:] == -1).all() and sorted(ids[5][:6].tolist()) == list(range(64, 70))
    assert ids[6].tolist() == list(range(8))
    rows = [2, 3, 5, 7]
    check(logits[rows], None, 8, flags, 1.0, (ids[rows], w[rows]))
    assert np.isfinite(w).all()
    if flags & REN:
        assert np.allclose(w[[2, 3, 4, 5, 6, 7]].sum(1), 1, atol=1e-5)


def test_renormalised_weights_of_very_small_scores():
    """Scores whose sigmoid underflows, and a bias that picks experts whose softmax underflows: the ratio is still that of the formula."""
    torch = torch_mod()
    logits = np.full((2, 40), -150.0, np.float32)
    logits[0, :8] = -150.0 + np.arange(8) / 8
    logits[1, 39] = 150.0
    bias = np.zeros(40, np.float32)
    bias[:8] = 1000.0
    for flags in (REN, SIG | REN):
        got = run(torch.from_numpy(logits).cuda(), torch.from_numpy(bias).cuda(), 8, flags, 1.0)
        check(logits, bias, 8, flags, 1.0, got)
        assert np.allclose(got[1].sum(1), 1, atol=1e-6)


def test_strided_rows_and_another_stream():
    torch = torch_mod()
    rng = np.random.default_rng(11)
    wide = torch.from_numpy(rng.standard_normal((50, 300)).astype(np.float32)).cuda()
    logits = wide[:, 7:7 + 90]
    ids = torch.full((50, 6), -7, dtype=torch.int32, device="cuda")
    w = torch.zeros(50, 6, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mw.mw_route(logits, None, 50, 90, 6, REN, 1.0, ids, w, logits_stride_bytes=wide.stride(0) * 4)
    side.synchronize()
    check(logits.cpu().numpy(), None, 6, REN, 1.0, (ids.cpu().numpy(), w.cpu().numpy()))


def test_refusals():
    torch = torch_mod()
    l, ids, w = torch.zeros(4, 16, device="cuda"), torch.zeros(4, 4, dtype=torch.int32, device="cuda"), torch.zeros(4, 4, device="cuda")

    def rc(logits=l, T=4, E=16, K=4, flags=0, i=ids, ww=w, stride=0, bias=None):
        return mw.mw_route(logits, bias, T, E, K, flags, 1.0, i, ww, logits_stride_bytes=stride, check=False)

    assert rc() == mw.MW_OK and rc(T=0) == mw.MW_OK
    for bad in (dict(T=-1), dict(E=0), dict(K=0), dict(K=17), dict(E=1025), dict(flags=4), dict(i=None), dict(ww=None), dict(stride=60), dict(stride=-64)):
        assert rc(**bad) == mw.MW_ERR_INVALID_ARG, bad
    assert mw.lib().mw_route(l.data_ptr(), 2, 0, None, 4, 16, 4, 0, 1.0, ids.data_ptr(), w.data_ptr(), None) == mw.MW_ERR_INVALID_ARG
    assert mw.lib().mw_route(l.data_ptr() + 2, 0, 0, None, 3, 16, 4, 0, 1.0, ids.data_ptr(), w.data_ptr(), None) == mw.MW_ERR_ALIGNMENT
    assert rc(stride=66) == mw.MW_ERR_ALIGNMENT
    assert rc(bias=l.data_ptr() + 1) == mw.MW_ERR_ALIGNMENT
    with pytest.raises(TypeError):
        mw.mw_route(l.double(), None, 4, 16, 4, 0, 1.0, ids, w)
    torch.cuda.synchronize()
