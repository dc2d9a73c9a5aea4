"""Log probabilities row by row: each value of each row within a bound that its own row sets.

x - m is exact to its own rounding, whatever the size of the logits, so the bound has no term in their size: under 400
roundings of S and T (a lane adds 32 numbers at most at a time, and the sums are joined), exponents off by |x - m| 2^-23,
which S weighs with e^(x - m) (their mean |x - m| is below log(vocab) < 12), and the roundings of x - m, log S and the
difference of the two."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.test_gpu_cache_ops import BF16, F32, _dev, _np, _rng

pytestmark = pytest.mark.gpu


def _check(x, given, k, got):
    lp, ent, tl, ti = (_np(t) for t in got)
    with np.errstate(divide="ignore", invalid="ignore"):
        w, h = oc.logprobs(_np(x))
    w = np.where(w <= -(2.0 ** 128 - 2.0 ** 103), -np.inf, w)          # the results are float32
    ids = oc.top(_np(x), k)
    assert np.array_equal(ti, ids)
    for r in range(x.shape[0]):
        for name, g, want in (("given", lp[r], w[r, given[r].cpu().numpy()]), ("top", tl[r], w[r, ids[r]])):
            fin = np.isfinite(want)
            assert np.array_equal(g[~fin], want[~fin], equal_nan=True), (r, name)
            off = np.abs(g[fin] - want[fin])
            assert (off <= 400 * 2.0 ** -24 + 2.0 ** -22 * (np.abs(want[fin]) + 12)).all(), (r, name, off.max())
        assert np.isnan(ent[r]) if np.isnan(h[r]) else abs(ent[r] - h[r]) <= 400 * 2.0 ** -24 + 2.0 ** -22 * (h[r] + 12) + h[r] * 400 * 2.0 ** -23, r


def _given(x, r):
    """The largest, a masked one if there is one, the ends and some others."""
    some = r.integers(0, x.shape[1], (x.shape[0], 4))
    ends = np.stack([x.argmax(1), x.argmin(1), np.zeros(len(x)), np.full(len(x), x.shape[1] - 1)], 1)
    return _dev(np.concatenate([some, ends], 1), torch.int32)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("vocab", [700, 8100, 20001, 152064])
def test_rows_far_from_zero_and_masked(gpu_lib, act, vocab):
    """Rows about 0, +-65536 (both sides of where the exponent is formed another way), +-70000, 1e6, -1e30, and rows
    masked with the type's lowest value or with -infinity, in part or wholly."""
    r = _rng(vocab, 13)
    low = torch.finfo(act).min
    x = r.normal(size=(14, vocab)) * 3
    for i, at in enumerate([0, 65530, -65530, 65544, -65544, 70000, -70000, 1e6, -1e30]):
        x[i] += at
    x[9, 5:] = low
    x[10, ::3] = low
    x[11] = low
    x[12, 1::2] = -np.inf
    x[13] = np.where(x[13] > 0, 3e38, -3e38)
    xt = _dev(x, F32).to(act)
    given = _given(_np(xt), r)
    _check(xt, given, 20, gpu_lib.logprobs(xt, given=given, n_top=20))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("vocab", [700, 9001, 152064])
@pytest.mark.parametrize("low", [-np.inf, None, -1e4])
def test_rows_of_few_tokens_left(gpu_lib, act, vocab, low):
    r = _rng(vocab, 15)
    x = np.full((8, vocab), torch.finfo(act).min if low is None else low)
    for i, n in enumerate((1, 5, 19, 31, 32, 40, 300)):
        at = (0, vocab - n, 77)[i % 3]
        x[i, at:at + n] = r.normal(size=n) + (0, 5e4, -2e5)[i % 3]
    x[7, 3] = 1.0
    xt = _dev(x, F32).to(act)
    given = _given(_np(xt), r)
    _check(xt, given, 32, gpu_lib.logprobs(xt, given=given, n_top=32))
