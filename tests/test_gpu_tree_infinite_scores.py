"""Rows of tree attention all of whose scores are -infinity have no softmax (NaN); a row that sees nothing is zero."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache_ops import Batch, _check_tree, _dev, _np, _rng

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])                # an e4m3 cache holds no infinity
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,n", [(2, 5), (8, 6), (24, 12)])
@pytest.mark.parametrize("ctx", [0, 20, 3000])
def test_rows_of_infinite_scores(gpu_lib, kind, d, n_q, n, ctx):
    nova = gpu_lib
    n_kv = 2
    bt = Batch(nova, [ctx, 7], [n, n], n_kv, d, kind, seed=ctx + n).fill(ctx + n, stale=float("nan"))
    c = bt.cache
    low = bt.k[0].copy()
    low[:, 0, 3] = -np.inf                                       # one KV head of the first sequence: every cached token
    low[ctx + 2:, 0, 3] = 1.0                                    # and the first two drafted ones
    for t in range(ctx + 2):
        blk, s = bt.place(0, t)
        c.k[0, blk, 0, s, 3] = float("-inf")
    for t in range(ctx + 2, ctx + n):
        blk, s = bt.place(0, t)
        c.k[0, blk, 0, s, 3] = 1.0
    bt.k[0] = low
    q = _dev(np.abs(_rng(n, n_q).normal(size=(bt.total, n_q, d))) + 0.25, c.dtype)   # no 0 times infinity
    masks = [1, 2, 0, 3, 0b10101, *[1 << 2] * (n - 5)] + [0] * n
    mask = torch.tensor(masks, dtype=torch.int64, device="cuda")
    out = nova.tree_attention(c, bt.desc, q, mask=mask)
    _check_tree(bt, q, masks, out, d ** -0.5)
    got, g = _np(out), n_q // n_kv
    assert np.isnan(got[[0, 1, 3], :g]).all() and np.isfinite(got[4:n]).all()
    assert (np.isnan(got[2, :g]).all() if ctx else (got[2] == 0).all())


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("n_q", [2, 24])
def test_rows_of_missing_blocks_see_nothing(gpu_lib, kind, n_q):
    """Tokens whose blocks do not exist are not seen, whatever the context says: zeros, one split and several."""
    nova = gpu_lib
    for ctx in (40, 3000):
        bt = Batch(nova, [ctx], [3], 2, 64, kind, seed=5).fill(5, stale=float("nan"))
        rows = nova.Rows(bt.desc.row_start, bt.desc.ctx, torch.full_like(bt.desc.tables, -1), rows=3, max_rows=3, max_ctx=bt.max_ctx)
        q = _dev(_rng(5).normal(size=(3, n_q, 64)), bt.cache.dtype)
        assert (nova.tree_attention(bt.cache, rows, q) == 0).all()
