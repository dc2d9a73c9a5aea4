"""Rows whose tokens lie outside 0 .. max_ctx - 1, and row starts that are not what they should be: what the operators
write, read and leave alone, element by element."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.test_gpu_cache_ops import F32, TYPES, Batch, _dev, _np, _rng, _tree_tolerance

pytestmark = pytest.mark.gpu

BIG = 1 << 30
N_Q, N_KV, D = 4, 2, 64


def _rows_of(starts, ctx, rows, max_rows):
    """(first row, rows, ctx) of every sequence as include/nova.h defines them."""
    out = []
    for b, c in enumerate(ctx):
        r0 = min(max(starts[b], 0), rows)
        out.append((r0, min(min(max(starts[b + 1], r0), rows) - r0, max_rows), c))
    return out


def _desc(nova, bt, starts, ctx, rows, max_rows, max_ctx):
    return nova.Rows(_dev(np.array(starts), torch.int32), _dev(np.array(ctx), torch.int32), bt.desc.tables, rows=rows,
                     max_rows=max_rows, max_ctx=max_ctx)


# tokens past the bound (wholly, in part, far past), before the sequence, and the last that fit; bounds inside a block
# and at its end
CTX = [30, 31, 33, 34, 50, BIG, -1, -3, -4, -BIG, 0, 16]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("max_ctx", [34, 32])
def test_rows_outside_the_sequence_are_not_kept(gpu_lib, kind, max_ctx):
    nova = gpu_lib
    n, batch = 4, len(CTX)
    bt = Batch(nova, [60] * batch, [0] * batch, N_KV, D, kind, seed=7).fill(7)
    starts = [n * b for b in range(batch + 1)]
    desc = _desc(nova, bt, starts, CTX, n * batch, n, max_ctx)
    r = _rng(7, max_ctx)
    x, y = (_dev(r.normal(size=(n * batch, N_KV, D)), bt.cache.dtype) for _ in "kv")
    if kind == "e4m3":
        xv, yv = oc.quantise(_np(x))[0], oc.quantise(_np(y))[0]
    else:
        xv, yv = _np(x), _np(y)
    q = _dev(r.normal(size=(n * batch, N_Q, D)), bt.cache.dtype)
    q_out = nova.kv_append(bt.cache, desc, x, y, q=q)
    assert torch.equal(q_out, q)                              # not rotated: every row comes back, kept or not
    for b, c in enumerate(CTX):
        for j in range(n):
            if 0 <= c + j < max_ctx:
                bt.k[b][c + j], bt.v[b][c + j] = xv[n * b + j], yv[n * b + j]
        for t in range(60):                                   # the kept rows, and every other token as it was
            k, v = bt.stored(b, t)
            assert np.array_equal(k, bt.k[b][t]) and np.array_equal(v, bt.v[b][t]), (c, t)
    k, v = nova.kv_gather(bt.cache, desc, dtype=F32)
    for b, c in enumerate(CTX):
        for j in range(n):
            held = 0 <= c + j < max_ctx
            for got, want in ((k, bt.k[b]), (v, bt.v[b])):
                assert np.array_equal(_np(got[n * b + j]), want[c + j] if held else np.zeros((N_KV, D))), (c, j)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n_q,n", [(4, 4), (24, 4), (24, 16)])
def test_tokens_outside_the_sequence_are_not_seen(gpu_lib, kind, n_q, n):
    nova = gpu_lib
    max_ctx, batch = 34, len(CTX)
    bt = Batch(nova, [60] * batch, [0] * batch, N_KV, D, kind, seed=9).fill(9)
    desc = _desc(nova, bt, [n * b for b in range(batch + 1)], CTX, n * batch, n, max_ctx)
    q = _dev(_rng(9, n_q).normal(size=(n * batch, n_q, D)), bt.cache.dtype)
    out = nova.tree_attention(bt.cache, desc, q)
    for b, c in enumerate(CTX):
        held, before = min(max(c + n, 0), max_ctx), min(max(c, 0), max_ctx)
        masks = [((2 << j) - 1) >> min(max(-c, 0), 64) for j in range(n)]
        k, v, qq = bt.k[b][:held], bt.v[b][:held], _np(q[n * b:n * b + n])
        want, size = oc.tree_attention(qq, k, v, before, masks, D ** -0.5)
        assert (np.abs(_np(out[n * b:n * b + n]) - want) <= _tree_tolerance(kind, qq, k, want, size, D ** -0.5, held)).all(), c


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("starts,ctx", [([0, -5, 8], [30, 30]), ([4, 2, BIG], [-7, BIG]), ([BIG, BIG, BIG], [30, 30]),
                                        ([-BIG, 4, 8], [BIG, -BIG]), ([3, 5, 4], [1, 30])])
def test_only_the_rows_are_written(gpu_lib, kind, starts, ctx):
    """Guards on all sides of every output, and the whole pool before and after."""
    nova = gpu_lib
    rows, max_rows, max_ctx = 10, 4, 34
    bt = Batch(nova, [30, 30], [4, 4], N_KV, D, kind, seed=59, pad_rows=2).fill(59)
    desc = _desc(nova, bt, starts, ctx, rows, max_rows, max_ctx)
    seqs = _rows_of(starts, ctx, rows, max_rows)
    mine = sorted({r for r0, n, _ in seqs for r in range(r0, r0 + n)})
    held = {bt.place(b, c + j) for b, (_, n, c) in enumerate(seqs) for j in range(n) if 0 <= c + j < max_ctx}
    dt = bt.cache.dtype

    def guarded(heads, dtype):
        whole = torch.full((rows + 8, heads + 2, D), 3.0, dtype=dtype, device="cuda")
        return whole, whole[4:4 + rows, 1:1 + heads]

    def check(whole, heads):
        part = whole.clone()
        part[torch.tensor([4 + r for r in mine], dtype=torch.long, device="cuda"), 1:1 + heads] = 3.0
        assert (part == 3.0).all()

    q = _dev(_rng(1).normal(size=(rows, N_Q, D)), dt)
    x = _dev(_rng(2).normal(size=(rows, N_KV, D)), dt)
    before = [t.clone() for t in (bt.cache.k, bt.cache.v)]
    whole, q_out = guarded(N_Q, dt)
    nova.kv_append(bt.cache, desc, x, x, q=q, q_out=q_out)
    check(whole, N_Q)
    assert all(torch.equal(q_out[r], q[r]) for r in mine)
    for blk in range(bt.blocks):
        keep = [s for s in range(16) if (blk, s) not in held]
        assert torch.equal(bt.cache.k[0, blk][:, keep], before[0][0, blk][:, keep])
        assert torch.equal(bt.cache.v[0, blk][:, :, keep], before[1][0, blk][:, :, keep])
    (wk, k_out), (wv, v_out) = guarded(N_KV, F32), guarded(N_KV, F32)
    for slots in (None, _dev(np.arange(rows), torch.int32)):
        nova.kv_gather(bt.cache, desc, slots=slots, k_out=k_out, v_out=v_out)
        check(wk, N_KV)
        check(wv, N_KV)
    for n_q in (N_Q, 24):
        whole, out = guarded(n_q, dt)
        nova.tree_attention(bt.cache, desc, q.repeat(1, n_q // N_Q, 1).contiguous(), out=out)
        check(whole, n_q)


def test_a_context_that_outgrows_its_graph(gpu_lib):
    """A captured append replayed with contexts that pass its bound: what was cached stays."""
    nova = gpu_lib
    bt = Batch(nova, [28, 20], [4, 4], N_KV, D, "e4m3", seed=3).fill(3)
    x = _dev(_rng(3).normal(size=(8, N_KV, D)), torch.bfloat16)
    ctx = bt.desc.ctx
    rows = nova.Rows(None, ctx, bt.desc.tables, max_rows=4, max_ctx=32)
    held = [bt.cache.k.clone(), bt.cache.v.clone()]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nova.kv_append(bt.cache, rows, x, x)
    ctx.copy_(_dev(np.array([32, 40]), torch.int32))
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(bt.cache.k, held[0]) and torch.equal(bt.cache.v, held[1])
        ctx += 1
    ctx.copy_(_dev(np.array([30, 28]), torch.int32))
    g.replay()
    want = oc.quantise(_np(x))[0]
    for b, c, n in ((0, 30, 2), (1, 28, 4)):
        for j in range(n):
            assert np.array_equal(bt.stored(b, c + j)[0], want[4 * b + j])
