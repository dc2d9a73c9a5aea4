"""Verify steps at the real widths (hidden 3584, 28/4 heads of 128; bf16, the fp32 mode stops at heads of 80), where the
QKV projection is cut into K slices on the whole GPU and is not on a partition: drafted trees and single rows against
the oracle, and single rows beside nova_llm_decode.

An 8-bit cache is checked in two parts.  What a step writes is compared with the oracle's K and V; what it answers,
with the oracle attending to the K and V that the cache holds.  In one part it could not be: a value next to the middle
of two 8-bit numbers goes either way with any other rounding before it, a whole step of 2^-3, and the oracle's own
logits move by 0.017 to 0.030 when only its projections are rounded to bf16 before they are quantised."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import cache as oc, vlm
from paper_2509_21301_amd import synth
from tests import stage_cases as sc
from tests.test_gpu_cache_ops import _signed, _tree_mask

pytestmark = pytest.mark.gpu

CFG = dataclasses.replace(synth.LLM_28, layers=2, inter=1024, vocab=4096, name="llm2_width")
# rows of each sequence, at most 8, 9 to 16 and more than 16 in all (the step's three forms), and the most
BATCHES = {3: [1, 1, 1], 7: [3, 0, 4], 13: [5, 1, 7], 20: [1] * 20, 32: [16, 3, 13]}


@pytest.fixture(scope="module")
def weights():
    w = synth.llm_weights(CFG, 0)
    return w, {k: np.asarray(v, np.float64) for k, v in w.items()}


def _step(w, ids, pos, n, kept, masks, held=None):
    """The oracle's step over drafted rows: (logits [rows, vocab], K and V of each layer); ``held``: K and V of the
    rows, per layer, to attend to instead."""
    x, out, store = w["embed"][ids], [], vlm.bf16_store
    starts = np.concatenate([[0], np.cumsum(n)])
    d = CFG.head_dim
    for l in range(CFG.layers):
        p = f"l{l}."
        q, k, v = vlm._qkv(store(vlm.rms_norm(x, w[p + "rms1.g"], CFG.eps)), w, l, CFG, pos, store)
        out.append((k, v))
        if held is not None:
            k, v = held[l]
        att = np.zeros(q.shape)
        for b, m in enumerate(n):
            at = slice(starts[b], starts[b] + m)
            kc, vc = kept[l][b]
            if m:
                att[at] = oc.tree_attention(q[at], np.concatenate([kc, k[at]]), np.concatenate([vc, v[at]]), len(kc), masks[at], d ** -0.5)[0]
        x = x + vlm.linear(store(att).reshape(len(ids), -1), w[p + "o.w"])
        x = x + vlm._mlp(x, w, l, CFG, store)
    return vlm.lm_head(x, w, CFG, store), out


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("cus", [256, 64])
@pytest.mark.parametrize("total", BATCHES)
def test_verify_at_real_width(gpu_lib, weights, kind, cus, total):
    nova = gpu_lib
    w, w64 = weights
    n = BATCHES[total]
    r = np.random.default_rng([total, cus])
    ctx = [int(c) for c in r.integers(0, 200, len(n))]
    ctx[0] = 700
    llm = nova.Llm(CFG, w)
    tables, pool = synth.block_tables([c + m for c, m in zip(ctx, n)], CFG.block, seed=6)
    tables_d = torch.from_numpy(tables).cuda()
    cache = nova.Cache(pool, CFG.n_kv, CFG.head_dim, dict(bf16=nova.CACHE_BF16, e4m3=nova.CACHE_E4M3)[kind], layers=CFG.layers)
    kept = []                                          # what is cached, written as it stands
    fill = nova.Rows(torch.from_numpy(np.concatenate([[0], np.cumsum(ctx)]).astype(np.int32)).cuda(), None, tables_d,
                     rows=sum(ctx), max_rows=max(ctx), max_ctx=max(ctx))
    for l in range(CFG.layers):
        k, v = (torch.from_numpy(r.normal(size=(sum(ctx), CFG.n_kv, CFG.head_dim))).cuda().to(torch.bfloat16) for _ in "kv")
        nova.kv_append(cache, fill, k, v, layer=l)
        kk, vv = k.double().cpu().numpy(), v.double().cpu().numpy()
        if kind == "e4m3":
            kk, vv = oc.quantise(kk)[0], oc.quantise(vv)[0]
        cut = np.cumsum(ctx)[:-1]
        kept.append(list(zip(np.split(kk, cut), np.split(vv, cut))))
    ids = r.integers(0, CFG.vocab, total).astype(np.int32)
    masks = [m for c in n for m in _tree_mask(c, r)]
    starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    pos = np.array([c + bin(masks[starts[b] + j]).count("1") - 1 for b, c in enumerate(ctx) for j in range(n[b])], np.int32)   # its depth
    ctx_d = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    rows = nova.Rows(torch.from_numpy(starts).cuda(), ctx_d, tables_d, rows=total, max_rows=max(n), max_ctx=max(c + m for c, m in zip(ctx, n)))
    ids_d, pos_d = torch.from_numpy(ids).cuda(), torch.from_numpy(pos).cuda()
    pools = None
    if kind == "bf16" and set(n) == {1}:
        pools = nova.KvPool(llm, pool)
        pools.k5.copy_(cache.k), pools.v5.copy_(cache.v)
    logits = torch.full((total, CFG.vocab), float("nan"), device="cuda")
    torch.cuda.synchronize()
    s = nova.set_stage_partition(nova.STAGE_DECODE, nova.make_cu_mask(cus)) if cus < 256 else None
    nxt = llm.verify(ids_d, pos_d, rows, cache, mask=torch.tensor(_signed(masks), dtype=torch.int64, device="cuda"), logits=logits, stream=s)
    torch.cuda.synchronize()
    stored = [[t.double().cpu().numpy() for t in nova.kv_gather(cache, rows, dtype=torch.float32, layer=l)] for l in range(CFG.layers)]
    want, kv = _step(w64, ids, pos, n, kept, masks, stored if kind == "e4m3" else None)
    got = logits.double().cpu().numpy()
    for j in range(total):
        assert vlm.max_rel_err(got[j], want[j]) < sc.TOL_BF16, j
    assert nxt.tolist() == got.argmax(-1).tolist()
    for l in range(CFG.layers):
        for g, x in zip(stored[l], kv[l]):                 # in 8 bits half a step more, of the largest value at most
            assert vlm.max_rel_err(g, x) < sc.TOL_BF16 + (2.0 ** -4 if kind == "e4m3" else 0.0), l
    if pools is not None:
        plain = torch.empty(total, CFG.vocab, device="cuda")
        torch.cuda.synchronize()
        llm.decode(ids_d, pos_d, tables_d, pools, rows.max_ctx, logits=plain, stream=s)
        torch.cuda.synchronize()
        plain = plain.double().cpu().numpy()
        for j in range(total):
            assert vlm.max_rel_err(got[j], plain[j]) < sc.TOL_BF16, j
