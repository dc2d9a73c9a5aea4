"""Prefill into a cache of any type at the real widths (28/4 heads of 128): the 16-bit cache is a KvPool's to the bit, and
the 8-bit one holds the 16-bit one's values, quantised."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2509_21301_amd import synth

pytestmark = pytest.mark.gpu

# (the head of a prefill is not cut along K, so it needs 64 rows of the vocabulary for each compute unit)
CFG = dataclasses.replace(synth.LLM_28, layers=2, inter=1024, vocab=16384, name="llm2_width")


@pytest.mark.parametrize("n_vis,n_text", [(0, 1), (0, 16), (64, 31), (300, 17)])
def test_prefill_keeps_what_a_16_bit_cache_keeps(gpu_lib, n_vis, n_text):
    nova = gpu_lib
    s = n_vis + n_text
    llm = nova.Llm(CFG, synth.llm_weights_torch(CFG, 0))
    tables, pool = synth.block_tables([s, 40], CFG.block, seed=n_text)
    table = torch.from_numpy(tables[0]).cuda()
    vis = torch.from_numpy(synth.vision_embeds(n_vis, CFG.hidden)).cuda().to(torch.bfloat16) if n_vis else None
    ids = torch.from_numpy(synth.text_ids(n_text, CFG.vocab)).cuda()
    kv = nova.KvPool(llm, pool)
    caches = [nova.Cache(pool, CFG.n_kv, CFG.head_dim, t, layers=CFG.layers) for t in (nova.CACHE_BF16, nova.CACHE_E4M3)]
    logits = [torch.empty(CFG.vocab, device="cuda") for _ in range(3)]
    got = [llm.prefill(vis, ids, table, c, logits=x) for c, x in zip([kv] + caches, logits)]
    assert torch.equal(caches[0].k, kv.k5) and torch.equal(caches[0].v, kv.v5)
    for x, g in zip(logits[1:], got[1:]):                      # the prompt attends to K and V as computed
        assert torch.equal(x, logits[0]) and torch.equal(g, got[0])
    rows = nova.Rows(None, None, table[None].contiguous(), max_rows=s, max_ctx=s)
    for l in range(CFG.layers):
        wide, narrow = (nova.kv_gather(c, rows, dtype=torch.float32, layer=l) for c in caches)
        for a, b in zip(wide, narrow):
            assert np.array_equal(b.double().cpu().numpy(), oc.quantise(a.double().cpu().numpy())[0]), l
        # blocks and slots of no token stay clear
        used = torch.zeros(pool, 16, dtype=torch.bool)
        for t in range(s):
            used[int(tables[0][t // 16]), t % 16] = True
        free = ~used.cuda()
        assert not caches[1].k[l].transpose(1, 2)[free].any() and not caches[1].v[l].permute(0, 3, 1, 2)[free].any()
