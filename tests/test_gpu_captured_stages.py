"""Prefill and decode captured into graphs: each graph keeps a workspace of its own, whatever runs between its replays."""
import pytest
import torch

from paper_2509_21301_amd import synth

pytestmark = pytest.mark.gpu

CFG = synth.TINY_LLM


@pytest.mark.parametrize("kind", ["pool", "e4m3"])
def test_graphs_and_larger_calls_between(gpu_lib, kind):
    nova = gpu_lib
    llm = nova.Llm(CFG, synth.llm_weights(CFG, 0))
    lengths = [24, 40, 400]
    tables, pool = synth.block_tables([n + 24 for n in lengths], CFG.block, seed=5)
    tables = torch.from_numpy(tables).cuda()
    kv = nova.KvPool(llm, pool) if kind == "pool" else nova.Cache(pool, CFG.n_kv, CFG.head_dim, layers=CFG.layers)
    ids = [torch.from_numpy(synth.text_ids(n, CFG.vocab, seed=n)).cuda() for n in lengths]
    outs = [torch.empty(CFG.vocab, device="cuda") for _ in lengths]
    calls = [lambda i=i: llm.prefill(None, ids[i], tables[i], kv, logits=outs[i]) for i in range(3)]
    if kind == "pool":
        pos = torch.tensor(lengths[:2], dtype=torch.int32, device="cuda")
        step = torch.empty(2, CFG.vocab, device="cuda")
        tok = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
        calls.append(lambda: llm.decode(tok, pos, tables[:2].contiguous(), kv, 64, logits=step))
        outs.append(step)
    for c in calls[:2] + calls[3:]:
        c()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    graphs = []
    for c in calls[:2] + calls[3:]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c()
        graphs.append(g)
    used = [0, 1] + [3] * (kind == "pool")
    for turn in range(3):
        calls[2]()                                          # a larger prompt: its workspace replaces the kept one
        if kind == "pool":
            big = torch.zeros(3, dtype=torch.int32, device="cuda")
            at = torch.tensor([30, 50, 410], dtype=torch.int32, device="cuda")
            llm.decode(big, at, tables, kv, 424)
        torch.cuda.synchronize()
        junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]
        for g, i in zip(graphs, used):
            outs[i].zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i]), (turn, i)
        assert all(torch.isnan(j).all() for j in junk)      # and nothing of theirs is written
        del junk
