"""The LLM on a cache of any type: prefill into it, and decode steps over trees of drafted tokens
(nova_llm_prefill_cache, nova_llm_verify), against the oracle decoding every path of the tree alone."""
import copy

import numpy as np
import pytest
import torch

from oracle import cache as oc, vlm
from paper_2509_21301_amd import synth
from tests import stage_cases as sc

pytestmark = pytest.mark.gpu

CFG = synth.TINY_LLM
PROMPTS = (96, 21)            # tokens of the two sequences
PARENTS = ([-1, 0, 0, 1, 1, 2, 4], [-1, 0, 1, 1])


class QuantKV(vlm.PagedKV):
    """The oracle's cache, holding what an 8-bit one stands for."""

    def write(self, l, table, pos, k, v):
        super().write(l, table, pos, oc.quantise(k)[0], oc.quantise(v)[0])


def _oracle(kind):
    w = synth.llm_weights(CFG, 0)
    store = vlm._keep if kind == "f32" else vlm.bf16_store
    tables, pool = synth.block_tables([p + 40 for p in PROMPTS], CFG.block, seed=5)
    kv = (QuantKV if kind == "e4m3" else vlm.PagedKV)(CFG.layers, pool, CFG.n_kv, CFG.block, CFG.head_dim)
    ids = [synth.text_ids(p, CFG.vocab, seed=20 + b) for b, p in enumerate(PROMPTS)]
    first = [vlm.llm_prefill(np.zeros((0, CFG.hidden)), i, w, CFG, kv=kv, table=tables[b], store=store) for b, i in enumerate(ids)]
    return dict(w=w, store=store, tables=tables, pool=pool, kv=kv, ids=ids, logits=[f[0] for f in first], tokens=[f[1] for f in first])


def _path(parents, j):
    out = []
    while j >= 0:
        out.append(j)
        j = parents[j]
    return out[::-1]


def _mask(parents):
    m = []
    for j, p in enumerate(parents):
        m.append((1 << j) | (m[p] if p >= 0 else 0))
    return m


def _along(ref, b, tokens, start):
    """Oracle logits after each of ``tokens`` fed to sequence b from position ``start`` (on a copy of the cache)."""
    kv = copy.deepcopy(ref["kv"])
    out = [vlm.llm_decode_step(np.array([t]), np.array([start + i]), ref["tables"][b:b + 1], kv, ref["w"], CFG, store=ref["store"])[0][0]
           for i, t in enumerate(tokens)]
    return out, kv


def _setup(nova, kind, ref):
    act = nova.ACT_F32 if kind == "f32" else nova.ACT_BF16
    llm = nova.Llm(CFG, ref["w"], act=act)
    cache = nova.Cache(ref["pool"], CFG.n_kv, CFG.head_dim, dict(f32=nova.CACHE_F32, bf16=nova.CACHE_BF16, e4m3=nova.CACHE_E4M3)[kind], layers=CFG.layers)
    tables = torch.from_numpy(ref["tables"]).cuda()
    logits = torch.empty(2, CFG.vocab, device="cuda")
    for b in range(2):
        llm.prefill(None, torch.from_numpy(ref["ids"][b]).cuda(), tables[b], cache, logits=logits[b])
    return llm, cache, tables, logits


# fp32: the exact mode's bound.  bf16: the stages' bound; the 8-bit cache's values are the oracle's own
# except where a bf16 rounding of k or v before the quantisation differs, which the same bound covers
TOL = dict(f32=sc.TOL_F32, bf16=sc.TOL_BF16, e4m3=sc.TOL_BF16)


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
def test_tree_rows_equal_their_paths(gpu_lib, kind):
    nova = gpu_lib
    ref = _oracle(kind)
    llm, cache, tables, logits = _setup(nova, kind, ref)
    for b in range(2):
        assert vlm.max_rel_err(logits[b].cpu().numpy(), ref["logits"][b]) < TOL[kind]
    r = np.random.default_rng(4)
    drafts = [r.integers(0, CFG.vocab, len(p)).astype(np.int32) for p in PARENTS]
    depth = [[len(_path(p, j)) - 1 for j in range(len(p))] for p in PARENTS]
    n = sum(map(len, PARENTS)) + 1                                   # and a row of no sequence
    ids = torch.from_numpy(np.concatenate(drafts + [[0]]).astype(np.int32)).cuda()
    pos = torch.tensor([PROMPTS[b] + d for b in range(2) for d in depth[b]] + [0], dtype=torch.int32, device="cuda")
    mask = torch.tensor(_mask(PARENTS[0]) + _mask(PARENTS[1]) + [0], dtype=torch.int64, device="cuda")
    rows = nova.Rows(torch.tensor([0, 7, 11], dtype=torch.int32, device="cuda"), torch.tensor(PROMPTS, dtype=torch.int32, device="cuda"),
                     tables, rows=n, max_rows=7, max_ctx=max(PROMPTS) + 7)
    out = torch.empty(n, CFG.vocab, device="cuda")
    nxt = llm.verify(ids, pos, rows, cache, mask=mask, logits=out)
    torch.cuda.synchronize()
    row = 0
    for b in range(2):
        for j in range(len(PARENTS[b])):
            want, _ = _along(ref, b, [drafts[b][i] for i in _path(PARENTS[b], j)], PROMPTS[b])
            got = out[row].cpu().numpy()
            assert vlm.max_rel_err(got, want[-1]) < TOL[kind], (b, j)
            assert int(nxt[row]) == int(np.argmax(got))
            row += 1


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
def test_single_rows_decode(gpu_lib, kind):
    """One row per sequence, no row_start and no mask: plain decode, step after step, fed seeded tokens; on the
    16-bit and 32-bit caches beside nova_llm_decode on a KvPool with the same weights."""
    nova = gpu_lib
    ref = _oracle(kind)
    llm, cache, tables, _ = _setup(nova, kind, ref)
    steps = 6
    feed = np.random.default_rng(6).integers(0, CFG.vocab, (steps, 2)).astype(np.int32)
    want = [_along(ref, b, feed[:, b], PROMPTS[b])[0] for b in range(2)]
    pool = None
    if kind != "e4m3":
        pool = nova.KvPool(llm, ref["pool"])
        for b in range(2):
            llm.prefill(None, torch.from_numpy(ref["ids"][b]).cuda(), tables[b], pool)
        assert torch.equal(pool.k5, cache.k) and torch.equal(pool.v5, cache.v)       # prefill writes the same
    ctx = torch.tensor(PROMPTS, dtype=torch.int32, device="cuda")
    rows = nova.Rows(None, ctx, tables, max_rows=1, max_ctx=max(PROMPTS) + steps)
    out, old = torch.empty(2, CFG.vocab, device="cuda"), torch.empty(2, CFG.vocab, device="cuda")
    for t in range(steps):
        ids = torch.from_numpy(feed[t]).cuda()
        llm.verify(ids, ctx, rows, cache, logits=out)
        if pool is not None:
            llm.decode(ids, ctx, tables, pool, max(PROMPTS) + steps, logits=old)
            assert vlm.max_rel_err(out.cpu().numpy(), old.double().cpu().numpy()) < TOL[kind]
        for b in range(2):
            assert vlm.max_rel_err(out[b].cpu().numpy(), want[b][t]) < TOL[kind], (t, b)
        ctx += 1


def test_speculative_decoding_keeps_the_greedy_tokens(gpu_lib):
    """A whole loop in fp32: draft a tree (good and bad guesses), verify it, score it, keep the longest accepted path,
    move its K and V behind the context, go on; the tokens are those of greedy decoding one at a time."""
    nova = gpu_lib
    ref = _oracle("f32")
    b, want = 0, 10
    toks, kv, pos = [ref["tokens"][b]], copy.deepcopy(ref["kv"]), PROMPTS[b]
    for t in range(want + 8):
        _, nx = vlm.llm_decode_step(np.array([toks[-1]]), np.array([pos + t]), ref["tables"][b:b + 1], kv, ref["w"], CFG)
        toks.append(int(nx[0]))
    llm, cache, tables, _ = _setup(nova, "f32", ref)
    r = np.random.default_rng(8)
    got, ctx = [toks[0]], PROMPTS[b]
    parents = [-1, 0, 0, 1, 2, 4]                                    # root: the last token; the true path is 0, 2, 4, 5
    mask = torch.tensor(_mask(parents), dtype=torch.int64, device="cuda")
    depth = np.array([len(_path(parents, j)) - 1 for j in range(6)])
    turn = 0
    while len(got) < want:
        at = len(got) - 1
        wrong = lambda t: int((t + 1 + r.integers(0, CFG.vocab - 1)) % CFG.vocab)  # noqa: E731
        good = toks[at:at + 4]
        guess = [good[0], wrong(good[1]), good[1], wrong(good[2]), good[2], good[3] if turn % 2 else wrong(good[3])]
        ids = torch.tensor(guess, dtype=torch.int32, device="cuda")
        ctx_t = torch.tensor([ctx], dtype=torch.int32, device="cuda")
        rows = nova.Rows(None, ctx_t, tables[b:b + 1].contiguous(), max_rows=6, max_ctx=ctx + 6)
        logits = torch.empty(6, CFG.vocab, device="cuda")
        nxt = llm.verify(ids, torch.from_numpy((ctx + depth).astype(np.int32)).cuda(), rows, cache, mask=mask, logits=logits)
        lp, ent, tl, ti = nova.logprobs(logits, given=nxt[:, None].contiguous(), n_top=3)
        nxt = nxt.tolist()
        assert ti[:, 0].tolist() == nxt and torch.equal(lp[:, 0], tl[:, 0]) and (ent > 0).all()
        path = [0]                                                   # the accepted path: children that the model itself chose
        while True:
            more = [j for j in range(6) if parents[j] == path[-1] and guess[j] == nxt[path[-1]]]
            if not more:
                break
            path.append(more[0])
        assert len(path) == (4 if turn % 2 else 3)
        got += [guess[j] for j in path[1:]] + [nxt[path[-1]]]
        keep = nova.Rows(None, ctx_t, tables[b:b + 1].contiguous(), max_rows=len(path), max_ctx=ctx + 6)
        slots = torch.tensor([ctx + j for j in path], dtype=torch.int32, device="cuda")
        for l in range(CFG.layers):
            k, v = nova.kv_gather(cache, keep, slots=slots, dtype=torch.float32, layer=l)
            nova.kv_append(cache, keep, k, v, layer=l)
        ctx += len(path)
        turn += 1
    assert got == toks[:len(got)]


def test_verify_in_a_graph(gpu_lib):
    """A captured step replayed with other tokens and contexts against the eager one."""
    nova = gpu_lib
    ref = _oracle("e4m3")
    llm, cache, tables, _ = _setup(nova, "e4m3", ref)
    ids = torch.tensor([5, 6, 7, 8], dtype=torch.int32, device="cuda")
    ctx = torch.tensor(PROMPTS, dtype=torch.int32, device="cuda")
    pos = torch.tensor([96, 97, 21, 22], dtype=torch.int32, device="cuda")
    rows = nova.Rows(None, ctx, tables, max_rows=2, max_ctx=128)
    nxt, logits = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, CFG.vocab, device="cuda")
    llm.verify(ids, pos, rows, cache, next_ids=nxt, logits=logits)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        llm.verify(ids, pos, rows, cache, next_ids=nxt, logits=logits)
    for t in range(4):
        ids += 11
        ctx += 1
        pos += 1
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        n1, l1 = nxt.clone(), logits.clone()
        llm.verify(ids, pos, rows, cache, next_ids=nxt, logits=logits)
        torch.cuda.synchronize()
        assert torch.equal(n1, nxt) and torch.equal(l1, logits), t


def test_two_graphs_and_a_larger_step_between(gpu_lib):
    """Captured steps keep workspaces of their own: another capture and a larger eager step between the replays
    change nothing."""
    nova = gpu_lib
    ref = _oracle("bf16")
    llm, cache, tables, _ = _setup(nova, "bf16", ref)
    ctx = torch.tensor(PROMPTS, dtype=torch.int32, device="cuda")

    def step(n):
        ids = torch.arange(2 * n, dtype=torch.int32, device="cuda") + 3
        pos = (ctx[:, None] + torch.arange(n, dtype=torch.int32, device="cuda")).flatten().contiguous()
        rows = nova.Rows(None, ctx, tables, max_rows=n, max_ctx=130)
        out = torch.empty(2 * n, CFG.vocab, device="cuda")
        return lambda: llm.verify(ids, pos, rows, cache, logits=out), out
    steps = [step(1), step(4)]
    want = []
    for s, out in steps:
        s()
        want.append(out.clone())
    torch.cuda.synchronize()
    graphs = []
    for s, _ in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s()
        graphs.append(g)
    big, _ = step(16)
    for _ in range(3):
        for g, (_, out), w in zip(graphs, steps, want):
            big()
            junk = torch.full((1 << 22,), float("nan"), device="cuda")
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)
            del junk


def test_model_checks(gpu_lib):
    nova = gpu_lib
    ref = _oracle("bf16")
    llm, cache, tables, _ = _setup(nova, "bf16", ref)
    rows = nova.Rows(None, None, tables, max_rows=1, max_ctx=16)
    one = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        llm.verify(one, one, rows, nova.Cache(8, CFG.n_kv, CFG.head_dim, layers=1))      # layers
    with pytest.raises(ValueError):
        llm.verify(one[:1], one, rows, cache)
    with pytest.raises(ValueError):
        llm.verify(one, one, rows, cache, logits=torch.empty(2, 7, device="cuda"))
    with pytest.raises(nova.NovaError) as e:
        llm.verify(one, one, rows, nova.Cache(8, CFG.n_kv, CFG.head_dim, nova.CACHE_F32, layers=CFG.layers))
    assert e.value.code == nova.EUNSUPPORTED
    with pytest.raises(ValueError):
        nova.tree_attention(cache, rows, torch.zeros(2, 4, 64, device="cuda"))           # fp32 q on a bf16 cache
    assert nova.kv_gather(cache, nova.Rows(one[:1].new_zeros(3), None, tables, rows=0))[0].shape == (0, CFG.n_kv, CFG.head_dim)
