"""The operators between two model calls together, as a serving program uses them: prompts with image positions, verify
steps, acceptance, kept rows and pages, forked and compacted sequences, adapters beside a projection; on streams and
captured into graphs."""
import numpy as np
import pytest
import torch

from oracle import steps as st
from oracle import vlm
from paper_2509_21301_amd import synth
from tests import stage_cases as sc
from tests.test_gpu_output_streams import _stream_of
from tests.test_gpu_verify import QuantKV

pytestmark = pytest.mark.gpu

CFG = synth.TINY_LLM
PAIRS = (12, 10, 10)                     # of 32: time, row and column
TOL = dict(f32=sc.TOL_F32, bf16=sc.TOL_BF16, e4m3=sc.TOL_BF16)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def _image_positions(before, gh, gw, after):
    """Text, an image of gh x gw tokens (time stands still), text again: [3, tokens]."""
    t = [(i, i, i) for i in range(before)]
    t += [(before, before + r, before + c) for r in range(gh) for c in range(gw)]
    go = before + max(gh, gw)
    return np.array(t + [(go + i,) * 3 for i in range(after)]).T


def _model(nova, kind):
    w = synth.llm_weights(CFG, 0)
    act = nova.ACT_F32 if kind == "f32" else nova.ACT_BF16
    type = dict(f32=nova.CACHE_F32, bf16=nova.CACHE_BF16, e4m3=nova.CACHE_E4M3)[kind]
    return w, nova.Llm(CFG, w, act=act), type


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("cyclic", [False, True])
def test_prompts_and_steps_with_image_positions(gpu_lib, kind, cyclic, monkeypatch):
    """Llm.prefill and Llm.verify with positions on three axes against the oracle's prefill and decode steps."""
    nova = gpu_lib
    w, llm, type = _model(nova, kind)
    pos = _image_positions(5, 6, 9, 20)
    n, steps = 70, 4
    freq = st.axes_frequencies(PAIRS, CFG.rope_theta, cyclic)
    # the oracle turns token number p by where it stands
    monkeypatch.setattr(vlm, "rope", lambda x, p, theta: st.rotate_axes(x, pos[:, np.asarray(p)], PAIRS, freq, cyclic))
    tables, pool = synth.block_tables([n + steps], CFG.block, seed=5)
    store = vlm._keep if kind == "f32" else vlm.bf16_store
    kv = (QuantKV if kind == "e4m3" else vlm.PagedKV)(CFG.layers, pool, CFG.n_kv, CFG.block, CFG.head_dim)
    vis = synth.normal((54, CFG.hidden), 3, "vis", std=0.5)
    vis = vlm.bf16_store(vis)
    ids = synth.text_ids(n - 54, CFG.vocab, seed=9)
    want, _ = vlm.llm_prefill(vis, ids, w, CFG, kv=kv, table=tables[0], store=store)
    rope = nova.Rope(CFG.head_dim, theta=CFG.rope_theta, axes=PAIRS, cyclic=cyclic)
    cache = nova.Cache(pool, CFG.n_kv, CFG.head_dim, type, layers=CFG.layers)
    tab, logits = _i32(tables), torch.empty(1, CFG.vocab, device="cuda")
    p = _i32(pos)
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    llm.prefill(torch.from_numpy(vis).cuda().to(dt), _i32(ids), tab[0], cache, logits=logits[0], rope=rope, pos=p[:, :n].contiguous())
    assert vlm.max_rel_err(logits[0].cpu().numpy(), want) < TOL[kind]
    feed = synth.text_ids(steps, CFG.vocab, seed=31)
    for i in range(steps):
        at = n + i
        want, _ = vlm.llm_decode_step(feed[i:i + 1], np.array([at]), tables, kv, w, CFG, store=store)
        rows = nova.Rows(None, _i32([at]), tab, max_rows=1, max_ctx=n + steps)
        llm.verify(_i32(feed[i:i + 1]), p[:, at:at + 1].contiguous(), rows, cache, logits=logits, rope=rope)
        assert vlm.max_rel_err(logits[0].cpu().numpy(), want[0]) < TOL[kind], i


def test_positions_that_count_tokens_are_the_models_own(gpu_lib):
    """Equal positions on every axis, and a rope without axes, give what the calls without positions give."""
    nova = gpu_lib
    _, llm, type = _model(nova, "bf16")
    ids, tab = _i32(synth.text_ids(40, CFG.vocab, seed=2)), _i32(np.arange(3)[None])
    out = []
    for rope, pos in [(None, None), (nova.Rope(CFG.head_dim, CFG.rope_theta), _i32(range(40))),
                      (nova.Rope(CFG.head_dim, CFG.rope_theta, axes=PAIRS), _i32([range(40)] * 3))]:
        cache = nova.Cache(3, CFG.n_kv, CFG.head_dim, type, layers=CFG.layers)
        logits = torch.empty(2, CFG.vocab, device="cuda")
        llm.prefill(None, ids, tab[0], cache, logits=logits[0], rope=rope, pos=pos)
        rows = nova.Rows(None, _i32([40]), tab, max_rows=1, max_ctx=48)
        at = _i32([40]) if rope is None or rope.n_axes == 0 else _i32([[40]] * 3)
        llm.verify(_i32([7]), at, rows, cache, logits=logits[1:], rope=rope)
        out.append(logits)
    # the angles are formed in two ways (a sine of a library's and a series), each to a few fp32 roundings, which bf16
    # roundings of q and k carry on: within the stages' bound
    for b in range(2):
        for x in out[1:]:
            assert vlm.max_rel_err(x[b].cpu().numpy(), out[0][b].cpu().numpy()) < TOL["bf16"]
    assert torch.equal(out[1], out[2])
    with pytest.raises(ValueError):
        llm.prefill(None, ids, tab[0], nova.KvPool(llm, 3), rope=nova.Rope(64), pos=_i32(range(40)))
    with pytest.raises(ValueError):
        llm.prefill(None, ids, tab[0], cache, pos=_i32(range(40)))
    with pytest.raises(ValueError):
        llm.prefill(None, ids, tab[0], cache, rope=nova.Rope(64))


class Sessions:
    """Sequences of the tiny decoder that draft, verify, accept and keep, all on the device."""

    def __init__(self, nova, kind, batch, width, blocks, seed):
        self.nova, self.batch, self.width = nova, batch, width
        _, self.llm, type = _model(nova, kind)
        self.cache = nova.Cache(blocks, CFG.n_kv, CFG.head_dim, type, layers=CFG.layers)
        self.pages = nova.Pages(blocks)
        self.tables = torch.full((batch, 8), -1, dtype=torch.int32, device="cuda")
        r = np.random.default_rng(seed)
        lens = r.integers(9, 40, batch)
        self.ctx = _i32(lens)
        assert self.pages.extend(self.tables, self.ctx).tolist() == [1] * batch
        for b, n in enumerate(lens):
            self.llm.prefill(None, _i32(r.integers(0, CFG.vocab, n)), self.tables[b], self.cache)
        self.ids = _i32(r.integers(0, CFG.vocab, batch * width))
        masks, up = [], [-1] + [int(r.integers(max(0, j - 2), j)) for j in range(1, width)]
        for j in range(width):
            masks.append((1 << j) | (masks[up[j]] if j else 0))
        self.mask = torch.tensor(masks * batch, device="cuda")
        self.depth = _i32([bin(m).count("1") - 1 for m in masks])
        self.temperature = torch.full((batch,), 0.9, device="cuda")
        self.u = torch.zeros(batch * width, device="cuda")
        self.logits = torch.zeros(batch * width, CFG.vocab, device="cuda")
        self.rows = nova.Rows(None, self.ctx, self.tables, max_rows=width, max_ctx=128)
        self.out = None

    def step(self, stream=None):
        """Pages for the drafts, the verify step, what it keeps and the new contexts."""
        nova, kw = self.nova, dict(stream=stream)
        done = self.pages.extend(self.tables, self.ctx + self.width, **kw)
        pos = (self.ctx[:, None] + self.depth).flatten()
        self.llm.verify(self.ids, pos, self.rows, self.cache, mask=self.mask, logits=self.logits, **kw)
        self.out = nova.accept(self.rows, self.ids, self.logits, self.u, mask=self.mask, temperature=self.temperature, **kw)
        ctx = nova.kv_keep(self.cache, self.rows, self.out[1], self.out[0], **kw)
        self.ctx.copy_(ctx)
        return done

    def draft(self, r):
        """New drafts behind the last token: half of them what the model would draw there."""
        last = self.out[2].gather(1, (self.out[0] - 1).long()[:, None]).int() if self.out is not None else self.ids.view(self.batch, -1)[:, :1]
        ids = _i32(r.integers(0, CFG.vocab, (self.batch, self.width)))
        ids[:, :1] = last
        self.ids.copy_(ids.flatten())
        self.u.copy_(torch.from_numpy(r.random(self.batch * self.width).astype(np.float32)))

    def state(self):
        return [self.cache.k, self.cache.v, self.tables, self.pages.refs, self.ctx, self.ids, self.u, self.logits] + ([self.cache.k_exp, self.cache.v_exp] if self.cache.k_exp is not None else [])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_speculative_steps_leave_what_plain_decoding_leaves(gpu_lib, kind):
    """After steps that draft trees, accept and keep, a session's cache holds what a plain decode of its tokens holds, and
    every step's tokens are what the oracle draws from the step's logits."""
    nova = gpu_lib
    s = Sessions(nova, kind, 3, 6, 24, seed=2)
    plain = Sessions(nova, kind, 3, 6, 24, seed=2)                       # the same prompts
    r = np.random.default_rng(7)
    first = s.ids.view(3, 6)[:, 0].tolist()
    fed = [[t] for t in first]                                           # tokens in each cache behind the prompt
    up = [(int(m) & ((1 << j) - 1)).bit_length() - 1 for j, m in enumerate(s.mask[:6].tolist())]
    kept = 0
    for i in range(6):
        s.draft(r)
        if i % 2:                                                         # a draft that is right: the draw behind row 0, and behind that one's row
            trial = [t.clone() for t in s.state()]
            s.step()
            tok = s.out[2][:, 0].clone()
            for t, v in zip(s.state(), trial):
                t.copy_(v)
            s.ids.view(3, 6)[:, 2] = tok                                  # row 2 hangs under row 0 or 1
            s.ids.view(3, 6)[:, 1] = tok
        ids, u = s.ids.view(3, 6).tolist(), s.u.view(3, 6).tolist()
        assert s.step().tolist() == [1] * 3
        n, path, tokens, _ = (t.tolist() for t in s.out)
        for b in range(3):
            wp, wt, _ = st.accept(s.logits[6 * b:6 * b + 6].double().cpu().numpy(), ids[b], u[b], s.mask[:6].tolist(), None, 0.9)
            assert path[b][:n[b]] == wp and tokens[b][:n[b]] == wt
            fed[b] += wt
            kept += n[b] - 1
            assert all(up[j] == p for p, j in zip(wp, wp[1:]))
    assert kept >= 9                                                      # the right drafts, at least
    # the plain session, a token at a time
    longest = max(len(f) for f in fed) - 1
    lens = plain.ctx.clone()
    assert plain.pages.extend(plain.tables, lens + longest).tolist() == [1] * 3
    for i in range(longest):
        ids = _i32([f[min(i, len(f) - 2)] for f in fed])
        rows = nova.Rows(None, lens + i, plain.tables, max_rows=1, max_ctx=128)
        plain.llm.verify(ids, lens + i, rows, plain.cache)
    for b, f in enumerate(fed):
        n = int(lens[b]) + len(f) - 1
        assert int(s.ctx[b]) == n
        got, want = [], []
        for x, c in ((s, got), (plain, want)):
            rows = nova.Rows(None, None, x.tables[b:b + 1].contiguous(), max_rows=n, max_ctx=n)
            for l in range(CFG.layers):
                c += nova.kv_gather(x.cache, rows, layer=l, dtype=torch.float32)
        for g, w in zip(got, want):
            # the same values up to the stages' bound, which may take an 8-bit number to its neighbour, a step of 2^-3
            assert vlm.max_rel_err(g.cpu().numpy(), w.cpu().numpy()) < sc.TOL_BF16 + (2.0 ** -3 if kind == "e4m3" else 0.0)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_captured_steps(gpu_lib, kind):
    """A whole step in a graph, replayed with the program's own work in between, equals the eager step every time."""
    nova = gpu_lib
    s, e = Sessions(nova, kind, 2, 5, 20, seed=4), Sessions(nova, kind, 2, 5, 20, seed=4)
    side = torch.cuda.Stream()
    keep = [t.clone() for t in s.state()]
    with torch.cuda.stream(side):
        s.step()
    side.synchronize()
    for t, v in zip(s.state(), keep):
        t.copy_(v)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        done = s.step()
    out = s.out
    other = torch.cuda.CUDAGraph()                                       # a second graph that lives beside it
    with torch.cuda.graph(other):
        s.step()
    s.out = None                                                         # nothing has run yet: the results hold nothing
    for t, v in zip(s.state(), keep):
        t.copy_(v)
    for i in range(5):
        for x in (s, e):
            x.draft(np.random.default_rng(50 + i))
        for t, v in zip(s.state(), e.state()):
            assert torch.equal(t, v)
        g.replay()
        s.out = out
        want = e.step()
        torch.cuda.synchronize()
        junk = torch.randn(1 << 20, device="cuda").sum().item()          # eager work and a synchronisation between replays
        assert junk == junk and torch.equal(done, want)
        for a, b in zip(s.out, e.out):
            assert torch.equal(a, b)
        for t, v in zip(s.state(), e.state()):
            assert torch.equal(t, v), i


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_forked_and_compacted_sessions_go_on_as_before(gpu_lib, kind):
    """A branch continues exactly as its source would, whatever the other does; moving the pool's pages changes no
    logits; what is given up is free again."""
    nova = gpu_lib
    _, llm, type = _model(nova, kind)
    blocks = 30
    cache, pages = nova.Cache(blocks, CFG.n_kv, CFG.head_dim, type, layers=CFG.layers), nova.Pages(blocks)
    tables = torch.full((5, 8), -1, dtype=torch.int32, device="cuda")
    pages.refs[:3] = 1                                                   # taken by others, free later
    assert pages.extend(tables, _i32([50, 33, 0, 0, 0])).tolist() == [1] * 5
    r = np.random.default_rng(5)
    for b, n in ((0, 50), (1, 33)):
        llm.prefill(None, _i32(r.integers(0, CFG.vocab, n)), tables[b], cache)

    def logits(row, ctx, token, t=tables):
        rows = nova.Rows(None, _i32([ctx]), t[row:row + 1].contiguous(), max_rows=1, max_ctx=128)
        out = torch.empty(1, CFG.vocab, device="cuda")
        llm.verify(_i32([token]), _i32([ctx]), rows, cache, logits=out)
        return out
    want = logits(0, 50, 11)
    assert pages.fork(cache, tables, _i32([0, 0, 1]), _i32([2, 3, 4]), _i32([50, 37, 32])).tolist() == [1, 1, 1]
    assert pages.extend(tables, _i32([60, 33, 60, 60, 60])).tolist() == [1] * 5
    assert torch.equal(logits(2, 50, 11), want)
    a = [logits(0, 51, 3), logits(2, 51, 3)]
    assert torch.equal(a[0], a[1])
    logits(3, 37, 99), logits(4, 32, 98)                                 # other branches write pages of their own
    b = [logits(0, 52, 4), logits(2, 52, 4)]
    assert torch.equal(b[0], b[1])
    pages.refs[:3] = 0
    pages.free(tables, _i32([1, 3]))
    pool = st.Pool(pages.refs.cpu().numpy(), tables.cpu().numpy())
    live, _ = pool.compact()
    assert pages.compact(cache, tables).tolist() == [live]
    assert pages.refs.tolist() == pool.refs.tolist() and tables.tolist() == pool.tables.tolist()
    assert int(tables.max()) == live - 1
    c = [logits(0, 53, 5), logits(2, 53, 5)]
    assert torch.equal(c[0], c[1]) and torch.equal(logits(2, 52, 4), b[0])
    pages.free(tables, _i32(range(5)))
    assert (pages.refs == 0).all()


def _projection(nova):
    """A layer's start for three users: a shared projection, their adapters on it, append with image positions, attention."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    n_q, n_kv, d, k = 4, 2, 64, 256
    n, rows = (n_q + 2 * n_kv) * d, [9, 1, 5]
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    starts = _i32(np.concatenate([[0], np.cumsum(rows)]))
    w = (rn(n, k) / 16).bfloat16()
    ad = nova.Adapters((rn(2, 24, k) / 16).bfloat16(), (rn(2, n, 24) / 5).bfloat16(), rn(2).abs())
    x = rn(15, k).bfloat16()
    tables = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    cache = nova.Cache(6, n_kv, d, nova.CACHE_BF16)
    desc = nova.Rows(starts, _i32([3, 0, 20]), tables, rows=15, max_rows=9, max_ctx=32)
    rope = nova.Rope(d, axes=(12, 10, 10), cyclic=True)
    pos = torch.arange(45, dtype=torch.int32, device="cuda").view(3, 15)
    which = _i32([1, -1, 0])
    out = torch.zeros(15, n, device="cuda")

    def run():
        out.zero_()
        nova.linear(nova.LINEAR_TILED, x, w, out)
        y = nova.lora(ad, desc, which, x, base=out)
        q, kk, v = y.view(15, -1, d).split([n_q, n_kv, n_kv], 1)
        q = nova.kv_append(cache, desc, kk, v, q=q, pos=pos, rope=rope, q_out=torch.empty(15, n_q, d, dtype=torch.bfloat16, device="cuda"))
        return y, nova.tree_attention(cache, desc, q), cache.k, cache.v
    return run, (x, w, ad, which, starts, rows)


def test_projection_with_adapters_feeds_the_cache(gpu_lib):
    """The projection and its adapters against float64, then what is appended and attended on top of it, eager and captured."""
    nova = gpu_lib
    run, (x, w, ad, which, starts, rows) = _projection(nova)
    y, att, k, v = run()
    xn, wn = x.double().cpu().numpy(), w.double().cpu().numpy()
    want = xn @ wn.T
    size = np.abs(xn) @ np.abs(wn).T
    err = (256 + 16) * 2.0 ** -24 * size
    for b, n in enumerate(rows):
        i, sl = int(which[b]), slice(int(starts[b]), int(starts[b]) + n)
        if i >= 0:
            d, terms, sz = st.lora(xn[sl], ad.a[i].double().cpu().numpy(), ad.b[i].double().cpu().numpy(), float(ad.scale[i]))
            want[sl] += d
            # fp32 sums of 256 and of three parts of 24 products, h in three bf16 parts
            err[sl] += (256 + 16) * 2.0 ** -24 * sz + (3 * 24 + 16) * 2.0 ** -24 * terms + 2.0 ** -23 * terms
    assert (np.abs(y.double().cpu().numpy() - want) <= err + 2.0 ** -23 * np.abs(want)).all()
    first = [t.clone() for t in (y, att, k, v)]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        out = run()
    for _ in range(3):
        k.zero_(), v.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, first):
            assert torch.equal(a, b)


# ----------------------------------------------------------------------------- streams, devices, concurrent calls
def _calls(nova):
    """Every call once: name -> (run(stream), its fresh results are to be on the call's stream)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tables = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    rows = nova.Rows(None, _i32([20, 33]), tables, max_rows=4, max_ctx=64)
    cache = nova.Cache(16, 2, 64, nova.CACHE_E4M3, layers=2)
    x, pos = torch.randn(8, 2, 64, generator=g, device="cuda"), _i32([range(8)] * 2)
    rope = nova.Rope(64, axes=(20, 12))
    logits, draft = torch.randn(2, 8, 500, generator=g, device="cuda").unbind(0)
    ids, u = _i32(range(8)), torch.rand(8, generator=g, device="cuda")
    path, n = _i32([[0, 2, 3, -1], [0, 1, -1, -1]]), _i32([3, 2])
    ad = nova.Adapters(torch.randn(2, 16, 64, generator=g, device="cuda").bfloat16(), torch.randn(2, 64, 16, generator=g, device="cuda").bfloat16())

    def pages(call):
        def run(s):
            with torch.cuda.stream(s or torch.cuda.current_stream()):
                p, t = nova.Pages.of(_i32([0, 2, 0, 1, 1] + [0] * 11)), _i32([[1, 3, -1], [1, 4, -1], [-1] * 3])
                src, dst, n = _i32([0]), _i32([2]), _i32([25])
                tok = _i32([17, 40, 3])
            return {"extend": lambda: [p.extend(t, tok, stream=s), t, p.refs],
                    "fork": lambda: [p.fork(cache, t, src, dst, n, stream=s), t, p.refs, cache.k],
                    "free": lambda: [p.free(t, src, stream=s), t, p.refs],
                    "compact": lambda: [p.compact(cache, t, stream=s), t, p.refs]}[call]()
        return run
    return dict(rotate=lambda s: [nova.rotate(x, pos, rope, stream=s)], accept=lambda s: list(nova.accept(rows, ids, logits, u, stream=s)),
                accept_draft=lambda s: list(nova.accept(rows, ids, logits, u, draft=draft, stream=s)),
                kv_keep=lambda s: [nova.kv_keep(cache, rows, path, n, stream=s)], kv_copy=lambda s: [nova.kv_copy(cache, _i32([1]), _i32([14]), stream=s), cache.k],
                lora=lambda s: [nova.lora(ad, rows, _i32([0, 1]), x[:, 0].contiguous().bfloat16(), stream=s)],
                **{c: pages(c) for c in ("extend", "fork", "free", "compact")})


@pytest.mark.parametrize("call", ["rotate", "accept", "accept_draft", "kv_keep", "kv_copy", "lora", "extend", "fork", "free", "compact"])
def test_calls_on_a_stream(gpu_lib, call):
    """The same results on a stream of the caller's, allocated on it."""
    nova = gpu_lib
    run = _calls(nova)[call]
    want = [None if t is None else t.clone() for t in run(None)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(side)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert (a is None and b is None) or torch.equal(a, b)
    if got[0] is not None:
        assert _stream_of(got[0]) == side.cuda_stream


def test_two_acceptances_at_once(gpu_lib):
    """Two streams that run acceptances, and adapters, of other inputs over the same time: workspaces of their own."""
    nova = gpu_lib
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    rows = nova.Rows(None, None, torch.zeros(4, 4, dtype=torch.int32, device="cuda"), max_rows=8, max_ctx=64)
    ad = nova.Adapters(torch.randn(3, 32, 512, generator=g, device="cuda").bfloat16(), torch.randn(3, 1024, 32, generator=g, device="cuda").bfloat16())
    sets = []
    for _ in range(2):
        logits, draft = torch.randn(2, 32, 30000, generator=g, device="cuda").unbind(0)
        sets.append((torch.randint(0, 30000, (32,), generator=g, device="cuda", dtype=torch.int32), logits * 3, torch.rand(32, generator=g, device="cuda"), draft * 3,
                     torch.randn(32, 512, generator=g, device="cuda").bfloat16(), _i32([0, 1, 2, 1])))

    def one(s, stream=None):
        return [*nova.accept(rows, s[0], s[1], s[2], draft=s[3], stream=stream), *nova.accept(rows, s[0], s[1], s[2], stream=stream),
                nova.lora(ad, rows, s[5], s[4], stream=stream)]
    want = [one(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(sets):
            got[i].append(one(s, streams[i]))
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        for o in many:
            for a, b in zip(o, w):
                assert torch.equal(a, b)
