"""The operators over the paged cache and the logits against their float64 definitions (oracle.cache).

Tolerances count roundings (half a step of bf16 is 2^-8 relative, of e4m3 2^-4, of fp32 2^-24) and
the fp32 sums, bounded term by term, so that nothing in them was measured."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2509_21301_amd import synth

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
TYPES = ["bf16", "f32", "e4m3"]


def _np(t):
    return t.detach().double().cpu().numpy()


def _rng(*seed):
    return np.random.default_rng(list(seed))


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


class Batch:
    """Sequences with cached tokens and new rows over a shuffled pool; K and V of every token in float64."""

    def __init__(self, nova, ctx, rows, n_kv, d, kind, seed, spare=5, pad_rows=0, base_block=0):
        r = _rng(seed, 1)
        self.nova, self.ctx, self.rows, self.n_kv, self.d, self.kind = nova, ctx, rows, n_kv, d, kind
        self.starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.total = int(self.starts[-1]) + pad_rows
        held = [c + n for c, n in zip(ctx, rows)]
        need = [-(-h // 16) for h in held]
        self.width = max(1, max(need))
        self.blocks = sum(need) + spare
        order = r.permutation(self.blocks) + base_block
        self.tables = np.full((len(ctx), self.width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.tables[b, :n] = order[at:at + n]
            at += n
        self.type = dict(bf16=nova.CACHE_BF16, f32=nova.CACHE_F32, e4m3=nova.CACHE_E4M3)[kind]
        self.cache = nova.Cache(self.blocks + base_block, n_kv, d, self.type)
        self.max_ctx = max(1, max(held))
        self.desc = nova.Rows(_dev(self.starts, torch.int32), _dev(np.array(ctx), torch.int32), _dev(self.tables, torch.int32),
                              rows=self.total, max_rows=max(1, max(rows)), max_ctx=self.max_ctx)

    def place(self, b, t):
        return int(self.tables[b, t // 16]), t % 16

    def fill(self, seed, stale=0.0):
        """Every sequence's tokens (cached and new) written into the pool from the host, everything else ``stale``;
        self.k[b], self.v[b] [tokens, n_kv, d] hold the values as stored."""
        r = _rng(seed, 2)
        c = self.cache
        lead = (c.num_blocks, self.n_kv)
        k, v = np.full(lead + (16, self.d), stale), np.full(lead + (self.d, 16), stale)
        ke, ve = np.full(lead + (16,), 127), np.full(lead + (16,), 127)
        self.k, self.v = [], []
        for b, (x, n) in enumerate(zip(self.ctx, self.rows)):
            kk, vv = (r.normal(size=(x + n, self.n_kv, self.d)) * np.exp(0.5 * r.normal(size=(x + n, self.n_kv, 1))) for _ in "kv")
            if self.kind == "e4m3":
                (kk, ek), (vv, ev) = oc.quantise(kk), oc.quantise(vv)
            else:
                kk, vv = (torch.from_numpy(a).to(F32 if self.kind == "f32" else BF16).double().numpy() for a in (kk, vv))
                ek = ev = np.zeros(kk.shape[:2], int)
            for t in range(x + n):
                blk, s = self.place(b, t)
                k[blk, :, s], v[blk, :, :, s] = kk[t] / np.ldexp(1.0, ek[t])[:, None], vv[t] / np.ldexp(1.0, ev[t])[:, None]
                ke[blk, :, s], ve[blk, :, s] = ek[t] + 127, ev[t] + 127
            self.k.append(kk)
            self.v.append(vv)
        for dst, src in ((c.k, k), (c.v, v)):
            if self.kind == "e4m3":
                dst[0].copy_(_dev(src, F32).to(torch.float8_e4m3fn).view(torch.uint8))
            else:
                dst[0].copy_(_dev(src, dst.dtype))
        if self.kind == "e4m3":
            c.k_exp[0].copy_(_dev(ke, torch.uint8))
            c.v_exp[0].copy_(_dev(ve, torch.uint8))
        return self

    def put(self, b, t, k, v):
        """One token's K and V [n_kv, d] in the pool and in self.k, self.v."""
        c, (blk, s) = self.cache, self.place(b, t)
        if self.kind == "e4m3":
            (k, ek), (v, ev) = oc.quantise(k), oc.quantise(v)
            c.k_exp[0, blk, :, s], c.v_exp[0, blk, :, s] = _dev(ek + 127, torch.uint8), _dev(ev + 127, torch.uint8)
            c.k[0, blk, :, s] = _dev(k / np.ldexp(1.0, ek)[:, None], F32).to(torch.float8_e4m3fn).view(torch.uint8)
            c.v[0, blk, :, :, s] = _dev(v / np.ldexp(1.0, ev)[:, None], F32).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            c.k[0, blk, :, s], c.v[0, blk, :, :, s] = _dev(k, c.k.dtype), _dev(v, c.v.dtype)
        self.k[b][t], self.v[b][t] = k, v

    def stored(self, b, t):
        """What the pool holds of a token now: (k [n_kv, d], v [n_kv, d]) in float64."""
        c, (blk, s) = self.cache, self.place(b, t)
        k, v = c.k[0, blk, :, s], c.v[0, blk, :, :, s]
        if self.kind != "e4m3":
            return _np(k), _np(v)
        ek, ev = (np.ldexp(1.0, e[0, blk, :, s].cpu().numpy().astype(int) - 127)[:, None] for e in (c.k_exp, c.v_exp))
        return _np(k.contiguous().view(torch.float8_e4m3fn)) * ek, _np(v.contiguous().view(torch.float8_e4m3fn)) * ev


# ----------------------------------------------------------------------------- append
ROPES = [dict(rot=0), dict(), dict(interleaved=True), dict(rot=16, theta=1e6), dict(rot=48, interleaved=True, mscale=1.25),
         dict(rot=32, factor=4.0), dict(factor=8.0, orig_ctx=4096, mscale=1.2), dict(interleaved=True, factor=32.0, orig_ctx=64, alpha=1.0, beta=4.0)]


def _check_append(bt, q, k, v, pos, rope, act_out, q_out, row0_of):
    d = bt.d
    freq = oc.rope_frequencies(rope["rot"], rope["theta"], rope["factor"], rope["orig_ctx"], rope["alpha"], rope["beta"]) if rope["rot"] else np.zeros(0)
    turn = lambda x, p: oc.rotate(x, p, rope["rot"], freq, rope["interleaved"], rope["mscale"])  # noqa: E731
    for b, n in enumerate(bt.rows):
        if n == 0:
            continue
        sl = slice(row0_of(b), row0_of(b) + n)
        p = pos[sl]
        # fp32 rotation: sines and cosines within 3 roundings, two products and a sum: 8 in all of |a| + |b|
        fp = 8 * 2.0 ** -24 * abs(rope["mscale"]) if rope["rot"] else 0.0
        if q is not None:
            want = turn(_np(q[sl]), p)
            pair = np.abs(_np(q[sl])).max(-1, keepdims=True) * 2
            assert (np.abs(_np(q_out[sl]) - want) <= HALF[act_out] * np.abs(want) + 2 * fp * pair).all(), "q"
        wk, wv = turn(_np(k[sl]), p), _np(v[sl])
        for j in range(n):
            gk, gv = bt.stored(b, bt.ctx[b] + j)
            for got, want, err in ((gk, wk[j], 2 * fp * 2 * np.abs(_np(k[sl][j])).max(-1, keepdims=True)), (gv, wv[j], 0.0)):
                if bt.kind == "e4m3":
                    e = oc.quantise(want)[1]
                    # half a step of 4 significant bits, or of the smallest numbers; an fp32 error may move the maximum over a scale's border
                    tol = 2.0 ** -4 * np.abs(want) + np.ldexp(2.0 ** -9, e)[:, None] + err
                else:
                    tol = HALF[F32 if bt.kind == "f32" else BF16] * np.abs(want) + err
                assert (np.abs(got - want) <= tol).all(), (b, j, np.abs(got - want).max())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("which", range(len(ROPES)))
def test_append(gpu_lib, kind, which):
    nova = gpu_lib
    d, n_kv, n_q = [(64, 2, 4), (128, 4, 28), (128, 1, 3)][which % 3]
    rope = dict(dict(rot=d, theta=1e4, interleaved=False, factor=1.0, orig_ctx=0, alpha=1.0, beta=32.0, mscale=1.0), **ROPES[which])
    act = F32 if which % 2 else BF16
    ctx, rows = [0, 15, 16, 37, 5, 100000 % 700], [1, 2, 33, 0, 16, 12]
    bt = Batch(nova, ctx, rows, n_kv, d, kind, seed=which, pad_rows=3).fill(which, stale=0.5)
    r = _rng(which, 7)
    qkv = _dev(r.normal(size=(bt.total, n_q + 2 * n_kv, d)) * np.exp(r.normal(size=(1, n_q + 2 * n_kv, d))), act)
    q, k, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
    pos = r.integers(0, [50, 100000, 1 << 30][which % 3], bt.total)
    before = [t.clone() for t in (bt.cache.k, bt.cache.v)]
    act_out = F32 if which % 4 == 1 else BF16 if which % 4 == 3 else act
    q_out = torch.full((bt.total, n_q, d), 7.0, dtype=act_out, device="cuda")
    rope_h = nova.Rope(**rope) if rope["rot"] else None
    got = nova.kv_append(bt.cache, bt.desc, k, v, q=q, pos=_dev(pos, torch.int32), rope=rope_h, q_out=q_out)
    torch.cuda.synchronize()
    assert got is q_out
    _check_append(bt, q, k, v, pos, rope, act_out, q_out, lambda b: int(bt.starts[b]))
    assert (q_out[bt.starts[-1]:] == 7.0).all()                      # rows behind the last sequence
    new = {bt.place(b, c + j) for b, (c, n) in enumerate(zip(ctx, rows)) for j in range(n)}
    for blk in range(bt.blocks):                                     # every other slot as it was
        keep = [s for s in range(16) if (blk, s) not in new]
        assert torch.equal(bt.cache.k[0, blk][:, keep], before[0][0, blk][:, keep])
        assert torch.equal(bt.cache.v[0, blk][:, :, keep], before[1][0, blk][:, :, keep])


def test_append_defaults_in_place_and_without_q(gpu_lib):
    """No row_start (equal rows), no ctx, positions from the tokens, q rotated in place; then k and v alone."""
    nova = gpu_lib
    r = _rng(11)
    n_q, n_kv, d = 4, 2, 64
    bt = Batch(nova, [0, 0, 0], [19, 19, 19], n_kv, d, "bf16", seed=3)
    bt.desc = nova.Rows(None, None, _dev(bt.tables, torch.int32), max_rows=19, max_ctx=19)
    q = _dev(r.normal(size=(57, n_q, d)), BF16)
    k, v = (_dev(r.normal(size=(57, n_kv, d)), BF16) for _ in "kv")
    q0 = q.clone()
    rope = dict(rot=64, theta=1e4, interleaved=False, factor=1.0, orig_ctx=0, alpha=1.0, beta=32.0, mscale=1.0)
    nova.kv_append(bt.cache, bt.desc, k, v, q=q, rope=nova.Rope(64), q_out=q)
    pos = np.tile(np.arange(19), 3)
    _check_append(bt, q0, k, v, pos, rope, BF16, q, lambda b: 19 * b)
    first = [t.clone() for t in (bt.cache.k, bt.cache.v)]
    bt.cache.k.zero_(), bt.cache.v.zero_()
    assert nova.kv_append(bt.cache, bt.desc, k, v, rope=nova.Rope(64)) is None
    assert torch.equal(bt.cache.k, first[0]) and torch.equal(bt.cache.v, first[1])


def test_append_extremes_in_8_bits(gpu_lib):
    """Zeros, tiny and huge rows, borders of the scale, and NaN and infinities (stored as NaN, the rest of the row kept)."""
    nova = gpu_lib
    x = np.ones((16, 1, 64), np.float32)
    x[0] = 0
    x[1] *= 1e-38
    x[2] *= 3.3e38
    x[3, 0, 1:] = 0
    x[4, 0, 5] = 448
    x[5, 0, 5] = np.nextafter(np.float32(448), np.float32(449))
    x[6, 0, 5] = 1e-3 * 2.0 ** 20
    x[7, 0, 7], x[7, 0, 8], x[7, 0, 9] = np.nan, np.inf, -np.inf
    x[8] = np.nan
    x[9, 0] = np.linspace(-1, 1, 64)
    x[10, 0] = np.ldexp(1.0, -np.arange(64))
    x[11, 0] = -np.ldexp(1.1, -np.arange(64))
    bt = Batch(nova, [0], [16], 1, 64, "e4m3", seed=1)
    t = _dev(x, F32)
    nova.kv_append(bt.cache, bt.desc, t, t)
    for j in range(16):
        with np.errstate(invalid="ignore"):
            want, e = oc.quantise(x[j].astype(np.float64))
        for got in bt.stored(0, j):
            assert np.array_equal(got, want, equal_nan=True), j
    blk, _ = bt.place(0, 0)
    assert bt.cache.k_exp[0, blk, 0, 0] == 127 - 100


# ----------------------------------------------------------------------------- gather
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,n_kv", [(64, 2), (128, 4), (128, 3)])
@pytest.mark.parametrize("picked", [False, True])
def test_gather(gpu_lib, kind, d, n_kv, picked):
    nova = gpu_lib
    held = [40, 1, 0, 129, 16]
    bt = Batch(nova, held, [0] * 5, n_kv, d, kind, seed=d + n_kv).fill(9, stale=3.0)
    n = [7, 1, 0, 50, 16] if picked else [40, 1, 0, 129, 16]
    starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(starts[-1]) + 2
    r = _rng(d, n_kv)
    slots = np.concatenate([r.integers(0, max(1, h), m) for h, m in zip(held, n)] + [[0, 0]]).astype(np.int32)
    desc = nova.Rows(_dev(starts, torch.int32), None, _dev(bt.tables, torch.int32), rows=total, max_rows=129, max_ctx=129)
    for out in (BF16, F32):
        wide = torch.full((total, n_kv + 1, d), 5.0, dtype=out, device="cuda")
        k_out = wide[:, :n_kv]                                       # a pitch of its own
        v_out = torch.full((total, n_kv, d), 5.0, dtype=out, device="cuda")
        nova.kv_gather(bt.cache, desc, slots=_dev(slots, torch.int32) if picked else None, k_out=k_out, v_out=v_out)
        for b in range(5):
            at = slots[starts[b]:starts[b + 1]] if picked else np.arange(n[b])
            for want, got in ((bt.k[b], k_out), (bt.v[b], v_out)):
                w = want[at] if len(want) else np.zeros((0, n_kv, d))
                w = torch.from_numpy(w).to(out).double().numpy()     # an f32 cache rounds to bf16 once; the others are exact
                assert np.array_equal(_np(got[starts[b]:starts[b + 1]]), w), (kind, b)
        assert (v_out[starts[-1]:] == 5.0).all() and (wide[:, n_kv] == 5.0).all()


def test_gather_from_ctx_and_missing_blocks(gpu_lib):
    """Rows that start inside a block, and table entries that name no block, which read as zeros and are not written."""
    nova = gpu_lib
    bt = Batch(nova, [60, 60], [0, 0], 2, 64, "e4m3", seed=5).fill(5)
    tables = bt.tables.copy()
    tables[1, 1], tables[1, 2] = -1, 1 << 30
    desc = nova.Rows(None, _dev(np.array([21, 10]), torch.int32), _dev(tables, torch.int32), max_rows=39, max_ctx=60)
    k, v = nova.kv_gather(bt.cache, desc, dtype=F32)
    assert np.array_equal(_np(k[:39]), bt.k[0][21:60]) and np.array_equal(_np(v[:39]), bt.v[0][21:60])
    w = bt.v[1][10:49].copy()
    w[16 - 10:48 - 10] = 0
    assert np.array_equal(_np(v[39:]), w)
    slots = _dev(np.array([59, -1, 64, 0, 20, 59, 1 << 30, 3]), torch.int32)
    desc = nova.Rows(None, None, _dev(tables, torch.int32), max_rows=4, max_ctx=60)
    k, _ = nova.kv_gather(bt.cache, desc, slots=slots, dtype=F32)
    zero = np.zeros((2, 64))
    assert np.array_equal(_np(k), np.stack([bt.k[0][59], zero, zero, bt.k[0][0], zero, bt.k[1][59], zero, bt.k[1][3]]))
    before = bt.cache.k.clone()
    desc = nova.Rows(None, _dev(np.array([48, 16]), torch.int32), _dev(tables, torch.int32), max_rows=12, max_ctx=60)
    one = torch.ones(24, 2, 64, dtype=BF16, device="cuda")
    nova.kv_append(bt.cache, desc, one, one)                        # sequence 1's rows fall on a missing block
    changed = (bt.cache.k != before).flatten(2).any(-1)[0].nonzero().flatten().tolist()
    assert changed == [int(tables[0, 3])]


@pytest.mark.parametrize("kind", TYPES)
def test_accepted_tokens_move_unchanged(gpu_lib, kind):
    """Gather of the accepted tokens and append behind the context: the same stored values at their new slots."""
    nova = gpu_lib
    ctx, rows = [13, 30], [12, 9]
    bt = Batch(nova, ctx, rows, 2, 64, kind, seed=21).fill(21)
    accepted = [[0, 3, 4, 11], [0, 1, 8]]
    slots = np.concatenate([c + np.array(a) for c, a in zip(ctx, accepted)]).astype(np.int32)
    starts = np.array([0, 4, 7], np.int32)
    desc = nova.Rows(_dev(starts, torch.int32), _dev(np.array(ctx), torch.int32), _dev(bt.tables, torch.int32), rows=7, max_rows=4, max_ctx=bt.max_ctx)
    k, v = nova.kv_gather(bt.cache, desc, slots=_dev(slots, torch.int32), dtype=F32 if kind == "f32" else BF16)
    nova.kv_append(bt.cache, desc, k, v)
    for b in range(2):
        for j, a in enumerate(accepted[b]):
            gk, gv = bt.stored(b, ctx[b] + j)
            assert np.array_equal(gk, bt.k[b][ctx[b] + a]) and np.array_equal(gv, bt.v[b][ctx[b] + a])


# ----------------------------------------------------------------------------- tree attention
def _tree_mask(n, r):
    m = []
    for j in range(n):
        up = int(r.integers(max(0, j - 3), j)) if j else -1
        m.append((1 << j) | (m[up] if up >= 0 else 0))
    return m


def _signed(m):
    return [x - (1 << 64) if x >= 1 << 63 else x for x in m]


def _tree_tolerance(kind, q, k, out, size, scale, tokens):
    """|out| rounds once; every p by half a bf16 step (not in fp32); a score's fp32 sum of D products and its
    exponential move p by their error relative, twice (p and the sum of p); sums over the tokens in fp32."""
    d = q.shape[-1]
    top = np.abs(q).max() * np.abs(k).max() * d * abs(scale) if k.size else 0.0
    score = np.sqrt((q ** 2).sum(-1)).max() * np.sqrt((k ** 2).sum(-1)).max() * abs(scale) if k.size else 0.0
    es = (d + 4) * 2.0 ** -24 * min(top, score * np.sqrt(d)) + 2.0 ** -22 * max(1.0, 2 * score)
    p = 2 * es + (tokens + 16) * 2.0 ** -24 + (0 if kind == "f32" else 2.0 ** -8)
    return HALF[F32 if kind == "f32" else BF16] * np.abs(out) * 1.01 + p * size + 1e-30


def _check_tree(bt, q, masks, out, scale, skip=()):
    for b, n in enumerate(bt.rows):
        if n == 0:
            continue
        sl = slice(int(bt.starts[b]), int(bt.starts[b]) + n)
        m = [(2 << j) - 1 for j in range(n)] if masks is None else masks[sl]
        with np.errstate(invalid="ignore"):
            want, size = oc.tree_attention(_np(q[sl]), bt.k[b], bt.v[b], bt.ctx[b], m, scale)
        fin = np.isfinite(bt.k[b])
        tol = _tree_tolerance(bt.kind, _np(q[sl]), np.where(fin, bt.k[b], 0), np.where(np.isfinite(want), want, 0), np.where(np.isfinite(size), size, 0), scale, bt.ctx[b] + n)
        got = _np(out[sl])
        assert np.array_equal(np.isnan(got), np.isnan(want)), b
        inf = np.isinf(want)
        assert np.array_equal(got[inf], want[inf])
        ok = np.isfinite(want)
        off = np.abs(got[ok] - want[ok])
        assert (off <= tol[ok]).all(), (b, off.max())


HEADS = [(4, 2, 64), (28, 4, 128), (3, 3, 64), (16, 1, 128), (40, 2, 64)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("heads", range(len(HEADS)))
@pytest.mark.parametrize("size", range(4))
def test_tree_attention(gpu_lib, kind, heads, size):
    nova = gpu_lib
    n_q, n_kv, d = HEADS[heads]
    ctx, rows = [([0, 1, 15, 16], [1, 3, 2, 5]), ([63, 64, 65, 200, 7], [17, 0, 1, 16, 8]), ([500], [64]),
                 ([1000, 0, 259], [1, 1, 1])][size]
    r = _rng(heads, size)
    bt = Batch(nova, ctx, rows, n_kv, d, kind, seed=heads * 10 + size, pad_rows=2).fill(heads, stale=float("nan"))
    act = bt.cache.dtype
    wide = _dev(r.normal(size=(bt.total, n_q + 2, d)), act)
    q = wide[:, 1:n_q + 1]                                           # a view of a wider row
    masks = None
    if (heads + size) % 2:
        masks = [m for n in rows for m in _tree_mask(n, r)] + [0, 0]
    mask = None if masks is None else torch.tensor(_signed(masks), dtype=torch.int64, device="cuda")
    scale = None if size else 0.3
    out = torch.full((bt.total, n_q, d), 9.0, dtype=act, device="cuda")
    nova.tree_attention(bt.cache, bt.desc, q, mask=mask, out=out, scale=scale)
    _check_tree(bt, q, masks, out, d ** -0.5 if scale is None else scale)
    assert (out[bt.starts[-1]:] == 9.0).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n_q,n_kv,d", [(28, 4, 128), (4, 2, 64)])
def test_tree_long_context_splits(gpu_lib, kind, n_q, n_kv, d):
    """Contexts that are cut into splits of unequal use, one sequence far shorter than the bound."""
    nova = gpu_lib
    ctx, rows = [4000, 3], [9, 2]
    bt = Batch(nova, ctx, rows, n_kv, d, kind, seed=31).fill(31)
    q = _dev(_rng(31).normal(size=(bt.total, n_q, d)) * 2, bt.cache.dtype)
    out = nova.tree_attention(bt.cache, bt.desc, q)
    _check_tree(bt, q, None, out, d ** -0.5)
    again = nova.tree_attention(bt.cache, bt.desc, q)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [1, 5, 40])
def test_tree_where_splits_begin(gpu_lib, kind, n):
    """Contexts about the lengths from which they are cut, in one, two or more steps a split, alone, beside a shorter
    sequence, and with a bound on the length that is larger than any."""
    nova = gpu_lib
    n_q, n_kv, d = 8, 2, 64
    for ctx in (60, 127, 190, 256, 300, 511, 512, 700, 1100):
        for other in (None, 17):
            ctxs = [ctx] if other is None else [ctx, other]
            bt = Batch(nova, ctxs, [n] * len(ctxs), n_kv, d, kind, seed=ctx).fill(ctx, stale=float("nan"))
            q = _dev(_rng(ctx, n).normal(size=(bt.total, n_q, d)), bt.cache.dtype)
            _check_tree(bt, q, None, nova.tree_attention(bt.cache, bt.desc, q), d ** -0.5)
            most = 16 * bt.desc.tables.shape[1]
            loose = nova.Rows(bt.desc.row_start, bt.desc.ctx, bt.desc.tables, rows=bt.total, max_rows=64, max_ctx=max(most, 64))
            _check_tree(bt, q, None, nova.tree_attention(bt.cache, loose, q), d ** -0.5)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,n", [(14, 3), (14, 5), (14, 9)])
def test_tree_waves_that_share_a_step(gpu_lib, kind, d, n_q, n):
    """21 to 63 rows of a KV head over steps enough that two waves each take half of a step's tokens: random masks, a
    sequence that ends inside the first half of a step, a drafted value that is not finite."""
    nova = gpu_lib
    n_kv, ctx = 2, [4100, 1033, 70, 0, 2047]
    r = _rng(d, n)
    bt = Batch(nova, ctx, [n] * 5, n_kv, d, kind, seed=61).fill(61, stale=float("nan"))
    bad = bt.v[1][1033 + 1].copy()
    bad[0, 3], bad[1, d - 1] = np.nan, np.nan
    bt.put(1, 1033 + 1, bt.k[1][1033 + 1], bad)
    masks = [m for _ in ctx for m in _tree_mask(n, r)]
    masks[0] = 0
    q = _dev(r.normal(size=(bt.total, n_q, d)) * 2, bt.cache.dtype)
    mask = torch.tensor(_signed(masks), dtype=torch.int64, device="cuda")
    for desc in (bt.desc, nova.Rows(None, bt.desc.ctx, bt.desc.tables, max_rows=n, max_ctx=bt.max_ctx)):
        out = nova.tree_attention(bt.cache, desc, q, mask=mask)
        _check_tree(bt, q, masks, out, d ** -0.5)
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(nova.tree_attention(bt.cache, desc, q, mask=mask)))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("ctx", [0, 30, 2000])
@pytest.mark.parametrize("n_q,n", [(4, 20), (2, 14)])
def test_tree_unseen_tokens_have_no_effect(gpu_lib, kind, ctx, n_q, n):
    """NaN and infinities in drafted tokens reach the rows that see them, in the dimensions concerned, and no others;
    a row that sees nothing is zero; a row may see itself only, or not even that."""
    nova = gpu_lib
    n_kv, d = 2, 64
    bt = Batch(nova, [ctx], [n], n_kv, d, kind, seed=41).fill(41)
    masks = [1 << j for j in range(n)]
    masks[3] = 0
    masks[5] = (1 << 5) | (1 << 8)
    masks[6] = (1 << 6) | (1 << 9)
    masks[7] = (1 << 7) | (1 << 10)
    # token 8: a NaN in K and V; 9: an infinity in a dimension of V, another in one head; 10: both kinds in one head
    bad = np.nan if kind == "e4m3" else np.inf
    c = bt.cache
    odd = {t: (bt.k[0][ctx + t].copy(), bt.v[0][ctx + t].copy()) for t in (8, 9, 10)}
    odd[8][0][0, 3] = np.nan
    odd[8][1][:, 5] = np.nan
    odd[9][1][:, 7], odd[9][1][1, 60] = bad, -bad
    odd[10][1][1, 11], odd[10][1][1, 63] = bad, np.nan
    for t, (kk, vv) in odd.items():
        bt.put(0, ctx + t, kk, vv)
    q = _dev(_rng(41).normal(size=(n, n_q, d)), c.dtype)
    out = nova.tree_attention(c, bt.desc, q, mask=torch.tensor(masks, dtype=torch.int64, device="cuda"))
    got = _np(out)
    clean_rows = [j for j in range(n) if j not in (5, 6, 7, 8, 9, 10)]
    assert np.isfinite(got[clean_rows]).all()
    if ctx == 0:
        assert (got[3] == 0).all()
    _check_tree(bt, q, masks, out, d ** -0.5)


def test_tree_large_scores(gpu_lib):
    """Scores far from zero, all far below, and one that dwarfs the rest."""
    nova = gpu_lib
    for kind, shift in (("bf16", 1.0), ("bf16", -1.0), ("e4m3", 1.0), ("f32", -1.0)):
        bt = Batch(nova, [70], [4], 1, 64, kind, seed=51)
        bt.fill(51)
        q = _dev(np.full((4, 2, 64), 300.0 * shift), bt.cache.dtype)
        bt.cache.k[0].copy_(bt.cache.k[0].abs() if kind != "e4m3" else bt.cache.k[0] & 0x7F)
        bt.k[0] = np.abs(bt.k[0])
        out = nova.tree_attention(bt.cache, bt.desc, q)
        _check_tree(bt, q, None, out, 64 ** -0.5)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-20])
def test_tree_any_scale(gpu_lib, kind, scale):
    """A negative scale prefers the least similar token, none at all averages what is seen; one tile of rows and more."""
    nova = gpu_lib
    for n_q, rows in ((4, [3, 2]), (24, [5, 9])):
        bt = Batch(nova, [90, 7], rows, 2, 64, kind, seed=55).fill(55, stale=float("nan"))
        q = _dev(_rng(55).normal(size=(bt.total, n_q, 64)), bt.cache.dtype)
        _check_tree(bt, q, None, nova.tree_attention(bt.cache, bt.desc, q, scale=scale), scale)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n_q,rows", [(8, 1), (40, 3)])
def test_tree_many_steps_of_a_workgroup(gpu_lib, kind, n_q, rows):
    """On 8 compute units a workgroup walks through more blocks than its table registers hold at a time."""
    nova = gpu_lib
    bt = Batch(nova, [20000], [rows], 8, 64, kind, seed=57).fill(57)
    q = _dev(_rng(57).normal(size=(rows, n_q, 64)), bt.cache.dtype)
    torch.cuda.synchronize()
    s = nova.set_stage_partition(nova.STAGE_DECODE, nova.make_cu_mask(8))
    out = nova.tree_attention(bt.cache, bt.desc, q, stream=s)
    s.synchronize()
    _check_tree(bt, q, None, out, 0.125)


@pytest.mark.parametrize("kind", TYPES)
def test_many_sequences(gpu_lib, kind):
    """More sequences than a wave has lanes, some without rows, through append, gather and attention."""
    nova = gpu_lib
    r = _rng(58)
    ctx, rows = [int(x) for x in r.integers(0, 40, 150)], [int(x) for x in r.integers(0, 5, 150)]
    rows[64], rows[127], rows[149] = 0, 30, 2
    bt = Batch(nova, ctx, rows, 2, 64, kind, seed=58, pad_rows=4).fill(58)
    q = _dev(r.normal(size=(bt.total, 4, 64)), bt.cache.dtype)
    _check_tree(bt, q, None, nova.tree_attention(bt.cache, bt.desc, q), 0.125)
    k, v = nova.kv_gather(bt.cache, bt.desc, dtype=F32)
    for b, n in enumerate(rows):
        at = slice(int(bt.starts[b]), int(bt.starts[b]) + n)
        assert np.array_equal(_np(k[at]), bt.k[b][ctx[b]:]) and np.array_equal(_np(v[at]), bt.v[b][ctx[b]:])
    bt.cache.k.zero_(), bt.cache.v.zero_()
    nova.kv_append(bt.cache, bt.desc, k, v)
    for b, n in enumerate(rows):
        for j in range(n):
            # the values, not the bytes: a largest value that was rounded to 224 2^e is kept as 448 2^(e - 1) now
            gk, gv = bt.stored(b, ctx[b] + j)
            assert np.array_equal(gk, bt.k[b][ctx[b] + j]) and np.array_equal(gv, bt.v[b][ctx[b] + j])
    assert int((bt.cache.v[0] != 0).any(1).any(1).sum()) <= sum(rows)


def test_contents_outside_the_bounds_are_clamped(gpu_lib):
    """Row starts, contexts and block ids that are not what they should be change no memory but the calls' own."""
    nova = gpu_lib
    big = 1 << 30
    for kind in TYPES:
        bt = Batch(nova, [30, 30], [4, 4], 2, 64, kind, seed=59, pad_rows=2).fill(59)
        guard = torch.full((12, 4, 64), 3.0, dtype=bt.cache.dtype, device="cuda")
        for starts, ctx in (([0, -5, 8], [30, 30]), ([4, 2, big], [-7, big]), ([big, big, big], [30, 30]), ([-big, 4, 8], [big, -big])):
            desc = nova.Rows(torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(ctx, dtype=torch.int32, device="cuda"),
                             bt.desc.tables, rows=10, max_rows=4, max_ctx=34)
            x = torch.ones(10, 2, 64, dtype=bt.cache.dtype, device="cuda")
            nova.kv_append(bt.cache, desc, x, x, q=guard[:10], q_out=guard[:10])
            nova.kv_gather(bt.cache, desc, k_out=torch.empty_like(x))
            nova.tree_attention(bt.cache, desc, guard[:10], out=guard[:10].clone())
        torch.cuda.synchronize()
        assert (guard[10:] == 3.0).all()


def test_tree_missing_blocks(gpu_lib):
    """Tokens of blocks that the table does not name are not seen."""
    nova = gpu_lib
    for kind in TYPES:
        bt = Batch(nova, [100, 40], [3, 2], 2, 64, kind, seed=61).fill(61)
        tables = bt.tables.copy()
        tables[0, 2], tables[1, :] = -5, bt.cache.num_blocks
        bt.desc = nova.Rows(bt.desc.row_start, bt.desc.ctx, _dev(tables, torch.int32), rows=5, max_rows=3, max_ctx=103)
        q = _dev(_rng(61).normal(size=(5, 4, 64)), bt.cache.dtype)
        out = nova.tree_attention(bt.cache, bt.desc, q)
        keep = [t for t in range(103) if t // 16 != 2]
        k, v = bt.k[0][keep], bt.v[0][keep]
        want, size = oc.tree_attention(_np(q[:3]), k, v, 84, [1, 3, 7], 0.125)
        tol = _tree_tolerance(kind, _np(q[:3]), k, want, size, 0.125, 103)
        assert (np.abs(_np(out[:3]) - want) <= tol).all()
        assert (out[3:] == 0).all()


def test_far_blocks(gpu_lib):
    """Blocks past 4 GB of each of K and V (32 bits of byte offset)."""
    nova = gpu_lib
    base = (1 << 32) // (4 * 16 * 128) + 10                          # e4m3: 8 KB a block
    bt = Batch(nova, [50], [20], 4, 128, "e4m3", seed=71, base_block=base)
    assert bt.cache.k.numel() > 1 << 32
    r = _rng(71)
    full = nova.Rows(None, None, _dev(bt.tables, torch.int32), max_rows=70, max_ctx=70)
    k, v = (_dev(r.normal(size=(70, 4, 128)), BF16) for _ in "kv")
    nova.kv_append(bt.cache, full, k, v)
    gk, gv = nova.kv_gather(bt.cache, full, dtype=F32)
    bt.k, bt.v = [oc.quantise(_np(k))[0]], [oc.quantise(_np(v))[0]]
    assert np.array_equal(_np(gk), bt.k[0]) and np.array_equal(_np(gv), bt.v[0])
    q = _dev(r.normal(size=(20, 28, 128)), BF16)
    _check_tree(bt, q, None, nova.tree_attention(bt.cache, bt.desc, q), 128 ** -0.5)
    assert not bt.cache.k[0, :1000].any()


# ----------------------------------------------------------------------------- log probabilities
def _check_logprobs(x, given, k, got):
    lp, ent, tl, ti = got
    w, h = oc.logprobs(_np(x))
    # results are float32: what is beyond its range by half a step (2^128 - 2^103, as -6e38 is) rounds to -infinity
    w = np.where(w <= -(2.0 ** 128 - 2.0 ** 103), -np.inf, w)
    # a lane adds at most 32 numbers a time and their sums are joined: under 400 roundings of S and T, and of
    # x - m and log S one each; exponents are off by |x - m| 2^-23, which S weighs with e^(x - m) |x - m| < 0.4 (T: < 0.6)
    tol = lambda v: 400 * 2.0 ** -24 + 2.0 ** -22 * (np.abs(v) + 12 + np.abs(_np(x)).max(initial=0.0, where=np.isfinite(_np(x))))  # noqa: E731
    if given is not None:
        want = np.take_along_axis(w, given.cpu().numpy().astype(int), 1)
        fin = np.isfinite(want)
        assert (np.abs(_np(lp)[fin] - want[fin]) <= tol(want[fin])).all() and np.array_equal(_np(lp)[~fin], want[~fin])
    assert (np.abs(_np(ent) - h) <= tol(h) + h * 400 * 2.0 ** -23).all()
    if k:
        ids = oc.top(_np(x), k)
        assert np.array_equal(ti.cpu().numpy(), ids)
        want = np.take_along_axis(w, ids, 1)
        fin = np.isfinite(want)
        assert (np.abs(_np(tl)[fin] - want[fin]) <= tol(want[fin])).all() and np.array_equal(_np(tl)[~fin], want[~fin])
    else:
        assert tl is None and ti is None


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,n,k", [(1, 1, 1, 1), (3, 33, 2, 32), (1, 4096, 1, 5), (2, 2047, 0, 32), (5, 2049, 1, 20), (1, 152064, 1, 20),
                                            (32, 32001, 4, 8), (2, 70001, 1, 0), (300, 5000, 1, 0), (4, 8192, 3, 1)])
def test_logprobs(gpu_lib, act, rows, vocab, n, k):
    r = _rng(rows, vocab)
    x = _dev(r.normal(size=(rows, vocab)) * 3, act)
    given = _dev(r.integers(0, vocab, (rows, n)), torch.int32) if n else None
    _check_logprobs(x, given, k, gpu_lib.logprobs(x, given=given, n_top=k))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("vocab", [100, 4097, 20000])
def test_logprobs_ties_and_masked_tokens(gpu_lib, act, vocab):
    """Equal logits go to the lowest ids (all equal, two values, signed zeros); -infinity has probability 0."""
    r = _rng(vocab)
    x = np.zeros((6, vocab))
    x[1] = r.integers(0, 2, vocab)
    x[2] = np.where(r.random(vocab) < 0.5, 0.0, -0.0)
    x[3] = np.where(np.arange(vocab) % 97 == 5, r.normal(size=vocab), -np.inf)
    x[4], x[4, vocab - 1] = -np.inf, 2.0
    x[5] = -1e4 + r.integers(0, 3, vocab) * 64
    xt = _dev(x, act)
    given = _dev(np.stack([np.arange(6) % vocab, np.full(6, vocab - 1)], 1), torch.int32)
    with np.errstate(divide="ignore"):
        _check_logprobs(xt, given, 32, gpu_lib.logprobs(xt, given=given, n_top=32))


@pytest.mark.parametrize("vocab", [700, 20001])
def test_logprobs_of_masked_rows(gpu_lib, vocab):
    """Logits masked with the type's lowest value, some of a row or all of it, and rows far from zero."""
    r = _rng(vocab, 3)
    for act in (F32, BF16):
        low = torch.finfo(act).min
        x = torch.from_numpy(r.normal(size=(6, vocab)) * 3).cuda()
        x[0, 5:] = low
        x[1] = low
        x[2, ::3] = low
        x[3] += 1e6
        x[4] = torch.where(x[4] > 0, 3e38, -3e38)
        x[5] -= 70000
        x = x.to(act)
        given = torch.tensor([[0, vocab - 1]] * 6, dtype=torch.int32, device="cuda")
        got = gpu_lib.logprobs(x, given=given, n_top=8)
        _check_logprobs(x, given, 8, got)
        # x - m is exact to its own rounding: the size of the logits themselves costs nothing where the unmasked are near
        w, h = oc.logprobs(_np(x[:4]))
        want = np.take_along_axis(w, got[3][:4].cpu().numpy().astype(int), 1)
        assert (np.abs(_np(got[2][:4]) - want) <= 400 * 2.0 ** -24 + 2.0 ** -22 * (np.abs(want) + 12))[[0, 2, 3]].all()
        assert (np.abs(_np(got[1][:4]) - h) <= 400 * 2.0 ** -24 + 2.0 ** -22 * (h + 12) + h * 400 * 2.0 ** -23).all()


@pytest.mark.parametrize("vocab", [700, 9001, 152064])
def test_logprobs_of_few_tokens_left(gpu_lib, vocab):
    """Rows masked but for 0 to 300 tokens side by side, which may be fewer than the alternatives asked for; and rows
    whose largest logits are all in groups that a few lanes of a wave look at."""
    r = _rng(vocab, 5)
    for act in (F32, BF16):
        for low in (-np.inf, torch.finfo(act).min, -1e4):
            x = np.full((8, vocab), low)
            for i, n in enumerate((1, 5, 19, 31, 32, 40, 300)):
                at = (0, vocab - n, 77)[i % 3]
                x[i, at:at + n] = r.normal(size=n)
            if low == -np.inf:
                x[7, 0] = 1.0                                     # a row of nothing else has no distribution
            xt = _dev(x, act)
            given = torch.tensor([[0, vocab - 1]] * 8, dtype=torch.int32, device="cuda")
            with np.errstate(divide="ignore"):
                for k in (32, 7):
                    _check_logprobs(xt, given, k, gpu_lib.logprobs(xt, given=given, n_top=k))
        x = r.normal(size=(3, vocab))
        x[:, (np.arange(vocab) // 64) % 64 < 19] += 10
        x[2] = np.round(x[2])
        xt = _dev(x, act)
        _check_logprobs(xt, None, 20, gpu_lib.logprobs(xt, n_top=20))


def test_logprobs_odd_values_ids_and_pitch(gpu_lib):
    nova = gpu_lib
    x = torch.randn(5, 3001, device="cuda")
    x[0, 7], x[1, 9], x[2] = float("nan"), float("inf"), float("-inf")
    lp, ent, tl, ti = nova.logprobs(x, given=torch.tensor([[7], [9], [0], [0], [0]], dtype=torch.int32, device="cuda"), n_top=2)
    assert torch.isnan(lp[:3]).all() and torch.isnan(ent[:3]).all() and torch.isnan(tl[:3]).all()
    assert ti[0, 0] == 7 and ti[1, 0] == 9 and ti[2].tolist() == [0, 1]
    assert torch.isfinite(lp[3:]).all() and torch.isfinite(ent[3:]).all()
    lp, _, _, _ = nova.logprobs(x[3:], given=torch.tensor([[-1, 3001], [5, 1 << 30]], dtype=torch.int32, device="cuda"))
    assert lp[0].tolist() == [float("-inf")] * 2 and torch.isfinite(lp[1, 0]) and lp[1, 1] == float("-inf")
    for act in (F32, BF16):                                          # rows at odd addresses
        wide = torch.randn(4, 5003, device="cuda").to(act)
        part = wide[:, 3:4004]
        _check_logprobs(part, None, 10, nova.logprobs(part, n_top=10))


# ----------------------------------------------------------------------------- streams and graphs
def test_ops_on_a_stream_and_in_a_graph(gpu_lib):
    """The chain append, attention, gather, log probabilities on a side stream; captured once and replayed with
    other inputs, lengths and tables, against the eager calls."""
    nova = gpu_lib
    n_q, n_kv, d = 28, 4, 128
    r = _rng(81)
    bt = Batch(nova, [1500, 33], [5, 3], n_kv, d, "e4m3", seed=81).fill(81)
    qkv = _dev(r.normal(size=(8, n_q + 2 * n_kv, d)), BF16)
    mask = torch.tensor(_tree_mask(5, r) + _tree_mask(3, r), dtype=torch.int64, device="cuda")
    rope = nova.Rope(d)
    given = _dev(r.integers(0, n_q * d, (8, 1)), torch.int32)

    def chain(stream=None):
        q = nova.kv_append(bt.cache, bt.desc, qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:], q=qkv[:, :n_q], rope=rope, stream=stream)
        att = nova.tree_attention(bt.cache, bt.desc, q, mask=mask, stream=stream)
        k, v = nova.kv_gather(bt.cache, bt.desc, stream=stream)
        return (q, att, k, v) + nova.logprobs(att.view(8, -1), given=given, n_top=5, stream=stream)
    eager = chain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = chain(side)                                                # on `side` while another stream is current
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, got))
    with torch.cuda.stream(side):
        chain()
    side.synchronize()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = chain()
    for turn in range(4):
        qkv.copy_(_dev(r.normal(size=tuple(qkv.shape)), BF16))
        bt.desc.ctx.copy_(_dev(np.array([1500 - 200 * turn, 33 - turn]), torch.int32))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in held]
        want = chain()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want)), turn


def test_concurrent_calls_on_two_streams(gpu_lib):
    """Two chains at once, each with its own workspace, give what each gives alone."""
    nova = gpu_lib
    bts = [Batch(nova, [3000, 10], [7, 4], 4, 128, kind, seed=91 + i).fill(91 + i) for i, kind in enumerate(("bf16", "e4m3"))]
    qs = [_dev(_rng(92 + i).normal(size=(11, 28, 128)), BF16) for i in range(2)]
    x = torch.randn(16, 30000, device="cuda")
    alone = [nova.tree_attention(bt.cache, bt.desc, q) for bt, q in zip(bts, qs)]
    lp = nova.logprobs(x, n_top=8)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            outs[i].append((nova.tree_attention(bts[i].cache, bts[i].desc, qs[i], stream=s), nova.logprobs(x, n_top=8, stream=s)))
    torch.cuda.synchronize()
    for i in range(2):
        for o, l in outs[i]:
            assert torch.equal(o, alone[i])
            assert all(torch.equal(a, b) for a, b in zip(l[1:], lp[1:]))


def test_on_a_partition_stream(gpu_lib):
    """A stage's compute-unit partition changes the split of the context, not what is asked for."""
    nova = gpu_lib
    bt = Batch(nova, [2500], [6], 4, 128, "e4m3", seed=101).fill(101)
    q = _dev(_rng(101).normal(size=(6, 28, 128)), BF16)
    torch.cuda.synchronize()
    s = nova.set_stage_partition(nova.STAGE_DECODE, nova.make_cu_mask(64))
    out = nova.tree_attention(bt.cache, bt.desc, q, stream=s)
    s.synchronize()
    _check_tree(bt, q, None, out, 128 ** -0.5)


def test_logits_past_32_bits(gpu_lib):
    """More than 2^32 bytes of logits: the last rows are those of a call of their own."""
    nova = gpu_lib
    x = torch.randn(15000, 152064, dtype=BF16, device="cuda")
    given = torch.full((15000, 1), 152063, dtype=torch.int32, device="cuda")
    got = nova.logprobs(x, given=given, n_top=3)
    some = nova.logprobs(x[-5:], given=given[-5:], n_top=3)
    assert torch.equal(got[3][-5:], some[3])
    for a, b in zip(got[:3], some[:3]):
        assert (a[-5:] - b).abs().max() < 1e-4                       # cut into other parts: other orders of the sums
    _check_logprobs(x[-5:], given[-5:], 3, some)


def test_vocab_of_the_framework(gpu_lib):
    """The real head's logits of a full batch."""
    x = torch.randn(32, synth.LLM_28.vocab, device="cuda") * 3
    given = torch.randint(0, synth.LLM_28.vocab, (32, 1), dtype=torch.int32, device="cuda")
    _check_logprobs(x, given, 20, gpu_lib.logprobs(x, given=given, n_top=20))
