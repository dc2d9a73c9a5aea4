"""The operators between two model calls against their float64 definitions (oracle.steps).

Tolerances count roundings (half a step of bf16 is 2^-8 relative, of e4m3 2^-4, of fp32 2^-24) and fp32 sums, bounded
term by term, so that nothing in them was measured.  Whole numbers, and what is moved, are equal."""
import numpy as np
import pytest
import torch

from oracle import steps as st

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


def _i32(a):
    return _dev(np.asarray(a, np.int32), torch.int32)


def _signed(masks):
    return [m - (1 << 64) if m >= 1 << 63 else m for m in masks]


# ----------------------------------------------------------------------------- rotary positions with several axes
AXES = [dict(pairs=(16, 24, 24)), dict(pairs=(24, 20, 20), cyclic=True), dict(pairs=(8, 8), own_freqs=True),
        dict(pairs=(0, 3, 13), cyclic=True, own_freqs=True), dict(pairs=(32,)), dict(pairs=(5, 1, 20, 6), interleaved=True),
        dict(pairs=(10, 22), cyclic=True, interleaved=True, own_freqs=True, factor=4.0, mscale=1.25),
        dict(pairs=(7, 9), factor=8.0, orig_ctx=4096, theta=1e6), dict(pairs=(20, 20), own_freqs=True)]


def _rope_of(nova, a):
    args = {k: v for k, v in a.items() if k != "pairs"}
    scaling = {k: a[k] for k in ("factor", "orig_ctx") if k in a}
    freq = st.axes_frequencies(a["pairs"], a.get("theta", 1e4), a.get("cyclic", False), a.get("own_freqs", False), **scaling)

    def turn(x, pos):
        return st.rotate_axes(x, pos, a["pairs"], freq, a.get("cyclic", False), a.get("interleaved", False), a.get("mscale", 1.0))
    # sines and cosines within 3 roundings, two products and a sum: 8 of each of the pair's members
    return nova.Rope(2 * sum(a["pairs"]), axes=a["pairs"], **args), turn, 8 * 2.0 ** -24 * a.get("mscale", 1.0)


def _rotate_tol(x, want, out, fp):
    return HALF[out] * np.abs(want) + 2 * fp * 2 * np.abs(_np(x)).max(-1, keepdims=True)


@pytest.mark.parametrize("which", range(len(AXES)))
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
def test_rotate(gpu_lib, which, types):
    nova = gpu_lib
    a = AXES[which]
    rope, turn, fp = _rope_of(nova, a)
    rot = 2 * sum(a["pairs"])
    r = _rng(which, 1)
    for rows, heads, d in [(1, 1, rot), (3, 5, rot + 8), (17, 2, 128), (33, 32, 136 if which % 2 else 256)]:
        if d < rot:
            continue
        wide = _dev(r.normal(size=(rows, heads + 2, d)), types[0])          # a view of a packed projection
        x = wide[:, 1:1 + heads]
        pos = r.integers(0, [60, 100000, 1 << 30][which % 3], size=(len(a["pairs"]), rows))
        big = torch.full((rows, heads + 1, d), 7.0, dtype=types[1], device="cuda")
        out = nova.rotate(x, _i32(pos), rope, out=big[:, :heads])
        want = turn(_np(x), pos)
        assert (np.abs(_np(out) - want) <= _rotate_tol(x, want, types[1], fp)).all(), (rows, heads, d)
        assert (big[:, heads:] == 7.0).all()
        if types[0] == types[1]:                                            # in place, and out of the caller's sight
            beside = wide[:, [0, heads + 1]].clone()
            assert torch.equal(nova.rotate(x.contiguous(), _i32(pos), rope), out)
            nova.rotate(x, _i32(pos), rope, out=x)
            assert torch.equal(x, out) and torch.equal(wide[:, [0, heads + 1]], beside)


def test_rotate_back(gpu_lib):
    """Positions below 0 turn the other way: there and back is where it was, up to the two rotations' roundings."""
    nova = gpu_lib
    for a in (AXES[0], AXES[5]):
        rope, _, fp = _rope_of(nova, dict(a, mscale=1.0))
        x = torch.randn(50, 3, 2 * sum(a["pairs"]), device="cuda")
        pos = torch.randint(0, 1 << 20, (len(a["pairs"]), 50), device="cuda", dtype=torch.int32)
        y = nova.rotate(nova.rotate(x, pos, rope), -pos, rope)
        assert ((y - x).abs() <= 4 * 2 * fp * 2 * x.abs().amax(-1, keepdim=True)).all()


def test_rotate_many_rows(gpu_lib):
    """Rows beyond one workgroup's, its last workgroup in part, and 900 heads (more than a group)."""
    nova = gpu_lib
    a = AXES[-1]
    rope, turn, fp = _rope_of(nova, a)
    r = _rng(5)
    for rows, heads, d in [(9001, 3, 80), (8500, 1, 80), (2, 900, 80)]:
        x = torch.randn(rows, heads, d, device="cuda").to(BF16)
        pos = np.stack([np.arange(rows) // 97, np.arange(rows) % 97])
        out = nova.rotate(x, _i32(pos), rope)
        at = np.unique(np.concatenate([[0, rows - 1], r.integers(0, rows, 200)]))
        want = turn(_np(x[at]), pos[:, at])
        assert (np.abs(_np(out[at]) - want) <= _rotate_tol(x[at], want, BF16, fp)).all()
        assert torch.equal(out, torch.cat([nova.rotate(x[i:i + 500], _i32(pos[:, i:i + 500]), rope) for i in range(0, rows, 500)]))


def test_rotate_one_axis_is_the_plain_rope(gpu_lib):
    nova = gpu_lib
    x = torch.randn(40, 4, 64, device="cuda")
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    plain = nova.rotate(x, pos, nova.Rope(48))
    assert torch.equal(plain, nova.rotate(x, pos[None], nova.Rope(48, axes=(24,))))
    assert torch.equal(plain, nova.rotate(x, pos.expand(3, 40).contiguous(), nova.Rope(48, axes=(8, 6, 10), cyclic=True)))
    assert nova.rotate(x[:0], pos[:0], nova.Rope(48)).shape == (0, 4, 64)
    assert torch.equal(nova.rotate(x, pos, nova.Rope(0)), x)


def _paged(nova, ctx, rows, n_kv, d, kind, seed, layers=1, pad_rows=0, fill=True):
    """Sequences over a shuffled pool filled with random contents."""
    r = _rng(seed, 3)
    held = [c + n for c, n in zip(ctx, rows)]
    need = [-(-h // 16) for h in held]
    blocks, width = sum(need) + 4, max(1, max(need))
    tables = np.full((len(ctx), width), -1, np.int64)
    order, at = r.permutation(blocks), 0
    for b, n in enumerate(need):
        tables[b, :n] = order[at:at + n]
        at += n
    type = dict(bf16=nova.CACHE_BF16, f32=nova.CACHE_F32, e4m3=nova.CACHE_E4M3)[kind]
    c = nova.Cache(blocks, n_kv, d, type, layers=layers)
    if fill:
        _fill(c, r)
    starts = np.concatenate([[0], np.cumsum(rows)])
    desc = nova.Rows(_i32(starts), _i32(ctx), _i32(tables), rows=int(starts[-1]) + pad_rows, max_rows=max(1, max(rows)), max_ctx=max(1, max(held)))
    return c, desc, tables, starts


def _fill(c, r):
    for t in (c.k, c.v):
        if t.dtype == torch.uint8:
            t.copy_(torch.from_numpy(r.integers(0, 256, size=tuple(t.shape), dtype=np.uint8)))
        else:
            t.copy_(torch.from_numpy(r.normal(size=tuple(t.shape)).astype(np.float32)))
    for t in (c.k_exp, c.v_exp):
        if t is not None:
            t.copy_(torch.from_numpy(r.integers(100, 150, size=tuple(t.shape), dtype=np.uint8)))


def _arrays(c):
    return [t for t in (c.k, c.v, c.k_exp, c.v_exp) if t is not None]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("which", [0, 1, 3, 5, 6])
def test_append_axes(gpu_lib, kind, which):
    nova = gpu_lib
    a = AXES[which]
    rope, turn, fp = _rope_of(nova, a)
    d, n_kv, n_q = (64, 2, 4) if sum(a["pairs"]) <= 32 and which % 2 else (128, 3, 6)
    act = F32 if which % 2 else BF16
    ctx, rows = [0, 15, 37, 5], [1, 18, 0, 12]
    c, desc, tables, starts = _paged(nova, ctx, rows, n_kv, d, kind, which, pad_rows=2)
    r = _rng(which, 9)
    qkv = _dev(r.normal(size=(desc.rows, n_q + 2 * n_kv, d)) * np.exp(r.normal(size=(1, n_q + 2 * n_kv, d))), act)
    q, k, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
    pos = r.integers(0, 100000, size=(len(a["pairs"]), desc.rows))
    got = nova.kv_append(c, desc, k, v, q=q, pos=_i32(pos), rope=rope, q_out=torch.full_like(q, 7.0, memory_format=torch.contiguous_format))
    n = int(starts[-1])
    want = turn(_np(q), pos)
    assert (np.abs(_np(got[:n]) - want[:n]) <= _rotate_tol(q, want, act, fp)[:n]).all() and (got[n:] == 7.0).all()
    # The cache against the definition.  (Not bit by bit against rows turned by nova.rotate: whether a c - b s is one
    # fused operation or two is each kernel's own, and moves the result by a rounding of 2^-24 of a product.)
    wk, wv = turn(_np(k), pos), _np(v)
    for b, m in enumerate(rows):
        for j in range(m):
            blk, s = tables[b, (ctx[b] + j) // 16], (ctx[b] + j) % 16
            row = starts[b] + j
            for held, exps, w, err in ((c.k[0, blk, :, s], c.k_exp, wk[row], 2 * fp * 2 * np.abs(_np(k[row])).max(-1, keepdims=True)),
                                       (c.v[0, blk, :, :, s], c.v_exp, wv[row], 0.0)):
                if kind == "e4m3":
                    scale = np.ldexp(1.0, exps[0, blk, :, s].cpu().numpy().astype(int) - 127)[:, None]
                    have = _np(held.contiguous().view(torch.float8_e4m3fn)) * scale
                    # half a step of 4 significant bits or of the smallest numbers, of the scale that is kept
                    tol = 2.0 ** -4 * np.abs(w) + 2.0 ** -9 * scale + err
                    assert (np.abs(w).max(-1) <= 448 * scale[:, 0] + np.ravel(err)).all()
                else:
                    have, tol = _np(held), HALF[F32 if kind == "f32" else BF16] * np.abs(w) + err
                assert (np.abs(have - w) <= tol).all(), (b, j)


def test_append_axes_default_positions(gpu_lib):
    """Without positions every axis counts the token's number: the plain rope."""
    nova = gpu_lib
    k, v = torch.randn(2, 19, 2, 64, device="cuda")
    out = []
    for rope in (nova.Rope(64), nova.Rope(64, axes=(10, 12, 10))):
        c, desc, _, _ = _paged(nova, [5], [19], 2, 64, "f32", 4)
        nova.kv_append(c, desc, k, v, rope=rope)
        out.append(c)
    assert torch.equal(out[0].k, out[1].k) and torch.equal(out[0].v, out[1].v)


# ----------------------------------------------------------------------------- acceptance
def _accept_case(rows, vocab, seed, act, kind, spread=3.0):
    r = _rng(seed, 5)
    n = sum(rows)
    starts = np.concatenate([[0], np.cumsum(rows)])
    logits = _dev(r.normal(size=(n + 2, vocab)) * spread, act)
    draft = _dev(_np(logits)[np.maximum(np.arange(n + 2) - 1, 0)] + 0.7 * r.normal(size=(n + 2, vocab)), act) if kind == "draft" else None
    masks, ids, t = [], np.zeros(n + 2, np.int64), []
    for b, m in enumerate(rows):
        t.append([0.7, 1.0, 0.0, 1.6][b % 4])
        seen = []
        for j in range(m):
            up = -1 if j == 0 else j - 1 if kind != "tree" else int(r.integers(max(0, j - 3), j))
            seen.append((1 << j) | (seen[up] if up >= 0 else 0))
            p = st.distribution(_np((draft if draft is not None else logits)[starts[b] + (j if draft is not None else max(up, 0))]), max(t[-1], 0.05))
            ids[starts[b] + j] = st.draw(p, r.random())
        masks += seen
    masks += [0, 0]
    return starts, logits, draft, ids, (masks if kind == "tree" else None), np.array(t), r.random(n + 2).astype(np.float32)


def _check_accept(nova, rows, starts, logits, draft, ids, masks, t, u, tables=None):
    batch, width = len(rows), max(1, max(rows))
    desc = nova.Rows(_i32(starts), None, _i32(np.zeros((batch, 4))), rows=len(ids), max_rows=width, max_ctx=64)
    temp = None if t is None else _dev(t, F32)
    got = nova.accept(desc, _i32(ids), logits, _dev(u, F32), mask=None if masks is None else torch.tensor(_signed(masks), device="cuda"),
                      draft=draft, temperature=temp)
    n_keep, path, tokens, lp = (x.cpu().numpy() for x in got)
    lg, dr = _np(logits), None if draft is None else _np(draft)
    kept = 0
    for b, n in enumerate(rows):
        sl = slice(starts[b], starts[b] + n)
        if n == 0:
            assert n_keep[b] == 0 and (path[b] == -1).all() and (tokens[b] == -1).all() and (lp[b] == 0).all()
            continue
        wp, wt, wl = st.accept(lg[sl], ids[sl], u[sl].astype(float), None if masks is None else masks[sl], None if dr is None else dr[sl],
                               1.0 if t is None else t[b])
        k = len(wp)
        kept += k - 1
        assert n_keep[b] == k and list(path[b, :k]) == wp and list(tokens[b, :k]) == wt, (b, n_keep[b], path[b], tokens[b], wp, wt)
        assert (path[b, k:] == -1).all() and (tokens[b, k:] == -1).all() and (lp[b, k:] == 0).all()
        # 64-bit sums, rounded once to fp32
        wl = np.array(wl)
        assert np.array_equal(np.isnan(lp[b, :k]), np.isnan(wl))
        ok = ~np.isnan(wl)
        assert (np.abs(lp[b, :k][ok] - wl[ok]) <= 2.0 ** -24 * np.abs(wl[ok]) + 1e-9).all()
    return kept


@pytest.mark.parametrize("kind", ["tree", "chain", "draft"])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("vocab", [1, 2, 33, 4095, 4096, 4097, 20001])
def test_accept(gpu_lib, kind, act, vocab):
    rows = [5, 1, 0, 12, 3, 7, 2]
    case = _accept_case(rows, vocab, vocab, act, kind, spread=6.0 if vocab > 1000 else 2.0)
    kept = _check_accept(gpu_lib, rows, *case)
    assert kept > 0 or vocab > 4000


@pytest.mark.parametrize("kind", ["tree", "chain", "draft"])
def test_accept_at_the_real_vocabulary(gpu_lib, kind):
    """152064 logits, 64 rows of one sequence, nearly flat distributions (the running sums have many borders)."""
    rows = [64, 3]
    _check_accept(gpu_lib, rows, *_accept_case(rows, 152064, 3, F32, kind, spread=0.5))


@pytest.mark.parametrize("kind", ["tree", "draft"])
def test_accept_many_chunks(gpu_lib, kind):
    """More chunks than lanes (700001 logits: 86), equal large logits among them, a greedy sequence."""
    rows = [3, 2, 2]
    starts, logits, draft, ids, masks, t, u = _accept_case(rows, 700001, 12, F32, kind, spread=1.0)
    logits[3] = 0.0
    logits[3, [5, 650000, 700000]] = 40.0
    u[3] = 0.6
    _check_accept(gpu_lib, rows, starts, logits, draft, ids, masks, t, u)


def test_accept_keeps_everything_when_draft_and_target_agree(gpu_lib):
    nova = gpu_lib
    rows = [6, 6]
    starts, logits, _, ids, _, t, u = _accept_case(rows, 5000, 1, F32, "chain")
    draft = logits[torch.arange(len(ids)).sub(1).clamp(min=0)].contiguous()
    u[:] = np.float32(0.99999)
    assert _check_accept(nova, rows, starts, logits, draft, ids, None, np.array([1.0, 0.6]), u) == 10
    assert _check_accept(nova, rows, starts, logits, draft, ids, None, None, u) == 10


@pytest.mark.parametrize("kind", ["tree", "chain", "draft"])
def test_accept_rows_without_a_distribution(gpu_lib, kind):
    """NaN, infinities, masked rows and temperatures that give no distribution; logits masked but for one or two."""
    rows = [4] * 10
    starts, logits, draft, ids, masks, t, u = _accept_case(rows, 3000, 7, F32, kind)
    t = np.array([1.0] * 7 + [-1.0, np.nan, np.inf])
    logits[0, 17] = float("nan")
    logits[4, 2999] = float("inf")
    logits[8] = float("-inf")
    logits[13, 5] = float("nan")                       # behind the first row of sequence 3
    logits[16:20] = float("-inf")                      # all but one: certain
    logits[16:20, 11] = -3.0
    ids[16:20] = 11
    if draft is not None:
        draft[21] = float("-inf")                      # a draft row of nothing
        draft[25, 3] = float("nan")
        draft[17:20] = float("-inf")
        draft[17:20, 11] = 5.0
    logits[20:28, ::2] = float("-inf")
    with np.errstate(invalid="ignore"):
        _check_accept(gpu_lib, rows, starts, logits, draft, ids, masks, t, u)


@pytest.mark.parametrize("kind", ["chain", "draft"])
def test_accept_numbers_at_the_ends(gpu_lib, kind):
    """u of 0, just below 1, 1, above, negative and NaN; ids outside the vocabulary; probabilities that underflow."""
    rows = [3] * 8
    starts, logits, draft, ids, masks, _, u = _accept_case(rows, 4099, 8, F32, kind)
    for i, x in enumerate([0.0, np.nextafter(np.float32(1), np.float32(0)), 1.0, 7.0, -1.0, np.nan, 0.5, 1e-38]):
        u[3 * i:3 * i + 3] = x
    ids[4], ids[7], ids[10] = -1, 4099, 1 << 30
    logits[3] = -torch.arange(4099, device="cuda").float() * 50
    logits[18:21] = 3e38 * torch.sign(logits[18:21])
    _check_accept(gpu_lib, rows, starts, logits, draft, ids, masks, np.array([1.0, 0.01, 1.0, 1.0, 30.0, 1.0, 1e-30, 2.0]), u)


def test_accept_ties_and_temperature_zero(gpu_lib):
    rows = [4, 4]
    starts, logits, draft, ids, masks, _, u = _accept_case(rows, 9000, 9, BF16, "chain")
    logits[:] = torch.floor(logits.float()).to(BF16)
    top = logits[:8].float().amax(-1, keepdim=True)
    first = (logits[:8].float() == top).int().argmax(-1).cpu().numpy()
    ids[1:4] = first[0:3]
    _check_accept(gpu_lib, rows, starts, logits, None, ids, None, np.zeros(2), u)
    _check_accept(gpu_lib, rows, starts, logits, logits, ids, None, np.zeros(2), u)


def test_accept_odd_pitch_and_mixed_types(gpu_lib):
    """Logit rows at any element's address, a bf16 draft of an fp32 target and the reverse, equal rows without row_start."""
    nova = gpu_lib
    vocab, r = 4999, _rng(4)
    for act, dact in ((F32, BF16), (BF16, F32)):
        wide = _dev(r.normal(size=(12, vocab + 7)) * 4, act)
        dwide = _dev(_np(wide)[np.maximum(np.arange(12) - 1, 0)] + 0.3 * r.normal(size=(12, vocab + 7)), dact)
        logits, draft = wide[:, 3:3 + vocab], dwide[:, 3:3 + vocab]
        ids, u = r.integers(0, vocab, 12), r.random(12).astype(np.float32)
        for j in range(12):
            ids[j] = st.draw(st.distribution(_np(draft[j]), 1.0), r.random())
        desc = nova.Rows(None, None, _i32(np.zeros((3, 4))), max_rows=4, max_ctx=64)
        n_keep, path, tokens, _ = nova.accept(desc, _i32(ids), logits, _dev(u, F32), draft=draft)
        for b in range(3):
            sl = slice(4 * b, 4 * b + 4)
            wp, wt, _ = st.accept(_np(logits[sl]), ids[sl], u[sl].astype(float), None, _np(draft[sl]))
            assert n_keep[b] == len(wp) and tokens[b, :len(wp)].tolist() == wt and path[b, :len(wp)].tolist() == wp


def test_accept_draws_what_the_target_would(gpu_lib):
    """The tokens that come out are distributed as the target's: 6000 sequences over a vocabulary of 12, chi-squared."""
    nova = gpu_lib
    r, n = _rng(1), 6000
    p, q = _dev(r.normal(size=(1, 12)) * 1.5, F32), _dev(r.normal(size=(1, 12)) * 1.5, F32)
    logits = p.expand(2 * n, 12).contiguous()
    draft = q.expand(2 * n, 12).contiguous()
    pq = st.distribution(_np(q)[0], 1.0)
    ids = np.zeros(2 * n, np.int64)
    ids[1::2] = r.choice(12, size=n, p=pq)
    desc = nova.Rows(None, None, _i32(np.zeros((n, 4))), max_rows=2, max_ctx=64)
    _, _, tokens, _ = nova.accept(desc, _i32(ids), logits, _dev(r.random(2 * n), F32), draft=draft)
    seen = np.bincount(tokens[:, 0].cpu().numpy(), minlength=12)
    want = n * st.distribution(_np(p)[0], 1.0)
    # 11 degrees of freedom: 31.3 is passed by chance once in 1000 (the seed is fixed)
    assert ((seen - want) ** 2 / want).sum() < 31.3


# ----------------------------------------------------------------------------- kept rows
def _kept(arrays, tables, ctx, path, n_keep, e4m3):
    """What a keep leaves of a cache's arrays (host copies), from the copies before it."""
    out = [a.clone() for a in arrays]
    blocks = arrays[0].shape[1]
    for b, p in enumerate(path):
        for i, j in enumerate(p[:n_keep[b]]):
            frm, to = ctx[b] + j, ctx[b] + i
            if j < 0 or tables[b][frm // 16] not in range(blocks) or tables[b][to // 16] not in range(blocks):
                continue
            fb, fs, tb, ts = tables[b][frm // 16], frm % 16, tables[b][to // 16], to % 16
            for n, (a, o) in enumerate(zip(arrays, out)):
                if n == 1:
                    o[:, tb, :, :, ts] = a[:, fb, :, :, fs]
                else:
                    o[:, tb, :, ts] = a[:, fb, :, fs]
    return out


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("d,n_kv,layers", [(64, 2, 3), (128, 4, 2), (128, 3, 1)])
def test_keep(gpu_lib, kind, d, n_kv, layers):
    nova = gpu_lib
    ctx, rows = [0, 15, 100, 7, 30, 64, 5], [64, 12, 9, 0, 1, 33, 6]
    c, desc, tables, _ = _paged(nova, ctx, rows, n_kv, d, kind, d + n_kv, layers=layers)
    before = [a.cpu().clone() for a in _arrays(c)]
    r = _rng(6)
    path = np.full((7, 64), -1)
    # ascending, in reverse, with a row twice, in place, of the whole tree, and beyond the rows
    for b, p in enumerate([sorted(r.choice(64, 20, replace=False)), [0, 3, 4, 11], [0, 8, 7, 6, 1, 1], [], [0], list(range(32, -1, -1)), [0, 2, 5, 6, 99, -7]]):
        path[b, :len(p)] = p
    n_keep = np.array([20, 4, 6, 3, 1, 33, 6])
    got = nova.kv_keep(c, desc, _i32(path), _i32(n_keep))
    kept = np.minimum(n_keep, rows)
    assert got.tolist() == [x + n for x, n in zip(ctx, kept)]
    legal = [[j if 0 <= j < rows[b] else -1 for j in p] for b, p in enumerate(path)]
    for a, w in zip(_arrays(c), _kept(before, tables, ctx, legal, kept, kind == "e4m3")):
        assert torch.equal(a.cpu(), w)
    again = [a.clone() for a in _arrays(c)]
    assert nova.kv_keep(c, desc, None, _i32([-5, 99, 0, 1, 1, 2, 3])).tolist() == [0, 27, 100, 7, 31, 66, 8]
    for a, w in zip(_arrays(c), again):
        assert torch.equal(a, w)


def test_keep_missing_blocks_and_bounds(gpu_lib):
    """Table entries that name no block, tokens past max_ctx, contexts outside the sequence."""
    nova = gpu_lib
    for kind in TYPES:
        ctx, rows = [14, 14, 14], [8, 8, 8]
        c, desc, tables, _ = _paged(nova, ctx, rows, 2, 64, kind, 3)
        tables[0, 1], tables[1, 0] = 1 << 29, -1
        desc = nova.Rows(None, _i32([14, 14, 20]), _i32(tables), max_rows=8, max_ctx=22)
        before = [a.cpu().clone() for a in _arrays(c)]
        path = np.array([[0, 1, 7, 6, 0, 0, 0, 0], [0, 3, 4, 5, 6, 7, 0, 0], [1, 2, 0, 0, 0, 0, 0, 0]])
        out = torch.zeros(3, dtype=torch.int32, device="cuda")
        assert nova.kv_keep(c, desc, _i32(path), _i32([4, 6, 2]), ctx_out=out) is out
        assert out.tolist() == [18, 20, 22]
        want = _kept(before, tables, [14, 14, 20], [[-1] * 8, [-1, -1, 4, 5, 6, 7, 0, 0], [1, -1, 0, 0, 0, 0, 0, 0]], [4, 6, 2], False)
        for a, w in zip(_arrays(c), want):
            assert torch.equal(a.cpu(), w), kind


# ----------------------------------------------------------------------------- pages
def _pool(nova, blocks, kind="bf16", layers=2, n_kv=2, d=64, seed=1):
    c = nova.Cache(blocks, n_kv, d, dict(bf16=nova.CACHE_BF16, f32=nova.CACHE_F32, e4m3=nova.CACHE_E4M3)[kind], layers=layers)
    _fill(c, _rng(seed))
    return c


def _same(pages, tables, pool):
    assert pages.refs.tolist() == pool.refs.tolist() and tables.tolist() == pool.tables.tolist()


def _moved(c, before, copies):
    for a, b in zip(_arrays(c), before):
        w = b.clone()
        for x, y in copies:
            w[:, y] = b[:, x]
        assert torch.equal(a, w)


@pytest.mark.parametrize("kind", TYPES)
def test_copy(gpu_lib, kind):
    nova = gpu_lib
    for n_kv, d in ((2, 64), (3, 128)):
        a, b = _pool(nova, 9, kind, 3, n_kv, d), _pool(nova, 20, kind, 3, n_kv, d, seed=2)
        before = [x.clone() for x in _arrays(b)]
        src, dst = [0, 8, 3, 3, 9, -1, 1, 1 << 30], [19, 0, 7, 8, 1, 2, 20, 3]
        nova.kv_copy(a, _i32(src), _i32(dst), to=b)
        for x, y, w in zip(_arrays(a), _arrays(b), before):
            for s, t in [(0, 19), (8, 0), (3, 7), (3, 8)]:
                w[:, t] = x[:, s]
            assert torch.equal(y, w)
        before = [x.clone() for x in _arrays(a)]
        nova.kv_copy(a, _i32([2, 5, 7]), _i32([1, 5, 0]))
        _moved(a, before, [(2, 1), (7, 0)])
        nova.kv_copy(a, _i32([]), _i32([]))


def test_extend(gpu_lib):
    nova = gpu_lib
    r = _rng(2)
    for blocks, batch, width in [(1, 1, 1), (50, 7, 9), (5000, 40, 130), (9000, 1500, 7), (40011, 50, 700)]:
        refs = (r.random(blocks) < 0.3) * r.integers(1, 4, blocks)
        tables = np.full((batch, width), -1)
        tables[r.random((batch, width)) < 0.2] = 0
        tables[r.random((batch, width)) < 0.1] = blocks + 5                     # names no block
        pages, t = nova.Pages.of(_i32(refs)), _i32(tables)
        for step in range(3):
            pool = st.Pool(pages.refs.cpu().numpy(), t.cpu().numpy())
            tokens = r.integers(-5, 16 * width + (40 if step else 0), batch)
            done = nova.Pages.extend(pages, t, _i32(tokens))
            assert done.tolist() == pool.extend(tokens)
            _same(pages, t, pool)
    pages = nova.Pages(40)
    t = torch.full((2, 30), -1, dtype=torch.int32, device="cuda")
    assert pages.extend(t, _i32([17, 1 << 30])).tolist() == [1, 0] and t[0].tolist() == [0, 1] + [-1] * 28
    assert pages.extend(t, _i32([0, 480])).tolist() == [1, 1] and pages.extend(t, _i32([160, 480])).tolist() == [1, 1]
    assert pages.extend(t, _i32([161, 480])).tolist() == [0, 1] and (pages.refs == 1).all()


@pytest.mark.parametrize("kind", TYPES)
def test_fork_and_free(gpu_lib, kind):
    nova = gpu_lib
    r = _rng(3)
    c, pages = _pool(nova, 60, kind, 3), nova.Pages(60)
    t = torch.full((12, 8), -1, dtype=torch.int32, device="cuda")
    assert pages.extend(t, _i32([100, 16, 37] + [0] * 9)).tolist() == [1] * 12
    src, dst, n = [0, 0, 1, 2, 0, 2], [3, 4, 5, 6, 7, 8], [100, 99, 16, 1, 0, 33]
    for src, dst, n in [(src, dst, n), ([3, 6, 0], [9, 10, 11], [97, 1, 112])]:
        pool = st.Pool(pages.refs.cpu().numpy(), t.cpu().numpy())
        before = [a.clone() for a in _arrays(c)]
        want, copies = pool.fork(src, dst, n)
        assert pages.fork(c, t, _i32(src), _i32(dst), _i32(n)).tolist() == want
        _same(pages, t, pool)
        _moved(c, before, copies)
    for seqs, keep in [([0, 4], None), ([3, 3, 9], [40, 33, 0]), ([0, 40, -1, 8], [0, 0, 0, 17]), (list(range(12)), None)]:
        pool = st.Pool(pages.refs.cpu().numpy(), t.cpu().numpy())
        pool.free(seqs, keep)
        pages.free(t, _i32(seqs), None if keep is None else _i32(keep))
        _same(pages, t, pool)
    assert (pages.refs == 0).all() and (t == -1).all()


def test_fork_refusals_and_exhaustion(gpu_lib):
    """Requests that name a row twice, a target that is a source, rows and lengths that do not exist, a pool that is full."""
    nova = gpu_lib
    c, pages = _pool(nova, 12), nova.Pages(12)
    t = torch.full((9, 6), -1, dtype=torch.int32, device="cuda")
    pages.extend(t, _i32([90, 20] + [0] * 7))
    for src, dst, n in [([0, 0, 1, 1], [2, 2, 0, 3], [5, 6, 7, 20]), ([0, 9, -1, 0, 0, 4, 0], [9, 4, 5, -3, 6, 7, 8], [1, 1, 1, 1, 200, 16, -4]),
                        ([0] * 5, [4, 5, 6, 7, 8], [17, 18, 32, 19, 20]), ([0, 0], [1, 4], [95, 33])]:
        pool = st.Pool(pages.refs.cpu().numpy(), t.cpu().numpy())
        before = [a.clone() for a in _arrays(c)]
        want, copies = pool.fork(src, dst, n)
        assert pages.fork(c, t, _i32(src), _i32(dst), _i32(n)).tolist() == want
        _same(pages, t, pool)
        _moved(c, before, copies)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("blocks", [1, 2, 37, 1023, 3001, 5003, 20011])
def test_compact(gpu_lib, kind, blocks):
    nova = gpu_lib
    r = _rng(blocks)
    layers, n_kv, d = (3, 2, 64) if blocks < 100 else (1, 1, 64)
    for share in (0.0, 0.4, 0.9, 1.0):
        c = _pool(nova, blocks, kind, layers, n_kv, d)
        used = r.random(blocks) < share
        refs = np.where(used, r.integers(1, 4, blocks), 0)
        tables = r.integers(-2, blocks + 2, (5, 11))
        pool = st.Pool(refs, tables)
        before = [a.clone() for a in _arrays(c)]
        live, copies = pool.compact()
        pages, t = nova.Pages.of(_i32(refs)), _i32(tables)
        refs_out, tables_out = torch.full_like(pages.refs, 99), torch.full_like(t, 99)
        assert pages.compact(c, t, refs_out=refs_out, tables_out=tables_out).tolist() == [live]
        assert refs_out.tolist() == pool.refs.tolist() and tables_out.tolist() == pool.tables.tolist()
        assert pages.refs.tolist() == refs.tolist() and t.tolist() == tables.tolist()
        _moved(c, before, copies)
        for a, b in zip(_arrays(c), before):                                    # again, in place
            a.copy_(b)
        assert pages.compact(c, t).tolist() == [live]
        _same(pages, t, pool)
        _moved(c, before, copies)


# ----------------------------------------------------------------------------- adapters
def _check_lora(out, x, base, a, b, scale, which, starts, rows, types):
    k, rank = a.shape[2], a.shape[1]
    x_parts = 0.0 if types[0] == BF16 else 2.0 ** -16 if types[1] == BF16 else 2.0 ** -23
    h_parts = 2.0 ** -16 if types[1] == BF16 else 2.0 ** -23
    for s, n in enumerate(rows):
        if n == 0:
            continue
        sl = slice(int(starts[s]), int(starts[s]) + n)
        want = np.zeros((n, b.shape[1])) if base is None else _np(base[sl])
        err = np.zeros_like(want)
        if 0 <= which[s] < a.shape[0]:
            i = which[s]
            delta, terms, size = st.lora(_np(x[sl]), _np(a[i]), _np(b[i]), 1.0 if scale is None else float(scale[i]))
            # fp32 sums of k and of rank products (three parts each at most), the parts' rests, scale and base
            err = ((k + 16) * 2.0 ** -24 + x_parts) * size + ((3 * rank + 16) * 2.0 ** -24 + h_parts) * (terms + (k + 16) * 2.0 ** -24 * size)
            want = want + delta
        got = _np(out[sl])
        tol = HALF[types[1]] * (np.abs(want) + err) + err + 2.0 ** -24 * np.abs(want) + 1e-30
        assert (np.abs(got - want) <= tol).all(), (s, n, np.abs(got - want).max(), (np.abs(got - want) / tol).max())


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 128])
def test_lora(gpu_lib, types, rank):
    nova = gpu_lib
    r = _rng(rank, 2)
    for rows, k, n_out in [([1, 1, 1, 1, 1], 256, 512), ([3, 1, 0, 17, 16, 40], 1032, 72), ([70, 0, 129, 64, 1], 264, 328), ([1], 8, 8)]:
        batch, total = len(rows), sum(rows)
        starts = np.concatenate([[0], np.cumsum(rows)])
        which = (np.arange(batch) * 2 + 1) % 5 - (np.arange(batch) == 1) * 9             # the second has none, and 3 and 4 are none
        a, b = _dev(r.normal(size=(3, rank, k)) / np.sqrt(k), BF16), _dev(r.normal(size=(3, n_out, rank)), BF16)
        scale = r.normal(size=3)
        x = _dev(r.normal(size=(total + 2, k + 16)), types[0])[:, 8:8 + k]
        wide = _dev(r.normal(size=(total + 2, n_out + 8)), types[1])
        base = wide[:, 8:]
        desc = nova.Rows(_i32(starts), None, _i32(np.zeros((batch, 1))), rows=total + 2, max_rows=max(rows), max_ctx=16)
        ad = nova.Adapters(a, b, _dev(scale, F32))
        scale = _np(ad.scale)
        out = torch.full((total + 2, n_out), 5.0, dtype=types[1], device="cuda")
        assert nova.lora(ad, desc, _i32(which), x, base=base, out=out) is out
        _check_lora(out, x, base, a, b, scale, which, starts, rows, types)
        assert (out[total:] == 5.0).all()                                               # rows behind the last sequence
        again = base.clone()
        keep = again[total:].clone()
        nova.lora(ad, desc, _i32(which), x, base=again, out=again)                      # onto base itself
        assert torch.equal(again[:total], out[:total]) and torch.equal(again[total:], keep)
        plain = nova.lora(nova.Adapters(a, b), desc, _i32(which), x, dtype=types[1])    # no base, no scale
        _check_lora(plain, x, None, a, b, None, which, starts, rows, types)
        assert torch.equal(nova.lora(ad, desc, _i32(which), x, base=base)[:total], out[:total])


@pytest.mark.parametrize("rows,k,n_out,rank", [([1] * 32, 3584, 4608, 16), ([300, 5, 211], 3584, 1024, 64), ([900], 18944, 256, 128)])
def test_lora_at_real_widths(gpu_lib, rows, k, n_out, rank):
    nova = gpu_lib
    r = _rng(k, n_out)
    starts = np.concatenate([[0], np.cumsum(rows)])
    a, b = _dev(r.normal(size=(4, rank, k)) / np.sqrt(k), BF16), _dev(r.normal(size=(4, n_out, rank)), BF16)
    x, base = _dev(r.normal(size=(sum(rows), k)), BF16), _dev(r.normal(size=(sum(rows), n_out)), BF16)
    which = np.arange(len(rows)) % 5 - 1
    desc = nova.Rows(_i32(starts), None, _i32(np.zeros((len(rows), 1))), rows=sum(rows), max_rows=max(rows), max_ctx=16 if max(rows) < 16 else 16)
    out = nova.lora(nova.Adapters(a, b), desc, _i32(which), x, base=base)
    _check_lora(out, x, base, a, b, None, which, starts, rows, (BF16, BF16))


def test_lora_keeps_sequences_apart(gpu_lib):
    """NaN and infinities in one sequence's rows or adapter leave the others alone; rows beyond max_rows are left out."""
    nova = gpu_lib
    r = _rng(8)
    rows = [3, 20, 2]
    starts = [0, 3, 23, 25]
    a, b = _dev(r.normal(size=(3, 16, 64)), BF16), _dev(r.normal(size=(3, 64, 16)), BF16)
    x = _dev(r.normal(size=(25, 64)), BF16)
    desc = nova.Rows(_i32(starts), None, _i32(np.zeros((3, 1))), rows=25, max_rows=20, max_ctx=16)
    want = nova.lora(nova.Adapters(a, b), desc, _i32([0, 1, 2]), x)
    x2, a2 = x.clone(), a.clone()
    x2[5], a2[2, 3, 7] = float("nan"), float("inf")
    got = nova.lora(nova.Adapters(a2, b), desc, _i32([0, 1, 2]), x2)
    fine = [i for i in range(23) if i != 5]
    assert torch.equal(got[fine], want[fine]) and got[5].isnan().all() and not got[23:].isfinite().any()
    x2[5] = 0.0
    x2[5, 3] = float("inf")
    assert torch.equal(nova.lora(nova.Adapters(a, b), desc, _i32([0, 1, 2]), x2)[5].isfinite(), torch.zeros(64, dtype=torch.bool, device="cuda"))
    short = nova.Rows(_i32(starts), None, _i32(np.zeros((3, 1))), rows=25, max_rows=5, max_ctx=16)
    out = torch.full_like(want, 3.0)
    nova.lora(nova.Adapters(a, b), short, _i32([0, 1, 2]), x, out=out)
    assert torch.equal(out[:8], want[:8]) and (out[8:23] == 3.0).all() and torch.equal(out[23:], want[23:])


# ----------------------------------------------------------------------------- offsets beyond 32 bits
def test_far_rows(gpu_lib):
    """Rows, logits and outputs whose elements lie past 2^32: the last ones against the same rows by themselves."""
    nova = gpu_lib
    rope = nova.Rope(32, axes=(8, 8))
    x = torch.zeros(70000, 1 << 16, dtype=BF16, device="cuda")                            # 4.6e9 elements
    x[-3:, :64] = torch.randn(3, 64, device="cuda")
    pos = _i32(np.stack([np.arange(70000) % 97, np.arange(70000) % 89]))
    rows = x[:, :64].unflatten(1, (2, 32))
    want = nova.rotate(rows[-3:].contiguous(), pos[:, -3:].contiguous(), rope)
    nova.rotate(rows, pos, rope, out=rows)
    assert torch.equal(rows[-3:], want)
    del x, rows
    n, vocab = 32768, 152064                                                              # 5.0e9 logits
    logits = torch.zeros(n, vocab, dtype=BF16, device="cuda")
    logits[-64:] = (torch.randn(64, vocab, device="cuda") * 4).to(BF16)
    ids, u = torch.randint(0, vocab, (n,), device="cuda", dtype=torch.int32), torch.rand(n, device="cuda")
    ids[-63] = logits[-64].argmax()
    temperature = torch.full((512,), 0.0, device="cuda")
    temperature[-1] = 0.2
    tables = torch.zeros(512, 4, dtype=torch.int32, device="cuda")
    got = nova.accept(nova.Rows(None, None, tables, max_rows=64, max_ctx=64), ids, logits, u, temperature=temperature)
    want = nova.accept(nova.Rows(None, None, tables[:1], max_rows=64, max_ctx=64), ids[-64:].contiguous(), logits[-64:], u[-64:].contiguous(),
                       temperature=temperature[-1:].contiguous())
    for a, b in zip(got, want):
        assert torch.equal(a[-1:], b)
    wp, wt, _ = st.accept(_np(logits[-64:]), ids[-64:].tolist(), u[-64:].double().tolist(), t=0.2)
    assert got[1][-1, :len(wp)].tolist() == wp and got[2][-1, :len(wt)].tolist() == wt
    del logits, got, want
    n, wide = 120000, 37888                                                               # 4.5e9 results
    ad = nova.Adapters(torch.randn(2, 8, 16, device="cuda").to(BF16), torch.randn(2, wide, 8, device="cuda").to(BF16))
    x = torch.randn(n, 16, device="cuda").to(BF16)
    many = nova.Rows(_i32([0, 100000, n]), None, tables[:2], rows=n, max_rows=n, max_ctx=64)
    out = nova.lora(ad, many, _i32([0, 1]), x)
    few = nova.Rows(_i32([0, 32 * 4]), None, tables[:1], rows=128, max_rows=128, max_ctx=64)
    assert torch.equal(out[-32:], nova.lora(ad, few, _i32([1]), x[-128:].contiguous())[-32:])


def test_far_blocks(gpu_lib):
    """A pool of more than 2^32 bytes of K: copies, forks, kept rows and a compaction among its last blocks."""
    nova = gpu_lib
    blocks = 140000
    c = nova.Cache(blocks, 4, 128, nova.CACHE_F32)
    last = c.k[0, -6:], c.v[0, -6:]
    for t in last:
        t.normal_()
    k0, v0 = (t.clone() for t in last)
    nova.kv_copy(c, _i32([blocks - 1]), _i32([blocks - 6]))
    assert torch.equal(c.k[0, -6], k0[5]) and torch.equal(c.v[0, -6], v0[5])
    tables = _i32([[blocks - 4, blocks - 3, -1], [-1, -1, -1]])
    desc = nova.Rows(None, _i32([10, 10]), tables, max_rows=12, max_ctx=32)
    ctx = nova.kv_keep(c, desc, _i32([[0, 3, 11] + [-1] * 9, [-1] * 12]), _i32([3, 0]))
    assert ctx.tolist() == [13, 10]
    assert torch.equal(c.k[0, -4, :, 11], k0[2, :, 13]) and torch.equal(c.k[0, -4, :, 12], k0[3, :, 5])
    assert torch.equal(c.v[0, -4, :, :, 11], v0[2, :, :, 13]) and torch.equal(c.v[0, -4, :, :, 12], v0[3, :, :, 5])
    pages = nova.Pages(blocks)
    pages.refs[:-2] = 1
    pages.refs[-4:-2] = 1
    pages.refs[7] = 0
    assert pages.fork(c, tables, _i32([0]), _i32([1]), _i32([20])).tolist() == [1]
    assert tables[1].tolist() == [blocks - 4, 7, -1] and torch.equal(c.k[0, 7], c.k[0, -3]) and torch.equal(c.v[0, 7], c.v[0, -3])
    pages.refs[3] = 0
    kept = c.k[0, -3].clone(), c.v[0, -3].clone()
    assert pages.compact(c, tables).tolist() == [blocks - 3]
    assert tables.tolist() == [[blocks - 4, 3, -1], [blocks - 4, 7, -1]]
    assert torch.equal(c.k[0, 3], kept[0]) and torch.equal(c.v[0, 3], kept[1])
