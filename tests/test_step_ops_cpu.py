"""The operators between two model calls without a GPU: the library's refusals (made before any device work, so the
addresses here are never read), workspace sizes, the binding's checks, and the oracle's own definitions."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import steps as st
from paper_2509_21301_amd import nova, synth
from tests.test_cache_ops_cpu import FAKE, _cache, _rope, _rows

LIB = nova.lib


def _axes(**kw):
    a = dict(n_axes=3, pairs=(16, 10, 6, 0), cyclic=0, own_freqs=0)
    a.update(kw)
    return nova.RopeAxesC(a["n_axes"], (C.c_int * 4)(*a["pairs"]), a["cyclic"], a["own_freqs"])


def _ref(x):
    return None if x is None else C.byref(x)


# ----------------------------------------------------------------------------- rotary positions with several axes
BAD_AXES = [_axes(n_axes=0), _axes(n_axes=5), _axes(pairs=(16, 10, 5, 0)), _axes(pairs=(16, 17, -1, 0)), _axes(n_axes=2),
            _axes(pairs=(1 << 31 - 1, 1 << 30, 1 << 30, 0))]


def test_append_axes_refusals():
    def call(rope=_rope(), axes=_axes(), r=None):
        return LIB.nova_kv_append_axes(C.byref(_cache()), C.byref(r or _rows(rows=0)), _ref(rope), _ref(axes), FAKE, 0, FAKE, 256, 4, FAKE, 128,
                                       FAKE, 128, FAKE + 4096, 0, 256, None)
    assert call() == nova.OK and call(axes=None) == nova.OK and call(rope=None, axes=None) == nova.OK
    assert call(axes=_axes(pairs=(0, 0, 32, 0), cyclic=1, own_freqs=1)) == nova.OK
    assert call(rope=None) == nova.EINVAL
    for bad in BAD_AXES:
        assert call(axes=bad) == nova.EINVAL
    assert call(rope=_rope(rot=48)) == nova.EINVAL                       # the axes have 32 pairs


def test_rotate_refusals():
    def call(rope=_rope(), axes=_axes(), pos=FAKE, rows=5, heads=3, d=80, t=0, x=FAKE, xp=240, ot=0, o=FAKE + 8192, op=240):
        return LIB.nova_rotate(_ref(rope), _ref(axes), pos, rows, heads, d, t, x, xp, ot, o, op, None)
    assert call(rows=0) == nova.OK and call(rows=0, axes=None, d=256) == nova.OK
    for bad in BAD_AXES:
        assert call(axes=bad) == nova.EINVAL
    for bad in [dict(rope=None), dict(rows=-1), dict(heads=0), dict(t=2), dict(ot=-1), dict(pos=None), dict(pos=FAKE + 2), dict(x=None), dict(x=FAKE + 8),
                dict(xp=232), dict(xp=241), dict(o=None), dict(op=238), dict(o=FAKE, op=480), dict(o=FAKE, ot=1), dict(rope=_rope(rot=24)),
                dict(d=56), dict(rope=_rope(theta=-1.0))]:
        assert call(**bad) == nova.EINVAL, bad
    for bad in [dict(d=76), dict(d=264), dict(heads=8193, xp=8193 * 80, op=8193 * 80), dict(rows=(1 << 25) + 1)]:
        assert call(**bad) == nova.EUNSUPPORTED, bad


# ----------------------------------------------------------------------------- acceptance
def test_accept_refusals_and_workspace():
    need = LIB.nova_accept_workspace_bytes(C.byref(_rows()), 20000, 1)
    assert need > LIB.nova_accept_workspace_bytes(C.byref(_rows()), 20000, 0) > 0

    def call(r=None, ids=FAKE, mask=None, x=FAKE, t=1, xp=20000, d=FAKE, dt=1, dp=20000, vocab=20000, temp=None, u=FAKE, out=(FAKE,) * 4, ws=FAKE, n=need):
        return LIB.nova_accept(_ref(_rows(**(r or {}))), ids, mask, x, t, xp, d, dt, dp, vocab, temp, u, *out, ws, n, None)
    for bad in [dict(r=dict(batch=0)), dict(r=dict(batch=65536)), dict(r=dict(rows=-1)), dict(r=dict(max_rows=0)), dict(r=dict(row_start=None, rows=5)),
                dict(r=dict(row_start=FAKE + 2)), dict(ids=None), dict(ids=FAKE + 1), dict(x=None), dict(x=FAKE + 2), dict(xp=19999), dict(t=5), dict(dt=5),
                dict(d=FAKE + 2), dict(dp=19999), dict(vocab=0), dict(temp=FAKE + 1), dict(u=None), dict(u=FAKE + 3), dict(ws=None), dict(ws=FAKE + 16),
                dict(d=None, mask=FAKE + 4)] + [dict(out=(FAKE,) * i + (None,) + (FAKE,) * (3 - i)) for i in range(4)] + [dict(out=(FAKE, FAKE, FAKE + 2, FAKE))]:
        assert call(**bad) == nova.EINVAL, bad
    for bad in [dict(mask=FAKE), dict(r=dict(max_rows=65)), dict(vocab=(1 << 21) + 1, xp=1 << 22, dp=1 << 22), dict(r=dict(rows=1 << 22)),
                dict(r=dict(rows=(1 << 25) + 1))]:
        assert call(**bad) == nova.EUNSUPPORTED, bad
    assert call(n=need - 1) == nova.ENOSPACE
    for bad in [dict(max_rows=65), dict(batch=0), dict(rows=(1 << 24) // 3 + 1)]:     # 20000 logits are 3 chunks
        assert LIB.nova_accept_workspace_bytes(C.byref(_rows(**bad)), 20000, 0) == 0
    assert LIB.nova_accept_workspace_bytes(C.byref(_rows()), 0, 0) == 0 and LIB.nova_accept_workspace_bytes(None, 100, 0) == 0


# ----------------------------------------------------------------------------- kept rows, copies, pages
def test_keep_refusals():
    def call(c=None, layers=3, r=None, path=FAKE, n=FAKE + 256, out=FAKE + 512):
        return LIB.nova_kv_keep(C.byref(c or _cache()), layers, C.byref(r or _rows(ctx=FAKE + 1024)), path, n, out, None)
    for bad in [dict(c=_cache(type=9)), dict(c=_cache(v=None)), dict(layers=0), dict(r=_rows(tables=None)), dict(r=_rows(max_rows=65, max_ctx=64)),
                dict(n=None), dict(n=FAKE + 2), dict(path=FAKE + 1), dict(out=FAKE + 3), dict(out=FAKE + 1024), dict(out=FAKE + 1020), dict(out=FAKE + 260), dict(out=FAKE + 4)]:
        assert call(**bad) == nova.EINVAL, bad
    assert call(r=_rows(max_ctx=65)) == nova.ENOKV
    for bad in [dict(r=_rows(max_rows=65, max_ctx=1000, max_blocks=70)), dict(layers=1 << 24), dict(c=_cache(n_kv=8192), layers=2000)]:
        assert call(**bad) == nova.EUNSUPPORTED, bad


def test_copy_refusals():
    def call(a=None, b=None, layers=2, f=FAKE, t=FAKE, n=4):
        return LIB.nova_kv_copy(C.byref(a or _cache()), C.byref(b or _cache(num_blocks=20)), layers, f, t, n, None)
    assert call(n=0) == nova.OK
    for bad in [dict(a=_cache(num_blocks=0)), dict(b=_cache(k=FAKE + 16)), dict(b=_cache(type=nova.CACHE_BF16)), dict(b=_cache(n_kv=3)),
                dict(b=_cache(head_dim=128)), dict(layers=0), dict(n=-1), dict(f=None), dict(t=FAKE + 2)]:
        assert call(**bad) == nova.EINVAL, bad


def _pages(**kw):
    a = dict(refs=FAKE, num_blocks=8)
    a.update(kw)
    return nova.PagesC(a["refs"], a["num_blocks"])


def test_pages_refusals():
    need = LIB.nova_pages_workspace_bytes(C.byref(_pages()), 5, 7)
    assert need > 0 and LIB.nova_pages_workspace_bytes(None, 5, 7) == 0 and LIB.nova_pages_workspace_bytes(C.byref(_pages(num_blocks=0)), 5, 7) == 0
    assert LIB.nova_pages_workspace_bytes(C.byref(_pages()), 0, 7) == 0 and LIB.nova_pages_workspace_bytes(C.byref(_pages()), 5, -1) == 0
    far = 1 << 24

    def extend(p=None, t=far, w=4, b=5, tok=FAKE, done=FAKE, ws=FAKE, n=need):
        return LIB.nova_pages_extend(_ref(p or _pages()), t, w, b, tok, done, ws, n, None)

    def fork(p=None, c=None, layers=2, t=far, w=4, b=5, src=FAKE, dst=FAKE, tok=FAKE, n=7, done=FAKE, ws=FAKE, nb=need):
        return LIB.nova_pages_fork(_ref(p or _pages()), C.byref(c or _cache()), layers, t, w, b, src, dst, tok, n, done, ws, nb, None)

    def free(p=None, t=far, w=4, b=5, seqs=FAKE, tok=None, n=3):
        return LIB.nova_pages_free(_ref(p or _pages()), t, w, b, seqs, tok, n, None)

    def compact(p=None, c=None, layers=2, t=far, w=4, b=5, ro=FAKE, to=far, live=None, ws=FAKE, n=need):
        return LIB.nova_pages_compact(_ref(p or _pages()), C.byref(c or _cache()), layers, t, w, b, ro, to, live, ws, n, None)
    common = [dict(p=_pages(refs=None)), dict(p=_pages(refs=FAKE + 2)), dict(p=_pages(num_blocks=0)), dict(t=None), dict(t=far + 1), dict(w=0), dict(b=0), dict(b=65536)]
    for call in (extend, fork, free, compact):
        for bad in common:
            assert call(**bad) == nova.EINVAL, (call, bad)
        assert call(w=(1 << 26) + 1) == nova.EUNSUPPORTED
    for call in (extend, fork, compact):
        assert call(ws=None) == nova.EINVAL and call(ws=FAKE + 16) == nova.EINVAL
    assert extend(n=100) == nova.ENOSPACE and fork(nb=100) == nova.ENOSPACE and compact(n=100) == nova.ENOSPACE
    assert extend(tok=None) == nova.EINVAL and extend(done=FAKE + 2) == nova.EINVAL
    assert fork(n=0) == nova.OK and free(n=0) == nova.OK
    for bad in [dict(src=None), dict(dst=FAKE + 2), dict(tok=None), dict(done=None), dict(n=-1), dict(n=65536), dict(layers=0), dict(c=_cache(num_blocks=9)), dict(c=_cache(type=4))]:
        assert fork(**bad) == nova.EINVAL, bad
    for bad in [dict(seqs=None), dict(seqs=FAKE + 1), dict(tok=FAKE + 1), dict(n=-1), dict(n=65536)]:
        assert free(**bad) == nova.EINVAL, bad
    for bad in [dict(ro=None), dict(to=None), dict(ro=FAKE + 1), dict(live=FAKE + 2), dict(ro=FAKE + 4), dict(to=far + 4), dict(to=FAKE + 4), dict(ro=far),
                dict(ro=FAKE + 256, to=FAKE + 256), dict(layers=0), dict(c=_cache(num_blocks=9))]:
        assert compact(**bad) == nova.EINVAL, bad


# ----------------------------------------------------------------------------- adapters
def _adapters(**kw):
    a = dict(a=FAKE, b=FAKE, scale=None, n=3, rank=16, k=256, n_out=512)
    a.update(kw)
    return nova.AdaptersC(*a.values())


def test_lora_refusals_and_workspace():
    need = LIB.nova_lora_workspace_bytes(C.byref(_adapters()), C.byref(_rows()))
    assert need >= 6 * 16 * 4 and need % 256 == 0
    assert LIB.nova_lora_workspace_bytes(C.byref(_adapters(rank=12)), C.byref(_rows())) == 0
    assert LIB.nova_lora_workspace_bytes(C.byref(_adapters()), C.byref(_rows(batch=0))) == 0

    def call(d=None, r=None, which=FAKE, xt=0, x=FAKE, xp=256, ot=0, base=FAKE, bp=512, out=FAKE + 65536, op=512, ws=FAKE, n=need):
        return LIB.nova_lora(C.byref(d or _adapters()), C.byref(r or _rows()), which, xt, x, xp, ot, base, bp, out, op, ws, n, None)
    assert call(r=_rows(rows=0)) == nova.OK
    for bad in [dict(d=_adapters(n=0)), dict(d=_adapters(k=-8)), dict(d=_adapters(a=None)), dict(d=_adapters(b=FAKE + 8)), dict(d=_adapters(scale=FAKE + 2)),
                dict(r=_rows(batch=0)), dict(r=_rows(row_start=None, rows=7)), dict(which=None), dict(which=FAKE + 2), dict(xt=3), dict(ot=7), dict(x=None),
                dict(x=FAKE + 8), dict(xp=248), dict(xp=257), dict(base=FAKE + 4), dict(bp=504), dict(out=None), dict(op=508), dict(out=FAKE, op=520),
                dict(ws=None), dict(ws=FAKE + 32)]:
        assert call(**bad) == nova.EINVAL, bad
    for bad in [dict(d=_adapters(rank=136)), dict(d=_adapters(rank=12)), dict(d=_adapters(k=260)), dict(d=_adapters(n_out=500)),
                dict(d=_adapters(k=(1 << 24) + 8)), dict(r=_rows(rows=(1 << 25) + 1))]:
        assert call(**bad) == nova.EUNSUPPORTED, bad
    assert call(n=need - 1) == nova.ENOSPACE


# ----------------------------------------------------------------------------- the model with positions of the rows' own
def test_stage_refusals():
    h = C.c_void_p()
    d = nova.LlmDescC(nova.llm_config_c(synth.TINY_LLM, nova.ACT_BF16), FAKE, FAKE, FAKE)
    nova._check(LIB.nova_llm_create(C.byref(d), C.byref(h)))
    c, r = _cache(), _rows()
    need = LIB.nova_llm_verify_workspace_bytes(h, C.byref(c), C.byref(r))

    def verify(rope=_rope(), axes=_axes(), pos=FAKE, n=need - 1):
        return LIB.nova_llm_verify_axes(h, FAKE, _ref(rope), _ref(axes), pos, None, C.byref(r), C.byref(c), FAKE, None, FAKE, n, None)

    def prefill(rope=_rope(), axes=_axes(), pos=FAKE, n_text=10):
        return LIB.nova_llm_prefill_axes(h, None, 0, FAKE, n_text, FAKE, C.byref(c), _ref(rope), _ref(axes), pos, FAKE, None, FAKE, 0, None)
    for call in (verify, prefill):
        assert call() == nova.ENOSPACE and call(axes=None) == nova.ENOSPACE          # every other check passes
        for bad in [dict(rope=None), dict(rope=_rope(rot=80)), dict(pos=None), dict(pos=FAKE + 2)] + [dict(axes=a) for a in BAD_AXES]:
            assert call(**bad) == nova.EINVAL, (call, bad)
    assert prefill(n_text=0) == nova.EINVAL and prefill(n_text=129) == nova.ENOKV
    LIB.nova_llm_destroy(h)


# ----------------------------------------------------------------------------- the binding
def test_binding_checks():
    i32 = dict(dtype=torch.int32)
    for kw in [dict(axes=()), dict(axes=(1, 2, 3, 4, 5)), dict(cyclic=True), dict(own_freqs=True)]:
        with pytest.raises(ValueError):
            nova.Rope(64, **kw)
    rope = nova.Rope(64, axes=(16, 10, 6))
    for bad in [torch.zeros(6, **i32), torch.zeros(2, 6, **i32), torch.zeros(3, 7, **i32), torch.zeros(3, 6), torch.zeros(6, 3, **i32).T]:
        with pytest.raises(ValueError):
            rope._check_pos(bad, 6)
    rope._check_pos(torch.zeros(3, 6, **i32), 6), rope._check_pos(None, 6), nova.Rope(64)._check_pos(torch.zeros(6, **i32), 6)
    t = torch.zeros(2, 4, **i32)
    r, c = nova.Rows(None, None, t, max_rows=3), nova.Cache(8, 2, 64, layers=2, device="cpu")
    x, ids, u = torch.zeros(6, 100), torch.zeros(6, **i32), torch.zeros(6)
    with pytest.raises(ValueError):
        nova.accept(r, ids, x, u)                                             # not on a GPU
    with pytest.raises(ValueError):
        nova.rotate(torch.zeros(6, 2, 64), torch.zeros(3, 6, **i32), rope)
    with pytest.raises(ValueError):
        nova.kv_keep(c, r, torch.zeros(2, 3, **i32), torch.zeros(2, **i32))
    p = nova.Pages(8, device="cpu")
    assert p.refs.tolist() == [0] * 8
    for bad in [torch.zeros(8), torch.zeros(2, 4, **i32), torch.zeros(0, **i32), torch.zeros(16, **i32)[::2]]:
        with pytest.raises(ValueError):
            nova.Pages.of(bad)
    for bad in [t.long(), t[0], torch.zeros(4, 2, **i32).T]:
        with pytest.raises(ValueError):
            p.extend(bad, torch.zeros(2, **i32))
    with pytest.raises(ValueError):
        p.extend(t, torch.zeros(2, **i32))                                    # not on a GPU
    bf = dict(dtype=torch.bfloat16)
    for a, b in [(torch.zeros(2, 8, 64), torch.zeros(2, 16, 8, **bf)), (torch.zeros(2, 8, 64, **bf), torch.zeros(3, 16, 8, **bf)),
                 (torch.zeros(2, 8, 64, **bf), torch.zeros(2, 16, 16, **bf)), (torch.zeros(2, 8, 64, **bf)[:, :, ::2], torch.zeros(2, 16, 8, **bf))]:
        with pytest.raises(ValueError):
            nova.Adapters(a, b)
    ad = nova.Adapters(torch.zeros(2, 8, 64, **bf), torch.zeros(2, 16, 8, **bf))
    assert (ad.n, ad.rank, ad.k, ad.n_out) == (2, 8, 64, 16)
    with pytest.raises(ValueError):
        nova.Adapters(ad.a, ad.b, scale=torch.zeros(1))
    with pytest.raises(ValueError):
        nova.lora(ad, r, torch.zeros(2, **i32), torch.zeros(6, 64, **bf))


# ----------------------------------------------------------------------------- the oracle's definitions
def test_oracle_axes():
    assert st.pair_axes((2, 0, 3)).tolist() == [0, 0, 2, 2, 2]
    assert st.pair_axes((4, 2, 1), cyclic=True).tolist() == [0, 1, 2, 0, 1, 0, 0]
    f = st.axes_frequencies((4, 2), 1e4, own_freqs=True)
    assert np.allclose(f, [1, 1e-1, 1e-2, 1e-3, 1, 1e-2])
    assert np.array_equal(st.axes_frequencies((4, 4), 1e4), oc.rope_frequencies(16, 1e4))
    r = np.random.default_rng(1)
    x, pos = r.normal(size=(5, 2, 24)), r.integers(0, 99, 5)
    freq = oc.rope_frequencies(16, 1e4)
    for inter in (False, True):                       # equal positions on every axis are the plain embedding
        y = st.rotate_axes(x, np.stack([pos] * 3), (3, 4, 1), freq, cyclic=True, interleaved=inter, mscale=1.1)
        assert np.allclose(y, oc.rotate(x, pos, 16, freq, inter, 1.1)) and np.array_equal(y[..., 16:], x[..., 16:])


def test_oracle_accept_keeps_the_target_distribution():
    """Over every draft token and a fine grid of numbers, what comes out first is distributed as the target's p."""
    r = np.random.default_rng(2)
    l, d = r.normal(size=7) * 1.5, r.normal(size=7) * 1.5
    p, q = st.distribution(l, 0.8), st.distribution(d, 0.8)
    got, n = np.zeros(7), 400
    grid = (np.arange(n) + 0.5) / n
    for x in range(7):
        for u in grid:
            path, tokens, _ = st.accept(np.stack([l, l]), [0, x], [0.0, u], draft=np.stack([d, d]), t=0.8)
            if len(path) == 2:
                got[x] += q[x] / n
            else:                                                         # the rest is drawn: average over its own number
                rest = np.maximum(p - q, 0)
                got += q[x] / n * rest / rest.sum()
    assert np.abs(got - p).max() < 2.0 / n


def test_oracle_pages_keep_their_counts():
    """Whatever is called, a count is the number of entries that name the block."""
    r = np.random.default_rng(3)
    pool = st.Pool(np.zeros(40, int), np.full((6, 9), -1))
    for _ in range(60):
        what = r.integers(0, 4)
        if what == 0:
            pool.extend(r.integers(0, 120, 6))
        elif what == 1:
            dst = int(r.integers(0, 6))
            pool.free([dst])
            pool.fork([int(r.integers(0, 6))], [dst], [int(r.integers(0, 100))])
        elif what == 2:
            pool.free([int(r.integers(0, 6))], [int(r.integers(0, 80))])
        else:
            live, _ = pool.compact()
            assert (pool.refs[:live] > 0).all() and (pool.refs[live:] == 0).all()
        assert np.array_equal(pool.refs, np.bincount(pool.tables[pool.tables >= 0], minlength=40))
