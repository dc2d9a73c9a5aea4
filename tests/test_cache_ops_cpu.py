"""The cache and logit operators without a GPU: sizes, the binding's checks and the library's refusals
(made before any device work, so the addresses here are never read), and the oracle's own definitions."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2509_21301_amd import nova, synth

FAKE = 1 << 20
LIB = nova.lib


def _cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_exp=FAKE, v_exp=FAKE, num_blocks=8, n_kv=2, head_dim=64, type=nova.CACHE_E4M3)
    a.update(kw)
    return nova.CacheC(*a.values())


def _rows(**kw):
    a = dict(row_start=FAKE, ctx=FAKE, tables=FAKE, max_blocks=4, batch=2, rows=6, max_rows=3, max_ctx=64)
    a.update(kw)
    return nova.RowsC(*a.values())


def _rope(**kw):
    a = dict(rot=64, interleaved=0, theta=1e4, factor=1.0, orig_ctx=0, alpha=1.0, beta=32.0, mscale=1.0)
    a.update(kw)
    return nova.RopeC(*a.values())


def _append(c=None, r=None, rope=None, **kw):
    a = dict(pos=None, t=0, q=FAKE, qp=256, n_q=4, k=FAKE, kp=128, v=FAKE, vp=128, out=FAKE + 4096, ot=0, op=256)
    a.update(kw)
    return LIB.nova_kv_append(C.byref(c or _cache()), C.byref(r or _rows()), C.byref(rope or _rope()), a["pos"], a["t"], a["q"], a["qp"],
                              a["n_q"], a["k"], a["kp"], a["v"], a["vp"], a["out"], a["ot"], a["op"], None)


def test_cache_bytes():
    e = C.c_size_t()
    assert LIB.nova_cache_bytes(nova.CACHE_E4M3, 100, 4, 128, C.byref(e)) == 100 * 4 * 16 * 128 and e.value == 100 * 4 * 16
    assert LIB.nova_cache_bytes(nova.CACHE_BF16, 100, 4, 128, C.byref(e)) == 100 * 4 * 16 * 256 and e.value == 0
    assert LIB.nova_cache_bytes(nova.CACHE_F32, 1 << 20, 4, 64, None) == (1 << 20) * 4 * 16 * 256
    for bad in [(3, 8, 2, 64), (2, 0, 2, 64), (2, 8, 0, 64), (2, 8, 2, 80)]:
        assert LIB.nova_cache_bytes(*bad, C.byref(e)) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(c=_cache(type=7)), nova.EINVAL), (dict(c=_cache(head_dim=80)), nova.EUNSUPPORTED), (dict(c=_cache(k=None)), nova.EINVAL),
    (dict(c=_cache(k=FAKE + 64)), nova.EINVAL), (dict(c=_cache(k_exp=None)), nova.EINVAL), (dict(c=_cache(num_blocks=0)), nova.EINVAL),
    (dict(r=_rows(batch=0)), nova.EINVAL), (dict(r=_rows(tables=None)), nova.EINVAL), (dict(r=_rows(max_ctx=65)), nova.ENOKV),
    (dict(r=_rows(row_start=None)), None), (dict(r=_rows(row_start=None, rows=5)), nova.EINVAL), (dict(r=_rows(max_rows=65)), nova.EINVAL),
    (dict(r=_rows(rows=-1)), nova.EINVAL), (dict(r=_rows(ctx=FAKE + 2)), nova.EINVAL),
    (dict(rope=_rope(rot=24)), nova.EINVAL), (dict(rope=_rope(rot=80)), nova.EINVAL), (dict(rope=_rope(theta=0.0)), nova.EINVAL),
    (dict(rope=_rope(factor=0.0)), nova.EINVAL), (dict(rope=_rope(orig_ctx=4096, beta=1.0)), nova.EINVAL),
    (dict(rope=_rope(mscale=float("nan"))), nova.EINVAL),
    (dict(t=2), nova.EINVAL), (dict(ot=5), nova.EINVAL), (dict(k=None), nova.EINVAL), (dict(v=FAKE + 8), nova.EINVAL),
    (dict(kp=64), nova.EINVAL), (dict(vp=129), nova.EINVAL), (dict(q=FAKE + 4), nova.EINVAL), (dict(out=None), nova.EINVAL),
    (dict(n_q=0), nova.EINVAL), (dict(out=FAKE, ot=1), nova.EINVAL), (dict(out=FAKE, op=512), nova.EINVAL), (dict(pos=FAKE + 1), nova.EINVAL),
])
def test_append_refusals(kw, code):
    if code is None:                        # a call of no rows passes every check and launches nothing
        kw = dict(kw, r=_rows(row_start=FAKE, rows=0))
        assert _append(**kw) == nova.OK
        return
    assert _append(**kw) == code and LIB.nova_last_error()


def test_gather_refusals():
    def call(c=None, r=None, slots=None, t=0, k=FAKE, kp=128, v=FAKE, vp=128):
        return LIB.nova_kv_gather(C.byref(c or _cache()), C.byref(r or _rows()), slots, t, k, kp, v, vp, None)
    assert call(r=_rows(rows=0)) == nova.OK
    assert call(c=_cache(type=-1)) == nova.EINVAL
    assert call(t=9) == nova.EINVAL
    assert call(k=None) == nova.EINVAL
    assert call(vp=120) == nova.EINVAL
    assert call(slots=FAKE + 2) == nova.EINVAL
    assert call(r=_rows(max_rows=100)) == nova.EINVAL                     # consecutive tokens do not fit
    assert call(r=_rows(max_rows=100, rows=0), slots=FAKE) == nova.OK     # picked ones may repeat


def test_tree_refusals_and_workspace():
    def call(c=None, r=None, mask=None, q=FAKE, qp=256, n_q=4, scale=0.1, o=FAKE, op=256, ws=FAKE, n=1 << 30):
        return LIB.nova_tree_attention(C.byref(c or _cache()), C.byref(r or _rows()), mask, q, qp, n_q, scale, o, op, ws, n, None)
    assert call(r=_rows(rows=0)) == nova.OK
    assert call(n_q=3) == nova.EINVAL and call(n_q=0) == nova.EINVAL
    assert call(r=_rows(max_rows=65, max_ctx=1000, max_blocks=70)) == nova.EUNSUPPORTED
    assert call(q=FAKE + 8) == nova.EINVAL and call(op=128) == nova.EINVAL and call(mask=FAKE + 4) == nova.EINVAL
    assert call(scale=float("inf")) == nova.EINVAL
    long = _rows(max_blocks=256, max_ctx=4096)
    need = LIB.nova_tree_attention_workspace_bytes(C.byref(_cache()), C.byref(long), 4)
    assert need >= 6 * 4 * 2 * 64 * 4 and need % 256 == 0
    assert call(r=long, n=need - 1) == nova.ENOSPACE and call(r=long, ws=None) == nova.EINVAL and call(r=long, ws=FAKE + 16) == nova.EINVAL
    assert LIB.nova_tree_attention_workspace_bytes(C.byref(_cache(head_dim=96)), C.byref(long), 4) == 0


def test_logprobs_refusals_and_workspace():
    def call(x=FAKE, t=1, pitch=20000, rows=2, vocab=20000, given=FAKE, n=1, lp=FAKE, ent=FAKE, top=4, tl=FAKE, ti=FAKE, ws=FAKE, nb=1 << 30):
        return LIB.nova_logprobs(x, t, pitch, rows, vocab, given, n, lp, ent, top, tl, ti, ws, nb, None)
    assert call(rows=0) == nova.OK
    for bad in [dict(t=4), dict(x=None), dict(x=FAKE + 2), dict(pitch=19999), dict(vocab=0), dict(rows=-1), dict(n=-1), dict(given=None), dict(lp=None),
                dict(top=-1), dict(top=5, vocab=4, pitch=4), dict(tl=None), dict(ti=None), dict(ent=FAKE + 1), dict(ws=None), dict(ws=FAKE + 8)]:
        assert call(**bad) == nova.EINVAL, bad
    assert call(top=33) == nova.EUNSUPPORTED
    assert call(vocab=(1 << 21) + 1, pitch=1 << 22) == nova.EUNSUPPORTED
    need = LIB.nova_logprobs_workspace_bytes(2, 20000, 4)
    assert need > 0 and call(nb=need - 1) == nova.ENOSPACE
    assert LIB.nova_logprobs_workspace_bytes(2, 20000, 33) == 0
    assert LIB.nova_logprobs_workspace_bytes(2, 4096, 4) == 0     # a short row is one workgroup


def test_stage_refusals():
    h = C.c_void_p()
    cfg = synth.TINY_LLM
    d = nova.LlmDescC(nova.llm_config_c(cfg, nova.ACT_BF16), FAKE, FAKE, FAKE)
    nova._check(LIB.nova_llm_create(C.byref(d), C.byref(h)))
    c, r = _cache(), _rows()
    need = LIB.nova_llm_verify_workspace_bytes(h, C.byref(c), C.byref(r))
    assert need > 0

    def verify(c=c, r=r, ids=FAKE, pos=FAKE, mask=None, out=FAKE, ws=FAKE, n=need):
        return LIB.nova_llm_verify(h, ids, pos, mask, C.byref(r), C.byref(c), out, None, ws, n, None)
    assert verify(c=_cache(n_kv=4)) == nova.EINVAL
    assert verify(c=_cache(type=nova.CACHE_F32)) == nova.EUNSUPPORTED
    assert verify(r=_rows(rows=33, max_rows=33)) == nova.EINVAL
    assert verify(r=_rows(rows=0)) == nova.EINVAL
    assert verify(pos=None) == nova.EINVAL and verify(mask=FAKE + 4) == nova.EINVAL
    assert verify(ws=None) == nova.EINVAL and verify(n=need - 1) == nova.ENOSPACE
    pre = lambda c=c, n_text=10: LIB.nova_llm_prefill_cache(h, None, 0, FAKE, n_text, FAKE, C.byref(c), FAKE, None, FAKE, 0, None)  # noqa: E731
    assert pre(n_text=0) == nova.EINVAL and pre(n_text=129) == nova.ENOKV and pre() == nova.ENOSPACE
    assert pre(c=_cache(head_dim=128)) == nova.EINVAL
    LIB.nova_llm_destroy(h)


def test_binding_checks():
    with pytest.raises(ValueError):
        nova.Cache(4, 2, 96, device="cpu")
    with pytest.raises(ValueError):
        nova.Cache(4, 2, 64, type=9, device="cpu")
    c = nova.Cache(4, 2, 64, layers=3, device="cpu")
    assert c.k.shape == (3, 4, 2, 16, 64) and c.v_exp.shape == (3, 4, 2, 16) and c.dtype == torch.bfloat16
    with pytest.raises(ValueError):
        nova.Cache.of(c.k, c.v)                                  # no exponents
    with pytest.raises(ValueError):
        nova.Cache.of(c.k, c.k, c.k_exp, c.v_exp)                # V in K's layout
    i32 = dict(dtype=torch.int32)
    t = torch.zeros(2, 4, **i32)
    with pytest.raises(ValueError):
        nova.Rows(torch.zeros(3, **i32), None, t)                # how many rows?
    with pytest.raises(ValueError):
        nova.Rows(torch.zeros(2, **i32), None, t, rows=4)        # row_start has batch + 1 entries
    with pytest.raises(ValueError):
        nova.Rows(None, torch.zeros(2), t)
    with pytest.raises(ValueError):
        nova.Rows(None, None, t.long())
    r = nova.Rows(None, None, t, max_rows=3)
    assert r.rows == 6 and r.max_ctx == 64
    k = torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        nova.kv_append(c, r, k, k)                               # not on a GPU
    for bad in [k[:5], k.half(), k[:, :, ::2], k.transpose(0, 1)]:
        with pytest.raises(ValueError):
            nova._check_rows_of("k", bad, 6, 2, 64)
    assert nova._check_rows_of("k", torch.zeros(6, 8, 64)[:, 2:4], 6, 2, 64) == (nova.ACT_F32, 512)
    x = torch.zeros(2, 10)
    for bad in [dict(n_top=-1), dict(given=torch.zeros(2, 1)), dict(given=torch.zeros(3, 1, **i32))]:
        with pytest.raises(ValueError):
            nova.logprobs(x, **bad)
    with pytest.raises(ValueError):
        nova.logprobs(x.T)
    with pytest.raises(ValueError):
        nova.logprobs(x)


def test_sizes_beyond_a_launch():
    """More heads, rows or tokens than a grid or an index holds are refused by each entry."""
    big = dict(rows=1 << 26, max_rows=1 << 26, max_ctx=1 << 26, max_blocks=1 << 23, batch=1)
    long = dict(max_ctx=(1 << 30) + 1, max_blocks=1 << 27)
    for kw in (dict(c=_cache(n_kv=8193)), dict(n_q=8193, qp=8193 * 64, op=8193 * 64), dict(r=_rows(**big)), dict(r=_rows(**long))):
        assert _append(**kw) == nova.EUNSUPPORTED, kw
    for c, r in ((_cache(n_kv=8193), _rows()), (_cache(), _rows(**big)), (_cache(), _rows(**long))):
        assert LIB.nova_kv_gather(C.byref(c), C.byref(r), FAKE, 0, FAKE, 1 << 20, FAKE, 1 << 20, None) == nova.EUNSUPPORTED
    for n_q, r in ((8194, _rows()), (4, _rows(**long))):
        assert LIB.nova_tree_attention(C.byref(_cache()), C.byref(r), None, FAKE, 1 << 20, n_q, 0.1, FAKE, 1 << 20, FAKE, 1 << 40,
                                       None) == nova.EUNSUPPORTED
    assert LIB.nova_logprobs(FAKE, 1, 64, (1 << 23) + 1, 64, None, 0, None, FAKE, 0, None, None, None, 0, None) == nova.EUNSUPPORTED
    t = torch.zeros(2, 4, dtype=torch.int32)
    for kw in (dict(max_ctx=(1 << 32) + 16), dict(max_rows=1 << 31), dict(rows=-1)):
        with pytest.raises(ValueError):
            nova.Rows(None, None, t, **kw)


def test_cache_of_tensors_on_two_devices():
    c = nova.Cache(4, 2, 64, device="cpu")
    for kw in (dict(v=c.v.to("meta")), dict(k_exp=c.k_exp.to("meta")), dict(v_exp=c.v_exp.to("meta"))):
        with pytest.raises(ValueError):
            nova.Cache.of(**{**dict(k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp), **kw})


def test_oracle_quantiser_against_torch():
    """The oracle's e4m3 rounding is torch's, and writing back what was read changes nothing."""
    g = np.random.default_rng(3)
    x = g.normal(size=(200, 64)) * np.exp(g.normal(size=(200, 1)) * 8)
    x[0], x[1, 1:] = 0.0, 0.0
    y, e = oc.quantise(x.astype(np.float32))
    s = np.ldexp(1.0, e)[:, None]
    t = torch.from_numpy((x.astype(np.float32) / s).astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t * s, y)
    assert np.abs(y / s).max() <= 448 and (np.abs(x).max(-1) > 224 * s[:, 0])[2:].all()
    again, _ = oc.quantise(y)
    assert np.array_equal(again, y)


def test_oracle_frequencies():
    f = oc.rope_frequencies(128, 1e4)
    assert f[0] == 1 and np.allclose(oc.rope_frequencies(128, 1e4, factor=4), f / 4)
    b = oc.rope_frequencies(128, 1e4, factor=8, orig_ctx=4096)
    turns = 4096 * f / (2 * np.pi)
    assert np.array_equal(b[turns >= 32], f[turns >= 32]) and np.allclose(b[turns <= 1], f[turns <= 1] / 8)
    assert (np.diff(b) < 0).all()
