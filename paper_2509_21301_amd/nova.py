"""Python binding of libnova (ctypes).  Argument marshalling only: every step of the three stages
runs in the HIP kernels behind the C ABI declared in ``include/nova.h``.

PyTorch provides device memory, pinned host memory and streams.  The library must be built
(``python -m paper_2509_21301_amd.build``); importing this module without it raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnova.so")

OK, EINVAL, ENOKV, EHIP, EUNSUPPORTED, ENOSPACE = 0, -1, -2, -3, -4, -5
STAGE_ENCODE, STAGE_PREFILL, STAGE_DECODE = 0, 1, 2
ACT_BF16, ACT_F32 = 0, 1
CACHE_BF16, CACHE_F32, CACHE_E4M3 = 0, 1, 2
KIND_GEMM, KIND_ATTN, KIND_GEMV, KIND_DECODE_ATTN, KIND_MISC = 0, 1, 2, 3, 4
KIND_NAMES = {KIND_GEMM: "gemm", KIND_ATTN: "attention", KIND_GEMV: "thin_gemm", KIND_DECODE_ATTN: "decode_attention",
              KIND_MISC: "misc"}


class NovaError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libnova error {code}: {msg}")
        self.code = code


class VitConfigC(C.Structure):
    _fields_ = [("hidden", C.c_int), ("heads", C.c_int), ("mlp", C.c_int), ("layers", C.c_int), ("patch", C.c_int),
                ("merge", C.c_int), ("out_hidden", C.c_int), ("image_h", C.c_int), ("image_w", C.c_int),
                ("eps", C.c_float), ("act", C.c_int)]


class VitDescC(C.Structure):
    _fields_ = [("cfg", VitConfigC), ("embed", C.c_void_p), ("head", C.c_void_p), ("layers", C.c_void_p),
                ("host_layers", C.c_void_p), ("slots", C.c_void_p), ("n_slots", C.c_int)]


class LlmConfigC(C.Structure):
    _fields_ = [("hidden", C.c_int), ("n_q", C.c_int), ("n_kv", C.c_int), ("head_dim", C.c_int), ("inter", C.c_int),
                ("vocab", C.c_int), ("layers", C.c_int), ("block", C.c_int), ("rope_theta", C.c_float),
                ("eps", C.c_float), ("act", C.c_int)]


class LlmDescC(C.Structure):
    _fields_ = [("cfg", LlmConfigC), ("embed", C.c_void_p), ("layers", C.c_void_p), ("head", C.c_void_p)]


class KvC(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("num_blocks", C.c_int)]


class CacheC(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("num_blocks", C.c_int), ("n_kv", C.c_int), ("head_dim", C.c_int), ("type", C.c_int)]


class RowsC(C.Structure):
    _fields_ = [("row_start", C.c_void_p), ("ctx", C.c_void_p), ("tables", C.c_void_p), ("max_blocks", C.c_int),
                ("batch", C.c_int), ("rows", C.c_int), ("max_rows", C.c_int), ("max_ctx", C.c_int)]


class RopeC(C.Structure):
    _fields_ = [("rot", C.c_int), ("interleaved", C.c_int), ("theta", C.c_float), ("factor", C.c_float),
                ("orig_ctx", C.c_int), ("alpha", C.c_float), ("beta", C.c_float), ("mscale", C.c_float)]


# symbol -> (restype, argtypes); mirrors include/nova.h
_SIG = {
    "nova_last_error": (C.c_char_p, []),
    "nova_init": (C.c_int, [C.c_int]),
    "nova_shutdown": (None, []),
    "nova_device_cus": (C.c_int, []),
    "nova_vit_embed_layout": (C.c_int, [C.POINTER(VitConfigC), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "nova_vit_layer_layout": (C.c_int, [C.POINTER(VitConfigC), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "nova_vit_head_layout": (C.c_int, [C.POINTER(VitConfigC), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "nova_vit_create": (C.c_int, [C.POINTER(VitDescC), C.POINTER(C.c_void_p)]),
    "nova_vit_destroy": (None, [C.c_void_p]),
    "nova_vit_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int]),
    "nova_vit_encode": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "nova_prefetch_layer": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "nova_vit_offload_state": (C.c_int, [C.c_void_p, C.POINTER(C.c_int), C.POINTER(C.c_ulonglong)]),
    "nova_llm_layer_layout": (C.c_int, [C.POINTER(LlmConfigC), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "nova_llm_head_layout": (C.c_int, [C.POINTER(LlmConfigC), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "nova_llm_create": (C.c_int, [C.POINTER(LlmDescC), C.POINTER(C.c_void_p)]),
    "nova_llm_destroy": (None, [C.c_void_p]),
    "nova_kv_bytes": (C.c_size_t, [C.c_void_p, C.c_int]),
    "nova_llm_prefill_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int]),
    "nova_llm_decode_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int, C.c_int]),
    "nova_llm_prefill": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.POINTER(KvC),
                                   C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "nova_llm_decode": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int,
                                  C.POINTER(KvC), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "nova_llm_decode_noalloc": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int,
                                          C.POINTER(KvC), C.c_void_p, C.c_void_p, C.c_void_p]),
    "nova_cache_bytes": (C.c_size_t, [C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_size_t)]),
    "nova_kv_append": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int64, C.c_int,
                                 C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.c_int64, C.c_void_p]),
    "nova_kv_gather": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                 C.c_void_p]),
    "nova_tree_attention_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_void_p, C.c_int]),
    "nova_tree_attention": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_float,
                                      C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "nova_logprobs_workspace_bytes": (C.c_size_t, [C.c_int, C.c_int, C.c_int]),
    "nova_logprobs": (C.c_int, [C.c_void_p, C.c_int, C.c_int64, C.c_int, C.c_int, C.c_void_p, C.c_int, C.c_void_p,
                                C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "nova_llm_prefill_cache": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "nova_llm_verify_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "nova_llm_verify": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "nova_linear": (C.c_int, [C.c_int, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "nova_make_cu_mask": (C.c_int, [C.c_int, C.c_int, C.POINTER(C.c_uint32)]),
    "nova_set_stage_partition": (C.c_int, [C.c_int, C.POINTER(C.c_uint32), C.c_int, C.POINTER(C.c_void_p)]),
    "nova_cu_probe": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int]),
    "nova_timing_enable": (C.c_int, [C.c_int]),
    "nova_timing_read": (C.c_int, [C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int)]),
}


def _load():
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2509_21301_amd.build`")
    lib = C.CDLL(LIB_PATH)
    for name, (res, args) in _SIG.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


lib = _load()


def _check(rc):
    if rc != OK:
        raise NovaError(rc, lib.nova_last_error().decode())
    return rc


def init(device: int = 0):
    _check(lib.nova_init(device))


def device_cus() -> int:
    return lib.nova_device_cus()


def _ptr(t) -> int | None:
    if t is None:
        return None
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:      # the handle itself: building a Stream object costs as much as a kernel launch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


# ----------------------------------------------------------------------------- layouts
def _layout(fn, cfg, n):
    off = (C.c_size_t * n)()
    size = C.c_size_t()
    _check(fn(C.byref(cfg), off, C.byref(size)))
    return list(off), size.value


def vit_config_c(cfg, act=ACT_BF16) -> VitConfigC:
    return VitConfigC(cfg.hidden, cfg.heads, cfg.mlp, cfg.layers, cfg.patch, cfg.merge, cfg.out_hidden, cfg.image_h,
                      cfg.image_w, cfg.eps, act)


def llm_config_c(cfg, act=ACT_BF16) -> LlmConfigC:
    return LlmConfigC(cfg.hidden, cfg.n_q, cfg.n_kv, cfg.head_dim, cfg.inter, cfg.vocab, cfg.layers, cfg.block,
                      cfg.rope_theta, cfg.eps, act)


def vit_layouts(cfg, act=ACT_BF16):
    c = vit_config_c(cfg, act)
    return (_layout(lib.nova_vit_embed_layout, c, 3), _layout(lib.nova_vit_layer_layout, c, 12),
            _layout(lib.nova_vit_head_layout, c, 4))


def llm_layouts(cfg, act=ACT_BF16):
    c = llm_config_c(cfg, act)
    return _layout(lib.nova_llm_layer_layout, c, 6), _layout(lib.nova_llm_head_layout, c, 2)


def _round(x, m):
    return (x + m - 1) // m * m


# ----------------------------------------------------------------------------- weight packing
def _bf16(a, device) -> torch.Tensor:
    """bf16 copy of a bf16-exact float array (numpy or torch)."""
    t = torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a
    return t.to(device=device, dtype=torch.bfloat16)


class _Blob:
    def __init__(self, nbytes, device, pin=False):
        if pin:
            self.t = torch.zeros(nbytes // 2, dtype=torch.bfloat16, pin_memory=True)
        else:
            self.t = torch.zeros(nbytes // 2, dtype=torch.bfloat16, device=device)

    def view(self, off, shape):
        n = int(np.prod(shape))
        return self.t[off // 2: off // 2 + n].view(*shape)


def _put(blob, off, src, shape, device):
    """Copy src (rows x cols) into the top-left corner of a zero region of `shape`."""
    v = blob.view(off, shape)
    s = _bf16(src, v.device)
    if s.dim() == 1:
        v[: s.shape[0]].copy_(s)
    else:
        v[: s.shape[0], : s.shape[1]].copy_(s)


def pack_vit(cfg, w, act=ACT_BF16, device="cuda", layer_range=None, pin_layers=False):
    """Pack ViT weights (dict name -> array, as synth.vit_weights gives) into the three blob kinds.

    Returns (embed blob, list-of-layers blob (all layers back to back), head blob) as bf16 tensors.
    """
    (eo, eb), (lo, lb), (ho, hb) = vit_layouts(cfg, act)
    H, I, P = cfg.hidden, _round(cfg.mlp, 256), _round(cfg.patch_dim, 64)
    emb = _Blob(eb, device)
    _put(emb, eo[0], w["patch.w"], (H, P), device)
    _put(emb, eo[1], w["patch.b"], (H,), device)
    _put(emb, eo[2], w["pos"], (cfg.n_patches, H), device)
    layers = list(range(cfg.layers)) if layer_range is None else list(layer_range)
    lay = _Blob(lb * len(layers), device, pin=pin_layers)
    for i, l in enumerate(layers):
        p = f"l{l}."
        base = i * lb
        specs = [("ln1.g", (H,)), ("ln1.b", (H,)), ("qkv.w", (3 * H, H)), ("qkv.b", (3 * H,)), ("o.w", (H, H)),
                 ("o.b", (H,)), ("ln2.g", (H,)), ("ln2.b", (H,)), ("fc1.w", (I, H)), ("fc1.b", (I,)),
                 ("fc2.w", (H, I)), ("fc2.b", (H,))]
        for j, (nm, shp) in enumerate(specs):
            _put(lay, base + lo[j], w[p + nm], shp, device)
    head = _Blob(hb, device)
    m2 = cfg.merge * cfg.merge
    _put(head, ho[0], w["merge.ln.g"], (H,), device)
    _put(head, ho[1], w["merge.ln.b"], (H,), device)
    _put(head, ho[2], w["merge.w"], (cfg.out_hidden, m2 * H), device)
    _put(head, ho[3], w["merge.b"], (cfg.out_hidden,), device)
    return emb.t, lay.t, head.t, lb


def pack_llm(cfg, w, act=ACT_BF16, device="cuda"):
    """Pack LLM weights into (embed table, layers blob, head blob)."""
    (lo, lb), (ho, hb) = llm_layouts(cfg, act)
    H, I, d = cfg.hidden, _round(cfg.inter, 256), cfg.head_dim
    lay = _Blob(lb * cfg.layers, device)
    for l in range(cfg.layers):
        p, base = f"l{l}.", l * lb
        _put(lay, base + lo[0], w[p + "rms1.g"], (H,), device)
        qkv = np.concatenate([w[p + "q.w"], w[p + "k.w"], w[p + "v.w"]], 0) if isinstance(w[p + "q.w"], np.ndarray) \
            else torch.cat([w[p + "q.w"], w[p + "k.w"], w[p + "v.w"]], 0)
        _put(lay, base + lo[1], qkv, ((cfg.n_q + 2 * cfg.n_kv) * d, H), device)
        _put(lay, base + lo[2], w[p + "o.w"], (H, cfg.n_q * d), device)
        _put(lay, base + lo[3], w[p + "rms2.g"], (H,), device)
        gu = lay.view(base + lo[4], (I // 8, 2, 8, H))
        gate = torch.zeros(I, H, dtype=torch.bfloat16, device=gu.device)
        up = torch.zeros(I, H, dtype=torch.bfloat16, device=gu.device)
        gate[: cfg.inter] = _bf16(w[p + "gate.w"], gu.device)
        up[: cfg.inter] = _bf16(w[p + "up.w"], gu.device)
        gu[:, 0].copy_(gate.view(I // 8, 8, H))
        gu[:, 1].copy_(up.view(I // 8, 8, H))
        _put(lay, base + lo[5], w[p + "down.w"], (H, I), device)
    head = _Blob(hb, device)
    _put(head, ho[0], w["norm.g"], (H,), device)
    _put(head, ho[1], w["lm_head.w"], (cfg.vocab, H), device)
    embed = _bf16(w["embed"], device).contiguous()
    return embed, lay.t, head.t, lb


def act_dtype(act):
    return torch.float32 if act == ACT_F32 else torch.bfloat16


# ----------------------------------------------------------------------------- models
class Vit:
    """Vision encoder handle.  With n_slots > 0 the layers stay in pinned host memory and are
    streamed through n_slots device slots."""

    def __init__(self, cfg, weights, act=ACT_BF16, device="cuda", n_slots=0, blobs=None):
        self.cfg, self.act, self.device = cfg, act, device
        if blobs is None:
            blobs = pack_vit(cfg, weights, act, device, pin_layers=n_slots > 0)
        self.embed, self.layers, self.head, self.layer_bytes = blobs
        self.slots = None
        desc = VitDescC(vit_config_c(cfg, act), _ptr(self.embed), _ptr(self.head), None, None, None, 0)
        if n_slots > 0:
            if self.layers.is_cuda:
                raise ValueError("offload needs the layer blob in pinned host memory")
            self.slots = torch.zeros(n_slots * self.layer_bytes // 2, dtype=torch.bfloat16, device=device)
            desc.host_layers = _ptr(self.layers)
            desc.slots = _ptr(self.slots)
            desc.n_slots = n_slots
            self.slots_n = n_slots
        else:
            desc.layers = _ptr(self.layers)
        h = C.c_void_p()
        _check(lib.nova_vit_create(C.byref(desc), C.byref(h)))
        self.h = h
        self._ws = {}

    def workspace(self, batch, stream=None):
        if batch not in self._ws:
            n = lib.nova_vit_workspace_bytes(self.h, batch)
            self._ws[batch] = _empty(self.embed, n, torch.uint8, stream)
        return self._ws[batch]

    def out_shape(self, batch):
        return (batch, self.cfg.n_out, self.cfg.out_hidden)

    def encode(self, pixels, out=None, stream=None):
        """pixels: bf16 [B, H, W, 3] on the device -> act-type [B, n_out, out_hidden]."""
        assert pixels.dtype == torch.bfloat16 and pixels.is_cuda and pixels.is_contiguous()
        b = pixels.shape[0]
        if out is None:
            out = _empty(self.embed, self.out_shape(b), act_dtype(self.act), stream)
        ws = self.workspace(b, stream)
        _check(lib.nova_vit_encode(self.h, _ptr(pixels), b, _ptr(out), _ptr(ws), ws.numel(), _stream(stream)))
        return out

    def prefetch(self, layer, stream=None):
        _check(lib.nova_prefetch_layer(self.h, layer, None if stream is None else stream.cuda_stream))

    def offload_state(self):
        """(logical layer held by each physical slot, layer copies issued so far)."""
        k = C.c_int * self.slots_n
        sl, n = k(), C.c_ulonglong()
        _check(lib.nova_vit_offload_state(self.h, sl, C.byref(n)))
        return list(sl), n.value

    def __del__(self):
        h = getattr(self, "h", None)
        if h is not None and h.value and lib is not None:
            lib.nova_vit_destroy(h)
            self.h = None


class KvPool:
    def __init__(self, llm, num_blocks, device="cuda"):
        n = lib.nova_kv_bytes(llm.h, num_blocks)
        dt = act_dtype(llm.act)
        el = n // torch.tensor([], dtype=dt).element_size()
        self.k = torch.zeros(el, dtype=dt, device=device)
        self.v = torch.zeros(el, dtype=dt, device=device)
        self.num_blocks = num_blocks
        self.c = KvC(_ptr(self.k), _ptr(self.v), num_blocks)
        cfg = llm.cfg
        self.k5 = self.k.view(cfg.layers, num_blocks, cfg.n_kv, cfg.block, cfg.head_dim)
        self.v5 = self.v.view(cfg.layers, num_blocks, cfg.n_kv, cfg.head_dim, cfg.block)


class Llm:
    def __init__(self, cfg, weights, act=ACT_BF16, device="cuda", blobs=None):
        self.cfg, self.act, self.device = cfg, act, device
        if blobs is None:
            blobs = pack_llm(cfg, weights, act, device)
        self.embed, self.layers, self.head, self.layer_bytes = blobs
        desc = LlmDescC(llm_config_c(cfg, act), _ptr(self.embed), _ptr(self.layers), _ptr(self.head))
        h = C.c_void_p()
        _check(lib.nova_llm_create(C.byref(desc), C.byref(h)))
        self.h = h
        self._ws = {}
        self._retired = []

    def _workspace(self, key, nbytes, stream=None):
        if torch.cuda.is_current_stream_capturing():
            # memory of the graph's own: a later, larger call would free the one that is kept here, and two graphs
            # would share it
            return _empty(self.embed, nbytes, torch.uint8, stream)
        t = self._ws.get(key)
        if t is None or t.numel() < nbytes:
            if t is not None:
                # the old buffer may still be read by work queued earlier by this stage; keep it
                # until an event recorded now on this call's stream has completed (the library
                # orders a stage's new partition stream after its earlier ones), so the caching
                # allocator cannot hand it out while the GPU still uses it
                ev = torch.cuda.Event()
                ev.record(stream if stream is not None else torch.cuda.current_stream())
                self._retired.append((t, ev))
            t = _empty(self.embed, nbytes, torch.uint8, stream)
            self._ws[key] = t
        if self._retired:
            self._retired = [(b, e) for b, e in self._retired if not e.query()]
        return t

    def reserve(self, prefill_tokens=0, decode_batch=0, decode_ctx=0):
        """Size the prefill and decode workspaces once for the largest calls to come, so that no
        later call grows them (a serving worker then never waits on a buffer swap)."""
        if prefill_tokens > 0:
            self._workspace("prefill", lib.nova_llm_prefill_workspace_bytes(self.h, prefill_tokens))
        if decode_batch > 0 and decode_ctx > 0:
            # the attention split count falls with the batch, so the largest need is not always at
            # the largest batch
            need = max(lib.nova_llm_decode_workspace_bytes(self.h, b, decode_ctx) for b in range(1, decode_batch + 1))
            self._workspace("decode", need)

    def prefill(self, vis, ids, table, kv, logits=None, next_id=None, stream=None):
        n_vis = 0 if vis is None else vis.shape[0]
        n_text = ids.shape[0]
        ws = self._workspace("prefill", lib.nova_llm_prefill_workspace_bytes(self.h, n_vis + n_text), stream)
        if next_id is None:
            next_id = _empty(self.embed, 1, torch.int32, stream)
        if isinstance(kv, Cache):
            kv._check_layers(self.cfg.layers)
            _check_device(kv.device, vis, ids, table, next_id, logits)
            _check_vector("table", table, torch.int32, (n_vis + n_text + 15) // 16)
            _check(lib.nova_llm_prefill_cache(self.h, _ptr(vis), n_vis, _ptr(ids), n_text, _ptr(table), kv.layer(0),
                                              _ptr(next_id), _ptr(logits), _ptr(ws), ws.numel(), _stream(stream)))
            return next_id
        _check(lib.nova_llm_prefill(self.h, _ptr(vis), n_vis, _ptr(ids), n_text, _ptr(table), C.byref(kv.c),
                                    _ptr(next_id), _ptr(logits), _ptr(ws), ws.numel(), _stream(stream)))
        return next_id

    def decode(self, ids, pos, tables, kv, max_ctx, next_ids=None, logits=None, stream=None):
        b = ids.shape[0]
        # one decode workspace for every batch size: a larger one serves a smaller step as well
        ws = self._workspace("decode", lib.nova_llm_decode_workspace_bytes(self.h, b, max_ctx), stream)
        if next_ids is None:
            next_ids = _empty(self.embed, b, torch.int32, stream)
        _check(lib.nova_llm_decode(self.h, _ptr(ids), _ptr(pos), _ptr(tables), tables.shape[1], b, max_ctx,
                                   C.byref(kv.c), _ptr(next_ids), _ptr(logits), _ptr(ws), ws.numel(),
                                   _stream(stream)))
        return next_ids

    def verify(self, ids, pos, rows, cache, mask=None, next_ids=None, logits=None, stream=None):
        """A decode step over drafted tokens on a ``Cache``: ids, pos int32 [rows.rows] (at most 32 rows), ``mask``
        int64 [rows] as for ``tree_attention``; the greedy id after every row.  One row per sequence decodes.  Rows
        behind the last sequence need valid ids too; what comes back for them means nothing."""
        cache._check_layers(self.cfg.layers)
        _check_device(cache.device, rows.tables, ids, pos, mask, next_ids, logits)
        for what, t, dt in (("ids", ids, torch.int32), ("pos", pos, torch.int32), ("mask", mask, torch.int64)):
            _check_vector(what, t, dt, rows.rows)
        if logits is not None and (logits.dtype != torch.float32 or not logits.is_contiguous() or
                                   logits.shape != (rows.rows, self.cfg.vocab)):
            raise ValueError(f"logits must be contiguous float32 {(rows.rows, self.cfg.vocab)}")
        # memory of the call's own, as the operators take it
        n = lib.nova_llm_verify_workspace_bytes(self.h, cache.layer(0), rows.ref)
        ws = _empty(cache.k, max(n, 256), torch.uint8, stream)
        if next_ids is None:
            next_ids = _empty(self.embed, rows.rows, torch.int32, stream)
        _check_vector("next_ids", next_ids, torch.int32, rows.rows)
        _check(lib.nova_llm_verify(self.h, _ptr(ids), _ptr(pos), _ptr(mask), rows.ref, cache.layer(0), _ptr(next_ids),
                                   _ptr(logits), _ptr(ws), ws.numel(), _stream(stream)))
        return next_ids

    def decode_noalloc(self, ids, pos, tables, kv, max_ctx, next_ids, logits=None, stream=None):
        """The same step with the library's static scratch as workspace (no allocation in the
        library; outputs are the caller's)."""
        _check(lib.nova_llm_decode_noalloc(self.h, _ptr(ids), _ptr(pos), _ptr(tables), tables.shape[1], ids.shape[0],
                                           max_ctx, C.byref(kv.c), _ptr(next_ids), _ptr(logits), _stream(stream)))
        return next_ids

    def __del__(self):
        h = getattr(self, "h", None)
        if h is not None and h.value and lib is not None:
            lib.nova_llm_destroy(h)
            self.h = None


# ----------------------------------------------------------------------------- operators over the paged cache
_CACHE_DTYPE = {CACHE_BF16: torch.bfloat16, CACHE_F32: torch.float32, CACHE_E4M3: torch.uint8}
_ACT = {torch.bfloat16: ACT_BF16, torch.float32: ACT_F32}


def _check_vector(what, t, dtype, n):
    if t is not None and (t.dtype != dtype or t.dim() != 1 or t.shape[0] < n or not t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous {dtype} vector of {n} entries, got {t.dtype} {tuple(t.shape)}")


def _check_rows_of(what, t, rows, heads, d):
    """Rows [rows, heads, d], heads and dimensions contiguous; returns (type, pitch)."""
    act, st = _ACT.get(t.dtype), t.stride()
    if act is not None and t.shape == (rows, heads, d) and st[2] == 1 and (st[1] == d or heads == 1):
        return act, st[0] if rows > 1 else heads * d
    if act is None:
        raise ValueError(f"{what} must be bfloat16 or float32, got {t.dtype}")
    raise ValueError(f"{what} must be rows {(rows, heads, d)} with contiguous heads, got {tuple(t.shape)} strides {st}")


def _check_device(dev, *tensors):
    """Every tensor lives on the device of index ``dev``, the current one (the library launches there)."""
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors on {t.device} and on device {dev}")
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise ValueError(f"tensors on device {dev}, which is not the current one")


def _empty(like, shape, dtype, stream):
    """Memory on the stream that a call runs on: what the allocator hands out may still be in use by work queued on its
    own stream, and what is freed after the call is reused behind it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _dense_like(t, stream):
    """Contiguous memory of t's shape and type, as ``_empty`` (a third faster)."""
    if stream is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    with torch.cuda.stream(stream):
        return torch.empty_like(t, memory_format=torch.contiguous_format)


def _stream_on(dev, stream):
    """``_stream`` for a call whose tensors are known to be on the current device."""
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


class Cache:
    """Paged K/V pool of ``layers`` layers: CACHE_BF16 or CACHE_F32 (a ``KvPool``'s layout) or CACHE_E4M3 (8 bits per
    value and a power-of-two scale per token and head).  ``k`` [layers, num_blocks, n_kv, 16, head_dim], ``v``
    [layers, num_blocks, n_kv, head_dim, 16], ``k_exp``, ``v_exp`` [layers, num_blocks, n_kv, 16] (E4M3)."""

    def __init__(self, num_blocks, n_kv, head_dim, type=CACHE_E4M3, layers=1, device="cuda"):
        if type not in _CACHE_DTYPE:
            raise ValueError(f"unknown cache type {type}")
        if lib.nova_cache_bytes(type, num_blocks, n_kv, head_dim, None) == 0 or layers < 1:
            raise ValueError(f"unsupported cache: {layers} layers of {num_blocks} blocks, {n_kv} heads of {head_dim}")
        k = torch.zeros(layers, num_blocks, n_kv, 16, head_dim, dtype=_CACHE_DTYPE[type], device=device)
        v = torch.zeros(layers, num_blocks, n_kv, head_dim, 16, dtype=_CACHE_DTYPE[type], device=device)
        e = (None, None)
        if type == CACHE_E4M3:
            e = tuple(torch.full((layers, num_blocks, n_kv, 16), 127, dtype=torch.uint8, device=device) for _ in "kv")
        self._own(k, v, *e)

    @classmethod
    def of(cls, k, v, k_exp=None, v_exp=None):
        """A cache on tensors in hand, with or without the layer dimension (a ``KvPool``'s k5 and v5, say)."""
        self = cls.__new__(cls)
        self._own(*(t if t is None or t.dim() == n else t.unsqueeze(0) for t, n in ((k, 5), (v, 5), (k_exp, 4), (v_exp, 4))))
        return self

    def _own(self, k, v, k_exp, v_exp):
        types = {t: n for n, t in _CACHE_DTYPE.items()}
        if k.dtype not in types or v.dtype != k.dtype or k.dim() != 5 or k.shape[3] != 16:
            raise ValueError(f"k must be bfloat16, float32 or uint8 [layers, blocks, n_kv, 16, head_dim], got {k.dtype} {tuple(k.shape)}")
        layers, nb, n_kv, _, d = k.shape
        if v.shape != (layers, nb, n_kv, d, 16) or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError(f"k and v must be contiguous, v {(layers, nb, n_kv, d, 16)}: got {tuple(v.shape)}")
        if any(t is not None and t.device != k.device for t in (v, k_exp, v_exp)):
            raise ValueError("k, v and their exponents must be on one device")
        self.type = types[k.dtype]
        if self.type == CACHE_E4M3:
            for t in (k_exp, v_exp):
                if t is None or t.dtype != torch.uint8 or t.shape != (layers, nb, n_kv, 16) or not t.is_contiguous():
                    raise ValueError(f"an 8-bit cache needs contiguous uint8 k_exp and v_exp {(layers, nb, n_kv, 16)}")
        else:
            k_exp = v_exp = None
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.num_blocks, self.n_kv, self.head_dim, self.layers = nb, n_kv, d, layers
        self.device = k.get_device()
        self.dtype = torch.float32 if self.type == CACHE_F32 else torch.bfloat16      # of q and the attention's output
        e = [(None, None) if k_exp is None else (_ptr(k_exp[i]), _ptr(v_exp[i])) for i in range(layers)]
        self._c = [CacheC(_ptr(k[i]), _ptr(v[i]), *e[i], nb, n_kv, d, self.type) for i in range(layers)]
        self._ref = [C.addressof(c) for c in self._c]

    def layer(self, i):
        return self._ref[i]

    def _check_layers(self, n):
        if self.layers != n:
            raise ValueError(f"a cache of {self.layers} layers for a model of {n}")


class Rows:
    """Which rows of a call belong to which sequence: ``row_start`` int32 [batch + 1] (None: max_rows rows each), ``ctx``
    int32 [batch] tokens cached before them (None: 0), ``tables`` int32 [batch, max_blocks].  Row j of sequence b is
    its token ctx[b] + j.  ``rows``, ``max_rows`` (of one sequence) and ``max_ctx`` (cached and new tokens of one
    sequence) bound what the device arrays may hold when a call runs; the arrays may change between calls.  Tokens
    outside 0 .. max_ctx - 1 do not exist: a row there is neither kept nor seen."""

    def __init__(self, row_start, ctx, tables, rows=None, max_rows=1, max_ctx=None):
        if tables.dtype != torch.int32 or tables.dim() != 2 or not tables.is_contiguous():
            raise ValueError(f"tables must be contiguous int32 [batch, max_blocks], got {tables.dtype} {tuple(tables.shape)}")
        batch, max_blocks = tables.shape
        if rows is None:
            if row_start is not None:
                raise ValueError("rows is needed beside row_start")
            rows = batch * max_rows
        if max_ctx is None:
            max_ctx = 16 * max_blocks
        for what, t, n in (("row_start", row_start, batch + 1), ("ctx", ctx, batch)):
            _check_vector(what, t, torch.int32, n)
            if t is not None and t.device != tables.device:
                raise ValueError(f"{what} on {t.device}, tables on {tables.device}")
        if any(not 0 <= n < 1 << 31 for n in (rows, max_rows, max_ctx)):
            raise ValueError(f"rows {rows}, max_rows {max_rows} and max_ctx {max_ctx} must be 32-bit sizes")
        self.row_start, self.ctx, self.tables = row_start, ctx, tables
        self.batch, self.rows, self.max_rows, self.max_ctx = batch, rows, max_rows, max_ctx
        self._c = RowsC(_ptr(row_start), _ptr(ctx), _ptr(tables), max_blocks, batch, rows, max_rows, max_ctx)
        self.ref = C.addressof(self._c)
        self._ws = {}

    def _tree_bytes(self, cache, n_q):
        """Workspace of an attention over these rows (its sizes are fixed, so it is asked for once)."""
        key = (cache.type, cache.n_kv, cache.head_dim, n_q)
        n = self._ws.get(key)
        if n is None:
            n = self._ws[key] = lib.nova_tree_attention_workspace_bytes(cache.layer(0), self.ref, n_q)
        return n


class Rope:
    """Rotary embedding of the first ``rot`` dimensions, half-split or ``interleaved`` pairs; ``factor`` and
    ``orig_ctx`` (with ``alpha``, ``beta``) scale it for longer contexts, ``mscale`` multiplies sines and cosines."""

    def __init__(self, rot, theta=10000.0, interleaved=False, factor=1.0, orig_ctx=0, alpha=1.0, beta=32.0, mscale=1.0):
        self._c = RopeC(rot, int(interleaved), theta, factor, orig_ctx, alpha, beta, mscale)
        self.ref = C.addressof(self._c)


def kv_append(cache, rows, k, v, q=None, pos=None, rope=None, q_out=None, layer=0, stream=None):
    """Rotate q and k (``rope`` None: not) at ``pos`` (int32 [rows]; None: the rows' token numbers) and write k and v
    behind their sequences' contexts in ``cache``, in its type.  k, v [rows, n_kv, head_dim], q [rows, n_q, head_dim],
    bf16 or fp32, may be views of one packed projection.  Returns the rotated q (``q_out``, which may be q itself)."""
    n, d = rows.rows, cache.head_dim
    _check_device(cache.device, rows.tables, k, v, q, pos, q_out)
    act, k_pitch = _check_rows_of("k", k, n, cache.n_kv, d)
    act_v, v_pitch = _check_rows_of("v", v, n, cache.n_kv, d)
    _check_vector("pos", pos, torch.int32, n)
    n_q = q_pitch = out_pitch = act_out = 0
    act_q = act
    if q is not None:
        n_q = q.shape[1] if q.dim() == 3 else 0
        act_q, q_pitch = _check_rows_of("q", q, n, n_q, d)
        if q_out is None:
            q_out, act_out, out_pitch = _dense_like(q, stream), act_q, n_q * d
        else:
            act_out, out_pitch = _check_rows_of("q_out", q_out, n, n_q, d)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if act_v != act or act_q != act:
        raise ValueError("q, k and v must have one type")
    _check(lib.nova_kv_append(cache.layer(layer), rows.ref, rope.ref if rope is not None else None, _ptr(pos), act, _ptr(q), q_pitch,
                              n_q, k.data_ptr(), k_pitch, v.data_ptr(), v_pitch, _ptr(q_out), act_out, out_pitch,
                              _stream_on(cache.device, stream)))
    return q_out


def kv_gather(cache, rows, slots=None, k_out=None, v_out=None, dtype=torch.bfloat16, layer=0, stream=None):
    """Cached rows as dense K and V [rows, n_kv, head_dim] in ``dtype``: the sequences' tokens ctx[b] + j, or ``slots``
    (int32 [rows], token numbers in the row's sequence).  Rows behind the last sequence are left as they were."""
    n, d = rows.rows, cache.head_dim
    _check_vector("slots", slots, torch.int32, n)
    _check_device(cache.device, rows.tables, slots, k_out, v_out)
    dtype = k_out.dtype if k_out is not None else v_out.dtype if v_out is not None else dtype
    act = act_v = _ACT.get(dtype)
    k_pitch = v_pitch = cache.n_kv * d
    if k_out is not None:
        act, k_pitch = _check_rows_of("k_out", k_out, n, cache.n_kv, d)
    if v_out is not None:
        act_v, v_pitch = _check_rows_of("v_out", v_out, n, cache.n_kv, d)
    if act is None or act != act_v:
        raise ValueError("k_out and v_out must have one type, bfloat16 or float32")
    if k_out is None:
        k_out = _empty(cache.k, (n, cache.n_kv, d), dtype, stream)
    if v_out is None:
        v_out = _empty(cache.k, (n, cache.n_kv, d), dtype, stream)
    _check(lib.nova_kv_gather(cache.layer(layer), rows.ref, _ptr(slots), act, k_out.data_ptr(), k_pitch, v_out.data_ptr(), v_pitch,
                              _stream_on(cache.device, stream)))
    return k_out, v_out


def tree_attention(cache, rows, q, mask=None, out=None, scale=None, layer=0, stream=None):
    """Attention of each sequence's rows (at most 64 drafted tokens, appended before) over its cache: a row sees the
    context and the drafted tokens i whose bit i is set in ``mask`` (int64 [rows]; None: those up to its own).
    q [rows, n_q, head_dim] in ``cache.dtype``; returns ``out`` of the same shape and type."""
    n, d = rows.rows, cache.head_dim
    _check_device(cache.device, rows.tables, q, mask, out)
    _check_vector("mask", mask, torch.int64, n)
    n_q = q.shape[1] if q.dim() == 3 else 0
    act, q_pitch = _check_rows_of("q", q, n, n_q, d)
    act_out, out_pitch = act, n_q * d
    if out is None:
        out = _dense_like(q, stream)
    else:
        act_out, out_pitch = _check_rows_of("out", out, n, n_q, d)
    if q.dtype != cache.dtype or act_out != act:
        raise ValueError(f"q and out must be {cache.dtype}")
    nbytes = rows._tree_bytes(cache, n_q)
    ws = _empty(q, nbytes, torch.uint8, stream) if nbytes else None
    _check(lib.nova_tree_attention(cache.layer(layer), rows.ref, _ptr(mask), q.data_ptr(), q_pitch, n_q,
                                   d ** -0.5 if scale is None else scale, out.data_ptr(), out_pitch, _ptr(ws), nbytes,
                                   _stream_on(cache.device, stream)))
    return out


@functools.lru_cache(maxsize=256)
def _logprobs_bytes(rows, vocab, n_top):
    return lib.nova_logprobs_workspace_bytes(rows, vocab, n_top)


def logprobs(logits, given=None, n_top=0, stream=None):
    """Of logit rows [rows, vocab] (fp32 or bf16): (log probabilities of ``given`` int32 [rows, n] or None, entropies
    [rows], the ``n_top`` (at most 32) largest log probabilities [rows, n_top] and their ids, or None)."""
    act = _ACT.get(logits.dtype)
    if act is None or logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError(f"logits must be float32 or bfloat16 [rows, vocab] with contiguous rows, got {logits.dtype} {tuple(logits.shape)}")
    if n_top < 0:
        raise ValueError(f"n_top {n_top} is negative")
    rows, vocab = logits.shape
    n_given = 0
    if given is not None:
        if given.dtype != torch.int32 or given.dim() != 2 or given.shape[0] != rows or not given.is_contiguous():
            raise ValueError(f"given must be contiguous int32 [{rows}, n], got {given.dtype} {tuple(given.shape)}")
        n_given = given.shape[1]
    dev = logits.get_device()
    _check_device(dev, given)
    n_top = min(n_top, vocab)
    # one allocation for what is returned, cut into dense matrices
    buf = _empty(logits, rows * (n_given + 1 + 2 * n_top), torch.float32, stream)
    at = rows * n_given
    lp = buf.as_strided((rows, n_given), (n_given, 1), 0) if given is not None else None
    entropy = buf.as_strided((rows,), (1,), at)
    at += rows
    top_lp = top_ids = None
    if n_top:
        top_lp = buf.as_strided((rows, n_top), (n_top, 1), at)
        top_ids = buf.as_strided((rows, n_top), (n_top, 1), at + rows * n_top).view(torch.int32)
    nbytes = _logprobs_bytes(rows, vocab, n_top)
    ws = _empty(logits, nbytes, torch.uint8, stream) if nbytes else None
    _check(lib.nova_logprobs(logits.data_ptr(), act, logits.stride(0) if rows > 1 else vocab, rows, vocab, _ptr(given), n_given, _ptr(lp),
                             entropy.data_ptr(), n_top, _ptr(top_lp), _ptr(top_ids), _ptr(ws), nbytes, _stream_on(dev, stream)))
    return lp, entropy, top_lp, top_ids


# ----------------------------------------------------------------------------- linear co-run study
LINEAR_TILED, LINEAR_TILED_SMALL, LINEAR_THIN, LINEAR_THIN_VALU = 0, 1, 2, 3


def linear(variant: int, x, w, out, stream=None):
    """out (fp32 [M, N]) += x (bf16 [M, K]) w (bf16 [N, K])^T with the chosen kernel variant."""
    m, k = x.shape
    n = w.shape[0]
    _check(lib.nova_linear(variant, _ptr(x), m, k, _ptr(w), n, _ptr(out), _stream(stream)))
    return out


# ----------------------------------------------------------------------------- partitions & timing
def make_cu_mask(n_cus: int, first_slot: int = 0) -> list[int]:
    m = (C.c_uint32 * 8)()
    _check(lib.nova_make_cu_mask(n_cus, first_slot, m))
    return list(m)


def set_stage_partition(stage: int, mask) -> torch.cuda.ExternalStream:
    arr = (C.c_uint32 * len(mask))(*mask)
    s = C.c_void_p()
    _check(lib.nova_set_stage_partition(stage, arr, len(mask), C.byref(s)))
    return torch.cuda.ExternalStream(s.value)


def cu_probe(stream, n_workgroups: int = 4096):
    """(xcd, shader engine, cu) of the CU each probe workgroup ran on, as a set."""
    out = torch.zeros(n_workgroups, dtype=torch.int32, device="cuda")
    _check(lib.nova_cu_probe(_stream(stream), _ptr(out), n_workgroups))
    stream = stream or torch.cuda.current_stream()
    stream.synchronize()
    v = out.cpu().numpy().astype(np.uint32)
    return {(int(x >> 16), int((x >> 8) & 0xff), int(x & 0xff)) for x in v}


def timing_enable(on: bool = True):
    _check(lib.nova_timing_enable(1 if on else 0))


def timing_read(kind: int):
    ms = C.c_double()
    n = C.c_int()
    _check(lib.nova_timing_read(kind, C.byref(ms), C.byref(n)))
    return ms.value, n.value
