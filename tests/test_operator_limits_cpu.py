"""The largest sizes that the library accepts, without a GPU: the checks come before any device work, so the addresses
here are never read."""
import ctypes as C

from paper_2509_21301_amd import nova, synth

FAKE = 1 << 20
LIB = nova.lib


def test_logit_rows_fit_a_grid():
    """A row of the joining kernel is a workgroup of 512 threads, and a grid has fewer than 2^32 threads."""
    def call(rows):
        return LIB.nova_logprobs(FAKE, 1, 152064, rows, 152064, None, 0, None, FAKE, 4, FAKE, FAKE, FAKE, 0, None)
    assert call(1 << 23) == nova.EUNSUPPORTED
    assert call((1 << 23) - 1) == nova.ENOSPACE                       # accepted, but for its workspace
    assert ((1 << 23) - 1) * 512 < 1 << 32


def test_prompts_past_32_bits():
    """A prompt whose length wraps to a negative number is refused, and its workspace is not 0 bytes of it."""
    cfg = synth.TINY_LLM
    h = C.c_void_p()
    d = nova.LlmDescC(nova.llm_config_c(cfg, nova.ACT_BF16), FAKE, FAKE, FAKE)
    nova._check(LIB.nova_llm_create(C.byref(d), C.byref(h)))
    cache = nova.CacheC(FAKE, FAKE, FAKE, FAKE, (1 << 31) - 1, cfg.n_kv, cfg.head_dim, nova.CACHE_E4M3)
    kv = nova.KvC(FAKE, FAKE, (1 << 31) - 1)
    for n_vis, n_text in ((1 << 30, 1 << 30), ((1 << 31) - 1, 1), ((1 << 31) - 1, (1 << 31) - 1), (0, (1 << 31) - 1)):
        assert LIB.nova_llm_prefill_cache(h, FAKE, n_vis, FAKE, n_text, FAKE, C.byref(cache), FAKE, None, FAKE, 0, None) < 0
        assert b"prompt" in LIB.nova_last_error()
        assert LIB.nova_llm_prefill(h, FAKE, n_vis, FAKE, n_text, FAKE, C.byref(kv), FAKE, None, FAKE, 0, None) < 0
        assert b"prompt" in LIB.nova_last_error()
    LIB.nova_llm_destroy(h)
