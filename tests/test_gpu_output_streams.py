"""Where a model call allocates its output and its workspace: on the stream that the call runs on, so that memory freed
on another stream, which queued work there may still use, is not written behind that work's back."""
import pytest
import torch

from paper_2509_21301_amd import synth

pytestmark = pytest.mark.gpu

CFG = synth.TINY_LLM


def _stream_of(t):
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's")


@pytest.mark.parametrize("call", ["prefill", "prefill_cache", "decode", "verify"])
def test_outputs_are_allocated_on_the_call_stream(gpu_lib, call):
    nova = gpu_lib
    llm = nova.Llm(CFG, synth.llm_weights(CFG, 0))
    tables, pool = synth.block_tables([48, 48], CFG.block, seed=5)
    tables = torch.from_numpy(tables).cuda()
    kv = nova.KvPool(llm, pool)
    cache = nova.Cache(pool, CFG.n_kv, CFG.head_dim, nova.CACHE_BF16, layers=CFG.layers)
    prompt = torch.from_numpy(synth.text_ids(20, CFG.vocab, seed=3)).cuda()
    ids, pos = torch.tensor([3, 4], dtype=torch.int32, device="cuda"), torch.tensor([20, 20], dtype=torch.int32, device="cuda")
    rows = nova.Rows(None, pos, tables, max_rows=1, max_ctx=40)
    run = dict(prefill=lambda s: llm.prefill(None, prompt, tables[0], kv, stream=s),
               prefill_cache=lambda s: llm.prefill(None, prompt, tables[0], cache, stream=s),
               decode=lambda s: llm.decode(ids, pos, tables, kv, 40, stream=s),
               verify=lambda s: llm.verify(ids, pos, rows, cache, stream=s))[call]
    want = run(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = run(side)
    side.synchronize()
    assert torch.equal(got, want)
    assert _stream_of(got) == side.cuda_stream
    assert _stream_of(want) == torch.cuda.current_stream().cuda_stream
    if call in ("prefill", "decode"):                       # a partition's stream is no stream of torch's
        s = nova.set_stage_partition(nova.STAGE_DECODE, nova.make_cu_mask(64))
        got = run(s)
        s.synchronize()
        assert torch.equal(got, want) and _stream_of(got) == s.cuda_stream


def test_first_calls_allocate_on_their_stream(gpu_lib):
    """The encoder's output, and the workspaces that models keep."""
    nova = gpu_lib
    side = torch.cuda.Stream()
    vit = nova.Vit(synth.TINY_VIT, synth.vit_weights(synth.TINY_VIT, 0))
    llm = nova.Llm(CFG, synth.llm_weights(CFG, 0))
    kv = nova.KvPool(llm, 8)
    table = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    pixels = torch.from_numpy(synth.image(1, 32, 32)).cuda().to(torch.bfloat16)
    prompt = torch.from_numpy(synth.text_ids(20, CFG.vocab, seed=3)).cuda()
    at = torch.tensor([20], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    vis = vit.encode(pixels, stream=side)
    first = llm.prefill(None, prompt, table[0], kv, stream=side)
    llm.decode(first, at, table, kv, 32, stream=side)
    side.synchronize()
    for t in (vis, vit.workspace(1), llm._ws["prefill"], llm._ws["decode"]):
        assert _stream_of(t) == side.cuda_stream
    assert torch.equal(vit.encode(pixels), vis)
