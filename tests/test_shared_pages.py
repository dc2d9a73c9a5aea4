"""Rows turned back to fewer tokens: a page that several rows name is never gone on in by one of them."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import steps as st
from paper_2509_21301_amd import nova as nova_
from tests.test_cache_ops_cpu import FAKE

# rows of 40, 32 and 20 tokens: row 1 shares two pages with row 0, row 3 names a page twice
TABLES, REFS = [[0, 1, 2], [0, 1, -1], [3, 4, -1], [5, 5, -1]], [2, 2, 1, 1, 1, 2, 0, 0]
# (rows, tokens) -> served, tables, counts
CASES = dict(
    inside_shared=(([1], [20]), [0], TABLES, REFS),
    at_a_border=(([1], [16]), [1], [[0, 1, 2], [0, -1, -1], [3, 4, -1], [5, 5, -1]], [2, 1, 1, 1, 1, 2, 0, 0]),
    own_page=(([2, 0], [17, 33]), [1, 1], TABLES, REFS),
    own_first_page=(([2], [5]), [1], [[0, 1, 2], [0, 1, -1], [3, -1, -1], [5, 5, -1]], [2, 2, 1, 1, 0, 2, 0, 0]),
    both_at_once=(([0, 1], [20, 25]), [0, 0], TABLES, REFS),
    # the counts before the call decide, whatever the order
    one_goes=(([0, 1], [0, 20]), [1, 0], [[-1, -1, -1], [0, 1, -1], [3, 4, -1], [5, 5, -1]], [1, 1, 0, 1, 1, 2, 0, 0]),
    one_goes_last=(([1, 0], [20, 0]), [0, 1], [[-1, -1, -1], [0, 1, -1], [3, 4, -1], [5, 5, -1]], [1, 1, 0, 1, 1, 2, 0, 0]),
    twice=(([1, 1], [20, 16]), [0, 1], [[0, 1, 2], [0, -1, -1], [3, 4, -1], [5, 5, -1]], [2, 1, 1, 1, 1, 2, 0, 0]),
    twice_in_a_row=(([3, 3], [20, 4]), [0, 0], TABLES, REFS),
    outside=(([4, -1, 2], [1, 1, 0]), [0, 0, 1], [[0, 1, 2], [0, 1, -1], [-1, -1, -1], [5, 5, -1]], [2, 2, 1, 0, 0, 2, 0, 0]),
    beyond=(([1, 1], [47, (1 << 31) - 1]), [1, 1], TABLES, REFS),
    negative=(([2], [-(1 << 31)]), [1], [[0, 1, 2], [0, 1, -1], [-1, -1, -1], [5, 5, -1]], [2, 2, 1, 0, 0, 2, 0, 0]))


@pytest.mark.parametrize("name", CASES)
def test_oracle(name):
    (rows, tokens), served, tables, refs = CASES[name]
    pool = st.Pool(REFS, TABLES)
    assert pool.free(rows, tokens) == served and pool.tables.tolist() == tables and pool.refs.tolist() == refs


def test_refusals():
    def trim(p=nova_.PagesC(FAKE, 8), t=FAKE, w=4, b=5, seqs=FAKE, tok=FAKE, n=3, done=FAKE):
        return nova_.lib.nova_pages_trim(C.byref(p), t, w, b, seqs, tok, n, done, None)
    assert trim(n=0) == nova_.OK
    for bad in [dict(seqs=None), dict(tok=None), dict(done=None), dict(seqs=FAKE + 2), dict(tok=FAKE + 1), dict(done=FAKE + 3), dict(n=-1), dict(n=65536),
                dict(t=None), dict(w=0), dict(b=65536), dict(p=nova_.PagesC(None, 8))]:
        assert trim(**bad) == nova_.EINVAL, bad
    assert trim(w=(1 << 26) + 1) == nova_.EUNSUPPORTED
    # what would be refused without a word
    assert nova_.lib.nova_pages_free(C.byref(nova_.PagesC(FAKE, 8)), FAKE, 4, 5, FAKE, FAKE, 3, None) == nova_.EUNSUPPORTED


def _i32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_trim(gpu_lib, name):
    (rows, tokens), served, tables, refs = CASES[name]
    pages, t = gpu_lib.Pages.of(_i32(REFS)), _i32(TABLES)
    assert pages.free(t, _i32(rows), _i32(tokens)).tolist() == served
    assert t.tolist() == tables and pages.refs.tolist() == refs


@pytest.mark.gpu
def test_trim_many(gpu_lib):
    """2000 requests over 700 rows that share pages, twice as many pages as a workgroup has threads."""
    r = np.random.default_rng(4)
    blocks, tables = 3000, np.full((700, 600), -1)
    for b in range(700):
        n = r.integers(0, 600)
        tables[b, :n] = r.integers(0, blocks, n)
    refs = np.bincount(tables[tables >= 0], minlength=blocks)
    refs[r.random(blocks) < 0.3] = 1                          # pages that count as a row's own
    rows, tokens = r.integers(-2, 702, 2000), r.integers(-20, 9700, 2000)
    pages, t, pool = gpu_lib.Pages.of(_i32(refs)), _i32(tables), st.Pool(refs, tables)
    assert pages.free(t, _i32(rows), _i32(tokens)).tolist() == pool.free(rows, tokens)
    assert t.tolist() == pool.tables.tolist() and pages.refs.tolist() == pool.refs.tolist()
    assert gpu_lib.Pages.of(pages.refs).free(t, _i32([]), _i32([])).shape == (0,)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("back", [16, 20, 31])
def test_a_branch_turned_back_leaves_its_source_alone(gpu_lib, kind, back):
    """A branch of 32 tokens turned back and appended to: its source's K and V stay as they were, and so do the tokens
    that the branch keeps."""
    nova = gpu_lib
    type = dict(bf16=nova.CACHE_BF16, f32=nova.CACHE_F32, e4m3=nova.CACHE_E4M3)[kind]
    cache, pages = nova.Cache(8, 2, 64, type, layers=1), nova.Pages(8)
    tables = torch.full((3, 3), -1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(back)

    def rows(b, ctx, n):
        return nova.Rows(None, _i32([ctx]), tables[b:b + 1].clone(), max_rows=n, max_ctx=48)

    def append(b, ctx, n):
        nova.kv_append(cache, rows(b, ctx, n), *torch.randn(2, n, 2, 64, generator=g, device="cuda").bfloat16().unbind(0))

    assert pages.extend(tables, _i32([32, 0, 0])).tolist() == [1, 1, 1]
    append(0, 0, 32)
    assert pages.fork(cache, tables, _i32([0]), _i32([1]), _i32([32])).tolist() == [1]
    source = nova.kv_gather(cache, rows(0, 0, 32), dtype=torch.float32)
    served = pages.free(tables, _i32([1]), _i32([back]))
    branch = 1
    assert served.tolist() == [int(back == 16)]
    if back != 16:                                            # the row is as it was; its tokens go on in another
        assert tables[1].tolist() == tables[0].tolist() and pages.refs.tolist() == [2, 2] + [0] * 6
        assert pages.fork(cache, tables, _i32([1]), _i32([2]), _i32([back])).tolist() == [1]
        pages.free(tables, _i32([1]))
        branch = 2
    assert pages.extend(tables, _i32([36 if b == branch else 0 for b in range(3)])).tolist() == [1, 1, 1]
    append(branch, back, 36 - back)
    for a, b in zip(nova.kv_gather(cache, rows(0, 0, 32), dtype=torch.float32), source):
        assert torch.equal(a, b)
    for a, b in zip(nova.kv_gather(cache, rows(branch, 0, 36), dtype=torch.float32), source):
        assert torch.equal(a[:back], b[:back]) and not torch.equal(a[back:32], b[back:])
    pages.free(tables, _i32([0, branch]))
    assert (pages.refs == 0).all()
