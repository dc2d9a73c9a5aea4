"""Forks whose rows meet, by tables and counts written out: a row that is a request's source is never overwritten."""
import numpy as np
import pytest
import torch

from oracle import steps as st

# (requests (source, target, tokens), served, rows of the tables, counts) from START: three rows of a page or two
START = ([[0, 1, -1], [2, 3, -1], [4, -1, -1], [-1, -1, -1]], [1, 1, 1, 1, 1, 0, 0, 0])
CASES = dict(
    chain=([(0, 1, 32), (1, 2, 20)], [0, 1], [[0, 1, -1], [2, 3, -1], [2, 5, -1], [-1, -1, -1]], [1, 1, 2, 1, 1, 1, 0, 0]),
    chain_from_behind=([(1, 2, 20), (0, 1, 32)], [1, 0], [[0, 1, -1], [2, 3, -1], [2, 5, -1], [-1, -1, -1]], [1, 1, 2, 1, 1, 1, 0, 0]),
    swap=([(0, 1, 5), (1, 0, 5)], [0, 0], *START),
    itself=([(1, 1, 16), (0, 3, 17)], [0, 1], [[0, 1, -1], [2, 3, -1], [4, -1, -1], [0, 5, -1]], [2, 1, 1, 1, 1, 1, 0, 0]),
    # the source of a request that is refused is one all the same, and so is its target
    refused_source=([(0, 1, 16), (1, 9, 16)], [0, 0], *START),
    refused_target=([(-1, 3, 16), (0, 3, 16), (3, 2, 0)], [0, 0, 1], [[0, 1, -1], [2, 3, -1], [-1, -1, -1], [-1, -1, -1]], [1, 1, 1, 1, 1, 0, 0, 0]),
    twice=([(0, 3, 32), (1, 3, 32)], [1, 0], [[0, 1, -1], [2, 3, -1], [4, -1, -1], [0, 1, -1]], [2, 2, 1, 1, 1, 0, 0, 0]))


@pytest.mark.parametrize("name", CASES)
def test_oracle(name):
    requests, served, tables, refs = CASES[name]
    pool = st.Pool(START[1], START[0])
    done, _ = pool.fork(*(list(x) for x in zip(*requests)))
    assert done == served and pool.tables.tolist() == tables and pool.refs.tolist() == refs


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_fork(gpu_lib, name):
    nova = gpu_lib
    requests, served, tables, refs = CASES[name]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pages, t = nova.Pages.of(i32(START[1])), i32(START[0])
    cache = nova.Cache(8, 1, 64, nova.CACHE_BF16, layers=2)
    cache.k.normal_(), cache.v.normal_()
    before = cache.k.clone(), cache.v.clone()
    done = pages.fork(cache, t, *(i32(x) for x in zip(*requests)))
    assert done.tolist() == served and t.tolist() == tables and pages.refs.tolist() == refs
    # of the blocks only 5, the first that is free, is ever written: with a source's second page
    for x, y in zip((cache.k, cache.v), before):
        w = y.clone()
        if refs[5]:
            w[:, 5] = y[:, 3 if name != "itself" else 1]
        assert torch.equal(x, w)


@pytest.mark.gpu
def test_fork_many_rows(gpu_lib):
    """65535 rows, of which every other is a target and the last requests' targets are sources."""
    nova = gpu_lib
    n = 65535
    r = np.random.default_rng(3)
    tables = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
    tables[::2, 0] = torch.arange((n + 1) // 2, dtype=torch.int32, device="cuda")
    refs = torch.zeros((n + 1) // 2 + 40000, dtype=torch.int32, device="cuda")
    refs[:(n + 1) // 2] = 1
    src, dst = 2 * r.integers(0, n // 2, n // 2), 2 * np.arange(n // 2) + 1
    dst[-500:] -= 1
    lens = r.integers(0, 17, n // 2)
    pool = st.Pool(refs.cpu().numpy(), tables.cpu().numpy())
    seen = set(src.tolist())
    cache = nova.Cache(len(refs), 1, 64, nova.CACHE_E4M3)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    done = nova.Pages.of(refs).fork(cache, tables, i32(src), i32(dst), i32(lens))
    assert done.tolist() == [int(d not in seen) for d in dst.tolist()]
    free = iter(range((n + 1) // 2, len(refs)))
    want, counts = pool.tables, pool.refs
    for a, b, k in zip(src.tolist(), dst.tolist(), lens.tolist()):
        if b in seen:
            continue
        block = -1 if k == 0 else a // 2 if k == 16 else next(free)
        want[b] = [block, -1]
        if block >= 0:
            counts[block] += 1
    assert tables.tolist() == want.tolist() and refs.tolist() == counts.tolist()
