"""Acceptance at the largest grids that it takes: sequences times chunks of 8192 logits up to 2^24."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2509_21301_amd import nova as nova_
from tests.test_cache_ops_cpu import FAKE, _rows


def test_limits():
    """The check comes before any device work, so the addresses here are never read."""
    def call(batch, vocab):
        return nova_.lib.nova_accept(C.byref(_rows(batch=batch, rows=16, max_rows=16)), FAKE, None, FAKE, 1, vocab, FAKE, 1, vocab, vocab, None, FAKE,
                                     FAKE, FAKE, FAKE, FAKE, FAKE, 0, None)
    # 245 chunks: 16056075 workgroups of 512 threads, more than one grid dimension has; accepted, but for the workspace
    assert 65535 * 245 * 512 > 1 << 32 and call(65535, 2000000) == nova_.ENOSPACE
    assert call(65535, 1 << 21) == nova_.ENOSPACE
    assert nova_.lib.nova_accept(C.byref(_rows(batch=4, rows=1 << 15, max_rows=16)), FAKE, None, FAKE, 1, 1 << 21, FAKE, 1, 1 << 21, 1 << 21, None,
                                 FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0, None) == nova_.EUNSUPPORTED     # 2^16 rows with the draft's, 256 chunks


@pytest.mark.gpu
def test_more_workgroups_than_a_grid_dimension(gpu_lib):
    """65535 sequences, most of them without rows, of 135 chunks each: 2^32 threads and more."""
    from tests.test_gpu_step_ops import F32, _accept_case, _check_accept
    vocab = 1100000
    starts, logits, draft, ids, _, t, u = _accept_case([3, 2, 3], vocab, 5, F32, "draft", spread=1.0)
    rows = [0] * 65535
    rows[0], rows[40000], rows[65534] = 3, 2, 3
    assert len(rows) * -(-vocab // 8192) * 512 > 1 << 32
    temperature = np.ones(65535)
    temperature[[0, 40000, 65534]] = np.asarray(t)[:3]
    _check_accept(gpu_lib, rows, np.concatenate([[0], np.cumsum(rows)]), logits, draft, ids, None, temperature, u)
    torch.cuda.synchronize()
