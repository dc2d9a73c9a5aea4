"""Draws with a number of 0 from rows whose first weights underflow: the first token is the first one that has a weight."""
import numpy as np
import pytest
import torch

from tests.test_gpu_step_ops import F32, _check_accept, _dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["chain", "draft"])
@pytest.mark.parametrize("u", [0.0, -1.0, float("nan"), 2.0 ** -24, 0.9999])
def test_parts_whose_weights_underflow(gpu_lib, kind, u):
    """e^-746 is below half of the smallest 64-bit number, but a hundred of them are not, relative to their chunk's e^-700:
    the second 2048 tokens have a sum and no weight.  The tokens before them are masked."""
    x = np.full((4, 20000), -np.inf)
    x[:, 2061:2161] = -746.0
    x[:, 7000] = -700.0
    x[:, 17000] = 0.0
    assert np.exp(-746.0) == 0.0 and 100 * np.exp(-46.0) * np.exp(-700.0) > 0.0
    x[1, 4096:4196] = -746.0                                 # two such parts one after the other
    x[2, 2061:2161] = -745.0                                 # and one whose weights are the smallest numbers
    logits = _dev(x, F32)
    ids = np.full(4, 17000)
    draft = torch.zeros_like(logits) if kind == "draft" else None
    for t in (1.0, 0.5):                                     # at 0.5 nothing but the largest has a weight
        _check_accept(gpu_lib, [1, 1, 1, 1], np.arange(5), logits, draft, ids, None, np.full(4, t), np.full(4, u, np.float32))
    tokens = gpu_lib.accept(gpu_lib.Rows(None, None, torch.zeros(4, 1, dtype=torch.int32, device="cuda"), max_rows=1, max_ctx=16),
                            _dev(ids, torch.int32), logits, _dev(np.full(4, u), F32), draft=draft)[2]
    assert tokens.flatten().tolist() == ([17000] * 4 if u > 0 else [7000, 7000, 2061, 7000])
