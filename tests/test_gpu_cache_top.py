"""The largest numbers of an 8-bit cache: what is stored, read back and stored again."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.test_gpu_cache_ops import BF16, F32, Batch, _dev, _np, _rng

pytestmark = pytest.mark.gpu

TOP = 2.0 ** 128 - 2.0 ** 104                       # the largest float32


@pytest.mark.parametrize("d", [64, 128])
def test_largest_numbers_of_an_8_bit_cache(gpu_lib, d):
    """Finite rows of any size read back finite, within half a step, and are kept as they are when appended again."""
    nova = gpu_lib
    r = _rng(d, 128)
    x = np.zeros((20, 2, d), np.float32)
    tops = [TOP, -TOP, 3.3e38, 248 * 2.0 ** 120, np.nextafter(np.float32(248 * 2.0 ** 120), np.float32(0)), 240 * 2.0 ** 120,
            448 * 2.0 ** 119, np.nextafter(np.float32(448 * 2.0 ** 119), np.float32(np.inf)), 3e38, 1e38]
    for i, t in enumerate(tops):
        x[i, :, i % d] = t
        x[10 + i] = np.float32(t) * r.uniform(-1, 1, (2, d))
        x[10 + i, 1, 3] = t
    bt = Batch(nova, [0], [20], 2, d, "e4m3", seed=d)
    t = _dev(x, F32)
    nova.kv_append(bt.cache, bt.desc, t, t)
    want, _ = oc.quantise(x.astype(np.float64))
    assert np.abs(want).max() < TOP and (np.abs(want - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** (119 - 9)).all()
    for dtype in (F32, BF16):
        for got in nova.kv_gather(bt.cache, bt.desc, dtype=dtype):
            assert np.array_equal(_np(got), want)
    k, v = nova.kv_gather(bt.cache, bt.desc, dtype=BF16)
    nova.kv_append(bt.cache, bt.desc, k, v)
    for got, first in zip(nova.kv_gather(bt.cache, bt.desc, dtype=F32), (k, v)):
        assert np.array_equal(_np(got), _np(first))
