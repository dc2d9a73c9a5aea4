"""Adapters on numbers whose sums are exact in fp32, so that the result is the exact one rounded once: whole numbers below
2^24 in every sum, whatever its order, and bases that cancel all but the last bits of what the adapter gives."""
import numpy as np
import pytest
import torch

from tests.test_gpu_step_ops import BF16, F32, _dev, _i32, _np

pytestmark = pytest.mark.gpu


def _rows(nova, rows):
    starts = np.concatenate([[0], np.cumsum(rows)])
    return nova.Rows(_i32(starts), None, _i32(np.zeros((len(rows), 1))), rows=sum(rows), max_rows=max(rows), max_ctx=16)


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("rows", [[1, 5, 3], [40, 33], [200]])
@pytest.mark.parametrize("rank", [8, 16, 32, 64, 128])
def test_bases_that_cancel(gpu_lib, types, rows, rank):
    nova = gpu_lib
    r = np.random.default_rng([rank, rows[0], types[0] == F32])
    k, n_out, total = 64, 200, sum(rows)
    if types[0] == F32:                      # |A x| < 64 * 2^17 * 2 = 2^24
        x, a = r.integers(-(1 << 17) + 1, 1 << 17, (total, k)), r.integers(-2, 3, (2, rank, k))
    else:                                    # below 64 * 255 * 127 < 2^21
        x, a = r.integers(-255, 256, (total, k)), r.integers(-127, 128, (2, rank, k))
    b = np.zeros((2, n_out, rank))           # a power of two of one rank each
    np.put_along_axis(b, r.integers(0, rank, (2, n_out, 1)), np.ldexp(r.choice([-1.0, 1.0], (2, n_out, 1)), r.integers(-12, 5, (2, n_out, 1))), 2)
    scale = np.array([1.0, -0.5])
    which = np.arange(len(rows)) % 2
    of = np.repeat(which, rows)
    delta = np.stack([scale[i] * (b[i] @ (a[i] @ x[j])) for j, i in enumerate(of)])
    base = _dev(-delta, F32).to(BF16).to(types[1])       # its first 8 bits
    want = (_np(base) + delta)
    assert (np.abs(want) > 0).any() and (np.abs(want) <= 2.0 ** -7 * np.abs(delta)).all()
    ad = nova.Adapters(_dev(a, F32).to(BF16), _dev(b, F32).to(BF16), _dev(scale, F32))
    x = _dev(x, F32).to(types[0])
    got = nova.lora(ad, _rows(nova, rows), _i32(which), x, base=base)
    assert torch.equal(got, torch.from_numpy(want).cuda().to(F32).to(types[1]))
    got = nova.lora(ad, _rows(nova, rows), _i32(which), x, dtype=types[1])
    assert torch.equal(got, torch.from_numpy(delta).cuda().to(F32).to(types[1]))


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("rows", [[2, 1, 2], [35, 40], [160]])
def test_range_of_fp32(gpu_lib, out, rows):
    """x and h above the largest number of bf16, and infinities and NaN, which stay in their rows."""
    nova = gpu_lib
    total, k, big = sum(rows), 64, float(torch.finfo(F32).max)
    x, a, b = np.zeros((total, k)), np.zeros((1, 8, k)), np.zeros((1, 16, 8))
    a[0, 0, 0], a[0, 1, 1], a[0, 1, 2], b[0, :8, 0], b[0, 8:, 1] = 2.0 ** -100, 1.9921875, 1.5, 0.5, 2.0 ** -60
    x[0, 0] = big                            # one part of it would be infinite, rounded
    x[1, 1], x[1, 2] = 2.0 ** 127, 2.0 ** 119           # h = 2^127 (1.9921875 + 1.5 2^-8) = 2^127 1.998046875
    x[2, 0], x[3, 0], x[4, 1] = np.inf, -np.inf, np.nan
    want = np.zeros((total, 16))
    want[0, :8], want[1, 8:] = big * 2.0 ** -101, 2.0 ** 67 * 1.998046875
    want[2], want[3], want[4] = np.nan, np.nan, np.nan    # 0 times infinity in the other rank
    want[2, :8], want[3, :8] = np.nan, np.nan
    ad = nova.Adapters(_dev(a, F32).to(BF16), _dev(b, F32).to(BF16))
    got = nova.lora(ad, _rows(nova, rows), _i32(np.zeros(len(rows))), _dev(x, F32), dtype=out)
    assert torch.equal(torch.isnan(got[2:5]), torch.from_numpy(np.isnan(want[2:5])).cuda())
    keep = [0, 1, *range(5, total)]
    assert torch.equal(got[keep], torch.from_numpy(want[keep]).cuda().to(F32).to(out))
    # without zeros beside it an infinity is one: sign of h, then of B
    a[0] = 2.0 ** -10
    b[0] = 2.0 ** -3
    b[0, 3] = -1.0
    ad = nova.Adapters(_dev(a, F32).to(BF16), _dev(b, F32).to(BF16))
    x[0:2] = 0.0
    got = nova.lora(ad, _rows(nova, rows), _i32(np.zeros(len(rows))), _dev(x, F32), dtype=out).float()
    sign = torch.ones(16, device="cuda")
    sign[3] = -1
    assert torch.equal(got[2], sign * float("inf")) and torch.equal(got[3], -sign * float("inf")) and torch.isnan(got[4]).all()
    assert (got[[0, 1, *range(5, total)]] == 0).all()


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("rank", [8, 32, 64, 72])
def test_large_results(gpu_lib, types, rank):
    """More than 10^8 numbers of result, whose tiles are the largest; sequences that end inside them, and one without an adapter."""
    nova = gpu_lib
    g = torch.Generator(device="cuda")
    g.manual_seed(rank)
    rows, k, n_out = [9000, 40, 0, 3000, 1001], 72, 8192
    which, scale = [1, 0, 1, -1, 0], torch.tensor([1.0, -0.5], device="cuda")
    total = sum(rows)
    assert total * n_out > 10 ** 8
    whole = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda").to(F32)  # noqa: E731
    # sums of 72 numbers below 2^8, then of at most 72 of those times 3: below 2^22; in fp32 below 2^12, and two: below 2^21
    top = 1 << (12 if types[0] == F32 else 8)
    x, a, b = whole(1 - top, top, total, k).to(types[0]), whole(-1, 2, 2, rank, k).to(BF16), whole(-3, 4, 2, n_out, rank).to(BF16)
    if types[0] == F32:                      # two ranks of a column only
        b[:, :, 2:] = 0
    base = whole(-100, 101, total, n_out).to(types[1])
    got = nova.lora(nova.Adapters(a, b, scale), _rows(nova, rows), _i32(which), x, base=base)
    at = 0
    for n, i in zip(rows, which):
        sl = slice(at, at + n)
        at += n
        want = base[sl].double()
        if i >= 0:
            want = want + float(scale[i]) * ((x[sl].double() @ a[i].double().T.contiguous()) @ b[i].double().T.contiguous())
        assert torch.equal(got[sl], want.to(F32).to(types[1]))
