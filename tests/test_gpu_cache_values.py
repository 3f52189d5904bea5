"""What the operators around the paged cache give at values that an ordinary test does not meet: infinities among the visible values, angles whose sine or
cosine is small.  Needs an MI355X (-m gpu)."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_cache import BF16, F16, F32, HALF_STEP, SMALLEST, _close, _expect, _f64, _requests

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


# ---- infinite values

def _check_with_infinities(got, want, q, keys):
    """Elements that are not finite are the same ones; the others within what test_gpu_cache allows them."""
    out, lse, mass, most = want
    g, finite = _f64(got[0]), np.isfinite(out)
    assert np.array_equal(g[~finite], out[~finite], equal_nan=True)
    score = (q.shape[2] + 4) * 2.0 ** -24 * most
    weight = np.broadcast_to((2 * score + 2.0 ** -21 + 2.0 ** -16 + 2 * keys * 2.0 ** -24)[:, :, None], out.shape)
    off = 2 * weight[finite] * mass[finite]
    _close(g[finite], out[finite], HALF_STEP[q.dtype] * (np.abs(out[finite]) + off) + off + SMALLEST[q.dtype])
    none = lse == -np.inf
    _close(_f64(got[1])[~none], lse[~none], (score + 2.0 ** -21 + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(none, 0, lse)))[~none])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("heads, kv, dim, dtype", [(4, 4, 64, BF16), (8, 1, 128, F16), (16, 1, 64, BF16), (16, 1, 96, F16), (20, 1, 128, F16), (24, 2, 256, BF16), (12, 1, 80, F16)])
def test_infinite_values(dev, heads, kv, dim, dtype, wide):
    """The definition's: infinite where one of a sign is seen, however small its weight, NaN where both signs are; other elements and rows as ever.
    In a request of one token, of one tile, and of several shares."""
    lengths = [1, 20, 300, 2500]
    cache, q, table, length = _requests(dev, dim + heads, lengths, heads, kv, dim, 16, dtype, dtype, "tokens")
    v = cache.v
    place = lambda r, i: (table[r, i // 16].item(), i % 16)  # noqa: E731
    for r, n in enumerate(lengths):
        for i, d, x in ((0, 1, math.inf), (n - 1, 3, -math.inf), (n // 2, 4, math.inf), (n // 3, 4, -math.inf), (n - 1, 6, math.nan), (n // 2, dim - 1, math.inf)):
            v[(*place(r, i), slice(None), d)] = x
    # tokens whose weights are 2^-30 to 2^-100 of the largest
    q.abs_().add_(0.01)
    for r, i, below in ((2, 100, 30), (2, 101, 45), (3, 40, 60), (3, 2400, 100)):
        at = place(r, i)
        for h in range(kv):
            mean = _f64(q)[r, h * (heads // kv)].sum() * dim ** -0.5
            cache.k[(*at, h)] = -below * math.log(2) / mean
        v[(*at, slice(None), 8 + i % 7)] = math.inf
    if wide:
        table = torch.cat([table, torch.full((len(lengths), 3000), -1, dtype=torch.int32)], 1)
    got = dev.cache_attend(cache, q, table.cuda(), length.cuda())
    want = _expect(cache, q, table, length, dim ** -0.5)
    assert np.isposinf(want[0][:, :, 1]).all() and np.isnan(want[0][1:, :, 4]).all() and np.isfinite(want[0][:, :, 20]).all()
    _check_with_infinities(got, want, q, max(lengths))


def test_values_that_became_infinite_in_the_store(dev):
    """32-bit values beyond fp16's largest are infinite in the cache, and in what is read from it."""
    k, v = (torch.zeros((2, 16, 1, 64), dtype=F16, device="cuda") for _ in range(2))
    cache = dev.PagedCache(k, v)
    new = torch.zeros((3, 1, 64), device="cuda")
    new[1, 0, 5], new[2, 0, 7] = 1e6, -7e4
    dev.cache_append(cache, torch.zeros_like(new), new, torch.arange(3, device="cuda"))
    q = torch.ones((1, 2, 64), dtype=F16, device="cuda")
    out, lse = dev.cache_attend(cache, q, torch.tensor([[0]], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"))
    want = torch.zeros((1, 2, 64), device="cuda")
    want[..., 5], want[..., 7] = math.inf, -math.inf
    assert torch.equal(out.float(), want)


def test_scales_at_the_ends(dev):
    """What is stored in an 8-bit cache is the value over its head's scale whatever that is: an infinite one, the smallest and the largest normal numbers, 0."""
    scale = torch.tensor([math.inf, 2.0 ** -126, 2.0 ** 127, 0.0, -math.inf, 0.5], dtype=F32, device="cuda")
    x = torch.tensor([0.0, 1.0, -3.5, 448.0, 2.0 ** -126, 2.0 ** 127, 3e38, math.inf, -math.inf, math.nan, 1e-3, -2.0 ** 120, 5.0, 6.0, 7.0, 2.0 ** 125], dtype=F32, device="cuda")
    k, v = (torch.zeros((1, 1, 6, 16), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    rows = x.expand(1, 6, 16).contiguous()
    dev.cache_append(dev.PagedCache(k, v, scale, scale), rows, rows, torch.zeros(1, dtype=torch.int64, device="cuda"))
    want = (rows.double() / scale.double()[:, None]).clamp(-448, 448)[0].cpu()   # (every quotient is a number of the type or far from a tie, or none)
    got = k[0, 0].cpu()
    assert torch.equal(got.view(torch.uint8), v[0, 0].cpu().view(torch.uint8)) and torch.equal(got.float().isnan(), want.isnan())
    assert torch.equal(got.float().nan_to_num(0), want.to(torch.float8_e4m3fn).float().nan_to_num(0))


# ---- the bits of an angle

@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_where_a_sine_is_small(dev, interleaved):
    """Angles next to whole quarters of a turn: what is left of them is small, and has to have the bits that the 64-bit angle has, not those of a fraction of
    a turn in 32.  Sine and cosine at most 4 units of 2^-23 off (what OpenCL allows sinpi and cospi), the rest of the angle added by a product and a sum, the pair's
    products by 0 and 1 exact: under 16 * 2^-24 of the value, and 2^-39 for 1600 radians in 64 bits (3 roundings of 2^-53 of them)."""
    pairs, position = 512, 1000
    quarters = torch.arange(pairs, dtype=torch.float64) * (math.pi / 2) / position
    rope = dev.Rope(quarters.float().cuda(), None, interleaved)
    x = torch.zeros((1, 2, 2 * pairs), dtype=F32, device="cuda")
    first, second = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :pairs], x[..., pairs:])
    first[:, 0], second[:, 1] = 1, 1
    got = _f64(dev.rotary(x, rope, torch.tensor([position], dtype=torch.int32, device="cuda")))
    angle = position * quarters.float().double().numpy()
    c, s = np.cos(angle), np.sin(angle)
    want = np.zeros((1, 2, 2 * pairs))
    a, b = (want[..., 0::2], want[..., 1::2]) if interleaved else (want[..., :pairs], want[..., pairs:])
    a[0, 0], b[0, 0], a[0, 1], b[0, 1] = c, s, -s, c
    _close(got, want, 16 * 2.0 ** -24 * np.abs(want) + 2.0 ** -39)
