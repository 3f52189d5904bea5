"""Gates at the ends of their type's range in front of rows in 8 bits, against the formula in 64 bits.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from oracle import rows as oracle
from tests.test_gpu_cache import BF16, F16, F32, _f64
from tests.test_gpu_rows import U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


def _most(dtype):
    return torch.finfo(dtype).max


def _gates(dtype):
    ends = [-60.0, -69.0, -69.5, -80.0, -87.0, -87.5, -88.0, -95.0, -100.0, -110.0, -150.0, -180.0, -190.0, -250.0, -399.5, -400.5, -1000.0, 40.0, 88.0, 1000.0]
    far = [] if dtype == F16 else [-1e30, -2.3e38, -2.4e38, -3e38, 2.4e38, 3e38]
    return ends + far + [_most(dtype), -_most(dtype)]


def _check(dev, x, gate):
    """The exponential's argument, its power of two, sum, reciprocal and products take 17 u of a value at most.  Where what leads to it lies below 2^-126 each of three steps rounds to whole
    2^-149, times a gate of at most 400 behind them: 2^-139, or 2^-13 of the least scale."""
    got = dev.quantize(x.contiguous().cuda(), gate=gate.contiguous().cuda())
    with np.errstate(over="ignore"):
        y = oracle.gated(_f64(x), _f64(gate))
    assert (np.abs(y) <= 3.4e38).all()
    want, of = oracle.blocks(y, 1)
    t = y / of
    assert (np.abs(_f64(got.scale) - want) <= 17 * U * want).all()
    assert (np.abs(_f64(got.out) - t) <= (2.0 ** -4 * (1 + 36 * U) + 36 * U) * np.abs(t) + 2.0 ** -10 + 2.0 ** -13).all()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("size", [1.0, 1e-4, 1e4, 1e-30, 1e30, 3e38])
def test_gates_in_blocks_of_their_own(dev, size, dtype):
    """Every gate fills a row's first block by itself, so that the scale shows what becomes of it, and lies among ordinary ones in the second."""
    size = min(max(size, torch.finfo(dtype).tiny), _most(dtype))
    gates = _gates(dtype)
    g = torch.Generator().manual_seed(1)
    gate = torch.randn((len(gates), 256), generator=g, dtype=torch.float64)
    x = torch.randn((len(gates), 256), generator=g, dtype=torch.float64)
    x[:, :128] = size * (0.5 + 0.5 * torch.rand((len(gates), 128), generator=g, dtype=torch.float64))
    for i, v in enumerate(gates):
        gate[i, :128] = v
        gate[i, 130] = v
        if v > 1:   # (times such a gate a value of its own size has no place in 32 bits)
            x[i, :128] *= min(1.0, 1e38 / (v * size))
            x[i, 130] = min(1.0, 1e38 / v)
    _check(dev, x.to(dtype), gate.to(dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_no_larger_than_the_least_numbers(dev, dtype):
    """A gate of 2^-140 halves to what 32 bits hold less of; beside a large x the product is an ordinary number."""
    gate = torch.tensor([[2.0 ** -130], [2.0 ** -133], [-2.0 ** -132], [2.0 ** -127]], dtype=torch.float64).expand(4, 128).to(dtype)
    x = (torch.linspace(1.0, 1.9, 128, dtype=torch.float64) * 2.0 ** 126).expand(4, 128).to(dtype)
    _check(dev, x, gate)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_gates_that_are_infinite_or_nan(dev, dtype):
    """Each is NaN alone, and the others of its block are what they are without it."""
    g = torch.Generator().manual_seed(2)
    gate, x = (torch.randn((3, 300), generator=g).to(dtype) for _ in range(2))
    plain = dev.quantize(x.cuda(), gate=gate.cuda())
    at = torch.tensor([5, 131, 299])
    gate[0, at], gate[1, at], gate[2, at] = float("inf"), -float("inf"), float("nan")
    got = dev.quantize(x.cuda(), gate=gate.cuda())
    gate[:, at] = 0
    without = dev.quantize(x.cuda(), gate=gate.cuda())
    assert got.out[:, at].float().isnan().all() and torch.equal(got.scale, without.scale)
    rest = torch.ones(300, dtype=torch.bool)
    rest[at] = False
    assert torch.equal(got.out[:, rest].view(torch.uint8), without.out[:, rest].view(torch.uint8)) and not plain.out.float().isnan().any()


def test_a_mask_of_the_lowest_value(dev):
    """Gates of the type's lowest value: zeros that leave the rest of the row as it is, through the product that follows too."""
    g = torch.Generator().manual_seed(3)
    x, gate = torch.randn((5, 256), generator=g).to(BF16), torch.randn((5, 256), generator=g).to(BF16)
    hidden = torch.rand((5, 256), generator=g) < 0.3
    hidden[3] = True
    gate[hidden] = -_most(BF16)
    got = dev.quantize(x.cuda(), gate=gate.cuda())
    assert (got.out.float()[hidden.cuda()] == 0).all() and (got.scale[3] == 2.0 ** -126).all()
    w = dev.quantize(torch.randn((128, 256), generator=g).to(BF16).cuda(), tall=128)
    out = dev.gemm_scaled(got.out, got.scale, w.out, w.scale)
    assert out.isfinite().all() and (out[3] == 0).all() and (out[0] != 0).any()
