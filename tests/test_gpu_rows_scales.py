"""Products of scales at the ends of 32 bits in a product of rows in 8 bits: what the header says of them.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from oracle import rows as oracle
from tests.test_gpu_cache import BF16, E4M3, F32, HALF_STEP, SMALLEST, _f64
from tests.test_gpu_rows import U, _operands

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


# (one for each kernel: few rows, tiles, tiles of 256)
SIZES = [(7, 200, 400), (90, 600, 272), (389, 1003, 528), (2100, 4200, 144)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m, n, k", SIZES)
def test_small_products_of_scales(dev, m, n, k, dtype):
    """Rows whose scales' products are 2^-60, 2^-125, and, below what 32 bits hold whole, 2^-130 and 2^-140 (to 2^-150 each) and 2^-160 (nothing)."""
    a, sa, w, sw = _operands(m, m, n, k)
    powers = np.array([0, -65, -70, -80, -100])[np.arange(m) % 5]
    sa, sw = sa * torch.from_numpy(2.0 ** powers).float()[:, None], sw * 2.0 ** -60
    got = _f64(dev.gemm_scaled(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), dtype=dtype))
    want, mass = oracle.product(_f64(a), _f64(sa), _f64(w), _f64(sw))
    blocks = np.abs(_f64(a)).sum(1)[:, None] * 448   # (of at least the size of all blocks' sums together)
    off = (260 + sa.shape[1]) * U * mass + 2.0 ** -150 * blocks + sa.shape[1] * SMALLEST[F32]
    if dtype != F32:
        off += 7 * 2.0 ** -13 * oracle.largest_products(_f64(a), _f64(sa), _f64(w), _f64(sw), 8)
    assert (np.abs(got - want) <= HALF_STEP[dtype] * (np.abs(want) + off) + off + SMALLEST[dtype]).all()
    assert (got[powers == -100] == 0).all() and (got[powers == -65] != 0).mean() > 0.9 and (got[powers == -70] != 0).mean() > 0.9


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m, n, k", SIZES)
def test_large_products_of_scales(dev, m, n, k, dtype):
    """Up to 3.4e38 as any other; past it infinite, a block's sum of 0 NaN."""
    g = torch.Generator().manual_seed(k)
    a, w = ((torch.randint(0, 2, s, generator=g) * 2 - 1).float().mul(2.0 ** -9).to(E4M3) for s in ((m, k), (n, k)))
    across, down = -(-k // 128), -(-n // 128)
    sa, sw = torch.full((m, across), 2.0 ** 67), torch.full((down, across), 2.0 ** 60)
    sa[m // 2:] = 2.0 ** 68
    w.view(torch.uint8)[3] = 0
    got = _f64(dev.gemm_scaled(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), dtype=dtype))
    want, _ = oracle.product(_f64(a), _f64(sa), _f64(w), _f64(sw))   # (whole numbers of 2^109: exact)
    top = m // 2
    assert np.array_equal(got[:top], _f64(torch.from_numpy(want[:top]).to(dtype))) and (got[:top, 3] == 0).all()
    assert not np.isfinite(got[top:]).any() and np.isnan(got[top:, 3]).all()
