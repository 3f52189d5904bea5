"""The norm's gradient where sums are long, and where rows hold what 32 bits do not.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from oracle import rows as oracle
from tests.test_gpu_cache import BF16, F16, F32, HALF_STEP, SMALLEST, _close, _f64
from tests.test_gpu_rows import EPS, U, _check_grad, _rand, _rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


# (each a way that rows are held by lanes, and several rows to a workgroup: a last turn that some of its groups have no row in, parts to join)
MANY = [(F32, 1531, 0, 1001), (BF16, 5000, 0, 4096), (BF16, 12800, 0, 4096), (F32, 9000, 0, 4096), (BF16, 700, 40, 128), (BF16, 3000, 5, 40), (F16, 20001, 0, 200), (BF16, 40000, 0, 96),
        (F32, 3001, 0, 20001), (BF16, 2500, 0, 32768), (BF16, 33, 0, 128), (F16, 517, 0, 9000)]


def _shape(tokens, heads, dim):
    return (tokens, heads, dim) if heads else (tokens, dim)


@pytest.mark.parametrize("dtype, tokens, heads, dim", MANY)
def test_every_row_counts_once(dev, dtype, tokens, heads, dim):
    """Rows of 1 and -1 and an eps of 3: r is 1/2, and every sum a whole number of halves below 2^23.  A row lost or counted twice shows in every column."""
    rows = tokens * max(1, heads)
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = torch.where(torch.rand(_shape(tokens, heads, dim), device="cuda", generator=g) < 0.5, -1.0, 1.0).to(dtype)
    grad = torch.randint(-3, 8, (rows, 1), device="cuda", generator=g).to(dtype).expand(rows, dim).reshape(x.shape)
    dx, dw = dev.norm_grad(x, torch.ones(dim, dtype=dtype, device="cuda"), grad * x, 3.0)
    want = 0.5 * grad.reshape(rows, dim)[:, 0].double().sum()
    assert (dw.double() == want).all()
    # dx = r (grad x - x r^2 (grad dim) / dim) = x grad 3 / 8; 1 / dim is off by half a step, c / dim by a whole one
    off = 3 * U * 0.5 * grad.double().abs()
    exact = 0.375 * (grad * x).double()
    assert ((dx.double() - exact).abs() <= HALF_STEP[dtype] * (exact.abs() + off) + off).all()


@pytest.mark.parametrize("dtype, tokens, heads, dim", MANY)
def test_one_row_at_a_time(dev, dtype, tokens, heads, dim):
    """A gradient in one row alone, the first and last ones and some between: its own term, and rows of zeros elsewhere."""
    rows = tokens * max(1, heads)
    x = _rows_of(1, rows, dim, dtype)
    w = _rand(2, (dim,), dtype).cuda()
    mine = _rand(3, (1, dim), dtype, 0.1)
    for at in sorted({0, 1, rows // 2, rows * 2 // 3 + 1, rows - 16, rows - 2, rows - 1}):
        grad = torch.zeros((rows, dim), dtype=dtype, device="cuda")
        grad[at] = mine.cuda()[0]
        dx, dw = dev.norm_grad(x.view(_shape(tokens, heads, dim)), w, grad.view(_shape(tokens, heads, dim)), EPS)
        dx = dx.view(rows, dim)
        _check_grad((dx[at:at + 1], dw), x[at:at + 1].cpu(), w.cpu(), mine, EPS)
        dx[at] = 0
        assert not dx.any()


def test_rows_past_four_gigabytes(dev):
    """The last rows of 5.2 GB, a gradient in them alone and another weight than 1: what they are by themselves, their own terms the whole of the weight's gradient."""
    rows, dim, few = 160000, 16256, 50
    x = torch.empty((rows, dim), dtype=BF16, device="cuda").fill_(0.5)
    grad = torch.zeros((rows, dim), dtype=BF16, device="cuda")
    x[:few].normal_()
    x[-few:].normal_()
    grad[-few:].normal_()
    w = _rand(5, (dim,), BF16).cuda()
    last, its = x[-few:].clone(), grad[-few:].clone()
    dx, dw = dev.norm_grad(x, w, grad, EPS)
    _check_grad((dx[-few:], dw), last.cpu(), w.cpu(), its.cpu(), EPS)
    assert not dx[:-few].any()
    # in place, with what reaches the rows by other ways
    dx, again = dev.norm_grad(x, w, grad, EPS, extra=x, dx=grad)
    _check_grad((dx[-few:], again), last.cpu(), w.cpu(), its.cpu(), EPS, last.cpu())
    assert torch.equal(again, dw) and torch.equal(dx[:-few], x[:-few])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 300, 4096, 20000])
def test_rows_that_are_not_finite(dev, dim, dtype):
    """A row of zeros has a gradient; one whose squares pass 32 bits has none, and adds none to the weight's; an infinite element or a NaN makes its own row NaN, and of the weight's gradient its
    column (NaN in x: all of them).  Other rows are as ever."""
    x, g, w, e = (_rand(dim + i, (9, dim), dtype) for i in range(4))
    w = w[0].contiguous()
    x[2], x[4] = 0, x[4].double().clamp(-1, 1).to(dtype) * 1e25
    x[4, 0] = 1e25
    plain = [0, 1, 3, 5, 6, 7, 8]
    dx, dw = dev.norm_grad(x.cuda(), w.cuda(), g.cuda(), EPS, extra=e.cuda())
    assert torch.equal(dx[4].cpu(), e[4])
    rest = [i for i in range(9) if i != 4]
    _check_grad((dx[rest], dw), x[rest], w, g[rest], EPS, e[rest])
    for t, value, all_columns in ((x, float("inf"), False), (x, float("nan"), True), (g, float("inf"), False), (g, -float("inf"), False), (g, float("nan"), False)):
        a, b = x.clone(), g.clone()
        (a if t is x else b)[6, 5] = value
        one = dev.norm_grad(a.cuda(), w.cuda(), b.cuda(), EPS, extra=e.cuda())
        assert one[0][6].isnan().any() and not one[0][6].isfinite().all()
        assert torch.equal(one[0][plain[:4]], dx[plain[:4]]) and torch.equal(one[0][7:], dx[7:])
        assert one[1].isnan().all() if all_columns else not one[1][5].isfinite()
        if not all_columns:
            finite = torch.arange(dim) != 5
            assert one[1].cpu()[finite].isfinite().all()


@pytest.mark.parametrize("dim", [64, 1001, 17000])
def test_large_gradients_beside_large_rows(dev, dim):
    """grad h passes 32 bits, grad h r does not: the weight's gradient has it."""
    x, g, w = _rand(1, (5, dim), F32), _rand(2, (5, dim), F32, 1e-3), _rand(3, (dim,), F32)
    x[1] *= 1e14
    g[1, 7], w[7] = 1e30, 0   # (a weight of 0: nothing of it goes to the row)
    got = dev.norm_grad(x.cuda(), w.cuda(), g.cuda(), EPS)
    assert got[1].isfinite().all()
    _check_grad(got, x, w, g, EPS)


@pytest.mark.parametrize("eps", [1e-12, 1e-30, 1e-38, 2e-39, 1e-44])
@pytest.mark.parametrize("dim", [64, 1001, 17000])
def test_rows_of_zeros_and_a_small_eps(dev, dim, eps):
    """1 / eps may pass 32 bits where 1 / sqrt(eps) does not: dx = grad weight / sqrt(eps).  (eps is one of 32 bits.)"""
    eps = float(np.float32(eps))
    g, w = _rand(2, (5, dim), F32, 1e-3), _rand(3, (dim,), F32)
    dx, dw = dev.norm_grad(torch.zeros((5, dim), device="cuda"), w.cuda(), g.cuda(), eps)
    want = _f64(g) * _f64(w) / np.sqrt(eps)
    _close(_f64(dx), want, 4 * U * np.abs(want) + SMALLEST[F32])
    assert (dw == 0).all()
