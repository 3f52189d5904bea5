"""Elements in 8 bits are their quotient in 32 bits rounded to nearest even: the same bits as a division gives, at ties as well.  Needs an MI355X (-m gpu)."""
import pytest
import torch

from tests.test_gpu_cache import BF16, E4M3, F16, F32
from tests.test_gpu_rows import _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


def _divided(y, tall):
    """y [rows, columns], 32 bits: its elements and scales by divisions in 32 bits (on the CPU), and how many quotients of 32 bits are ties."""
    rows, columns = y.shape
    down, across = -(-rows // tall), -(-columns // 128)
    blocks = torch.nn.functional.pad(y, (0, across * 128 - columns, 0, down * tall - rows)).view(down, tall, across, 128)
    scale = (blocks.abs().amax((1, 3)) / 448).clamp(min=2.0 ** -126)
    quotient = (blocks / scale[:, None, :, None]).view(down * tall, across * 128)[:rows, :columns]
    step = torch.exp2(torch.floor(torch.log2(quotient.double().abs().clamp(min=2.0 ** -6))) - 3)
    return quotient.to(E4M3), scale, int(((quotient.double() / step) % 1 == 0.5).sum())


def _same_bits(got, y, tall, least_ties=0):
    q, scale, ties = _divided(y, tall)
    assert ties >= least_ties
    assert torch.equal(got.scale.cpu(), scale)
    assert torch.equal(got.out.cpu().view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("tall", [1, 128])
@pytest.mark.parametrize("dtype, rows, columns", [(BF16, 64, 2560), (BF16, 700, 1000), (F16, 300, 1288), (F32, 200, 1001), (BF16, 9000, 4160)])
def test_rows_of_16_bits_meet_ties(dev, dtype, rows, columns, tall):
    x = _rand(rows, (rows, columns), dtype)
    _same_bits(dev.quantize(x.cuda(), tall=tall), x.float(), tall, 0 if dtype == F32 else 10)


@pytest.mark.parametrize("power", [-149, -140, -126, -110, -100, -92, -80, -66, -65, -64, -63, -30, 60, 119])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scales_of_every_size(dev, dtype, power):
    """Down to blocks whose scale is the least one, and up to the largest."""
    x = (_rand(7, (64, 640), F32).clamp(-6, 6).double() * 2.0 ** (power + 6)).to(dtype)
    for tall in (1, 128):
        _same_bits(dev.quantize(x.cuda(), tall=tall), x.float(), tall)


@pytest.mark.parametrize("most", [1.0, 1.0078125, 1.296875, 1.3125, 1.75, 1.984375])
def test_every_number_of_16_bits_over_one_scale(dev, most):
    """All bf16 numbers up to `most` and down to zero, of both signs, in blocks that all hold `most`."""
    bits = torch.arange(1 << 15, dtype=torch.int32).to(torch.int16).view(BF16)
    x = bits[bits.float() <= most]
    x = torch.cat([x, -x])
    x = torch.nn.functional.pad(x.float(), (0, -x.numel() % 126)).view(-1, 126)
    x = torch.cat([x, torch.tensor([most, -0.0]).expand(x.shape[0], 2)], 1).to(BF16)
    _same_bits(dev.quantize(x.cuda()), x.float(), 1)


@pytest.mark.parametrize("dtype, tokens, dim", [(BF16, 5, 4096), (F16, 40, 256), (F32, 9, 1024), (BF16, 6000, 128), (BF16, 3000, 2048)])
def test_norm_into_8_bits(dev, dtype, tokens, dim):
    """Rows of 1 and -1 and an eps of 3: the norm is half the weight, to the bit."""
    x = torch.where(_rand(1, (tokens, dim), F32) < 0, -1.0, 1.0).to(dtype)
    w = _rand(2, (dim,), dtype)
    _same_bits(dev.norm(x.cuda(), w.cuda(), 3.0, eight=True), 0.5 * x.float() * w.float(), 1)


def test_behind_a_gate(dev):
    """Large gates: silu(gate) is the gate, to the bit."""
    gate, x = (100.0 + torch.arange(64 * 512).view(64, 512) % 100).to(BF16), _rand(3, (64, 512), F32).to(BF16)
    _same_bits(dev.quantize(x.cuda(), gate=gate.cuda()), x.float() * gate.float(), 1, 1)


@pytest.mark.parametrize("tall", [1, 128])
def test_scales_whose_reciprocal_is_hard_to_round(dev, tall):
    """Scales of all ones and others that a step of Newton's gets wrong: numbers around the ties of 8 bits over each."""
    scale = torch.tensor([0x3FFFFFFF, 0x3F869913, 0x3F87CC45, 0x3F8EFA43, 0x3FC23DC3, 0x3FD0DD0D, 0x3FEE4BC5], dtype=torch.int32).view(F32)
    q = torch.cat([torch.arange(2 ** -6, 2 ** -5, 2 ** -10), torch.arange(8, 16, 0.25), torch.arange(256, 448, 8)]).to(F32)
    rows = []
    for s in scale:
        x = torch.cat([q * s, torch.nextafter(q * s, torch.tensor(0.0)), torch.nextafter(q * s, torch.tensor(1e9))])
        x = torch.nn.functional.pad(x, (0, -x.numel() % 127)).view(-1, 127)
        most = next(m for m in (torch.nextafter(448 * s, torch.tensor(0.0)), 448 * s, torch.nextafter(448 * s, torch.tensor(1e9))) if m / 448 == s)
        x = torch.cat([x.clamp(max=float(most)), most.expand(x.shape[0], 1)], 1)
        rows.append(x if tall == 1 else torch.nn.functional.pad(x, (0, 0, 0, 128 - x.shape[0])))
    x = torch.cat(rows)
    assert set(scale.tolist()) == set(_divided(x, tall)[1].unique().tolist())
    for power in (0, -90):
        _same_bits(dev.quantize((x * 2.0 ** power).cuda(), tall=tall), x * 2.0 ** power, tall, 1)
