"""Types of rows that the Python calls take and refuse."""
import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device
from tests.test_cache_args import _refuses


@pytest.mark.parametrize("x", [torch.zeros((4, 64), dtype=torch.float64), torch.zeros((4, 64), dtype=torch.int32), torch.zeros(64), torch.zeros((2, 2, 2, 2)), None, [1.0]])
def test_a_workspace_for_what_is_no_row(x):
    assert "known type" in _refuses(B.AMAP_E_INVALID, device.norm_grad_workspace, x)


def test_a_workspace_for_rows_of_8_bits():
    _refuses(B.AMAP_E_INVALID, device.norm_grad_workspace, torch.zeros((4, 64), dtype=torch.float8_e4m3fn))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [("x",), ("w",), ("x", "w")])
def test_bf16_bits_in_16_bit_words(bits):
    """Rows or a weight as words of their bits: what the same call on bfloat16 gives."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r, w = torch.randn((37, 300), device="cuda", generator=g).bfloat16(), torch.randn((37, 300), device="cuda", generator=g).bfloat16(), torch.randn(300, device="cuda", generator=g).bfloat16()
    word = lambda t, name: t.view(torch.int16) if name in bits else t  # noqa: E731
    a, b, c = word(x, "x"), word(r, "x"), word(w, "w")
    same = lambda got, want: all(p.contiguous().view(torch.uint8).equal(q.contiguous().view(torch.uint8)) for p, q in zip(got, want) if q is not None)  # noqa: E731
    assert same(device.norm(a, c, residual=b), device.norm(x, w, residual=r)) and same(device.norm(a, c, eight=True), device.norm(x, w, eight=True))
    assert device.norm(a, c).out.dtype == a.dtype and same(device.norm_grad(a, c, b), device.norm_grad(x, w, r)) and same(device.quantize(a, gate=b), device.quantize(x, gate=r))
    assert same(device.norm(a, c.new_ones(300, dtype=torch.float32)), device.norm(x, w.new_ones(300, dtype=torch.float32)))


@pytest.mark.gpu
def test_weights_of_other_types():
    x = torch.ones((4, 64), dtype=torch.bfloat16, device="cuda")
    for dtype in (torch.float16, torch.float64, torch.int32, torch.float8_e4m3fn):
        _refuses(B.AMAP_E_INVALID, device.norm, x, torch.ones(64, device="cuda").to(dtype))
    _refuses(B.AMAP_E_INVALID, device.norm, x.half(), torch.ones(64, dtype=torch.int16, device="cuda"))
