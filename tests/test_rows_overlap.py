"""Rows in 8 bits whose tensors lie between one another's rows: taken where they share no element, as rows with their scales behind them, refused where they do."""
import os
import subprocess

import pytest
import torch

from paper_2002_12798_amd import binding as B
from tests.test_cache_args import AT, _refuses

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, U = B.AMAP_E_ALIAS, B.AMAP_E_UNSUPPORTED
E4, BF16 = B.AMAP_E4M3, B.AMAP_BF16


def test_whether_runs_share_a_byte(tmp_path):
    """The host's answer against every byte, built with the host's compiler."""
    exe = str(tmp_path / "rows_overlap_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2002_12798_amd", "csrc"), os.path.join(ROOT, "tests", "rows_overlap_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


# a buffer of 10 rows of 1024 bytes: 200 columns in 8 bits, their two scales, the same columns in 16 bits, a product.  Where all are apart, the
# refusal is that of x (a weight) which begins between two elements: it comes after those of overlaps.
PITCH = 1024


@pytest.mark.parametrize("out, scale, x, status", [
    (0, 200, 300, U), (8, 0, 300, U), (402, 604, 0, U), (824, 816, 4, U), (0, 200, 208, U),
    (0, 196, 300, A), (0, 200, 206, A), (101, 304, 300, A), (0, 1020, 300, A), (1000, 600, 100, A), (300, 0, 299, A), (200, 0, 399, A),
])
def test_rows_with_their_scales(out, scale, x, status):
    at = 5 * AT
    q, s = B.amap_rows(at + out, E4, PITCH), B.amap_scales(at + scale, PITCH // 4, 1)
    odd = x + 1 - x % 2   # (a place between two elements)
    _refuses(status, B.amap_quantize, B.amap_rows(at + odd, BF16, PITCH // 2), None, 10, 200, 1, q, s)
    heads = lambda t, type, es: B.amap_heads(at + t, type, 1, PITCH // es, 3)  # noqa: E731
    _refuses(status, B.amap_norm, heads(odd, BF16, 2), None, 10, 200, AT, BF16, 1e-6, None, heads(out, E4, 1), s)
    _refuses(status, B.amap_norm, B.amap_heads(9 * AT + 1, BF16, 1, 256, 0), heads(odd, BF16, 2), 10, 200, AT, BF16, 1e-6, None, heads(out, E4, 1), s)
    if x % 2 == 0:
        _refuses(status, B.amap_norm, B.amap_heads(9 * AT + 1, BF16, 1, 256, 0), B.amap_heads(8 * AT, BF16, 1, 256, 0), 10, 200, AT, BF16, 1e-6, heads(x, BF16, 2), heads(out, E4, 1), s)


@pytest.mark.parametrize("out, status", [(256, U), (512, U), (767, U), (199, A), (824, A), (7, A), (0, A)])
def test_a_product_beside_its_operand(out, status):
    """10 rows of 192 k and their two scales at 192 and 196 (w's 100 rows and scales elsewhere), 100 columns of 16 bits behind them."""
    at = 5 * AT
    a, s, y = B.amap_rows(at, E4, PITCH), B.amap_scales(at + 192, PITCH // 4, 1), B.amap_rows(at + out + 1 - out % 2, BF16, PITCH // 2)
    w, t = B.amap_rows(2 * AT, E4, 192), B.amap_scales(AT, 2, 1)
    _refuses(status, B.amap_gemm_scaled, a, s, w, t, 10, 100, 192, y)


@pytest.mark.gpu
def test_rows_and_scales_in_one_buffer():
    """The same bits as in tensors of their own, and nothing else of the buffer changes."""
    from paper_2002_12798_amd import device
    g = torch.Generator(device="cuda").manual_seed(1)
    for rows, columns in ((1, 128), (37, 96), (300, 336), (4500, 4096)):
        x, w = torch.randn((rows, columns), device="cuda", generator=g).bfloat16(), torch.randn(columns, device="cuda", generator=g).bfloat16()
        blocks, at = -(-columns // 128), columns + 16
        pitch = at + 4 * blocks + 16 - 4 * blocks % 16 + 2 * columns + 32
        room = torch.full((rows, pitch), 0x5A, dtype=torch.uint8, device="cuda")
        out, scale = room[:, :columns].view(torch.float8_e4m3fn), room[:, at:at + 4 * blocks].view(torch.float32)
        total = room[:, pitch - 2 * columns - 16:pitch - 16].view(torch.bfloat16)
        for call, more in ((lambda **k: device.quantize(x, **k), {}), (lambda **k: device.quantize(x, gate=x, **k), {}), (lambda **k: device.norm(x, w, eight=True, **k), {}),
                           (lambda **k: device.norm(x, w, residual=x, eight=True, **k), dict(total=total))):
            want, got = call(), call(out=out, scale=scale, **more)
            assert got.out is out and torch.equal(out.view(torch.uint8), want.out.view(torch.uint8)) and torch.equal(scale, want.scale)
            if more:
                assert torch.equal(total, want.total)
        used = torch.zeros(pitch, dtype=torch.bool)
        used[:columns] = used[at:at + 4 * blocks] = used[pitch - 2 * columns - 16:pitch - 16] = True
        assert (room[:, ~used.cuda()] == 0x5A).all()
        if columns % 16 == 0:
            v = device.quantize(torch.randn((200, columns), device="cuda", generator=g).bfloat16(), tall=128)
            y = device.quantize(x, out=out, scale=scale)
            assert torch.equal(device.gemm_scaled(y.out, y.scale, v.out, v.scale), device.gemm_scaled(out.contiguous(), scale.contiguous(), v.out, v.scale))
