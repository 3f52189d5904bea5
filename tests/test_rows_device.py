"""Rows on one device and a stream of another: refused."""
import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device
from tests.test_cache_args import _refuses


class On:
    """A tensor as far as its device goes."""

    def __init__(self, at):
        self.at = at

    def get_device(self):
        return self.at


def test_streams_of_the_current_device(monkeypatch):
    """The current stream and the null stream are the current device's; whose another one is the library finds out."""
    monkeypatch.setattr(device, "_get_device", lambda: 0)
    for stream in (None, 0, 1 << 20):
        device._one_device("amap_norm", stream, On(0), None, On(0))
        _refuses(B.AMAP_E_INVALID, device._one_device, "amap_norm", stream, On(0), On(1))
    for stream in (None, 0):
        assert "cuda:1" in _refuses(B.AMAP_E_INVALID, device._one_device, "amap_norm", stream, On(1), On(1))
    device._one_device("amap_norm", 1 << 20, On(1), On(1))


@pytest.mark.gpu
def test_the_native_way_asks_whose_the_null_stream_is():
    """Told that another device is current, it takes no call on the null stream, and goes on taking those of a stream that is named."""
    x, w = torch.ones((4, 128), dtype=torch.bfloat16, device="cuda"), torch.ones(128, dtype=torch.bfloat16, device="cuda")
    out, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(128, device="cuda")
    e, f = device.quantize(x), device.quantize(x, tall=128)
    y = torch.empty((4, 4), dtype=torch.bfloat16, device="cuda")
    room, named = torch.empty(16, dtype=torch.uint8, device="cuda"), torch.cuda.Stream().cuda_stream
    torch.cuda.synchronize()
    calls = [lambda s: device._native.norm(x, w, 1e-6, None, False, out, None, None, s), lambda s: device._native.norm_grad(x, w, x, 1e-6, None, dx, dw, room, s),
             lambda s: device._native.quantize(x, None, 1, e.out, e.scale, s), lambda s: device._native.gemm_scaled(e.out, e.scale, f.out, f.scale, torch.bfloat16, y, s)]

    def told(current):
        device._native.library(*(B.C.cast(getattr(B._L, name), B.C.c_void_p).value for name in ("amap_cache_assign", "amap_rotary", "amap_cache_append", "amap_cache_attend",
                                                                                               "amap_cache_attend_workspace")),
                               device.Assigned, device._raw_stream, current, torch.cuda.is_initialized, device._capturing)

    assert all(c(s) is not None for c in calls for s in (0, named))
    try:
        told(lambda: torch.cuda.current_device() + 1)
        assert all(c(0) is None and c(named) is not None for c in calls)
    finally:
        told(device._get_device)
    assert all(c(0) is not None for c in calls)
    torch.cuda.synchronize()
