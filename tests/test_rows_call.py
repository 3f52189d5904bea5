"""The native way from a Python call to the operators on a layer's rows: what it does not take, and that it gives what the way through ctypes gives."""
import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
NATIVE = ("norm", "norm_grad", "quantize", "gemm_scaled")


def test_calls_that_are_not_taken():
    """Tensors that are not on the GPU, other types, ranks and objects, no arguments: none reaches the library, none raises."""
    x, w, e, s = torch.zeros((4, 64), dtype=BF16), torch.zeros(64, dtype=BF16), torch.zeros((4, 64), dtype=E4M3), torch.zeros((4, 1))
    calls = device._native
    for a in ((), (None,) * 9, (x, w, 1e-6, None, False, None, None, None, None), (x, w, 1, None, False, None, None, None, None), (1, w, 1e-6, x, True, x, s, x, 0)):
        assert calls.norm(*a) is None
    for a in ((), (None,) * 9, (x, w, x, 1e-6, None, None, None, None, None), ("x",) * 9):
        assert calls.norm_grad(*a) is None
    for a in ((), (None,) * 6, (x, None, 1, None, None, None), (x, x, 1 << 70, None, None, 0)):
        assert calls.quantize(*a) is None
    for a in ((), (None,) * 7, (e, s, e, s, BF16, None, None), (e, s, e, s, "bf16", x, 0)):
        assert calls.gemm_scaled(*a) is None
    for a in ((), (1,) * 7, (1, 2, 3, 4, 5, int, tuple)):
        with pytest.raises(TypeError):
            calls.rows_library(*a)


def test_without_the_extension():
    for name in NATIVE:
        assert getattr(device._NoCalls, name)(1, 2) is None


def _same(a, b):
    if a is None or b is None:
        return a is b
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride() and torch.equal(a.view(raw) if a.element_size() > 1 else a.view(raw), b.view(raw))


@pytest.mark.gpu
def test_it_gives_what_the_other_way_gives(monkeypatch):
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s, dtype=BF16: torch.randn(s, device="cuda", generator=g).to(dtype)  # noqa: E731
    x, r, w, h = rand(37, 300), rand(37, 300), rand(300), rand(5, 3, 64)
    q, p = device.quantize(rand(37, 320)), device.quantize(rand(200, 320), tall=128)
    kept = dict(out=torch.empty((37, 300), dtype=E4M3, device="cuda"), scale=torch.empty((37, 3), device="cuda"), total=torch.empty_like(x))
    work = torch.empty(device.norm_grad_workspace(x), dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    calls = [
        lambda: device.norm(x, w), lambda: device.norm(x, w.float(), 1e-3, eight=True), lambda: device.norm(x, w, residual=r), lambda: device.norm(h, w[:64].contiguous()),
        lambda: device.norm(x, w, residual=r, eight=True), lambda: device.norm(x, w, residual=r, eight=True, stream=s, **kept), lambda: device.norm(x[:0], w, residual=r[:0], eight=True),
        lambda: device.norm(x, w, stream=s), lambda: device.norm(x, w, eight=True, out=kept["out"]),
        lambda: device.norm_grad(x, w, r), lambda: device.norm_grad(h, w[:64].contiguous(), h, extra=h), lambda: device.norm_grad(x, w, r, workspace=work),
        lambda: device.norm_grad(x, w, r, 1e-5, x, torch.empty_like(x), torch.empty(300, device="cuda"), work, s), lambda: device.norm_grad(x[:0], w, r[:0]),
        lambda: device.quantize(x), lambda: device.quantize(x, tall=128), lambda: device.quantize(x, gate=r), lambda: device.quantize(x, out=kept["out"], scale=kept["scale"], stream=s),
        lambda: device.quantize(x[:, :0]), lambda: device.quantize(x[:0]),
        lambda: (device.gemm_scaled(*q, *p),), lambda: (device.gemm_scaled(*q, *p, torch.float32),), lambda: (device.gemm_scaled(*q, *p, out=torch.empty((37, 200), device="cuda"), stream=s),),
        lambda: (device.gemm_scaled(q.out[:0], q.scale[:0], *p),),
    ]
    taken = []
    for name in NATIVE:
        f = getattr(device._native, name)
        monkeypatch.setattr(device, "_native_" + name, lambda *a, f=f: taken.append(f(*a)) or taken[-1])
    first = [[None if t is None else t.clone() for t in c()] for c in calls]
    types = [type(c()) for c in calls]
    assert sum(t is None for t in taken) <= 6   # (a stream of its own without outputs, one of two outputs: the other way)
    for name in NATIVE:
        monkeypatch.setattr(device, "_native_" + name, lambda *a: None)
    for c, want, kind in zip(calls, first, types):
        got = c()
        assert type(got) is kind and len(got) == len(want)
        for a, b in zip(got, want):
            assert (a is None and b is None) or _same(a, b.as_strided(a.shape, a.stride()) if b.stride() != a.stride() and a.shape == b.shape and b.numel() == 0 else b)


@pytest.mark.gpu
def test_refusals_and_gradients_of_the_native_way():
    x, w = torch.zeros((4, 64), dtype=BF16, device="cuda", requires_grad=True), torch.ones(64, dtype=BF16, device="cuda")
    y = device.norm(x, w, residual=x)
    assert not y.out.requires_grad and not y.total.requires_grad and not device.quantize(x).scale.requires_grad
    e, s = device.quantize(x)
    for call, status, say in ((lambda: device.norm(x, w, out=x.detach()[:, 1:]), B.AMAP_E_SHAPE, ""), (lambda: device.norm(x, w, 0.0), B.AMAP_E_INVALID, ""),
                              (lambda: device.norm(x, w[:7]), B.AMAP_E_SHAPE, "7"), (lambda: device.quantize(x, tall=3), B.AMAP_E_UNSUPPORTED, "3"),
                              (lambda: device.gemm_scaled(e[:, :40], s, e[:, :40], s), B.AMAP_E_SHAPE, ""), (lambda: device.gemm_scaled(e[:, :40], s, e[:, :40], s[:1]), B.AMAP_E_UNSUPPORTED, "16"),
                              (lambda: device.gemm_scaled(e, s, e, s[:1], dtype=torch.float64), B.AMAP_E_INVALID, ""), (lambda: device.norm(x.t(), w), B.AMAP_E_UNSUPPORTED, "contiguous"),
                              (lambda: device.norm(x.expand(1, 4, 64).permute(0, 2, 1), w[:4]), B.AMAP_E_UNSUPPORTED, "contiguous")):
        with pytest.raises(B.AmapError) as err:
            call()
        assert err.value.status == status and say in str(err.value), str(err.value)
