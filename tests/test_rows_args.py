"""The entry points for a layer's rows in 8 bits refuse what does not fit before anything is launched (no GPU: the addresses are never read)."""
import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device
from tests.test_cache_args import AT, _refuses

I, S, U, A = B.AMAP_E_INVALID, B.AMAP_E_SHAPE, B.AMAP_E_UNSUPPORTED, B.AMAP_E_ALIAS


def _heads(at=AT, type=B.AMAP_BF16, heads=1, token=256, head=64):
    return B.amap_heads(at, type, heads, token, head)


def _rows(at=AT, type=B.AMAP_BF16, stride=256):
    return B.amap_rows(at, type, stride)


def _scales(at=9 * AT, row=1, block=64):
    return B.amap_scales(at, row, block)


def _norm(**over):
    c = dict(x=_heads(), residual=_heads(2 * AT), tokens=10, dim=200, weight=3 * AT, weight_type=B.AMAP_BF16, eps=1e-6, total=_heads(4 * AT), out=_heads(5 * AT), scale=None)
    c.update(over)
    B.amap_norm(*c.values())


E4 = B.AMAP_E4M3
EIGHT = dict(out=_heads(5 * AT, E4), scale=_scales())


@pytest.mark.parametrize("over, status", [
    (dict(x=_heads(None)), I), (dict(x=None), I), (dict(out=None), I), (dict(weight=None), I), (dict(residual=None), I), (dict(tokens=-1), I), (dict(dim=0), I),
    (dict(x=_heads(type=E4)), I), (dict(residual=_heads(2 * AT, B.AMAP_F16)), I), (dict(out=_heads(5 * AT, B.AMAP_F32)), I), (dict(weight_type=B.AMAP_F16), I),
    (dict(eps=0.0), I), (dict(eps=-1.0), I), (dict(eps=float("nan")), I), (dict(eps=float("inf")), I),
    (dict(scale=_scales()), I), (dict(out=_heads(5 * AT, E4)), I), ({**EIGHT, "scale": _scales(None)}, I),
    (dict(dim=32769, **{n: _heads(i * AT, token=1 << 20) for i, n in ((1, "x"), (2, "residual"), (4, "total"), (5, "out"))}), U),
    ({**EIGHT, **{n: _heads(i * AT, heads=2, token=512) for i, n in ((1, "x"), (2, "residual"), (4, "total"))}, "out": _heads(5 * AT, E4, 2)}, U),
    (dict(x=_heads(AT + 1)), U), (dict(weight=3 * AT + 1), U), ({**EIGHT, "scale": _scales(9 * AT + 2)}, U),
    (dict(tokens=1 << 31), S), (dict(residual=_heads(2 * AT, heads=2)), S), (dict(out=_heads(5 * AT, heads=2)), S), (dict(out=_heads(5 * AT, token=199)), S),
    (dict(total=_heads(4 * AT, token=100)), S), (dict(x=_heads(token=-256)), S), ({**EIGHT, "scale": _scales(row=1, block=5)}, S), ({**EIGHT, "scale": _scales(row=0, block=1)}, S),
    (dict(out=_heads(AT + 2)), A), (dict(out=_heads(AT, token=512)), A), (dict(total=_heads(5 * AT)), A), (dict(out=_heads(3 * AT)), A), (dict(total=_heads(3 * AT)), A),
    (dict(out=_heads(2 * AT + 400)), A), ({**EIGHT, "out": _heads(AT, E4)}, A), ({**EIGHT, "scale": _scales(AT)}, A), ({**EIGHT, "scale": _scales(2 * AT)}, A),
    ({**EIGHT, "scale": _scales(3 * AT)}, A), ({**EIGHT, "scale": _scales(4 * AT)}, A), ({**EIGHT, "scale": _scales(5 * AT)}, A),
])
def test_norm(over, status):
    _refuses(status, lambda: _norm(**over))


def _grad(**over):
    c = dict(x=_heads(), tokens=50, dim=200, weight=3 * AT, weight_type=B.AMAP_BF16, eps=1e-6, grad=_heads(2 * AT), extra=_heads(4 * AT), dx=_heads(5 * AT), dweight=6 * AT,
             workspace=7 * AT, bytes=1 << 20)
    c.update(over)
    B.amap_norm_grad(*c.values())


@pytest.mark.parametrize("over, status", [
    (dict(x=None), I), (dict(x=_heads(None)), I), (dict(grad=None), I), (dict(dx=None), I), (dict(dweight=None), I), (dict(weight=None), I), (dict(grad=_heads(2 * AT, B.AMAP_F32)), I),
    (dict(extra=_heads(4 * AT, B.AMAP_F16)), I), (dict(dx=_heads(5 * AT, E4)), I), (dict(eps=0.0), I), (dict(workspace=None), I), (dict(bytes=B.amap_norm_grad_workspace(1, 50, 200, B.AMAP_BF16) - 1), I),
    (dict(dim=40000), U), (dict(workspace=7 * AT + 8), U), (dict(dweight=6 * AT + 2), U), (dict(dx=_heads(5 * AT + 1)), U),
    (dict(dx=_heads(5 * AT, heads=2)), S), (dict(dx=_heads(5 * AT, token=128)), S), (dict(tokens=1 << 31), S),
    (dict(dx=_heads(AT + 2)), A), (dict(dx=_heads(2 * AT, token=512)), A), (dict(dx=_heads(4 * AT + 64)), A), (dict(dx=_heads(3 * AT)), A), (dict(dweight=3 * AT), A),
    (dict(dweight=AT), A), (dict(dweight=2 * AT), A), (dict(dweight=4 * AT), A), (dict(dweight=5 * AT), A), (dict(dweight=7 * AT + 400), A), (dict(workspace=AT), A),
    (dict(workspace=5 * AT), A), (dict(workspace=3 * AT), A),
])
def test_norm_grad(over, status):
    _refuses(status, lambda: _grad(**over))


def test_what_workspace_the_gradient_takes():
    """None for rows that one workgroup takes, a part for each workgroup else; as much for more rows, up to a bound."""
    room = B.amap_norm_grad_workspace
    assert room(1, 0, 4096, B.AMAP_BF16) == room(1, 1, 4096, B.AMAP_BF16) == room(1, 4, 4096, B.AMAP_BF16) == room(1, 32, 200, B.AMAP_BF16) == 0
    assert room(1, 6, 4095, B.AMAP_BF16) == 2 * 4096 * 4
    assert room(1, 10 ** 7, 4096, B.AMAP_BF16) == room(1, 10 ** 6, 4096, B.AMAP_BF16) <= 1024 * 4096 * 4
    for args, status in (((0, 1, 1, B.AMAP_BF16), I), ((1, -1, 1, B.AMAP_BF16), I), ((1, 1, 1, E4), I), ((1, 1, 32769, B.AMAP_F32), U), ((2, 1 << 30, 64, B.AMAP_F32), S)):
        _refuses(status, room, *args)


def _quantize(**over):
    c = dict(x=_rows(), gate=_rows(2 * AT), rows=10, columns=200, tall=1, out=_rows(3 * AT, E4), scale=_scales())
    c.update(over)
    B.amap_quantize(*c.values())


@pytest.mark.parametrize("over, status", [
    (dict(x=None), I), (dict(x=_rows(None)), I), (dict(out=None), I), (dict(out=_rows(None, E4)), I), (dict(scale=None), I), (dict(scale=_scales(None)), I), (dict(rows=-1), I),
    (dict(columns=-1), I), (dict(x=_rows(type=E4)), I), (dict(out=_rows(3 * AT)), I), (dict(gate=_rows(2 * AT, B.AMAP_F16)), I), (dict(gate=_rows(None)), I),
    (dict(tall=2), U), (dict(tall=128), U), (dict(x=_rows(AT + 1)), U), (dict(gate=_rows(2 * AT + 1)), U), (dict(scale=_scales(9 * AT + 1)), U),
    (dict(rows=1 << 31), S), (dict(columns=1 << 31), S), (dict(out=_rows(3 * AT, E4, 100)), S), (dict(x=_rows(stride=-256)), S), (dict(scale=_scales(block=3)), S),
    (dict(rows=(1 << 31) - 1, columns=1, gate=None, x=_rows(stride=1), out=_rows(3 * AT, E4, 1), scale=_scales(row=1)), U),
    (dict(out=_rows(AT, E4)), A), (dict(out=_rows(2 * AT, E4)), A), (dict(scale=_scales(AT)), A), (dict(scale=_scales(2 * AT)), A), (dict(scale=_scales(3 * AT)), A),
])
def test_quantize(over, status):
    _refuses(status, lambda: _quantize(**over))


def _gemm(**over):
    c = dict(a=_rows(AT, E4), a_scale=_scales(2 * AT), w=_rows(3 * AT, E4), w_scale=_scales(4 * AT), m=20, n=300, k=256, out=_rows(5 * AT, stride=300))
    c.update(over)
    B.amap_gemm_scaled(*c.values())


@pytest.mark.parametrize("over, status", [
    ({n: None}, I) for n in ("a", "a_scale", "w", "w_scale", "out")
] + [
    (dict(a=_rows(None, E4)), I), (dict(w=_rows(None, E4)), I), (dict(out=_rows(None)), I), (dict(a_scale=_scales(None)), I), (dict(w_scale=_scales(None)), I),
    (dict(a=_rows(AT)), I), (dict(w=_rows(3 * AT)), I), (dict(out=_rows(5 * AT, E4)), I), (dict(m=-1), I), (dict(n=-1), I), (dict(k=-16), I),
    (dict(k=0), U), (dict(k=200), U), (dict(a=_rows(AT + 8, E4)), U), (dict(w=_rows(3 * AT + 8, E4)), U), (dict(a=_rows(AT, E4, 264)), U), (dict(w=_rows(3 * AT, E4, 264)), U),
    (dict(out=_rows(5 * AT + 1, stride=300)), U), (dict(a_scale=_scales(2 * AT + 1)), U), (dict(w_scale=_scales(4 * AT + 1)), U),
    (dict(a=_rows(AT, E4, 1 << 24)), U), (dict(w=_rows(3 * AT, E4, 1 << 24)), U), (dict(a_scale=_scales(2 * AT, 1 << 24)), U),
    (dict(m=(1 << 31) - 1, n=1, out=_rows(5 * AT, stride=1)), U), (dict(m=1 << 31), S), (dict(out=_rows(5 * AT, stride=299)), S), (dict(a=_rows(AT, E4, -256)), S), (dict(w_scale=_scales(4 * AT, -1)), S),
    (dict(out=_rows(AT, stride=300)), A), (dict(out=_rows(3 * AT, stride=300)), A), (dict(out=_rows(2 * AT, stride=300)), A), (dict(out=_rows(4 * AT, stride=300)), A),
])
def test_gemm_scaled(over, status):
    _refuses(status, lambda: _gemm(**over))


def test_nothing_to_do_is_no_call():
    _norm(tokens=0, x=_heads(None))
    _quantize(rows=0, x=_rows(None))
    _quantize(columns=0)
    _gemm(m=0)
    _gemm(n=0)


def test_tensors_that_do_not_fit():
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    e, s = torch.zeros((4, 64), dtype=torch.float8_e4m3fn), torch.zeros((4, 1))
    for call in (lambda: device.norm(x, w), lambda: device.norm_grad(x, w, x), lambda: device.quantize(x), lambda: device.gemm_scaled(e, s, e, s[:1])):
        assert "not on the GPU" in _refuses(I, call)
    for call in (lambda: device.norm(x[0], w), lambda: device.norm(x.double(), w), lambda: device.norm([1.0], w), lambda: device.quantize(x[None]), lambda: device.quantize(None),
                 lambda: device.norm_grad(x.long(), w, x), lambda: device.gemm_scaled(x.double(), s, e, s)):
        _refuses(I, call)
