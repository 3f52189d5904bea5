"""Norm, its gradient, rows and weights in 8 bits and their product against plain 64-bit forms (oracle/rows.py).  Needs an MI355X (-m gpu).

Tolerances count roundings of 32-bit arithmetic, u = 2^-24 each: the sum of a row's squares takes at most 32 additions in a lane, 6 over the lanes and 15 over
wavefronts, so with the mean, its root and the quotient r is off by 30 u, and y = h r w by 32 u; a scale by one more; the quotient that goes to 8 bits by the sum of both
and 3 for the reciprocal and the product."""
import numpy as np
import pytest
import torch

from oracle import rows as oracle
from tests.test_gpu_cache import BF16, E4M3, F16, F32, HALF_STEP, SMALLEST, _close, _f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NORM, SCALE = 33 * U, 35 * U
EIGHT = NORM + SCALE + 3 * U
EPS = 1e-6


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


def _rand(seed, shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g, dtype=torch.float64) * std
    x *= torch.exp(0.5 * torch.randn(shape[-1], generator=g, dtype=torch.float64))
    return x.to(dtype)


def _strided(x, how):
    """The same values on the GPU: "whole", with room between the rows ("room": an odd number of elements; "far": 16 bytes), or from an odd element on ("off")."""
    if how == "whole":
        return x.cuda()
    room = {"room": 3, "far": 16 // x.element_size(), "off": 5}[how]
    out = torch.full((*x.shape[:-1], x.shape[-1] + room), 7.0, device="cuda").to(x.dtype)
    out = out[..., 1:1 + x.shape[-1]] if how == "off" else out[..., :x.shape[-1]]
    out.copy_(x)
    return out


def _rounded(got, want, rel, dtype, mass=None):
    """got is want computed with an error of `rel` (of the value, or of `mass`), rounded once to dtype; what lies beyond the type's largest number and half a step is infinite
    there (fp16: from 65520 on)."""
    off = rel * (np.abs(want) if mass is None else mass)
    tol = HALF_STEP[dtype] * (np.abs(want) + off) + off + SMALLEST[dtype]
    g, most = _f64(got), torch.finfo(dtype).max * (1 + HALF_STEP[dtype] / 2)
    beyond = np.abs(want) - tol > most
    assert np.array_equal(g[beyond], np.sign(want[beyond]) * np.inf)
    border = ~beyond & (np.abs(want) + tol >= most) & np.isinf(g)
    _close(np.where(beyond | border, 0, g), np.where(beyond | border, 0, want), tol)


def _check_eight(q, scale, y, tall, rel=EIGHT, scale_rel=SCALE):
    """8 bits and scales of 64-bit values y that the kernel has with an error of about rel."""
    want, of = oracle.blocks(y, tall)
    _close(_f64(scale), want, scale_rel * want)
    t = y / of
    _close(_f64(q)[np.isfinite(y)], t[np.isfinite(y)], (2.0 ** -4 * (1 + rel) + rel) * np.abs(t[np.isfinite(y)]) + 2.0 ** -10)
    assert np.isnan(_f64(q)[~np.isfinite(y)]).all()


# ---- norm

DIMS = [1, 7, 8, 40, 64, 127, 128, 129, 200, 256, 257, 264, 512, 1001, 1024, 4096, 5000, 8192, 16384, 20001, 32768]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("dim", DIMS)
def test_norm(dev, dim, dtype):
    for tokens, residual, eight, how in ((1, False, False, "whole"), (3, True, False, "room"), (5, True, True, "off"), (4, False, True, "far")):
        x, w = _rand(dim, (tokens, dim), dtype), _rand(dim + 1, (dim,), dtype).abs() + 0.5
        w = w.to(dtype if tokens % 2 else F32)
        r = _rand(dim + 2, (tokens, dim), dtype, 3.0) if residual else None
        got = dev.norm(_strided(x, how), w.cuda(), EPS, residual=None if r is None else _strided(r, how), eight=eight)
        h = x
        if residual:
            h = (x.float() + r.float()).to(dtype)
            assert torch.equal(got.total.cpu(), h)
        else:
            assert got.total is None
        y = oracle.norm(_f64(h), _f64(w), EPS)
        if eight:
            assert got.scale.shape == (tokens, -(-dim // 128))
            _check_eight(got.out, got.scale, y, 1)
        else:
            assert got.scale is None
            _rounded(got.out, y, NORM, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens, dim", [(9000, 96), (5003, 300), (3001, 1000), (2600, 2048), (1500, 4104)])
def test_norm_of_many_rows(dev, tokens, dim, dtype):
    x, w = _rand(1, (tokens, dim), dtype), _rand(2, (dim,), dtype)
    got = dev.norm(x.cuda(), w.cuda(), EPS, eight=True)
    y = oracle.norm(_f64(x), _f64(w), EPS)
    _check_eight(got.out, got.scale, y, 1)
    _rounded(dev.norm(x.cuda(), w.cuda(), EPS).out, y, NORM, dtype)


@pytest.mark.parametrize("heads, dim", [(1, 64), (5, 40), (40, 128), (3, 256), (7, 80), (2, 1000)])
def test_norm_of_heads(dev, heads, dim):
    packed = _rand(heads, (37, heads + 2, dim), BF16).cuda()
    w = _rand(3, (dim,), BF16)
    before = packed.clone()
    got = dev.norm(packed[:, 1:1 + heads], w.cuda(), 1e-5).out
    y = oracle.norm(_f64(before[:, 1:1 + heads]), _f64(w), 1e-5)
    _rounded(got, y, NORM, BF16)
    # in place, inside the projection: nothing else of it changes
    out = packed[:, 1:1 + heads]
    assert dev.norm(out, w.cuda(), 1e-5, out=out).out is out
    assert torch.equal(out, got) and torch.equal(packed[:, 0], before[:, 0]) and torch.equal(packed[:, 1 + heads], before[:, 1 + heads])


@pytest.mark.parametrize("dim", [96, 1000, 5000])
def test_norm_in_place(dev, dim):
    """total in the residual or in x, out in x or in the residual: what the call gives with tensors of its own."""
    x, r, w = (_rand(i, (300, dim), BF16).cuda() for i in range(3))
    w = w[0].contiguous()
    want = dev.norm(x, w, EPS, residual=r)
    for total_in, out_in in (("r", "x"), ("x", "r"), ("r", None), (None, "x"), (None, "r")):
        a, b = x.clone(), r.clone()
        place = {"x": a, "r": b, None: None}
        got = dev.norm(a, w, EPS, residual=b, total=place[total_in], out=place[out_in])
        assert torch.equal(got.out, want.out) and torch.equal(got.total, want.total)
    a = r.clone()
    got = dev.norm(x, w, EPS, residual=a, total=a, eight=True)
    assert torch.equal(a, want.total)
    again = dev.norm(x, w, EPS, residual=r, eight=True)
    assert torch.equal(got.out.view(torch.uint8), again.out.view(torch.uint8)) and torch.equal(got.scale, again.scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 300, 4096])
def test_norm_of_extreme_rows(dev, dim, dtype):
    """Rows of zeros, tiny, infinite and NaN: the formula's, and beside them ordinary rows as ever."""
    x = _rand(dim, (7, dim), dtype).double()
    x[1] = 0
    x[2] *= 1e-18
    x[3, 5] = float("inf")
    x[4, 6] = float("nan")
    x[5] *= 1e15
    x = x.to(dtype)
    w = torch.ones(dim, dtype=dtype)
    got = dev.norm(x.cuda(), w.cuda(), EPS)
    with np.errstate(invalid="ignore"):
        y = oracle.norm(_f64(x), _f64(w), EPS)
    assert np.isnan(y[3, 5]) and (np.delete(y[3], 5) == 0).all() and np.isnan(y[4]).all()
    _rounded(got.out, y, NORM, dtype)
    eight = dev.norm(x.cuda(), w.cuda(), EPS, eight=True)
    _check_eight(eight.out, eight.scale, y, 1)
    assert (eight.scale[1] == 2.0 ** -126).all() and (eight.out[1].float() == 0).all()


def test_norm_of_no_rows(dev):
    for shape in ((0, 64), (0, 3, 64)):
        x = torch.empty(shape, dtype=BF16, device="cuda")
        w = torch.ones(64, dtype=BF16, device="cuda")
        assert dev.norm(x, w, EPS, residual=x).total.shape == shape
        dx, dw = dev.norm_grad(x, w, x, EPS)
        assert dx.shape == shape and torch.equal(dw, torch.zeros_like(dw))


# ---- its gradient

def _check_grad(got, x, w, g, eps, extra=None):
    """c is a sum of 55 roundings of its terms' sizes, r^3 is off by 90 u; the columns' sums by their terms' 33 u and one rounding a row, at most 16 groups and 16 parts."""
    dx, dw, (own, common), mass = oracle.norm_grad(_f64(x), _f64(w), _f64(g), eps, None if extra is None else _f64(extra))
    off = 40 * U * own + 160 * U * common + 2 * U * np.abs(dx)
    _close(_f64(got[0]), dx, HALF_STEP[x.dtype] * (np.abs(dx) + off) + off + SMALLEST[x.dtype])
    rows = x.numel() // x.shape[-1]
    _close(_f64(got[1]), dw, (70 + rows) * U * mass + SMALLEST[F32])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("dim", DIMS)
def test_norm_grad(dev, dim, dtype):
    for tokens, extra, how in ((1, False, "whole"), (3, True, "room"), (130, False, "off"), (40, True, "far")):
        x, g, w = _rand(dim, (tokens, dim), dtype), _rand(dim + 1, (tokens, dim), dtype, 0.1), _rand(dim + 2, (dim,), dtype)
        w = w.to(dtype if tokens % 2 else F32)
        e = _rand(dim + 3, (tokens, dim), dtype, 0.1) if extra else None
        got = dev.norm_grad(_strided(x, how), w.cuda(), _strided(g, how), EPS, extra=None if e is None else _strided(e, how))
        assert got[1].dtype == F32
        _check_grad(got, x, w, g, EPS, e)


@pytest.mark.parametrize("heads, dim, tokens", [(1, 64, 50), (5, 40, 3000), (40, 128, 700), (3, 256, 90), (7, 80, 1), (2, 1000, 300)])
def test_norm_grad_of_heads(dev, heads, dim, tokens):
    packed = _rand(heads, (tokens, heads + 2, dim), BF16)
    x, w, g = packed[:, 1:1 + heads], _rand(3, (dim,), BF16), _rand(4, (tokens, heads, dim), BF16)
    _check_grad(dev.norm_grad(packed.cuda()[:, 1:1 + heads], w.cuda(), g.cuda(), EPS), x, w, g, EPS)


@pytest.mark.parametrize("dim", [128, 1000, 17000])
def test_norm_grad_in_place_and_again(dev, dim):
    """dx in any tensor that is read; and the same bits at every call."""
    x, g, e = (_rand(i, (600, dim), BF16).cuda() for i in range(3))
    w = _rand(4, (dim,), BF16).cuda()
    want = dev.norm_grad(x, w, g, EPS, extra=e)
    for i in range(4):
        t = [x.clone(), g.clone(), e.clone()]
        got = dev.norm_grad(t[0], w, t[1], EPS, extra=t[2], dx=t[i] if i < 3 else None)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dim", [5, 130])
def test_norm_grad_against_differences(dev, dim):
    """In 32 bits against central differences of the 64-bit norm (steps of 1e-5: off by 1e-10 of the third derivative, and 2^-52 / 1e-5 of the value)."""
    x, g, w = _rand(1, (3, dim), F32), _rand(2, (3, dim), F32), _rand(3, (dim,), F32)
    dx, dw = (_f64(t) for t in dev.norm_grad(x.cuda(), w.cuda(), g.cuda(), 1e-3))
    f = lambda a, b: (oracle.norm(a, b, 1e-3) * _f64(g)).sum()  # noqa: E731
    d = 1e-5
    for i in range(3):
        for j in range(0, dim, 7):
            a = np.zeros((3, dim))
            a[i, j] = d
            want = (f(_f64(x) + a, _f64(w)) - f(_f64(x) - a, _f64(w))) / (2 * d)
            assert abs(dx[i, j] - want) < 1e-4 * max(1.0, abs(want))
    for j in range(0, dim, 7):
        a = np.zeros(dim)
        a[j] = d
        want = (f(_f64(x), _f64(w) + a) - f(_f64(x), _f64(w) - a)) / (2 * d)
        assert abs(dw[j] - want) < 1e-4 * max(1.0, abs(want))


# ---- to 8 bits

@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows, columns", [(1, 1), (1, 128), (3, 129), (16, 7), (17, 1000), (200, 300), (5, 4096), (1000, 64), (129, 256), (1, 30000), (2000, 2560)])
def test_quantize(dev, rows, columns, dtype):
    x = _rand(rows + columns, (rows, columns), dtype)
    for tall, how in ((1, "whole"), (128, "whole"), (1, "room"), (128, "off")):
        if rows * columns > 1e6 and how != "whole":
            continue
        got = dev.quantize(_strided(x, how), tall=tall)
        assert got.out.dtype == E4M3 and got.scale.shape == (-(-rows // tall), -(-columns // 128))
        _check_eight(got.out, got.scale, _f64(x), tall, 4 * U, U)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows, columns", [(1, 1), (3, 129), (17, 1000), (200, 384), (2000, 640), (1, 10240)])
def test_quantize_behind_a_gate(dev, rows, columns, dtype):
    """exp(-|g|): its argument in two parts, the power of two within 2 u, 4 for the parts; sum, reciprocal (2 u) and products 7 more."""
    both = _rand(rows, (rows, 2 * columns), dtype)
    both[:, :columns] *= 3
    both[0, 0], both[-1, columns - 1] = -60, 40
    gate, x = both.cuda()[:, :columns], both.cuda()[:, columns:]
    got = dev.quantize(x, gate=gate)
    _check_eight(got.out, got.scale, oracle.gated(_f64(x), _f64(gate)), 1, 36 * U, 17 * U)


def test_quantize_special_values(dev):
    """Every number of the type comes back as itself, ties go to the even one, what is infinite or NaN is NaN alone; a block of nothing finite has the least scale."""
    bits = torch.arange(256, dtype=torch.uint8).view(E4M3).float()
    number = bits[~bits.isnan()]
    x = torch.zeros((6, 256), dtype=F32)
    x[0, :number.numel()] = number           # both blocks hold 448: scales of 1, or the block's own
    x[0, 127], x[0, 255] = 448, -448
    tie = torch.arange(8, 16, dtype=F32) + 0.5   # between neighbours at 16 .. 32, in units of 2
    x[1, :8], x[1, 8] = 2 * tie, 448
    x[2, 0], x[2, 1], x[2, 2], x[2, 3] = float("inf"), float("nan"), -float("inf"), 7.0
    x[3, :128] = float("nan")
    x[4] = 1e-42
    x[4, 200] = 3e38
    x[5, 0], x[5, 1] = 463.9 * 2.0 ** -100, 448 * 2.0 ** -100
    for tall, of in ((1, x), (128, x[:1]), (128, x[1:2]), (128, x[2:3])):
        got = dev.quantize(of.cuda(), tall=tall)
        _check_eight(got.out, got.scale, _f64(of), tall, 4 * U, U)
    got = dev.quantize(x.cuda())
    q, s = got.out.float().cpu(), got.scale.cpu()
    assert (s[0] == 1).all() and torch.equal(q[0, :127], x[0, :127]) and torch.equal(q[0, 128:254], x[0, 128:254])
    assert torch.equal(q[1, :8], torch.tensor([16, 20, 20, 24, 24, 28, 28, 32], dtype=F32))
    assert q[2, :3].isnan().all() and q[2, 3] == 448 and (q[2, 4:] == 0).all()
    assert q[3, :128].isnan().all() and s[3, 0] == 2.0 ** -126 and (q[3, 128:] == 0).all()
    assert (q[4, :128] == 0).all() and s[4, 0] == 2.0 ** -126


# ---- the product

def _operands(seed, m, n, k, exact=False):
    g = torch.Generator().manual_seed(seed)
    if exact:   # whole numbers and scales of powers of two: every sum is a number of 24 bits
        a, w = (torch.randint(-3, 4, s, generator=g).float().to(E4M3) for s in ((m, k), (n, k)))
        sa, sw = (torch.exp2(torch.randint(-1, 2, s, generator=g).float()) for s in ((m, -(-k // 128)), (-(-n // 128), -(-k // 128))))
    else:
        a, w = ((torch.randn(s, generator=g) * 60).clamp(-448, 448).to(E4M3) for s in ((m, k), (n, k)))
        sa, sw = (0.01 + torch.rand(s, generator=g) for s in ((m, -(-k // 128)), (-(-n // 128), -(-k // 128))))
    return a, sa, w, sw


def _lying(t, order):
    """Scales on the GPU with rows ("rows") or blocks ("blocks") beside one another, or neither."""
    if order == "rows":
        return t.t().contiguous().cuda().t()
    if order == "blocks":
        return t.cuda()
    room = torch.full((t.shape[0] * 2, t.shape[1] * 3), 1e30, device="cuda")
    room[::2, ::3] = t.cuda()
    return room[::2, ::3]


def _check_product(got, a, sa, w, sw, exact, dtype):
    """A block's 128 products sum with at most 256 roundings, scales and sums over blocks add 3 and one a block.  With an out of 16 bits up to seven of eight neighbouring
    products are cut at 2^-13 of the largest."""
    want, mass = oracle.product(_f64(a), _f64(sa), _f64(w), _f64(sw))
    if exact:
        assert np.array_equal(_f64(got), _f64(torch.from_numpy(want).to(dtype)))
    else:
        off = (260 + sa.shape[1]) * U * mass
        if dtype != F32:
            off += 7 * 2.0 ** -13 * oracle.largest_products(_f64(a), _f64(sa), _f64(w), _f64(sw), 8)
        _rounded(got, want, 1.0, dtype, off)


SIZES = [(1, 1, 16), (1, 64, 128), (1, 4096, 4096), (2, 100, 144), (16, 128, 256), (17, 129, 272), (3, 5003, 2576), (33, 200, 1040), (64, 384, 4096), (64, 6144, 512), (65, 300, 640),
         (100, 1000, 1008), (128, 128, 128), (129, 257, 384), (200, 40, 8192), (389, 5003, 112), (500, 512, 2560), (1000, 130, 96), (700, 900, 1296), (1024, 1024, 1024), (2500, 1100, 400)]


@pytest.mark.parametrize("m, n, k", SIZES)
def test_gemm_scaled(dev, m, n, k):
    dtype = (BF16, F16, F32)[(m + n) % 3]
    for exact, order, dtype in ((True, "rows", F32), (True, "rows", BF16), (False, "blocks", dtype), (False, "blocks", F32)):
        a, sa, w, sw = _operands(m + n + k, m, n, k, exact)
        got = dev.gemm_scaled(a.cuda(), _lying(sa, order), w.cuda(), _lying(sw, order), dtype=dtype)
        assert got.shape == (m, n)
        _check_product(got, a, sa, w, sw, exact, dtype)


WAYS = {"few rows, 16 x 16": [(5, 300, 1296)], "few rows, 16 x 32": [(16, 6144, 1040)], "few rows, 32 x 32": [(72, 2700, 144), (397, 567, 160)], "tiles of 64 x 16": [(100, 2000, 4112)],
        "tiles of 64 x 32": [(87, 3512, 400)], "tiles of 64 x 32, four stages": [(183, 2637, 96), (51, 5178, 160)], "tiles of 64 x 64": [(256, 4096, 1040)],
        "tiles of 64 x 64, four stages": [(200, 3000, 400), (1100, 1030, 656)], "tiles of 128 x 128": [(389, 5003, 2576), (2500, 1100, 400)],
        "tiles of 256 x 128": [(1500, 5000, 272)], "tiles of 256 x 256": [(2100, 4200, 144), (4357, 4100, 80), (4352, 4352, 128), (4352, 4352, 256), (4352, 4352, 400), (4352, 4103, 512)]}


@pytest.mark.parametrize("way", WAYS)
def test_every_way_of_gemm_scaled(dev, way, monkeypatch, capfd):
    """Each is reached (a trace names it), takes whole and partial tiles, several of them to a workgroup, and gives the same bits at every call."""
    monkeypatch.setenv("AMAP_PLAN_TRACE", "1")
    for m, n, k in WAYS[way]:
        for exact, dtype in ((True, BF16), (True, F16), (False, F16)):
            a, sa, w, sw = (t.cuda() for t in _operands(m + k, m, n, k, exact))
            capfd.readouterr()
            got = dev.gemm_scaled(a, sa, w, sw, dtype=dtype)
            assert f"amap gemm scaled: {way}, {m} x {n} x {k}" in capfd.readouterr().err
            _check_product(got, a, sa, w, sw, exact, dtype)
            for _ in range(20):
                assert torch.equal(got.view(torch.int16), dev.gemm_scaled(a, sa, w, sw, dtype=dtype).view(torch.int16))


@pytest.mark.parametrize("way, m, n, k", [("few rows, 16 x 16", 1, 500, 1040), ("few rows, 16 x 32", 16, 6144, 1040), ("few rows, 32 x 32", 72, 2700, 144),
                                          ("tiles of 64 x 32, four stages", 87, 3512, 400), ("tiles of 64 x 64, four stages", 389, 5003, 272), ("tiles of 128 x 128", 2500, 1100, 400)])
def test_every_way_of_gemm_scaled_to_32_bits(dev, way, m, n, k, monkeypatch, capfd):
    monkeypatch.setenv("AMAP_PLAN_TRACE", "1")
    for exact in (True, False):
        a, sa, w, sw = (t.cuda() for t in _operands(m + k, m, n, k, exact))
        capfd.readouterr()
        got = dev.gemm_scaled(a, sa, w, sw, dtype=F32)
        assert f"amap gemm scaled: {way}, {m} x {n} x {k}" in capfd.readouterr().err
        _check_product(got, a, sa, w, sw, exact, F32)


@pytest.mark.parametrize("m, n, k", [(1, 130, 272), (20, 500, 528), (300, 260, 400), (1100, 1030, 656), (2100, 4203, 144)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_gemm_scaled_of_strided_operands(dev, m, n, k, dtype):
    """Rows with other things between them (NaN behind the last k, too), scales in no order, an out with room around it, which stays as it was."""
    a, sa, w, sw = _operands(7, m, n, k)

    def among_nan(t):
        room = torch.full((t.shape[0] + 1, k + 48), 0x7F, dtype=torch.uint8, device="cuda").view(E4M3)
        room.view(torch.uint8)[:-1, 16:16 + k] = t.view(torch.uint8).cuda()
        return room[:-1, 16:16 + k]

    room = torch.full((m + 2, n + 3), 5.0, dtype=dtype, device="cuda")
    out = room[1:-1, 1:-2]
    assert dev.gemm_scaled(among_nan(a), _lying(sa, ""), among_nan(w), _lying(sw, ""), out=out) is out
    _check_product(out, a, sa, w, sw, False, dtype)
    room[1:-1, 1:-2] = 5
    assert (room == 5).all()


@pytest.mark.parametrize("m, n, k", [(1, 64, 256), (40, 300, 400), (600, 520, 384)])
def test_gemm_scaled_special_values(dev, m, n, k):
    """NaN in a row of either operand, an infinite scale, scales at the ends: the formula's, and elsewhere as ever."""
    a, sa, w, sw = _operands(3, m, n, k)
    for t, row in ((a, m - 1), (w, 5)):
        t.view(torch.uint8)[row, k - 1] = 0x7F
    sa[0, 1] = float("inf")
    if m > 2:
        sa[1], sa[2, 0] = 0.0, 2.0 ** -126
    got = _f64(dev.gemm_scaled(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), dtype=F32))
    with np.errstate(invalid="ignore"):
        want, mass = oracle.product(_f64(a), _f64(sa), _f64(w), _f64(sw))
    whole = np.isfinite(want)
    assert whole.sum() == max(m - 2, 0) * (n - 1)
    _close(got[whole], want[whole], (260 + sa.shape[1]) * U * mass[whole] + 2.0 ** -149)
    assert np.isnan(got[-1]).all() and np.isnan(got[:, 5]).all()
    if m > 1:
        assert not np.isfinite(np.delete(got[0], 5)).any()


# ---- sizes that go past the caches

def _rows_of(seed, rows, columns, dtype, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((rows, columns), dtype=dtype, device="cuda")
    for part in x.split(4096):
        part.copy_(torch.randn(part.shape, device="cuda", generator=g) * std)
    return x


@pytest.mark.parametrize("rows", [4100, 16391])
def test_large_norm(dev, rows):
    """Stored past the caches, and loaded so as well: every 37th row, and all scales against those of the same rows by themselves (whose squares may be summed in another order: both are
    within SCALE of the definition's)."""
    x, r, w = _rows_of(1, rows, 4096, BF16), _rows_of(2, rows, 4096, BF16, 3.0), _rand(3, (4096,), BF16).cuda()
    h = (x.float() + r.float()).to(BF16)
    got, wide = dev.norm(x, w, EPS, residual=r, eight=True), dev.norm(x, w, EPS, residual=r)
    assert torch.equal(got.total, h) and torch.equal(wide.total, h)
    at = torch.arange(0, rows, 37, device="cuda")
    y = oracle.norm(_f64(h[at]), _f64(w), EPS)
    _check_eight(got.out[at], got.scale[at], y, 1)
    _rounded(wide.out[at], y, NORM, BF16)
    for part in torch.arange(rows, device="cuda").split(1000):
        few = dev.norm(h[part], w, EPS, eight=True)
        _close(_f64(got.scale[part]), _f64(few.scale), 2 * SCALE * (1 + SCALE) * _f64(few.scale))


@pytest.mark.parametrize("rows, dtype", [(5000, BF16), (12800, BF16), (9000, F32)])
def test_large_norm_grad(dev, rows, dtype):
    x, g, e, w = _rows_of(1, rows, 4096, dtype), _rows_of(2, rows, 4096, dtype, 0.1), _rows_of(3, rows, 4096, dtype, 0.1), _rand(3, (4096,), dtype).cuda()
    got = dev.norm_grad(x, w, g, EPS, extra=e)
    dw, mass = torch.zeros(4096, dtype=torch.float64, device="cuda"), torch.zeros(4096, dtype=torch.float64, device="cuda")
    for a, b in zip(x.split(1000), g.split(1000)):
        t = b.double() * a.double() / torch.sqrt(a.double().square().mean(-1, keepdim=True) + EPS)
        dw += t.sum(0)
        mass += t.abs().sum(0)
    _close(_f64(got[1]), _f64(dw), (70 + rows) * U * _f64(mass))
    at = torch.arange(0, rows, 41, device="cuda")
    dx, _, (own, common), _ = oracle.norm_grad(_f64(x[at]), _f64(w), _f64(g[at]), EPS, _f64(e[at]))
    off = 40 * U * own + 160 * U * common + 2 * U * np.abs(dx)
    _close(_f64(got[0][at]), dx, HALF_STEP[dtype] * (np.abs(dx) + off) + off + SMALLEST[dtype])


@pytest.mark.parametrize("rows, columns, gate, tall", [(8192, 10240, False, 1), (8192, 10240, True, 1), (6000, 4096, False, 1), (8192, 10240, False, 128), (12000, 4032, False, 128), (30000, 4100, False, 1)])
def test_large_quantize(dev, rows, columns, gate, tall):
    x = _rows_of(rows, rows, columns * (1 + gate), BF16)
    a, b = (x[:, columns:], x[:, :columns]) if gate else (x, None)
    got = dev.quantize(a, gate=b, tall=tall)
    step = 128 * tall
    for first in (0, (rows // 2) // step * step, (rows - 1) // step * step):
        part = slice(first, min(first + max(tall, 3), rows))
        y = _f64(a[part]) if b is None else oracle.gated(_f64(a[part]), _f64(b[part]))
        _check_eight(got.out[part], got.scale[first // tall:-(-part.stop // tall)], y, tall, 36 * U, 17 * U)


@pytest.mark.parametrize("rows, columns, apart, gate, tall", [(300, 1000, 0, False, 1), (300, 1000, 0, False, 128), (129, 1288, 1, True, 1), (1, 5000, 0, False, 128), (6100, 4080, 0, False, 128),
                                                              (4096, 4080, 0, False, 1), (16391, 10240, 8, False, 1), (16391, 10240, 8, False, 128), (9000, 10240, 3, True, 1)])
def test_quantize_rows_of_no_whole_lines(dev, rows, columns, apart, gate, tall):
    """Blocks of rows that begin inside a line of 128 bytes are taken in another order, and by 128 rows never loaded past the caches: the same bits as of rows that begin at lines, for every block."""
    lines = _rows_of(rows, rows, -(-columns // 64) * 64 * (1 + gate), BF16)
    half = lines.shape[1] // 2
    a, b = (lines[:, half:half + columns], lines[:, :columns]) if gate else (lines[:, :columns], None)
    want = dev.quantize(a, gate=b, tall=tall)
    room = [torch.empty((rows, columns + apart), dtype=BF16, device="cuda")[:, apart:] for _ in range(1 + gate)]
    for to, of in zip(room, (a, b)):
        to.copy_(of)
    out = torch.full((rows, columns), 0xFF, dtype=torch.uint8, device="cuda").view(E4M3)
    scale = torch.full((-(-columns // 128), -(-rows // tall)), -1.0, device="cuda").t()
    got = dev.quantize(room[0], gate=room[1] if gate else None, tall=tall, out=out, scale=scale)
    assert torch.equal(got.out.view(torch.uint8), want.out.view(torch.uint8)) and torch.equal(got.scale, want.scale)
    part = slice((rows - 1) // tall * tall, rows)
    y = _f64(a[part]) if b is None else oracle.gated(_f64(a[part]), _f64(b[part]))
    _check_eight(got.out[part], got.scale[part.start // tall:], y, tall, 36 * U, 17 * U)


# ---- together

def test_a_gated_layer(dev):
    """norm -> product -> gate -> product -> norm with the residual, all handed on in 8 bits: each step within its own tolerance of the 64-bit form of what it was given."""
    tokens, width, hidden = 77, 512, 1408
    x, r, w = _rand(1, (tokens, width), BF16).cuda(), _rand(2, (tokens, width), BF16).cuda(), _rand(3, (width,), BF16).cuda()
    up, down = (dev.quantize(_rand(i, s, BF16, s[1] ** -0.5).cuda(), tall=128) for i, s in ((4, (2 * hidden, width)), (5, (width, hidden))))
    y = dev.norm(x, w, EPS, residual=r, eight=True)
    _check_eight(y.out, y.scale, oracle.norm(_f64(y.total), _f64(w), EPS), 1)
    both = dev.gemm_scaled(y.out, y.scale, up.out, up.scale)
    _check_product(both, y.out, y.scale, up.out, up.scale, False, BF16)
    z = dev.quantize(both[:, hidden:], gate=both[:, :hidden])
    _check_eight(z.out, z.scale, oracle.gated(_f64(both[:, hidden:]), _f64(both[:, :hidden])), 1, 36 * U, 17 * U)
    out = dev.gemm_scaled(z.out, z.scale, down.out, down.scale)
    _check_product(out, z.out, z.scale, down.out, down.scale, False, BF16)
    end = dev.norm(out, w, EPS, residual=y.total, total=y.total)
    _rounded(end.out, oracle.norm(_f64(end.total), _f64(w), EPS), NORM, BF16)
