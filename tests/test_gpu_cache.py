"""The operators around the paged cache against plain loops in 64 bits (oracle/cache.py).  Needs an MI355X (-m gpu)."""
import math

import numpy as np
import pytest
import torch

from oracle import cache as oracle
from paper_2002_12798_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
HALF_STEP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24, E4M3: 2.0 ** -4}       # of a rounding, relative
SMALLEST = {BF16: 2.0 ** -134, F16: 2.0 ** -25, F32: 2.0 ** -150, E4M3: 2.0 ** -10}    # half a step below the normal numbers


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


def _f64(t):
    return t.detach().cpu().to(torch.float64 if t.dtype != E4M3 else torch.float32).double().numpy()


def _gpu(x, dtype=torch.int32):
    return torch.as_tensor(x, dtype=dtype).cuda()


def _close(got, want, tol):
    far = np.abs(got - want) > tol
    assert not far.any() and np.array_equal(np.isnan(got), np.isnan(want)), (int(far.sum()), far.size, np.abs(got - want).max())


# ---- block tables and slots

def _step(seed, requests, page, longest, fresh, lack=0, narrow=0, first=True):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, longest + 1, requests) if first else None
    new = rng.integers(0, fresh + 1, requests)
    have = -(-(cached if first else np.zeros(requests, int)) // page)
    total = -(-((cached if first else 0) + new) // page)
    width = max(1, int(total.max(initial=0)) - narrow)
    ids = rng.permutation(int(total.sum()) + 5)
    table = np.full((requests, width), -7)
    used = 0
    for r in range(requests):
        n = min(int(have[r]), width)
        table[r, :n] = ids[used:used + n]
        used += n
    free = ids[used:]
    return cached, new, table, free[:max(0, len(free) - 5 - lack)]


@pytest.mark.parametrize("requests, page, longest, fresh, spare, more", [
    (1, 16, 0, 1, 0, {}), (1, 1, 5, 3, 2, {}), (3, 16, 40, 0, 3, {}), (64, 16, 2000, 1, 0, {}), (65, 13, 300, 40, 7, {}), (513, 32, 100, 90, 64, {}),
    (1025, 7, 50, 3, 0, {}), (300, 16, 100, 40, 0, dict(lack=60)), (50, 8, 100, 60, 5, dict(narrow=4)), (40, 16, 0, 500, 1, dict(first=False)),
    (16384, 16, 64, 5, 100, {}), (8193, 128, 900, 2, 0, dict(lack=100)),
])
def test_assign(dev, requests, page, longest, fresh, spare, more):
    cached, new, table, free = _step(requests + page, requests, page, longest, fresh, **more)
    n = int(new.sum()) + spare
    t = _gpu(table)
    c = None if cached is None else _gpu(cached)
    for _ in range(2):   # the same call again gives the same
        a = dev.cache_assign(page, c, _gpu(new), t, _gpu(free), n)
    want = oracle.assign(page, cached, new, table, free, n)
    for got, w, name in zip((t, a.begin, a.length, a.slot, a.position, a.owner), want, ("table", "begin", "length", "slot", "position", "owner")):
        assert np.array_equal(got.cpu().numpy(), np.asarray(w).reshape(got.shape)), name
    assert a.taken.item() == want[6]


def test_assign_of_a_strided_table_and_wild_lengths(dev):
    """Rows further apart than the table is wide; negative lengths count as none; fewer places than tokens; no request at all."""
    wide = torch.full((4, 20), 99, dtype=torch.int32, device="cuda")
    table = wide[:, 3:9]
    before = table.cpu().numpy().copy()
    a = dev.cache_assign(4, _gpu([-5, 7, 0, 24]), _gpu([3, -2, 9, 2]), table, _gpu([11, 12, 13, 14, 15]), 6)
    want = oracle.assign(4, [-5, 7, 0, 24], [3, -2, 9, 2], before, [11, 12, 13, 14, 15], 6)
    assert np.array_equal(table.cpu().numpy(), want[0]) and a.slot.tolist() == want[3] and a.owner.tolist() == want[5] and a.begin.tolist() == want[1]
    assert (wide[:, :3] == 99).all() and (wide[:, 9:] == 99).all() and a.taken.item() == want[6]
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    a = dev.cache_assign(4, none, none, torch.empty((0, 3), dtype=torch.int32, device="cuda"), none, 3)
    assert a.begin.tolist() == [0] and a.slot.tolist() == [-1] * 3 and a.owner.tolist() == [-1] * 3 and a.taken.item() == 0


# ---- rotary positions

def _frequencies(axes):
    return torch.tensor([10000.0 ** (-i / n) for n in axes for i in range(n)], dtype=F32).cuda()


def _turn_tolerance(x, pairs, interleaved, dtype):
    """Half a step of the result's type, and in 32 bits: the fraction of a turn rounded to 2^-25 of two half turns (pi * 2^-25 of a radian), sine and
    cosine a few steps off, two products and a sum: together under 8 * 2^-24 of either element's size."""
    both = np.abs(x).copy()
    i = np.arange(2 * pairs)
    other = i ^ 1 if interleaved else (i + pairs) % (2 * pairs)
    both[..., :2 * pairs] += both[..., other]
    return lambda want: HALF_STEP[dtype] * (np.abs(want) + 8 * 2.0 ** -24 * both) + 8 * 2.0 ** -24 * both + SMALLEST[dtype]


@pytest.mark.parametrize("tokens, heads, dim, axes, interleaved, dtype, furthest", [
    (1, 1, 2, (1,), False, F32, 10), (1, 16, 64, (32,), False, BF16, 1000000), (33, 5, 80, (8, 16, 16), False, BF16, 64), (7, 3, 40, (20,), False, F16, 3000),
    (100, 4, 96, (8, 8, 8), False, F32, 100), (513, 2, 128, (64,), True, BF16, 500000), (20, 25, 72, (12, 12, 12), True, F16, 99), (9, 3, 6, (1, 1), False, BF16, 9),
    (9, 3, 7, (3,), False, F16, 9), (2000, 12, 64, (16, 16), True, F32, 4096), (64, 1, 256, (32, 32, 32, 32), False, F16, 77), (3, 2, 1024, (512,), False, BF16, 50),
    (5, 7, 30, (0, 15), False, F32, 50), (5, 7, 30, (13,), True, BF16, 50), (3001, 8, 64, (32,), False, BF16, 30000),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(dev, tokens, heads, dim, axes, interleaved, dtype, furthest, inverse):
    g = torch.Generator().manual_seed(tokens * dim)
    x = torch.randn((tokens, heads, dim), generator=g).to(dtype).cuda()
    position = torch.randint(-3, furthest, (len(axes), tokens), generator=g, dtype=torch.int32)
    rope = dev.Rope(_frequencies(axes), axes, interleaved)
    got = dev.rotary(x, rope, position.cuda(), inverse=inverse)
    want = oracle.turn(_f64(x), position.numpy(), rope.freq.cpu().numpy(), axes, interleaved, inverse)
    _close(_f64(got), want, _turn_tolerance(_f64(x), sum(axes), interleaved, dtype)(want))
    # in place, inside a wider tensor that begins at an odd place, the same positions for every axis
    whole = torch.full((tokens, heads + 2, dim + 3), 5.0, dtype=dtype, device="cuda")
    part = whole[:, 1:heads + 1, 1:dim + 1]
    part.copy_(x)
    if not interleaved:
        dev.rotary(part, rope, position[0].cuda(), out=part, inverse=inverse)
        want = oracle.turn(_f64(x), position[:1].numpy().repeat(len(axes), 0), rope.freq.cpu().numpy(), axes, interleaved, inverse)
        _close(_f64(part), want, _turn_tolerance(_f64(x), sum(axes), interleaved, dtype)(want))
        part.fill_(5.0)
        assert (whole == 5.0).all()


def test_rotary_gradient_by_differences(dev):
    """The gradient of sum(w * turn(x)) is w turned back: against the formula's and against differences of the 64-bit turn."""
    axes, rng = (5, 3, 4), np.random.default_rng(4)
    x, w, position = rng.standard_normal((6, 2, 26)), rng.standard_normal((6, 2, 26)), rng.integers(0, 200, (3, 6))
    freq = _frequencies(axes)
    rope = dev.Rope(freq, axes)
    got = _f64(dev.rotary(_gpu(w, F32), rope, _gpu(position), inverse=True))
    loss = lambda y: (w * oracle.turn(y, position, freq.cpu().numpy(), axes)).sum()  # noqa: E731
    step = 1e-3
    for t, h, d in [(0, 0, 0), (5, 1, 11), (3, 0, 12), (2, 1, 23), (4, 1, 24), (1, 0, 25)]:
        up, down = x.copy(), x.copy()
        up[t, h, d] += step
        down[t, h, d] -= step
        # (linear in x: differences are exact but for the 64-bit sums, w itself is rounded to 32 bits)
        assert abs((loss(up) - loss(down)) / (2 * step) - got[t, h, d]) < 1e-9 + 12 * 2.0 ** -24 * np.abs(w).max() * 2


# ---- the store into the cache

def _empty_cache(pages, page, heads, dim, dtype, order, seed=3):
    """k and v as [pages, page, heads, dim] in the memory order named, filled with numbers that a store must not touch."""
    shape = {"tokens": (pages, page, heads, dim), "heads": (pages, heads, page, dim), "both": (pages, page, heads, 2, dim)}[order]
    g = torch.Generator().manual_seed(seed)
    made = [torch.randn(shape, generator=g).to(dtype).cuda() for _ in range(1 if order == "both" else 2)]
    if order == "both":
        return made[0][:, :, :, 0], made[0][:, :, :, 1]
    return tuple(t.permute(0, 2, 1, 3) if order == "heads" else t for t in made)


@pytest.mark.parametrize("tokens, heads, kv, dim, page, order, dtype, to, axes", [
    (1, 2, 1, 64, 16, "tokens", BF16, BF16, (32,)), (37, 4, 4, 64, 16, "heads", F16, F16, ()), (50, 8, 2, 128, 24, "both", BF16, E4M3, (32, 32)),
    (19, 3, 3, 40, 1, "tokens", F32, BF16, (10,)), (700, 5, 5, 80, 32, "heads", BF16, BF16, (8, 16, 16)), (64, 7, 1, 96, 8, "tokens", F16, E4M3, ()),
    (11, 2, 2, 6, 5, "heads", F32, F16, (1, 2)), (2100, 2, 2, 256, 64, "both", F16, F16, (128,)), (9, 1, 1, 7, 3, "tokens", BF16, F16, (3,)),
])
def test_append(dev, tokens, heads, kv, dim, page, order, dtype, to, axes):
    g = torch.Generator().manual_seed(tokens + dim)
    packed = torch.randn((tokens, heads + 2 * kv, dim), generator=g).to(dtype).cuda()
    q, k, v = packed[:, :heads], packed[:, heads:heads + kv], packed[:, heads + kv:]
    pages = -(-tokens * 4 // (3 * page)) + 2
    ck, cv = _empty_cache(pages, page, kv, dim, to, order)
    before = [_f64(ck), _f64(cv)]
    slot = torch.randperm(pages * page, generator=g)[:tokens]
    if tokens > 4:
        slot[1], slot[3], slot[4] = -1, pages * page, -(1 << 40)   # none of these is in the cache
    scales = [torch.rand(kv, generator=g).add_(0.05).cuda() if to == E4M3 else None for _ in range(2)]
    rope, position = None, None
    if axes:
        rope, position = dev.Rope(_frequencies(axes), axes), torch.randint(0, 5000, (len(axes), tokens), generator=g, dtype=torch.int32).cuda()
    q_before = _f64(q)
    got_q = dev.cache_append(dev.PagedCache(ck, cv, *scales), k, v, slot.cuda(), rope, position, q if axes else None, q if axes and tokens % 2 else None)
    slot = slot.numpy()
    live = (slot >= 0) & (slot < pages * page)
    for got, was, x, scale, turned in ((ck, before[0], k, scales[0], axes), (cv, before[1], v, scales[1], ())):
        x = _f64(x)
        tol = np.zeros_like(x)
        by = 1.0 if scale is None else _f64(scale)[None, :, None]
        if turned:
            want = oracle.turn(x, position.cpu().numpy(), rope.freq.cpu().numpy(), axes)
            tol = _turn_tolerance(x, sum(axes), False, F32)(want) / by
        else:
            want = x
        want = want / by
        if to == E4M3:
            want = np.clip(want, -448, 448)
        tol = tol * (1 + 2.0 ** -20) + HALF_STEP[to] * (np.abs(want) + tol) + 2.0 ** -24 * np.abs(want) + SMALLEST[to]
        whole, allowed = was.copy(), np.zeros_like(was)
        whole[slot[live] // page, slot[live] % page] = want[live]
        allowed[slot[live] // page, slot[live] % page] = tol[live]
        _close(_f64(got), whole, allowed)
    if axes:
        want = oracle.turn(q_before, position.cpu().numpy(), rope.freq.cpu().numpy(), axes)
        _close(_f64(got_q), want, _turn_tolerance(q_before, sum(axes), False, dtype)(want))


def test_append_rounds_as_a_conversion_does(dev):
    """What is only stored has the bits of a conversion on the CPU: ties, numbers below the normal ones, overflow, infinities, NaN."""
    x = torch.tensor([0.0, -0.0, 1.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 2.0 ** -11, 447.0, 448.0, 464.0, 465.0, 1e4, -1e4, math.inf, -math.inf,
                      math.nan, 0.1, -0.3, 3.1e-3, 17.0, 19.0, 208.0, 2.0 ** -7, 2.0 ** -6 * 0.97, 240.0, 232.0, 5.5, -6.5, 1e-30, 6e-8], dtype=F32)
    for to in (E4M3, BF16, F16):
        k, v = (torch.zeros((2, 1, 1, 32), dtype=to, device="cuda") for _ in range(2))
        dev.cache_append(dev.PagedCache(k, v), x.view(1, 1, 32).cuda(), -x.view(1, 1, 32).cuda(), torch.tensor([1], device="cuda"))
        for got, want in ((k, x), (v, -x)):
            want = want.clamp(-448, 448).to(to) if to == E4M3 else want.to(to)
            got = got[1, 0, 0].cpu()
            nan = torch.isnan(want.float())
            raw = torch.uint8 if to == E4M3 else torch.int16
            assert torch.equal(torch.isnan(got.float()), nan) and torch.equal(got.view(raw)[~nan], want.view(raw)[~nan]), (to, got, want)


# ---- attention of one token

def _requests(dev, seed, lengths, heads, kv, dim, page, dtype, to, order, spare=2, window=0):
    """A filled cache with NaN wherever no request has a token, and everything a call takes."""
    g = torch.Generator().manual_seed(seed)
    n = len(lengths)
    need = [-(-v // page) for v in lengths]
    pages, width = sum(need) + spare, max(need) + 1
    k, v = _empty_cache(pages, page, kv, dim, F32, order, seed)
    ids = torch.randperm(pages, generator=g)
    table = torch.full((n, width), -1, dtype=torch.int32)
    used, filled = 0, torch.zeros((pages, page), dtype=torch.bool)
    for r, c in enumerate(need):
        table[r, :c] = ids[used:used + c]
        used += c
        for i in range(lengths[r]):
            if not window or i >= lengths[r] - window:
                filled[table[r, i // page], i % page] = True
        if window:
            table[r, :max(0, lengths[r] - window) // page] = -1   # given back
    caches = []
    for t in (k, v):
        t = t * (1.0 if to != E4M3 else 12.0)
        t[~filled.cuda()] = math.nan
        caches.append(t.to(to))
    scales = [torch.rand(kv, generator=g).mul_(0.1).add_(0.03).cuda() if to == E4M3 else None for _ in range(2)]
    q = torch.randn((n, heads, dim), generator=g).to(dtype).cuda()
    return dev.PagedCache(*caches, *scales), q, table, torch.tensor(lengths, dtype=torch.int32)


def _expect(cache, q, table, length, scale, window=0):
    k, v = _f64(cache.k), _f64(cache.v)
    if cache.k_scale is not None:
        k, v = k * _f64(cache.k_scale)[:, None], v * _f64(cache.v_scale)[:, None]
    return oracle.attend(_f64(q), k, v, table.numpy(), length.numpy(), cache.page_size, scale, window)


def _check(got, want, q, keys):
    """A score is a sum of dim products in 32 bits, at most (dim + 2) * 2^-24 of the sum of their sizes off; a weight twice that much, by relation to
    the largest, and the exponential's 2^-21 and the 2^-16 of a weight kept in two 16-bit parts; the sums over keys
    in 32 bits keys * 2^-24 at the most; the result half a step of its type."""
    out, lse, mass, most = want
    score = (q.shape[2] + 4) * 2.0 ** -24 * most
    weight = 2 * score + 2.0 ** -21 + 2.0 ** -16 + 2 * keys * 2.0 ** -24
    off = 2 * weight[:, :, None] * mass
    _close(_f64(got[0]), out, HALF_STEP[q.dtype] * (np.abs(out) + off) + off + SMALLEST[q.dtype])
    g, none = _f64(got[1]), lse == -np.inf
    assert np.array_equal(g == -np.inf, none)
    _close(g[~none], lse[~none], (score + 2.0 ** -21 + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(none, 0, lse)))[~none])


ATTEND = [
    # lengths, heads, kv, dim, page, types, order, window
    ([1], 1, 1, 64, 16, BF16, BF16, "tokens", 0),
    ([1, 2, 0, 31, 32, 33], 4, 4, 64, 16, BF16, BF16, "heads", 0),
    ([127, 128, 129, 0, 255, 257], 8, 2, 128, 16, F16, F16, "tokens", 0),
    ([500], 16, 16, 64, 16, BF16, BF16, "tokens", 0),
    ([1500, 3, 700], 32, 8, 128, 16, BF16, BF16, "both", 0),
    ([900, 64], 10, 2, 80, 7, BF16, BF16, "tokens", 0),
    ([333, 1, 77], 3, 3, 40, 1, F16, F16, "heads", 0),
    ([600, 11], 16, 1, 96, 128, F16, F16, "heads", 0),
    ([260, 19], 34, 2, 72, 24, BF16, BF16, "tokens", 0),
    ([400, 200], 12, 4, 256, 32, BF16, BF16, "heads", 0),
    ([401, 5], 9, 1, 192, 32, F16, F16, "both", 0),
    ([70, 300], 48, 1, 128, 16, BF16, BF16, "tokens", 0),
    ([350, 0, 20], 8, 8, 8, 16, BF16, BF16, "tokens", 0),
    ([700, 41, 64], 12, 12, 64, 32, BF16, E4M3, "heads", 0),
    ([513, 0, 100], 16, 2, 128, 16, F16, E4M3, "tokens", 0),
    ([300, 90], 20, 4, 256, 13, BF16, E4M3, "tokens", 0),
    ([129, 40], 5, 1, 80, 8, F16, E4M3, "both", 0),
    ([1000, 90, 100, 101, 0, 1], 4, 2, 64, 16, BF16, BF16, "tokens", 100),
    ([800, 7, 650], 16, 1, 96, 24, F16, F16, "heads", 1),
    ([900, 70], 6, 2, 128, 32, BF16, E4M3, "heads", 333),
    ([9000, 17], 4, 1, 64, 16, BF16, BF16, "tokens", 0),
    ([12345], 2, 2, 128, 64, F16, F16, "heads", 0),
]


@pytest.mark.parametrize("lengths, heads, kv, dim, page, dtype, to, order, window", ATTEND)
def test_attend(dev, lengths, heads, kv, dim, page, dtype, to, order, window):
    cache, q, table, length = _requests(dev, sum(lengths) + dim, lengths, heads, kv, dim, page, dtype, to, order, window=window)
    got = dev.cache_attend(cache, q, table.cuda(), length.cuda(), window=window)
    _check(got, _expect(cache, q, table, length, dim ** -0.5, window), q, max(lengths))


@pytest.mark.parametrize("lengths, heads, kv, dim, page, dtype, to, order, window", [c for c in ATTEND if max(c[0]) < 5000])
def test_attend_of_a_wide_table(dev, lengths, heads, kv, dim, page, dtype, to, order, window):
    """The same requests in a table that has room for long ones: other workgroups, the same result but for roundings."""
    cache, q, table, length = _requests(dev, sum(lengths) + dim, lengths, heads, kv, dim, page, dtype, to, order, window=window)
    wide = torch.full((len(lengths), -(-40000 // page)), -1, dtype=torch.int32)
    wide[:, :table.size(1)] = table
    got = dev.cache_attend(cache, q, wide.cuda(), length.cuda(), window=window)
    _check(got, _expect(cache, q, table, length, dim ** -0.5, window), q, max(lengths))


@pytest.mark.parametrize("requests, heads, kv, dim, dtype, to", [
    (300, 8, 8, 64, BF16, BF16), (40, 16, 2, 96, F16, F16), (150, 4, 4, 128, BF16, BF16), (2, 64, 2, 256, F16, F16), (37, 24, 1, 128, BF16, E4M3), (5, 3, 3, 256, F16, E4M3),
])
@pytest.mark.parametrize("longest", [31, 100, 300])
def test_attend_by_size(dev, requests, heads, kv, dim, dtype, to, longest):
    """From one wavefront to a segment to as many as a compute unit holds."""
    lengths = [int(v) for v in np.random.default_rng(longest + dim).integers(0, longest + 1, requests)] + [longest]
    cache, q, table, length = _requests(dev, longest, lengths, heads, kv, dim, 16, dtype, to, "tokens")
    _check(dev.cache_attend(cache, q, table.cuda(), length.cuda()), _expect(cache, q, table, length, dim ** -0.5), q, longest)


def test_attend_many_short_requests(dev):
    lengths = [int(v) for v in np.random.default_rng(5).integers(0, 90, 700)]
    cache, q, table, length = _requests(dev, 8, lengths, 4, 2, 64, 16, BF16, BF16, "tokens")
    _check(dev.cache_attend(cache, q, table.cuda(), length.cuda()), _expect(cache, q, table, length, 0.125), q, 90)


def test_attend_pages_that_are_not_there(dev):
    """Holes and ids outside the cache are left out, a row of nothing but those is empty, and a length beyond the table ends with it."""
    cache, q, table, length = _requests(dev, 9, [200, 90, 64, 300], 4, 2, 64, 16, BF16, BF16, "tokens")
    table[0, 3], table[0, 5], table[1, 0] = -1, cache.k.size(0), 2 ** 31 - 1
    table[2, :] = -2 ** 31
    length[3] = 2 ** 31 - 1
    table[3, -1] = -1
    length[1] = 90
    want = _expect(cache, q, table, length, 0.3)
    assert want[1][2, 0] == -np.inf
    _check(dev.cache_attend(cache, q, table.cuda(), length.cuda(), scale=0.3), want, q, 330)
    length[:] = torch.tensor([-1, -2 ** 31, 0, 0])
    out, lse = dev.cache_attend(cache, q, table.cuda(), length.cuda())
    assert (out == 0).all() and (lse == -math.inf).all()


def test_attend_extreme_scores(dev):
    """Scores far from one another and from zero, keys of -inf and of the type's lowest value, a row of nothing else, NaN where it is seen."""
    cache, q, table, length = _requests(dev, 10, [300, 200, 150, 100], 2, 2, 64, 16, BF16, BF16, "tokens")
    q.abs_().add_(0.01)
    k = cache.k
    k[table[0, 2].item(), 3] = -math.inf           # one token's keys: the score -inf
    k[table[1, :13].long().cuda()] = -math.inf      # all of a request's: its row is empty
    lowest = torch.finfo(BF16).min
    k[table[2, 1].item(), 2] = lowest
    k[table[2, 0].item(), 0] = 90.0                # over all others by some hundred
    k[table[3, 0].item(), 4, 1] = math.nan          # of the second head only
    want = _expect(cache, q, table, length, 0.125)
    out, lse = dev.cache_attend(cache, q, table.cuda(), length.cuda())
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all() and torch.isnan(out[3, 1]).all() and torch.isnan(lse[3, 1])
    _check((out[[0, 2]], lse[[0, 2]]), tuple(x[[0, 2]] for x in want), q[[0, 2]], 300)
    _check((out[3:, :1], lse[3:, :1]), tuple(x[3:, :1] for x in want), q[3:, :1], 300)


@pytest.mark.parametrize("heads, to", [(4, F16), (16, F16), (4, E4M3)])
def test_attend_many_small_weights_in_fp16(dev, heads, to):
    """One key's score is 17.5 over all others, whose weights are under half of fp16's smallest step: together they are the result, as that key's value is 0."""
    lengths, dim = [6000, 40], 64
    cache, q, table, length = _requests(dev, 14, lengths, heads, 1, dim, 16, F16, to, "tokens")
    q.fill_(1.0)
    by = 1.0 if to == F16 else cache.k_scale.item()
    for r, n in enumerate(lengths):
        for p in range(-(-n // 16)):
            cache.k[table[r, p], :min(16, n - 16 * p)] = 0
        at = table[r, 1].item()
        cache.k[at, 5] = 17.5 / 8 / by
        cache.v[at, 5] = 0
    _check(dev.cache_attend(cache, q, table.cuda(), length.cuda()), _expect(cache, q, table, length, dim ** -0.5), q, 6000)


def test_attend_strided_tensors(dev):
    """q inside a packed projection at an odd place, out inside a wider tensor, a table with rows further apart, no lse kept."""
    cache, q, table, length = _requests(dev, 11, [260, 45, 130], 8, 2, 80, 16, F16, F16, "heads")
    packed = torch.zeros((3, 11, 83), dtype=F16, device="cuda")
    inside = packed[:, 2:10, 1:81]
    inside.copy_(q)
    wide = torch.full((3, 10, 90), 3.0, dtype=F16, device="cuda")
    rows = torch.full((3, table.size(1) + 5), 2 ** 30, dtype=torch.int32, device="cuda")
    rows[:, 2:2 + table.size(1)] = table.cuda()
    out = wide[:, 1:9, 3:83]
    got = dev.cache_attend(cache, inside, rows[:, 2:2 + table.size(1)], length.cuda(), out=out)
    _check(got, _expect(cache, q, table, length, 80 ** -0.5), q, 260)
    out.fill_(3.0)
    assert (wide == 3.0).all()


def test_a_cache_past_32_bit_offsets(dev):
    """Pages whose rows begin past 2^31 elements and 2^32 bytes, written and read."""
    pages, page, kv, dim = 9300, 16, 128, 128   # 2.4e9 elements each
    k, v = (torch.empty((pages, page, kv, dim), dtype=BF16, device="cuda") for _ in range(2))
    cache = dev.PagedCache(k, v)
    g = torch.Generator().manual_seed(1)
    ids = [pages - 1, 0, 8200, pages - 2, 4100]
    lengths = [70, 5]
    table = torch.tensor([ids, [pages - 3] * 5], dtype=torch.int32)
    new = torch.randn((75, 2 * kv, dim), generator=g).to(BF16).cuda()
    at = [table[r, i // page].item() * page + i % page for r, n in enumerate(lengths) for i in range(n)]
    dev.cache_append(cache, new[:, :kv], new[:, kv:], torch.tensor(at, device="cuda"))
    q = torch.randn((2, kv, dim), generator=g).to(BF16).cuda()
    length = torch.tensor(lengths, dtype=torch.int32)
    got = dev.cache_attend(cache, q, table.cuda(), length.cuda())
    used = sorted({p for row in table.tolist() for p in row})
    small = dev.PagedCache(k[used], v[used])
    again = torch.tensor([[used.index(p) for p in row] for row in table.tolist()], dtype=torch.int32)
    for r, n in enumerate(lengths):
        for i in range(n, -(-n // page) * page):
            small.k[again[r, i // page], i % page] = 0   # (never written: not read by the oracle either, but it converts them)
            small.v[again[r, i // page], i % page] = 0
    for i, slot in enumerate(at):
        assert torch.equal(k[slot // page, slot % page], new[i, :kv]) and torch.equal(v[slot // page, slot % page], new[i, kv:])
    _check(got, _expect(small, q, again, length, dim ** -0.5), q, 70)


# ---- streams, graphs, and the step as a whole

def test_other_streams(dev):
    """A call on a stream of its own by argument, and by torch's current stream; what the call allocates is that stream's."""
    cache, q, table, length = _requests(dev, 12, [4000, 300], 8, 2, 64, 16, BF16, BF16, "tokens")
    table, length = table.cuda(), length.cuda()
    want = dev.cache_attend(cache, q, table, length)
    position, x = torch.arange(2, dtype=torch.int32, device="cuda"), q.clone()
    rope = dev.Rope(_frequencies((32,)))
    turned = dev.rotary(x, rope, position)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        got = dev.cache_attend(cache, q, table, length, stream=side.cuda_stream)
        y = dev.rotary(x, rope, position, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(y, turned)
        with torch.cuda.stream(side):
            got = dev.cache_attend(cache, q, table, length)
        side.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_step_in_a_graph(dev):
    """assign -> append -> attend captured once and replayed while the requests grow, each replay against the same step run eagerly."""
    n, kv, heads, dim, page, width = 5, 2, 4, 64, 4, 9
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((n * width + 3, page, kv, dim), generator=g).to(BF16).cuda() for _ in range(2))
    cache, rope = dev.PagedCache(k, v), dev.Rope(_frequencies((16, 16)), (16, 16))
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    cached, fresh = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda")
    pool = torch.randperm(n * width + 3, generator=g).int().cuda()
    free = pool.clone()
    qkv, out = torch.zeros((n, heads + 2 * kv, dim), dtype=BF16, device="cuda"), torch.zeros((n, heads, dim), dtype=BF16, device="cuda")
    lse, made = torch.zeros((n, heads), device="cuda"), dev.assigned_buffers(n, n)
    q_out = torch.empty((n, heads, dim), dtype=BF16, device="cuda")
    work = torch.empty(max(16, dev.attend_workspace(cache, heads, n, width)), dtype=torch.uint8, device="cuda")

    def step():
        a = dev.cache_assign(page, cached, fresh, table, free, n, out=made)
        dev.cache_append(cache, qkv[:, heads:heads + kv], qkv[:, heads + kv:], a.slot, rope, a.position, qkv[:, :heads], q_out)
        dev.cache_attend(cache, q_out, table, a.length, out=out, lse=lse, workspace=work)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    table.fill_(-1)
    for i in range(2 * page + 3):
        fresh.copy_(torch.tensor([1, 1, i % 2, 0, 1], dtype=torch.int32))
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        before = [t.clone() for t in (table, k, v)]
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (out, lse, table, k, v, *made)]
        for t, b in zip((table, k, v), before):
            t.copy_(b)
        for t in (out, lse, *made):
            t.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(replayed, (out, lse, table, k, v, *made)):
            assert torch.equal(a, b), i
        cached.copy_(made.length)
        rest = free[made.taken.item():].clone()
        free[:rest.numel()] = rest
    assert cached.tolist() == [11, 11, 5, 0, 11]


def test_refused_tensors(dev):
    """Types and shapes that do not fit, on the GPU."""
    cache, q, table, length = _requests(dev, 13, [40, 20], 4, 2, 64, 16, BF16, BF16, "tokens")
    t, n = table.cuda(), length.cuda()
    for call in (lambda: dev.cache_attend(cache, q[:, :3], t, n), lambda: dev.cache_attend(cache, q.half(), t, n), lambda: dev.cache_attend(cache, q, t.long(), n),
                 lambda: dev.cache_attend(cache, q, t, n[:1]), lambda: dev.cache_attend(cache, q[..., :32], t, n), lambda: dev.cache_attend(cache, q, t, n, out=q),
                 lambda: dev.cache_attend(cache, q, t, n, lse=torch.empty((2, 3), device="cuda")),
                 lambda: dev.rotary(q, dev.Rope(_frequencies((33,))), n), lambda: dev.rotary(q, dev.Rope(_frequencies((32,))), n[:1]),
                 lambda: dev.rotary(q, dev.Rope(_frequencies((16, 16)), (16, 16)), torch.zeros((3, 2), dtype=torch.int32, device="cuda")),
                 lambda: dev.cache_append(cache, q, q, torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: dev.cache_append(cache, q[:, :2], q[:, 2:], torch.zeros(3, dtype=torch.int64, device="cuda"))):
        with pytest.raises(B.AmapError):
            call()
