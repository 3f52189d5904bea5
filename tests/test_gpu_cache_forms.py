"""cache_attend over the sizes that decide which kernel takes a call and how it is cut: many requests to a lane of the shares' search, more requests than
workgroups, as many wavefronts to a segment as there are, more segments than a launch of one workgroup each can have.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache import BF16, E4M3, F16, _check, _expect, _f64, _requests

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2002_12798_amd import device
    device.require_gpu()
    return device


def _run(dev, seed, lengths, heads, kv, dim, page, dtype, to, order="tokens", width=None, window=0):
    """In a table of `width` entries a row, if it is wider than these requests need."""
    cache, q, table, length = _requests(dev, seed, lengths, heads, kv, dim, page, dtype, to, order, window=window)
    if width:
        wide = torch.full((len(lengths), width), -1, dtype=torch.int32)
        wide[:, :min(width, table.size(1))] = table[:, :width]
        table = wide
    got = dev.cache_attend(cache, q, table.cuda(), length.cuda(), window=window)
    again = dev.cache_attend(cache, q, table.cuda(), length.cuda(), window=window)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])   # nothing hangs on which workgroup comes first
    _check(got, _expect(cache, q, table, length, dim ** -0.5, window), q, max(lengths))


@pytest.mark.parametrize("requests", [64, 65, 128, 130, 321, 700])
@pytest.mark.parametrize("heads, kv, dim, dtype, to", [(4, 2, 64, BF16, BF16), (3, 3, 128, F16, E4M3)])
def test_shares_of_many_requests(dev, requests, heads, kv, dim, dtype, to):
    """Several requests to a lane of the search; at the ends of its runs requests that are empty, and one that is long."""
    rng, run = np.random.default_rng(requests), -(-requests // 64)
    lengths = [int(v) for v in rng.integers(0, 70, requests)]
    for i in range(0, requests, 3 * run):
        lengths[i] = 0
        lengths[i - 1] = 0
    lengths[run - 1], lengths[requests // 2], lengths[-1] = 1500, 900, 0
    _run(dev, requests, lengths, heads, kv, dim, 16, dtype, to, width=2500)


@pytest.mark.parametrize("some", [0, 1, 60])
def test_more_requests_than_workgroups(dev, some):
    """5000 requests, all but a few of them empty: more than 64 to a lane of the search, rows of nothing over all workgroups."""
    lengths = [0] * 5000
    for i, r in enumerate(np.random.default_rng(some).permutation(5000)[:some]):
        lengths[r] = 1 + 23 * i % 400
    lengths[4999] = lengths[0] = 33 if some else 0
    _run(dev, 5 + some, lengths, 4, 2, 64, 16, BF16, BF16, width=320)


@pytest.mark.parametrize("requests, heads, kv, dim, tokens, dtype, to", [
    (32, 8, 8, 64, 4096, BF16, E4M3),      # 13 wavefronts to a segment
    (32, 8, 8, 64, 3000, F16, E4M3),       # 10
    (32, 8, 8, 64, 2048, BF16, BF16),      # 7
    (32, 16, 8, 64, 1856, F16, F16),       # 6
    (32, 8, 8, 64, 1600, BF16, BF16),      # 5
    (32, 8, 8, 128, 1024, BF16, E4M3),     # 4
    (26, 20, 10, 96, 1300, F16, F16),      # 6, or as many as fit
])
def test_many_wavefronts_to_a_segment(dev, requests, heads, kv, dim, tokens, dtype, to):
    """The table says how many: requests that fill it, that end inside the last wavefront's first tile or before it, and none."""
    lengths = [tokens, 1, 0, tokens - 1, tokens // 2 + 1, 33, 320, 321, 319] + [int(v) for v in np.random.default_rng(tokens).integers(0, 90, requests - 9)]
    _run(dev, tokens + dim, lengths, heads, kv, dim, 16, dtype, to, width=-(-tokens // 16))


def test_more_segments_than_one_launch_takes(dev):
    """Over four million segments, of one token or none: the value itself and its score."""
    requests, kv, dim = 530000, 8, 8
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn((1000, 16, kv, dim), generator=g).to(BF16).cuda() for _ in range(2))
    q = torch.randn((requests, kv, dim), generator=g).to(BF16).cuda()
    table = torch.randint(0, 1000, (requests, 1), generator=g, dtype=torch.int32).cuda()
    length = torch.randint(0, 2, (requests,), generator=g, dtype=torch.int32).cuda()
    out, lse = dev.cache_attend(dev.PagedCache(k, v), q, table, length, scale=0.5)
    first, seen = table[:, 0].long(), length == 1
    assert torch.equal(out[seen], v[first[seen], 0]) and (out[~seen] == 0).all() and (lse[~seen] == -np.inf).all()
    products = q[seen].double() * k[first[seen], 0].double()
    # (dim products in 32 bits and one by the scale; into powers of two and out of them, two roundings each)
    far = (lse[seen].double() - 0.5 * products.sum(-1)).abs() - ((dim + 6) * 2.0 ** -24 * 0.5 * products.abs().sum(-1) + 2.0 ** -40)
    assert (far <= 0).all(), far.max().item()
