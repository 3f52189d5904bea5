"""Tensors of a call around the paged cache that have elements in common, where one is written: refused.  Tensors that only lie between one another's rows: taken."""
import os
import subprocess

import pytest
import torch

from paper_2002_12798_amd import binding as B
from tests.test_cache_args import AT, _cache, _refuses, _rope, _rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_whether_tensors_share_an_element(tmp_path):
    """The host's answer against every byte, built with the host's compiler."""
    exe = str(tmp_path / "overlap_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2002_12798_amd", "csrc"), os.path.join(ROOT, "tests", "overlap_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


# [10 tokens, 8 heads, 64] of 2 bytes: q, k and v are heads of it
HEAD, TOKEN = 128, 512


@pytest.mark.parametrize("q, heads, k, v", [
    (0, 2, 0, 6),      # q is k
    (0, 3, 2, 6),      # one head of q is k's first
    (3, 2, 2, 6),      # and k's last
    (2, 4, 0, 4),      # the same for v
    (0, 8, 0, 6),      # all of them
])
def test_queries_turned_in_place_over_keys_or_values(q, heads, k, v):
    at = lambda h, n: _rows(6 * AT + HEAD * h, heads=n, token=TOKEN)  # noqa: E731
    _refuses(B.AMAP_E_ALIAS, B.amap_cache_append, _cache(), at(k, 2), at(v, 2), 10, 7 * AT, _rope(), 7 * AT, 0, at(q, heads), at(q, heads))


@pytest.mark.parametrize("more", [dict(token=500), dict(token=TOKEN, head=68), dict(token=TOKEN)])
def test_queries_turned_in_place_between_other_strides(more):
    """Strides that differ from the keys' are not looked into, and a projection whose rows begin half a head off has elements in common."""
    off = 64 if more == dict(token=TOKEN) else 0
    q = _rows(6 * AT + off, heads=2, **more)
    _refuses(B.AMAP_E_ALIAS, B.amap_cache_append, _cache(), _rows(6 * AT + HEAD, token=TOKEN), _rows(5 * AT), 10, 7 * AT, _rope(), 7 * AT, 0, q, q)


def test_what_attend_writes():
    """Caches of 8 pages, 4 requests in a table of 8 entries a row 10 apart, 2 heads of 64: out, lse and the workspace each within one another and whatever is read."""
    need = B.amap_cache_attend_workspace(_cache(), 2, 4, 8)
    size = dict(k=2 * 2048 * 8, v=2 * 2048 * 8, q=2 * 128 * 4, table=4 * 38, length=16, out=2 * 128 * 4, lse=4 * 8, work=need)
    at = {n: (i + 2) * AT for i, n in enumerate(size)}

    def call(at, type=B.AMAP_BF16, **over):
        B.amap_cache_attend(_cache(k=at["k"], v=at["v"], type=type, **over), _rows(at["q"]), 4, at["table"], 10, 8, at["length"], 0.1, 0, _rows(at["out"]), at["lse"], at["work"], need)

    for n in ("out", "lse", "work"):
        for m in size:
            if m != n:   # (the workspace begins at a multiple of 16; out at its first element)
                for x in (at[m] + (size[m] - 4) // 16 * 16, at[m] - (size[n] - 4) // 16 * 16):
                    _refuses(B.AMAP_E_ALIAS, call, {**at, n: x})
        for scale in ("k_scale", "v_scale"):
            _refuses(B.AMAP_E_ALIAS, lambda: call({**at, n: 12 * AT}, B.AMAP_E4M3, **{scale: 12 * AT}))
    _refuses(B.AMAP_E_SHAPE, lambda: B.amap_cache_attend(_cache(), _rows(3 * AT), 1 << 29, 4 * AT, 1 << 40, 8, 5 * AT, 0.1, 0, _rows(6 * AT), None, 7 * AT, 1 << 40))


# keys and values in one buffer; 8 pages of 16 tokens, 2 heads of 64, 2 bytes
@pytest.mark.parametrize("over", [
    dict(v=AT + 2 * 64),                                                          # the second head of the keys is the first of the values
    dict(v=AT + 2 * 2048), dict(v=AT - 2 * 2048 * 7),                             # a page later; the keys' first page is the values' last
    dict(v=AT + 2 * 128 * 15), dict(v=AT + 2), dict(k=2 * AT + 126),
    dict(v=AT + 2 * 64, token_stride=256, page_stride=4096, head_stride=64),      # a token's heads beside one another, half of them in common
    dict(v=AT + 2 * 2048, page_stride=64, token_stride=512, head_stride=8192),    # heads outermost
])
def test_keys_and_values_of_one_buffer_that_overlap(over):
    _refuses(B.AMAP_E_ALIAS, B.amap_cache_append, _cache(**over), _rows(5 * AT), _rows(6 * AT), 10, 7 * AT)


@pytest.mark.gpu
def test_keys_and_values_of_one_buffer():
    """A token's keys beside its values, head by head or all of them, and whole pages of either: no element in common."""
    from paper_2002_12798_amd import device
    x = torch.randn((20, 4, 64)).half().cuda()
    slot = torch.randperm(48)[:20].cuda()
    for shape, k, v in (((3, 16, 2, 2, 64), lambda t: t[:, :, :, 0], lambda t: t[:, :, :, 1]), ((3, 16, 4, 64), lambda t: t[:, :, :2], lambda t: t[:, :, 2:]),
                        ((3, 2, 16, 2, 64), lambda t: t[:, 1], lambda t: t[:, 0]), ((6, 16, 2, 64), lambda t: t[3:], lambda t: t[:3])):
        buffer = torch.zeros(shape, dtype=torch.float16, device="cuda")
        device.cache_append(device.PagedCache(k(buffer), v(buffer)), x[:, :2], x[:, 2:], slot)
        assert torch.equal(k(buffer)[slot // 16, slot % 16], x[:, :2]) and torch.equal(v(buffer)[slot // 16, slot % 16], x[:, 2:])
        assert buffer.count_nonzero() == x.count_nonzero()


@pytest.mark.gpu
def test_queries_turned_in_place_beside_keys_and_values():
    """What is beside k and v, in front of them, between them or behind them, is taken and gives what a call into a tensor of its own gives."""
    from paper_2002_12798_amd import device
    g = torch.Generator().manual_seed(4)
    packed = torch.randn((33, 9, 64), generator=g).bfloat16().cuda()
    rope, position = device.Rope(torch.rand(32, generator=g).cuda()), torch.arange(33, dtype=torch.int32, device="cuda")
    slot = torch.randperm(48, generator=g)[:33].cuda()
    for q, heads, k, v in ((0, 5, 5, 7), (2, 5, 0, 7), (4, 5, 0, 2), (8, 1, 5, 2)):
        caches = [[torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
        want = device.cache_append(device.PagedCache(*caches[0]), packed[:, k:k + 2], packed[:, v:v + 2], slot, rope, position, packed[:, q:q + heads])
        x = packed.clone()
        part = x[:, q:q + heads]
        assert device.cache_append(device.PagedCache(*caches[1]), x[:, k:k + 2], x[:, v:v + 2], slot, rope, position, part, part) is part
        assert torch.equal(part, want) and torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])
        part.copy_(packed[:, q:q + heads])
        assert torch.equal(x, packed)


@pytest.mark.gpu
def test_outputs_beside_their_inputs():
    """Heads of one projection turned into, or attended into, other heads of it; the rest of it stays.  Outputs that share a head or part of one are refused."""
    from paper_2002_12798_amd import device
    g = torch.Generator().manual_seed(5)
    packed = torch.randn((21, 10, 64), generator=g).half().cuda()
    rope, position = device.Rope(torch.rand(32, generator=g).cuda()), torch.arange(21, dtype=torch.int32, device="cuda")
    k, v = (torch.randn((9, 16, 2, 64), generator=g).half().cuda() for _ in range(2))
    cache, table = device.PagedCache(k, v), torch.randint(0, 9, (21, 4), generator=g, dtype=torch.int32).cuda()
    length = torch.randint(0, 65, (21,), generator=g, dtype=torch.int32).cuda()
    calls = (lambda x, out: device.rotary(x, rope, position, out=out), lambda x, out: device.cache_attend(cache, x, table, length, out=out)[0],
             lambda x, out: device.cache_append(cache, packed[:, 8:], packed[:, 8:], torch.full((21,), -1, device="cuda"), rope, position, x, out))
    for call in calls:
        for of, to in ((0, 4), (4, 0), (2, 6), (0, 6)):
            x = packed.clone()
            want = call(x[:, of:of + 4].contiguous(), torch.empty((21, 4, 64), dtype=x.dtype, device="cuda"))
            call(x[:, of:of + 4], x[:, to:to + 4])
            assert torch.equal(x[:, to:to + 4], want)
            x[:, to:to + 4] = packed[:, to:to + 4]
            assert torch.equal(x, packed)
        for of, to in ((0, 3), (3, 0), (1, 2)):
            with pytest.raises(B.AmapError) as e:
                call(packed[:, of:of + 4], packed[:, to:to + 4])
            assert e.value.status == B.AMAP_E_ALIAS
        with pytest.raises(B.AmapError) as e:
            call(packed[:, :4, :], packed.view(-1)[4 * 64 - 2:].as_strided((21, 4, 64), packed.stride()))
        assert e.value.status == B.AMAP_E_ALIAS
