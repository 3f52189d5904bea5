"""The entry points around the paged cache refuse what does not fit before anything is launched (no GPU: the addresses are never read)."""
import ctypes as C

import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device

AT = 1 << 40


def _cache(**over):
    c = dict(k=AT, v=2 * AT, type=B.AMAP_BF16, n_pages=8, page_size=16, kv_heads=2, head_dim=64, page_stride=2048, token_stride=128, head_stride=64,
             k_scale=None, v_scale=None)
    c.update(over)
    return B.amap_cache(*[c[n] for n, _ in B.amap_cache._fields_])


def _rows(at=3 * AT, type=B.AMAP_BF16, heads=2, token=None, head=64):
    return B.amap_heads(at, type, heads, heads * head if token is None else token, head)


def _rope(pairs=32, axes=(32,), freq=4 * AT, interleaved=0):
    return B.amap_rope(freq, pairs, interleaved, len(axes), (C.c_int32 * 4)(*axes[:4]))


def _refuses(status, f, *a):
    with pytest.raises(B.AmapError) as e:
        f(*a)
    assert e.value.status == status, str(e.value)
    return str(e.value)


def _assign(**over):
    a = dict(requests=4, page_size=16, cached=AT, fresh=AT, free_pages=AT, n_free=9, table=AT, table_stride=8, table_width=8, begin=AT, length=AT, slot=AT,
             position=AT, owner=AT, n_tokens=32, taken=AT)
    a.update(over)
    return B.amap_assign(*[a[n] for n, _ in B.amap_assign._fields_])


@pytest.mark.parametrize("over, status", [
    (dict(page_size=0), B.AMAP_E_INVALID), (dict(requests=-1), B.AMAP_E_INVALID), (dict(fresh=None), B.AMAP_E_INVALID), (dict(slot=None), B.AMAP_E_INVALID),
    (dict(taken=None), B.AMAP_E_INVALID), (dict(free_pages=None), B.AMAP_E_INVALID), (dict(n_tokens=-1), B.AMAP_E_INVALID), (dict(table=None), B.AMAP_E_INVALID),
    (dict(table_stride=7), B.AMAP_E_SHAPE), (dict(n_tokens=1 << 31), B.AMAP_E_SHAPE), (dict(requests=16385), B.AMAP_E_UNSUPPORTED),
])
def test_assign(over, status):
    said = _refuses(status, B.amap_cache_assign, _assign(**over))
    assert status != B.AMAP_E_UNSUPPORTED or "16384" in said


def test_assign_to_arrays_that_overlap():
    """4 requests, 9 free pages, 32 tokens, a table of 4 rows of 8: every array a page apart, then one of those written within another."""
    names = ["cached", "fresh", "free_pages", "table", "begin", "length", "slot", "position", "owner", "taken"]
    size = dict(cached=16, fresh=16, free_pages=36, table=128, begin=20, length=16, slot=256, position=128, owner=128, taken=4)
    at = {n: AT + 4096 * i for i, n in enumerate(names)}
    for i, n in enumerate(names[3:]):
        for m in names:
            if m != n:
                _refuses(B.AMAP_E_ALIAS, B.amap_cache_assign, _assign(**{**at, n: at[m] + size[m] - 4}))
                _refuses(B.AMAP_E_ALIAS, B.amap_cache_assign, _assign(**{**at, n: at[m] - size[n] + 4}))


@pytest.mark.parametrize("x, out, dim, rope, position, status", [
    (_rows(), _rows(5 * AT), 64, _rope(33, (33,)), AT, B.AMAP_E_SHAPE),                       # more pairs than halves
    (_rows(), _rows(5 * AT), 64, _rope(32, (16, 15)), AT, B.AMAP_E_SHAPE),                    # axes that do not add up
    (_rows(), _rows(5 * AT), 64, _rope(32, (32,), None), AT, B.AMAP_E_INVALID),
    (_rows(), _rows(5 * AT), 64, _rope(0, (0,)), AT, B.AMAP_E_INVALID),
    (_rows(), _rows(5 * AT), 64, _rope(32, (64, -32)), AT, B.AMAP_E_INVALID),
    (_rows(), _rows(5 * AT), 64, _rope(), None, B.AMAP_E_INVALID),
    (_rows(), _rows(5 * AT, B.AMAP_F16), 64, _rope(), AT, B.AMAP_E_INVALID),
    (_rows(type=B.AMAP_E4M3), _rows(5 * AT, B.AMAP_E4M3), 64, _rope(), AT, B.AMAP_E_INVALID),
    (_rows(), _rows(5 * AT, heads=3), 64, _rope(), AT, B.AMAP_E_SHAPE),
    (_rows(), _rows(5 * AT, token=64), 64, _rope(), AT, B.AMAP_E_SHAPE),                      # rows of out over one another
    (_rows(), _rows(5 * AT, head=0), 64, _rope(), AT, B.AMAP_E_SHAPE),
    (_rows(), _rows(token=-128), 64, _rope(), AT, B.AMAP_E_SHAPE),
    (_rows(), _rows(3 * AT + 2), 64, _rope(), AT, B.AMAP_E_ALIAS),
    (_rows(), _rows(3 * AT, token=256), 64, _rope(), AT, B.AMAP_E_ALIAS),
    (_rows(3 * AT + 1), _rows(5 * AT), 64, _rope(), AT, B.AMAP_E_UNSUPPORTED),
    (_rows(3 * AT + 2), _rows(5 * AT), 64, _rope(interleaved=1), AT, B.AMAP_E_UNSUPPORTED),   # pairs across two accesses
    (_rows(head=4096), _rows(5 * AT, head=4096), 4096, _rope(), AT, B.AMAP_E_UNSUPPORTED),
    (_rows(token=1 << 60), _rows(5 * AT), 64, _rope(), AT, B.AMAP_E_SHAPE),
])
def test_rotary(x, out, dim, rope, position, status):
    _refuses(status, B.amap_rotary, x, out, 10, dim, rope, position, 0)


def test_no_tokens_is_no_call():
    B.amap_rotary(_rows(), _rows(5 * AT), 0, 64, _rope(), None, 0)
    B.amap_cache_append(_cache(), _rows(), _rows(5 * AT), 0, None)
    B.amap_cache_attend(_cache(), _rows(), 0, None, 0, 4, None, 0.1, 0, _rows(5 * AT), None, None, 0)


CACHES = [
    (dict(k=None), B.AMAP_E_INVALID), (dict(v=AT), B.AMAP_E_INVALID), (dict(type=B.AMAP_F32), B.AMAP_E_INVALID), (dict(n_pages=0), B.AMAP_E_INVALID),
    (dict(k_scale=AT), B.AMAP_E_INVALID), (dict(head_stride=32), B.AMAP_E_SHAPE), (dict(page_stride=1024), B.AMAP_E_SHAPE), (dict(n_pages=1 << 31), B.AMAP_E_SHAPE),
    (dict(page_stride=1 << 62), B.AMAP_E_SHAPE),
]


@pytest.mark.parametrize("over, status", CACHES)
def test_caches(over, status):
    c = _cache(**over)
    _refuses(status, B.amap_cache_append, c, _rows(), _rows(5 * AT), 10, AT)
    _refuses(status, B.amap_cache_attend, c, _rows(), 4, AT, 8, 8, AT, 0.1, 0, _rows(5 * AT), None, None, 0)
    _refuses(status, B.amap_cache_attend_workspace, c, 2, 4, 8)


@pytest.mark.parametrize("k, v, slot, rope, q, q_out, status", [
    (_rows(), _rows(5 * AT), None, None, None, None, B.AMAP_E_INVALID),
    (_rows(), _rows(5 * AT, B.AMAP_F16), AT, None, None, None, B.AMAP_E_INVALID),
    (_rows(heads=3), _rows(5 * AT), AT, None, None, None, B.AMAP_E_SHAPE),
    (_rows(), _rows(5 * AT), AT, None, _rows(6 * AT), _rows(7 * AT), B.AMAP_E_INVALID),        # q without a rope
    (_rows(), _rows(5 * AT), AT, _rope(), _rows(6 * AT), None, B.AMAP_E_INVALID),
    (_rows(), _rows(5 * AT), AT, _rope(), _rows(6 * AT, B.AMAP_F16), _rows(7 * AT, B.AMAP_F16), B.AMAP_E_INVALID),
    (_rows(AT + 64), _rows(5 * AT), AT, None, None, None, B.AMAP_E_ALIAS),
    (_rows(), _rows(5 * AT), AT, _rope(), _rows(6 * AT), _rows(2 * AT + 64), B.AMAP_E_ALIAS),
    (_rows(), _rows(5 * AT), AT, _rope(), _rows(6 * AT), _rows(5 * AT), B.AMAP_E_ALIAS),
])
def test_append(k, v, slot, rope, q, q_out, status):
    _refuses(status, B.amap_cache_append, _cache(), k, v, 10, slot, rope, AT, 0, q, q_out)


@pytest.mark.parametrize("over, args, status", [
    ({}, dict(heads=3), B.AMAP_E_SHAPE), ({}, dict(type=B.AMAP_F16), B.AMAP_E_INVALID), ({}, dict(type=B.AMAP_F32), B.AMAP_E_INVALID),
    ({}, dict(length=None), B.AMAP_E_INVALID), ({}, dict(table=None), B.AMAP_E_INVALID), ({}, dict(scale=float("nan")), B.AMAP_E_INVALID),
    ({}, dict(window=-1), B.AMAP_E_INVALID), ({}, dict(table_stride=-8), B.AMAP_E_SHAPE), ({}, {}, B.AMAP_E_INVALID), ({}, dict(out=3 * AT), B.AMAP_E_ALIAS), ({}, dict(out=AT), B.AMAP_E_ALIAS),
    ({}, dict(width=1 << 28, table_stride=1 << 28), B.AMAP_E_SHAPE), ({}, dict(requests=1 << 31), B.AMAP_E_SHAPE),
    (dict(head_dim=60), {}, B.AMAP_E_UNSUPPORTED), (dict(head_dim=264, head_stride=264, token_stride=528, page_stride=8448), {}, B.AMAP_E_UNSUPPORTED),
    (dict(token_stride=132), {}, B.AMAP_E_SHAPE), (dict(token_stride=132, page_stride=4096), {}, B.AMAP_E_UNSUPPORTED), (dict(k=AT + 8), {}, B.AMAP_E_UNSUPPORTED), (dict(type=B.AMAP_E4M3, head_dim=56), {}, B.AMAP_E_UNSUPPORTED),
])
def test_attend(over, args, status):
    a = dict(heads=2, type=B.AMAP_BF16, length=AT, table=AT, scale=0.1, window=0, table_stride=8, width=8, out=5 * AT, requests=4)
    a.update(args)
    _refuses(status, B.amap_cache_attend, _cache(**over), _rows(heads=a["heads"], type=a["type"]), a["requests"], a["table"], a["table_stride"], a["width"],
             a["length"], a["scale"], a["window"], _rows(a["out"], a["type"], a["heads"]), None, None, 0)


def test_what_workspace_a_call_takes():
    """None where no request can be longer than one tile; more for more workgroups, up to the chip's; 16-byte aligned."""
    room = lambda requests, width, **over: B.amap_cache_attend_workspace(_cache(**over), 2, requests, width)  # noqa: E731
    assert room(4, 2) == 0 and room(0, 100) == 0 and room(4, 0) == 0
    assert 0 < room(4, 8) < room(64, 8) <= room(64, 1 << 20) == room(1024, 1 << 20) - 8 * 2 * 960
    _refuses(B.AMAP_E_UNSUPPORTED, room, 1 << 20, 1 << 22)
    c, need = _cache(), room(4, 8)
    for at, size, status in ((None, 0, B.AMAP_E_INVALID), (6 * AT, need - 1, B.AMAP_E_INVALID), (6 * AT + 8, need, B.AMAP_E_UNSUPPORTED)):
        _refuses(status, B.amap_cache_attend, c, _rows(), 4, AT, 8, 8, AT, 0.1, 0, _rows(5 * AT), None, at, size)


def test_tensors_that_are_not_on_the_gpu():
    x, i, long = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: device.Rope(torch.zeros(32)), lambda: device.PagedCache(x[None], x[None]), lambda: device.rotary(x, None, i),
                 lambda: device.cache_assign(16, i, i, torch.zeros((4, 2), dtype=torch.int32), i, 4)):
        assert "not on the GPU" in _refuses(B.AMAP_E_INVALID, call)
    for call in (lambda: device.Rope([1.0]), lambda: device.PagedCache(x.float()[None], x.float()[None]), lambda: device.rotary(long, None, i),
                 lambda: device.cache_assign(16, i, long, i, i, 4)):
        _refuses(B.AMAP_E_INVALID, call)
