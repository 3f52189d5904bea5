"""Calls of cache_attend that threads issue on one cache and one stream: the workspace that the cache keeps is one call's own from its first launch to its last."""
import contextlib
import ctypes as C
import threading

import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device

ATTEND = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_float, C.c_int, C.c_void_p, C.c_void_p,
                     C.c_void_p, C.c_int64, C.c_void_p)


def test_the_way_through_ctypes_shows_a_workspace_behind_its_launches(monkeypatch):
    """On the CPU, the library's call replaced: while it runs no other thread may find the workspace that it was given."""
    seen = []
    monkeypatch.setattr(device, "_on_gpu", lambda t, *a: t)
    monkeypatch.setattr(device, "_native_attend", lambda *a: None)
    monkeypatch.setattr(device, "_made_on", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(device, "current_stream", lambda: 7)
    monkeypatch.setattr(device, "_capturing", lambda: False)
    monkeypatch.setattr(B, "amap_cache_attend", lambda *a: seen.append((a[11], {s: w.data_ptr() for s, w in cache._work.items()})))
    k, v = (torch.zeros((64, 16, 1, 64), dtype=torch.bfloat16) for _ in range(2))
    cache, q = device.PagedCache(k, v), torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    device.cache_attend(cache, q, torch.zeros((1, 64), dtype=torch.int32), torch.ones(1, dtype=torch.int32))
    (used, found), = seen
    assert used and used not in found.values() and cache._work[7].data_ptr() == used


def _requests(n, longest, pages, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((n, 8, 64), generator=g).bfloat16().cuda()
    table = torch.randint(0, pages, (n, -(-longest // 16)), generator=g, dtype=torch.int32).cuda()
    return q, table, torch.randint(1, longest + 1, (n,), generator=g, dtype=torch.int32).cuda()


@pytest.mark.gpu
def test_a_call_takes_the_kept_workspace_out():
    """The library's call replaced by one in which another call on the same cache and stream is made, as another thread's could be: that one has a workspace of its own."""
    k, v = (torch.randn((300, 16, 2, 64)).bfloat16().cuda() for _ in range(2))
    cache, (q, table, length) = device.PagedCache(k, v), _requests(2, 4000, 300, 1)
    want = device.cache_attend(cache, q, table, length)   # (makes the workspace that is kept)
    torch.cuda.synchronize()
    here = device.current_stream()
    kept, seen, got = cache._work[here], [], []

    @ATTEND
    def call(*a):
        seen.append((a[11], here in cache._work))
        with pytest.MonkeyPatch.context() as m:
            m.setattr(B, "amap_cache_attend", lambda *b: seen.append((b[11], here in cache._work)))
            device.cache_attend(cache, q, table, length)
        return 0

    at = [C.cast(getattr(B._L, name), C.c_void_p).value for name in ("amap_cache_assign", "amap_rotary", "amap_cache_append")]
    rest = (device.Assigned, device._raw_stream, device._get_device, torch.cuda.is_initialized, device._capturing)
    device._native.library(*at, C.cast(call, C.c_void_p).value, C.cast(B._L.amap_cache_attend_workspace, C.c_void_p).value, *rest)
    try:
        device.cache_attend(cache, q, table, length)
    finally:
        device._native_calls()
    assert len(seen) == 2 and seen[0] == (kept.data_ptr(), False) and seen[1][0] not in (None, kept.data_ptr()) and not seen[1][1]
    assert cache._work[here] is kept
    # an error on the way (lse of a wrong size) and a refusal put it back as well
    for more in (dict(lse=torch.empty((1, 8), device="cuda"), out=torch.empty_like(q)), dict(out=q)):
        with pytest.raises(B.AmapError):
            device.cache_attend(cache, q, table, length, **more)
        assert cache._work[here] is kept
    got = device.cache_attend(cache, q, table, length)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_threads_on_one_stream():
    """Calls of different sizes from four threads, on one cache and on the default stream that they share: each gives what it gives by itself."""
    k, v = (torch.randn((300, 16, 2, 64)).bfloat16().cuda() for _ in range(2))
    cache = device.PagedCache(k, v)
    calls = [_requests(n, longest, 300, n) for n, longest in ((1, 4700), (70, 3000), (3, 2000), (130, 1500))]
    want = [device.cache_attend(device.PagedCache(k, v), *c) for c in calls]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(len(calls))

    def work(i):
        start.wait()
        for _ in range(200):
            out, lse = device.cache_attend(cache, *calls[i])
            if not (torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])):
                wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong
