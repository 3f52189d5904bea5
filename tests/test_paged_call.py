"""The native way from a Python call to the operators around the paged cache (_amap_paged_call): what it does not take, and that it gives what the way
through ctypes gives."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import build, device

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_it_is_built_for_this_torch():
    from paper_2002_12798_amd import _amap_paged_call as calls
    assert calls.torch_version == torch.__version__ and os.path.realpath(calls.__file__) == os.path.realpath(build.PAGED_CALL)
    assert device._native is calls


def test_calls_that_are_not_taken():
    """Tensors that are not on the GPU, other types, ranks and objects, no arguments: none reaches the library, none raises."""
    x, i = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    calls = device._native
    for a in ((), (1,), (x, None, i, x, False, 0), (x, 7, i, None, False, None), (None,) * 6, ("x",) * 6, (x, object(), i, x, 0, 0)):
        assert calls.rotary(*a) is None
    for a in ((), (None,) * 9, (object(), x, x, i, None, None, None, None, 0)):
        assert calls.append(*a) is None
    for a in ((), (None,) * 10, (object(), x, i[None], i, None, 0, x, x, None, 0), (object(), x, i[None], i, 1, -1, x, x, None, 0)):
        assert calls.attend(*a) is None
    for a in ((), (None,) * 8, (16, i, i, i[None], i, 4, None, 0), (0, i, i, i[None], i, 4, None, 0), (1 << 70, i, i, i[None], i, 4, None, 0)):
        assert calls.assign(*a) is None


def test_an_interrupt_passes_through():
    class Cache:
        @property
        def _cache_at(self):
            raise KeyboardInterrupt

    # (asked for only after the tensors have been looked at, which are not on the GPU here: not reached)
    assert device._native.append(Cache(), *(torch.zeros((1, 1, 8)),) * 2, torch.zeros(1, dtype=torch.int64), None, None, None, None, 0) is None


WITHOUT = """
import sys
sys.modules["paper_2002_12798_amd._amap_paged_call"] = None
from paper_2002_12798_amd import device
assert device._native is device._NoCalls and device._native.rotary(1, 2) is None
"""


def test_without_the_extension():
    r = subprocess.run([sys.executable, "-W", "always", "-c", WITHOUT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "around the paged cache go through ctypes" in r.stderr, r.stderr


def test_a_build_that_lacks_something(monkeypatch, tmp_path, capfd):
    """A compiler that is not there, or does not take it: said, an old one removed, nothing raised."""
    monkeypatch.setattr(build, "PAGED_CALL", str(tmp_path / "_amap_paged_call.x.so"))
    (tmp_path / "_amap_paged_call.x.so").write_bytes(b"old")
    monkeypatch.setattr(build.shutil, "which", lambda name: None)
    assert build.build_paged_call() is None and not os.path.exists(build.PAGED_CALL)
    monkeypatch.undo()
    monkeypatch.setattr(build, "PAGED_CALL", str(tmp_path / "_amap_paged_call.x.so"))
    monkeypatch.setattr(build, "CSRC", str(tmp_path))   # (no source there)
    assert build.build_paged_call() is None and capfd.readouterr().err.count("through ctypes") == 2


# ---- on the GPU: the two ways side by side

def _both(monkeypatch, f):
    native = f()
    with monkeypatch.context() as m:
        for name in ("assign", "rotary", "append", "attend"):
            m.setattr(device, "_native_" + name, lambda *a: None)
        plain = f()
    torch.cuda.synchronize()
    for a, b in zip(native, plain):
        assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride() and torch.equal(a.float().nan_to_num(7e9), b.float().nan_to_num(7e9))
    return native


@pytest.mark.gpu
def test_both_ways_give_the_same(monkeypatch):
    g = torch.Generator().manual_seed(1)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v = (torch.randn((40, 16, 2, 64), generator=g).bfloat16().cuda() for _ in range(2))
    cache, rope = device.PagedCache(k, v), device.Rope(torch.rand(32, generator=g).cuda(), (20, 12))
    x = torch.randn((9, 8, 64), generator=g).bfloat16().cuda()
    position = torch.randint(0, 900, (2, 9), generator=g, dtype=torch.int32).cuda()

    def assign():
        table = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
        table[:, 0] = i32(7, 8, 9)
        return [table, *device.cache_assign(16, i32(3, 16, 9), i32(40, 1, 0), table, torch.arange(20, 40, dtype=torch.int32, device="cuda"), 44)]

    made = _both(monkeypatch, assign)
    slot = made[3][:9].contiguous()
    _both(monkeypatch, lambda: [device.rotary(x, rope, position), device.rotary(x[:, 1:5], rope, position[0], out=torch.zeros((9, 4, 64), dtype=x.dtype, device="cuda"), inverse=True)])
    _both(monkeypatch, lambda: [device.cache_append(cache, x[:, :2], x[:, 2:4], slot, rope, position, x[:, 4:]), k, v])
    _both(monkeypatch, lambda: [torch.zeros(1) if device.cache_append(cache, x[:, :2], x[:, 2:4], slot) is None else None, k, v])
    table = torch.arange(36, dtype=torch.int32, device="cuda").view(3, 12)
    for more in (dict(), dict(scale=0.3), dict(window=20), dict(out=torch.zeros((3, 8, 64), dtype=x.dtype, device="cuda"), lse=torch.zeros((3, 8), device="cuda")),
                 dict(workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))):
        _both(monkeypatch, lambda: device.cache_attend(cache, x[:3], table, i32(190, 0, 33), **more))
        _both(monkeypatch, lambda: device.cache_attend(cache, x[:3].view(torch.int16), table, i32(190, 0, 33)))
    with pytest.raises(B.AmapError) as e:   # the library's refusal, by the native way
        device.rotary(x, device.Rope(torch.rand(33).cuda()), position[0])
    assert e.value.status == B.AMAP_E_SHAPE
    with pytest.raises(B.AmapError):
        device.cache_attend(cache, x[:3], table, i32(1, 2, 3), out=x[:3])


@pytest.mark.gpu
def test_outputs_of_one_allocation():
    """What a call makes is as a user would make it: contiguous, of its own type, apart, without a gradient; odd sizes, no requests and no tokens among them."""
    k, v = (torch.randn((8, 16, 3, 40)).half().cuda() for _ in range(2))
    cache = device.PagedCache(k, v)
    for n in (0, 1, 3):
        q = torch.randn((n, 3, 40)).half().cuda().requires_grad_()
        table, length = torch.arange(2 * n, dtype=torch.int32, device="cuda").view(n, 2), torch.full((n,), 20, dtype=torch.int32, device="cuda")
        out, lse = device.cache_attend(cache, q, table, length)
        given = torch.empty_like(out), torch.empty((n, 3), device="cuda")
        device.cache_attend(cache, q, table, length, out=given[0], lse=given[1])
        for got, want in zip((out, lse), given):
            assert got.shape == want.shape and got.dtype == want.dtype and got.is_contiguous() and not got.requires_grad and torch.equal(got, want)
        before = lse.clone()
        out.zero_()
        assert torch.equal(lse, before)
    fresh, free = torch.tensor([3, 0], dtype=torch.int32, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    for tokens in (0, 3, 5):
        a = device.cache_assign(2, None, fresh, torch.full((2, 2), -1, dtype=torch.int32, device="cuda"), free, tokens)
        assert type(a) is device.Assigned and all(t.is_contiguous() for t in a) and a.slot.dtype == torch.int64
        assert a.begin.tolist() == [0, 3, 3] and a.length.tolist() == [3, 0] and a.taken.tolist() == [2]
        assert a.slot.tolist() == [0, 1, 2, -1, -1][:tokens] and a.position.tolist() == [0, 1, 2, -1, -1][:tokens] and a.owner.tolist() == [0, 0, 0, -1, -1][:tokens]


@pytest.mark.gpu
def test_the_workspace_that_a_cache_keeps():
    """One for each stream that it was called on, grown when a call needs more, none made while a graph is captured."""
    k, v = (torch.randn((64, 16, 1, 64)).bfloat16().cuda() for _ in range(2))
    cache = device.PagedCache(k, v)
    q, n = torch.randn((1, 4, 64)).bfloat16().cuda(), torch.tensor([1000], dtype=torch.int32, device="cuda")
    table = torch.arange(64, dtype=torch.int32, device="cuda")[None]
    want = device.cache_attend(cache, q, table[:, :20], n)
    here = device.current_stream()
    first = cache._work[here]
    out, lse = device.cache_attend(cache, q, table, n)
    assert cache._work[here].numel() > first.numel() and list(cache._work) == [here]
    kept = cache._work[here]
    again = device.cache_attend(cache, q, table, n)
    assert cache._work[here] is kept and torch.equal(again[0], out) and torch.equal(again[1], lse)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        device.cache_attend(cache, q, table, n)
    assert len(cache._work) == 2
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    before = dict(cache._work)
    with torch.cuda.graph(graph, stream=side):
        captured = device.cache_attend(cache, q, table, n)
    assert all(cache._work[s] is w for s, w in before.items()) and len(cache._work) == 2
    for _ in range(3):
        graph.replay()
        device.cache_attend(cache, q, table[:, :20], n)
        torch.cuda.synchronize()
        assert torch.equal(captured[0], out) and torch.equal(captured[1], lse)
    assert torch.equal(device.cache_attend(cache, q, table[:, :20], n)[0], want[0])


@pytest.mark.gpu
def test_a_decoder_layer_on_the_cache():
    """The example: prompts, then steps of one token.  What it differs by are the roundings between its products, half a step of bf16 each: of the keys and queries
    (a score is at most 64 of their products wide, scaled by 1 / 8), of the attention's output and of the layer's; 2^-8 of the largest times a few."""
    from paper_2002_12798_amd import decode_example
    assert decode_example.run() < 8 * 2.0 ** -8
    assert decode_example.run(requests=3, steps=3, heads=6, kv_heads=6, dim=80, longest=90, width=256) < 8 * 2.0 ** -8
