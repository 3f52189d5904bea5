"""PyTorch glue: device memory and streams only.  All data movement happens in
libamap.so; nothing here computes, and there is no CPU fallback."""
from __future__ import annotations

import contextlib
import operator
import warnings
from typing import NamedTuple

import numpy as np
import torch

from . import binding as B

_TORCH_DT = {2: torch.int16, 4: torch.int32}
_NP_DT = {2: np.uint16, 4: np.uint32}
_NP_SIGNED = {2: np.int16, 4: np.int32}


def require_gpu() -> torch.device:
    if not torch.cuda.is_available():
        raise RuntimeError("amap needs a GPU: the HIP path has no CPU fallback")
    return torch.device("cuda:0")


def to_device(bits: np.ndarray) -> torch.Tensor:
    """Opaque element bits (uint16 / uint32 ndarray) -> device tensor of the same bits."""
    es = bits.dtype.itemsize
    return torch.from_numpy(np.ascontiguousarray(bits).view(_NP_SIGNED[es])).to(require_gpu())


def to_host(t: torch.Tensor) -> np.ndarray:
    es = t.element_size()
    return t.cpu().numpy().view(_NP_DT[es])


def empty_dst(m, fill=None) -> torch.Tensor:
    info = B.amap_describe(m)
    shape = tuple(info.shape[k] for k in range(info.rank))
    t = torch.empty(shape, dtype=_TORCH_DT[info.elem_size], device=require_gpu())
    if fill is not None:
        t.fill_(fill)
    return t


# torch.cuda.current_stream() builds a Stream object (2.8 us); the handle alone is 0.2 us away
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# once CUDA is initialised: what torch.cuda.current_device() asks after its own check (0.2 against 0.1 us)
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


if _raw_stream is not None:
    B._call.torch(_raw_stream, _get_device, torch.cuda.is_initialized)
_execute, _execute_multi, _current_stream = B._call.execute, B._call.execute_multi, B._call.current_stream


def current_stream() -> int:
    handle = _current_stream()
    if handle is not None:
        return handle
    if _raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_get_device())


def execute(m, srcs, dst=None, kernel_id=None, stream=None) -> torch.Tensor:
    """dst <- map(srcs) on the current stream; returns dst (allocated if None)."""
    if dst is not None and kernel_id is None:
        st = _execute(m, srcs, dst, stream)
        if st == 0:
            return dst
        if st > 0:
            raise B.AmapError(st, "amap_execute")
    if dst is None:
        dst = empty_dst(m)
    ptrs = [0 if s is None else s.data_ptr() for s in srcs]
    B.amap_execute(ptrs, dst.data_ptr(), m, current_stream() if stream is None else stream, kernel_id)
    return dst


def execute_multi(maps, srcs, dsts=None, stream=None):
    """dsts[i] <- maps[i](srcs), all maps in shared launches; returns the dst tensors."""
    if dsts is not None:
        st = _execute_multi(maps, srcs, dsts, stream)
        if st == 0:
            return dsts
        if st > 0:
            raise B.AmapError(st, "amap_execute_multi")
    if dsts is None:
        dsts = [empty_dst(m) for m in maps]
    B.amap_execute_multi([0 if s is None else s.data_ptr() for s in srcs], [d.data_ptr() for d in dsts], maps,
                         current_stream() if stream is None else stream)
    return dsts


def gemm_fused(a_src: torch.Tensor, a_map, w: torch.Tensor, out=None, stream=None, out_map=None) -> torch.Tensor:
    """out = A x W with A read through a_map; with out_map the product is stored through
    that map (out then has out_map's dst shape)."""
    n = w.shape[1]
    if out is None:
        shape = (B.amap_describe(a_map).shape[0], n) if out_map is None else B.dst_shape(out_map)
        out = torch.empty(shape, dtype=torch.int16, device=require_gpu())
    st = current_stream() if stream is None else stream
    if out_map is None:
        B.amap_gemm_fused(a_src.data_ptr(), a_map, w.data_ptr(), n, out.data_ptr(), st)
    else:
        B.amap_gemm_fused_store(a_src.data_ptr(), a_map, w.data_ptr(), n, out_map, out.data_ptr(), st)
    return out


# ---- a paged key-value cache: block tables and slots, rotary positions, the store of fresh tokens, one token's attention

# (a tensor of 16-bit words holds bf16 bits, as everywhere in this package)
_ELEMENT = {torch.float32: B.AMAP_F32, torch.bfloat16: B.AMAP_BF16, torch.int16: B.AMAP_BF16, torch.float16: B.AMAP_F16, torch.float8_e4m3fn: B.AMAP_E4M3}

_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", torch.cuda.is_current_stream_capturing)


def _refused(what, why, status=B.AMAP_E_INVALID):
    return B.AmapError(status, f"{what}: {why}", said=False)


def _on_gpu(t, dtype, rank, what, name):
    """The tensor, on a GPU, of this type and rank, its last dimension contiguous."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.dim() != rank:
        raise _refused(what, f"{name} is no {dtype} tensor of {rank} dimension{'s' * (rank > 1)}")
    if not t.is_cuda:
        raise _refused(what, f"{name} is not on the GPU")
    if rank and t.size(-1) > 1 and t.stride(-1) != 1:
        raise _refused(what, f"{name} is not contiguous along its last dimension", B.AMAP_E_UNSUPPORTED)
    return t


def _rows(t, what, name):
    """A [tokens, heads, head_dim] tensor as the library takes it."""
    if not isinstance(t, torch.Tensor) or t.dtype not in _ELEMENT:
        raise _refused(what, f"{name} is no tensor of a known type")
    _on_gpu(t, t.dtype, 3, what, name)
    return B.amap_heads(t.data_ptr(), _ELEMENT[t.dtype], t.size(1), t.stride(0), t.stride(1))


class Rope:
    """Rotary positions: freq [pairs] (float32, on the GPU), the pairs of each axis, and which elements make a pair: (p, p + pairs), or
    (2p, 2p + 1) if interleaved."""

    def __init__(self, freq, axis_pairs=None, interleaved=False):
        self._freq = _on_gpu(freq, torch.float32, 1, "Rope", "freq")
        self.axis_pairs = (freq.numel(),) if axis_pairs is None else tuple(int(n) for n in axis_pairs)
        self.interleaved = bool(interleaved)
        if not 1 <= len(self.axis_pairs) <= B.AMAP_MAX_AXES or min(self.axis_pairs) < 0 or sum(self.axis_pairs) != freq.numel():
            raise _refused("Rope", f"axis_pairs {self.axis_pairs} are not the {freq.numel()} pairs", B.AMAP_E_SHAPE)
        self._c = B.amap_rope(freq.data_ptr(), freq.numel(), int(self.interleaved), len(self.axis_pairs), (B.C.c_int32 * B.AMAP_MAX_AXES)(*self.axis_pairs))
        self._rope_at = B.C.addressof(self._c)

    freq = property(operator.attrgetter("_freq"))   # (the library has its address)

    def _positions(self, position, tokens, what):
        """The address of [axes, tokens] or [tokens] int32 positions (the latter the same for all axes), and the step between axes."""
        if position is None:
            raise _refused(what, "a rope without positions")
        if isinstance(position, torch.Tensor) and position.dim() == 2:
            _on_gpu(position, torch.int32, 2, what, "position")
            if position.size(0) != len(self.axis_pairs) or position.size(1) != tokens:
                raise _refused(what, f"position is {tuple(position.shape)}, not {(len(self.axis_pairs), tokens)}", B.AMAP_E_SHAPE)
            return position.data_ptr(), position.stride(0)
        _on_gpu(position, torch.int32, 1, what, "position")
        if position.size(0) != tokens:
            raise _refused(what, f"position is {tuple(position.shape)}, not {(tokens,)}", B.AMAP_E_SHAPE)
        return position.data_ptr(), 0


class PagedCache:
    """Keys and values as [pages, page_size, kv_heads, head_dim] tensors of one type and one set of strides: any memory order with
    the elements of a head side by side (a heads-first cache is the permuted view of one).  float8_e4m3fn with a
    float32 scale per head, or none."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        for t, name in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or _ELEMENT.get(t.dtype, B.AMAP_F32) == B.AMAP_F32:
                raise _refused("PagedCache", f"{name} is no tensor of a cache's type")
            _on_gpu(t, t.dtype, 4, "PagedCache", name)
        if k.dtype != v.dtype or k.shape != v.shape or k.stride() != v.stride():
            raise _refused("PagedCache", "k and v differ in type, shape or strides", B.AMAP_E_SHAPE)
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t is not None and (_on_gpu(t, torch.float32, 1, "PagedCache", name).numel() != k.size(2) or k.dtype != torch.float8_e4m3fn):
                raise _refused("PagedCache", f"{name} is one scale per head of an 8-bit cache", B.AMAP_E_SHAPE)
        self._k, self._v, self._k_scale, self._v_scale = k, v, k_scale, v_scale
        self._c = B.amap_cache(k.data_ptr(), v.data_ptr(), _ELEMENT[k.dtype], k.size(0), k.size(1), k.size(2), k.size(3), k.stride(0), k.stride(1), k.stride(2),
                               None if k_scale is None else k_scale.data_ptr(), None if v_scale is None else v_scale.data_ptr())
        self._cache_at = B.C.addressof(self._c)
        # cache_attend's workspace on each stream that it has been called on: one call after the other uses it there.  A call takes it out while it issues its
        # launches, so that no call of another thread finds it before they are all on the stream.
        self._work = {}

    # (the library has their addresses)
    k, v, k_scale, v_scale = (property(operator.attrgetter(name)) for name in ("_k", "_v", "_k_scale", "_v_scale"))

    @property
    def page_size(self):
        return self._k.size(1)


class Assigned(NamedTuple):
    begin: torch.Tensor      # [requests + 1] int32: where each request's fresh tokens begin
    length: torch.Tensor     # [requests] int32: tokens after the step
    slot: torch.Tensor       # [n_tokens] int64: page * page_size + row, -1 where there is none
    position: torch.Tensor   # [n_tokens] int32
    owner: torch.Tensor      # [n_tokens] int32: the request
    taken: torch.Tensor      # [1] int32: pages needed from the list


def assigned_buffers(requests, n_tokens, like=None) -> Assigned:
    """Room for a step's assignment, for a program that keeps it from step to step (as a captured graph has to)."""
    dev = require_gpu() if like is None else like.device
    words = torch.empty(2 * requests + 2 + 4 * n_tokens, dtype=torch.int32, device=dev)
    slot, begin, length, position, owner, taken = words.split_with_sizes((2 * n_tokens, requests + 1, requests, n_tokens, n_tokens, 1))
    return Assigned(begin, length, slot.view(torch.int64), position, owner, taken)


class _NoCalls:
    """The extension's functions, none of which takes a call."""
    assign = rotary = append = attend = norm = norm_grad = quantize = gemm_scaled = staticmethod(lambda *args: None)


def _native_calls():
    """The calls on tensors as they are (amap_paged_call.cpp), if they are built for this torch and the library has what they call: their answer is the
    outputs or the library's status, or None for a call that they do not take, which goes the long way below; that says why."""
    if not hasattr(B._L, "amap_rotary") or _raw_stream is None:
        return _NoCalls
    try:
        from . import _amap_paged_call as calls
    except ImportError as e:
        warnings.warn(f"{e}: calls around the paged cache go through ctypes; run `python -c 'import __graft_entry__ as g; g.build()'`", RuntimeWarning)
        return _NoCalls
    if calls.torch_version != torch.__version__:
        warnings.warn(f"_amap_paged_call is built for torch {calls.torch_version}: calls around the paged cache go through ctypes", RuntimeWarning)
        return _NoCalls
    calls.library(*(B.C.cast(getattr(B._L, name), B.C.c_void_p).value for name in ("amap_cache_assign", "amap_rotary", "amap_cache_append", "amap_cache_attend",
                                                                                   "amap_cache_attend_workspace")),
                  Assigned, _raw_stream, _get_device, torch.cuda.is_initialized, _capturing)
    return calls


_native = _native_calls()
_native_assign, _native_rotary, _native_append, _native_attend = _native.assign, _native.rotary, _native.append, _native.attend


def _made_on(stream):
    """Where a tensor has to be made that `stream` is the first to use: memory of the current stream may still be in use there, and
    what is given back to it may be handed out before `stream` is done."""
    if stream is None or stream == current_stream():
        return contextlib.nullcontext()
    return torch.cuda.stream(torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream())


def cache_assign(page_size, cached, fresh, table, free_pages, n_tokens, out=None, stream=None) -> Assigned:
    """Pages, slots and positions for a step in which request r adds fresh[r] tokens to its cached[r] (None: none yet):
    new pages are taken from the head of free_pages into `table`, which is changed in place.  All int32.  What is made here is one buffer: whoever keeps one tensor of
    it from step to step (`length`, which the next step has as `cached`) keeps the others' memory too, or a clone.  `out` may not hold what the call reads."""
    what = "amap_cache_assign"
    done = _native_assign(page_size, cached, fresh, table, free_pages, n_tokens, out, stream)
    if done is not None:
        return done if type(done) is not int else B._check(done, what)
    n = _on_gpu(fresh, torch.int32, 1, what, "fresh").size(0)
    _on_gpu(table, torch.int32, 2, what, "table")
    _on_gpu(free_pages, torch.int32, 1, what, "free_pages")
    if cached is not None and _on_gpu(cached, torch.int32, 1, what, "cached").size(0) != n or table.size(0) != n:
        raise _refused(what, "cached, fresh and table are not of the same requests", B.AMAP_E_SHAPE)
    if out is None:
        with _made_on(stream):
            out = assigned_buffers(n, n_tokens, fresh)
    else:
        sizes = (n + 1, n, n_tokens, n_tokens, n_tokens, 1)
        for t, size, dtype, name in zip(out, sizes, (torch.int32, torch.int32, torch.int64, torch.int32, torch.int32, torch.int32), Assigned._fields):
            if _on_gpu(t, dtype, 1, what, name).size(0) != size:
                raise _refused(what, f"{name} holds {t.size(0)} entries, not {size}", B.AMAP_E_SHAPE)
    B.amap_cache_assign(B.amap_assign(n, page_size, None if cached is None else cached.data_ptr(), fresh.data_ptr(), free_pages.data_ptr(), free_pages.size(0),
                                      table.data_ptr(), table.stride(0), table.size(1), out.begin.data_ptr(), out.length.data_ptr(), out.slot.data_ptr(),
                                      out.position.data_ptr(), out.owner.data_ptr(), n_tokens, out.taken.data_ptr()),
                        current_stream() if stream is None else stream)
    return out


def rotary(x, rope, position, out=None, inverse=False, stream=None) -> torch.Tensor:
    """out = x [tokens, heads, head_dim] turned to its positions ([tokens] or [axes, tokens], int32); inverse: turned back.
    out may be x itself.  No gradient is recorded, whatever x asks for: that of x is the output's, turned back."""
    what = "amap_rotary"
    done = _native_rotary(x, rope, position, out, inverse, stream)
    if done is not None:
        return done if type(done) is not int else B._check(done, what)
    a = _rows(x, what, "x")
    if out is None:
        with _made_on(stream):
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    elif isinstance(out, torch.Tensor) and out.shape != x.shape:
        raise _refused(what, f"out is {tuple(out.shape)}, not {tuple(x.shape)}", B.AMAP_E_SHAPE)
    at, step = rope._positions(position, x.size(0), what)
    B.amap_rotary(a, _rows(out, what, "out"), x.size(0), x.size(2), rope._c, at, step, inverse, current_stream() if stream is None else stream)
    return out


def cache_append(cache, k, v, slot, rope=None, position=None, q=None, q_out=None, stream=None):
    """k and v [tokens, kv_heads, head_dim] into the cache at slot [tokens] (int64; outside the cache: left out), k turned by the
    rope on the way, if there is one, and q into q_out (allocated if None; returned)."""
    what = "amap_cache_append"
    done = _native_append(cache, k, v, slot, rope, position, q, q_out, stream)
    if done is not None:
        return (None if done is True else done) if type(done) is not int else B._check(done, what)
    a, b = _rows(k, what, "k"), _rows(v, what, "v")
    tokens, dim = k.size(0), cache.k.size(3)
    if v.size(0) != tokens or k.size(2) != dim or v.size(2) != dim or (q is not None and isinstance(q, torch.Tensor) and (q.size(0) != tokens or q.size(-1) != dim)):
        raise _refused(what, "k, v, q and the cache differ in tokens or head_dim", B.AMAP_E_SHAPE)
    if _on_gpu(slot, torch.int64, 1, what, "slot").size(0) != tokens:
        raise _refused(what, f"slot holds {slot.size(0)} entries, not {tokens}", B.AMAP_E_SHAPE)
    at, step = (None, 0) if rope is None else rope._positions(position, tokens, what)
    c = d = None
    if q is not None:
        c = _rows(q, what, "q")
        if q_out is None:
            with _made_on(stream):
                q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        elif isinstance(q_out, torch.Tensor) and q_out.shape != q.shape:
            raise _refused(what, f"q_out is {tuple(q_out.shape)}, not {tuple(q.shape)}", B.AMAP_E_SHAPE)
        d = _rows(q_out, what, "q_out")
    B.amap_cache_append(cache._c, a, b, tokens, slot.data_ptr(), None if rope is None else rope._c, at, step, c, d, current_stream() if stream is None else stream)
    return q_out


def cache_attend(cache, q, table, length, scale=None, window=0, out=None, lse=None, workspace=None, stream=None):
    """(out, lse): the attention of q [requests, heads, head_dim] over the first length[r] tokens (int32; window > 0: the last
    `window` of them) that table [requests, width] (int32) leads to.  scale: 1 / sqrt(head_dim) if None.  A request that sees nothing has
    rows of 0 and lse -inf; a visible value that is infinite or NaN counts as the formula has it.  No gradient is recorded.  workspace: a uint8 tensor
    of attend_workspace() bytes, for a program that keeps it; calls that may run at the same time, or that two threads issue on one stream at the
    same time, must not be given the same one."""
    what = "amap_cache_attend"
    done = _native_attend(cache, q, table, length, scale, window, out, lse, workspace, stream)
    if done is not None:
        return done if type(done) is not int else B._check(done, what)
    a = _rows(q, what, "q")
    n, heads, dim = q.shape
    _on_gpu(table, torch.int32, 2, what, "table")
    if _on_gpu(length, torch.int32, 1, what, "length").size(0) != n or table.size(0) != n or dim != cache.k.size(3):
        raise _refused(what, "q, table, length and the cache differ in requests or head_dim", B.AMAP_E_SHAPE)
    need, keep = attend_workspace(cache, heads, n, table.size(1)), False
    with _made_on(stream):
        if out is None:
            out = torch.empty((n, heads, dim), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((n, heads), dtype=torch.float32, device=q.device)
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
            keep = stream is None and not _capturing()   # (a graph's memory is the graph's)
    if isinstance(out, torch.Tensor) and out.shape != q.shape:
        raise _refused(what, f"out is {tuple(out.shape)}, not {tuple(q.shape)}", B.AMAP_E_SHAPE)
    if _on_gpu(lse, torch.float32, 2, what, "lse").shape != (n, heads) or not lse.is_contiguous():
        raise _refused(what, f"lse is no contiguous {(n, heads)}", B.AMAP_E_SHAPE)
    have = 0 if workspace is None else _on_gpu(workspace, torch.uint8, 1, what, "workspace").numel()
    B.amap_cache_attend(cache._c, a, n, table.data_ptr(), table.stride(0), table.size(1), length.data_ptr(), dim ** -0.5 if scale is None else scale, window,
                        _rows(out, what, "out"), lse.data_ptr(), None if workspace is None else workspace.data_ptr(), have,
                        current_stream() if stream is None else stream)
    if keep:   # (from here on: its launches are on the stream)
        cache._work[current_stream()] = workspace
    return out, lse


def attend_workspace(cache, heads, requests, table_width) -> int:
    """Bytes of workspace that cache_attend takes for such a call."""
    return B.amap_cache_attend_workspace(cache._c, heads, requests, table_width)


# ---- a layer's rows in 8 bits: the norm in front of a product, rows and weights with a scale for each block of 128, the product of them

class Normed(NamedTuple):
    out: torch.Tensor                # the norm, in x's type or (eight) float8_e4m3fn
    scale: torch.Tensor | None       # eight: [tokens, ceil(dim / 128)] float32
    total: torch.Tensor | None       # with a residual: x + residual


class Eight(NamedTuple):
    out: torch.Tensor                # [rows, columns] float8_e4m3fn
    scale: torch.Tensor              # [ceil(rows / tall), ceil(columns / 128)] float32


def _blocks(n):
    return -(-n // B.AMAP_SCALE_BLOCK)


def _made_scales(rows, blocks, beside):
    """Scales as the product likes to read them: those of one block of columns beside one another."""
    return torch.empty((blocks, rows), dtype=torch.float32, device=beside.device).t()


def _heads_or_rows(t, what, name, like=None, dtype=None):
    """A [tokens, heads, dim] or [tokens, dim] tensor as the library takes it; `like`: of the same shape (and type, unless another one is named)."""
    if not isinstance(t, torch.Tensor) or t.dim() not in (2, 3) or t.dtype not in _ELEMENT:
        raise _refused(what, f"{name} is no tensor of 2 or 3 dimensions and a known type")
    if like is not None and t.shape != like.shape:
        raise _refused(what, f"{name} is {tuple(t.shape)}, not {tuple(like.shape)}", B.AMAP_E_SHAPE)
    want = dtype if dtype is not None else t.dtype if like is None else like.dtype
    if _ELEMENT[t.dtype] != _ELEMENT[want]:
        raise _refused(what, f"{name} is of {t.dtype}, not of {want}")
    _on_gpu(t, t.dtype, t.dim(), what, name)
    if t.dim() == 3:
        return B.amap_heads(t.data_ptr(), _ELEMENT[t.dtype], t.size(1), t.stride(0), t.stride(1))
    return B.amap_heads(t.data_ptr(), _ELEMENT[t.dtype], 1, t.stride(0), 0)


def _matrix(t, what, name):
    if not isinstance(t, torch.Tensor) or t.dtype not in _ELEMENT:
        raise _refused(what, f"{name} is no tensor of a known type")
    _on_gpu(t, t.dtype, 2, what, name)
    return B.amap_rows(t.data_ptr(), _ELEMENT[t.dtype], t.stride(0))


def _scales(t, rows, blocks, what, name):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or t.dim() != 2:
        raise _refused(what, f"{name} is no torch.float32 tensor of 2 dimensions")
    if not t.is_cuda:
        raise _refused(what, f"{name} is not on the GPU")
    if tuple(t.shape) != (rows, blocks):
        raise _refused(what, f"{name} is {tuple(t.shape)}, not {(rows, blocks)}", B.AMAP_E_SHAPE)
    return B.amap_scales(t.data_ptr(), t.stride(0), t.stride(1))


def _norm_weight(weight, x, what):
    if not isinstance(weight, torch.Tensor) or _ELEMENT.get(weight.dtype) not in (_ELEMENT[x.dtype], B.AMAP_F32):
        raise _refused(what, f"weight is no tensor of {x.dtype} or torch.float32")
    if _on_gpu(weight, weight.dtype, 1, what, "weight").size(0) != x.size(-1):
        raise _refused(what, f"weight holds {weight.size(0)} elements, not {x.size(-1)}", B.AMAP_E_SHAPE)
    return weight.data_ptr(), _ELEMENT[weight.dtype]


def _one_device(what, stream, *tensors):
    """The tensors lie on one device, and a call without a stream of its own, or on the null stream, on the current one: that is whose streams these are."""
    at = {t.get_device() for t in tensors if t is not None}
    if len(at) > 1:
        raise _refused(what, f"tensors on several devices ({', '.join(f'cuda:{i}' for i in sorted(at))})")
    if not stream and at != {_get_device()}:
        raise _refused(what, f"tensors on cuda:{at.pop()} and a stream of cuda:{_get_device()}")


if _native is not _NoCalls:
    _native.rows_library(*(B.C.cast(getattr(B._L, name), B.C.c_void_p).value for name in ("amap_norm", "amap_norm_grad", "amap_norm_grad_workspace", "amap_quantize",
                                                                                          "amap_gemm_scaled")), Normed, Eight)
_native_norm, _native_norm_grad, _native_quantize, _native_gemm_scaled = _native.norm, _native.norm_grad, _native.quantize, _native.gemm_scaled


def norm(x, weight, eps=1e-6, residual=None, eight=False, out=None, scale=None, total=None, stream=None) -> Normed:
    """The root mean square norm of x [tokens, dim] or [tokens, heads, dim] (each head by itself), times weight [dim] (x's type or float32): with a residual, of
    total = x + residual, rounded to their type (and made here if it is not given).  eps > 0.  eight: out in float8_e4m3fn with a scale for each row's blocks of 128 (x [tokens, dim] only).
    out and total may each be x or residual themselves.  No gradient is recorded: norm_grad makes it.  What is made here in 8 bits lies in one buffer with its scales, and a total of up to
    1 MB beside it: whoever keeps one keeps the others' memory too, or a clone."""
    what = "amap_norm"
    done = _native_norm(x, weight, eps, residual, eight, out, scale, total, stream)
    if done is not None:
        return done if type(done) is not int else B._check(done, what)
    a = _heads_or_rows(x, what, "x")
    if x.dtype == torch.float8_e4m3fn or (eight and x.dim() != 2) or (scale is not None and not eight) or (total is not None and residual is None):
        raise _refused(what, "x of 8 bits" if x.dtype == torch.float8_e4m3fn else "eight is for x [tokens, dim]" if eight and x.dim() != 2 else
                       "a scale without eight" if scale is not None else "a total without a residual")
    dim, of = x.size(-1), torch.float8_e4m3fn if eight else x.dtype
    b = None if residual is None else _heads_or_rows(residual, what, "residual", x)
    at, kind = _norm_weight(weight, x, what)
    with _made_on(stream):
        if out is None:
            out = torch.empty(x.shape, dtype=of, device=x.device)
        if eight and scale is None:
            scale = _made_scales(x.size(0), _blocks(dim), x)
        if residual is not None and total is None:
            total = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    d = _heads_or_rows(out, what, "out", x, of)
    s = None if scale is None else _scales(scale, x.size(0), _blocks(dim), what, "scale")
    t = None if total is None else _heads_or_rows(total, what, "total", x)
    _one_device(what, stream, x, weight, residual, out, scale, total)
    B.amap_norm(a, b, x.size(0), dim, at, kind, eps, t, d, s, current_stream() if stream is None else stream)
    return Normed(out, scale, total)


def norm_grad(x, weight, grad, eps=1e-6, extra=None, dx=None, dweight=None, workspace=None, stream=None):
    """(dx, dweight): the gradient of norm(x, weight) (with a residual: of its total) from that of its output, all of x's shape and type; extra: what reaches x by
    other ways, added to dx.  dweight [dim] is float32, and the same at every call.  dx may be x, grad or extra themselves.  workspace: a uint8 tensor of
    norm_grad_workspace() bytes, for a program that keeps it; calls that may run at the same time must not be given the same one."""
    what = "amap_norm_grad"
    done = _native_norm_grad(x, weight, grad, eps, extra, dx, dweight, workspace, stream)
    if done is not None:
        return done if type(done) is not int else B._check(done, what)
    a = _heads_or_rows(x, what, "x")
    if x.dtype == torch.float8_e4m3fn:
        raise _refused(what, "x of 8 bits")
    b = _heads_or_rows(grad, what, "grad", x)
    c = None if extra is None else _heads_or_rows(extra, what, "extra", x)
    at, kind = _norm_weight(weight, x, what)
    need = norm_grad_workspace(x)
    with _made_on(stream):
        if dx is None:
            dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if dweight is None:
            dweight = torch.empty(x.size(-1), dtype=torch.float32, device=x.device)
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    d = _heads_or_rows(dx, what, "dx", x)
    if _on_gpu(dweight, torch.float32, 1, what, "dweight").size(0) != x.size(-1):
        raise _refused(what, f"dweight holds {dweight.size(0)} elements, not {x.size(-1)}", B.AMAP_E_SHAPE)
    have = 0 if workspace is None else _on_gpu(workspace, torch.uint8, 1, what, "workspace").numel()
    _one_device(what, stream, x, weight, grad, extra, dx, dweight, workspace)
    B.amap_norm_grad(a, x.size(0), x.size(-1), at, kind, eps, b, c, d, dweight.data_ptr(), None if workspace is None else workspace.data_ptr(), have,
                     current_stream() if stream is None else stream)
    return dx, dweight


def norm_grad_workspace(x) -> int:
    """Bytes of workspace that norm_grad takes for such rows."""
    if not isinstance(x, torch.Tensor) or x.dim() not in (2, 3) or x.dtype not in _ELEMENT:
        raise _refused("amap_norm_grad_workspace", "x is no tensor of 2 or 3 dimensions and a known type")
    return B.amap_norm_grad_workspace(x.size(1) if x.dim() == 3 else 1, x.size(0), x.size(-1), _ELEMENT[x.dtype])


def quantize(x, gate=None, tall=1, out=None, scale=None, stream=None) -> Eight:
    """x [rows, columns] in float8_e4m3fn, with a float32 scale for each block of `tall` (1: activations, 128: weights) rows and 128 columns: the block's largest value over
    448.  gate: silu(gate) * x instead (tall 1).  What is made here is one buffer."""
    what = "amap_quantize"
    done = _native_quantize(x, gate, tall, out, scale, stream)
    if done is not None:
        return done if type(done) is not int else B._check(done, what)
    a = _matrix(x, what, "x")
    b = None if gate is None else _matrix(gate, what, "gate")
    if gate is not None and gate.shape != x.shape:
        raise _refused(what, f"gate is {tuple(gate.shape)}, not {tuple(x.shape)}", B.AMAP_E_SHAPE)
    if tall not in (1, B.AMAP_SCALE_BLOCK):
        raise _refused(what, f"blocks of {tall} rows, not of 1 or 128", B.AMAP_E_UNSUPPORTED)
    rows, columns = x.shape
    with _made_on(stream):
        if out is None:
            out = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
        if scale is None:
            scale = _made_scales(-(-rows // tall), _blocks(columns), x)
    c = _matrix(out, what, "out")
    if out.shape != x.shape:
        raise _refused(what, f"out is {tuple(out.shape)}, not {tuple(x.shape)}", B.AMAP_E_SHAPE)
    d = _scales(scale, -(-rows // tall), _blocks(columns), what, "scale")
    _one_device(what, stream, x, gate, out, scale)
    B.amap_quantize(a, b, rows, columns, tall, c, d, current_stream() if stream is None else stream)
    return Eight(out, scale)


def gemm_scaled(a, a_scale, w, w_scale, dtype=torch.bfloat16, out=None, stream=None) -> torch.Tensor:
    """a [m, k] times w [n, k] transposed, both float8_e4m3fn with the scales that quantize gives (a: tall 1, w: tall 128), summed in 32 bits and rounded once to
    dtype (bfloat16, float16, float32; out's type if there is one).  For an out of 16 bits products of eight neighbouring k are summed to 2^-13 of their largest, which shows where a result is a hundred
    times smaller than its terms; a float32 one has the full sums.  k is a multiple of 16, and rows begin at multiples of 16 bytes."""
    what = "amap_gemm_scaled"
    done = _native_gemm_scaled(a, a_scale, w, w_scale, dtype, out, stream)
    if done is not None:
        return done if type(done) is not int else B._check(done, what)
    x, y = _matrix(a, what, "a"), _matrix(w, what, "w")
    m, k = a.shape
    n = w.size(0)
    if w.size(1) != k:
        raise _refused(what, f"a and w have {k} and {w.size(1)} columns", B.AMAP_E_SHAPE)
    s, t = _scales(a_scale, m, _blocks(k), what, "a_scale"), _scales(w_scale, _blocks(n), _blocks(k), what, "w_scale")
    if out is None:
        if dtype not in (torch.bfloat16, torch.float16, torch.float32):
            raise _refused(what, f"a product in {dtype}")
        with _made_on(stream):
            out = torch.empty((m, n), dtype=dtype, device=a.device)
    z = _matrix(out, what, "out")
    if tuple(out.shape) != (m, n):
        raise _refused(what, f"out is {tuple(out.shape)}, not {(m, n)}", B.AMAP_E_SHAPE)
    _one_device(what, stream, a, a_scale, w, w_scale, out)
    B.amap_gemm_scaled(x, s, y, t, m, n, k, z, current_stream() if stream is None else stream)
    return out
