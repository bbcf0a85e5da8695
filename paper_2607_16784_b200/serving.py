"""ctypes binding of libroomie.so's serving operators: the cache kernels of a resident language model.

Same names as the C entry points (roomie_rope -> rope, roomie_kv_append -> kv_append, ...), torch tensors in and out; every
step runs in the library's kernels and is only enqueued on the stream."""
from __future__ import annotations

import ctypes as C
import functools
import struct
from contextlib import contextmanager

import numpy as np
import torch
from torch.autograd import forward_ad

from .roomie import RoomieError, _check, _dll, _ptr

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_FORMATS = {"e4m3": 0, "int8": 1}
_LAYOUTS = {"hnd": 0, "nhd": 1}


# roomie_rows as bytes (data, type, token_stride, head_stride): a step's calls last a few microseconds on the GPU, and building a
# ctypes structure for each tensor cost as much again on the host
_pack_rows = struct.Struct("=Qi4xqq").pack
# a device's current stream as a number; the public way (1.2 us a call more) where torch has not got the short one
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


class _RopeTable(C.Structure):
    _fields_ = [("rotary_dim", C.c_uint32), ("interleaved", C.c_int32), ("amplitude", C.c_float), ("frequency", C.c_void_p)]


class _KVCache(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("layers", "num_pages", "page_tokens", "kv_heads", "head_dim")] + \
               [("format", C.c_int32), ("layout", C.c_int32), ("max_seqs", C.c_uint32), ("max_pages", C.c_uint32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("refs", C.c_void_p), ("pages", C.c_void_p),
                ("length", C.c_void_p), ("status", C.c_void_p)]


class _Launch(C.Structure):
    _fields_ = [("name", C.c_char * 32)] + \
               [(n, C.c_uint32) for n in ("grid_blocks", "block_threads", "regs_per_thread", "smem_per_block")] + \
               [("dur_us", C.c_float), ("gap_us", C.c_float)]


def _rows(t, what):
    """[tokens, heads, head_dim] with a unit last stride, as the library sees it."""
    kind = _TYPES.get(t.dtype)
    stride = t.stride()
    if kind is None or len(stride) != 3 or not t.is_cuda or (stride[2] != 1 and t.shape[2] > 1):
        raise ValueError(f"{what}: a [tokens, heads, head_dim] CUDA tensor of float32, float16 or bfloat16 whose last dimension is contiguous")
    return _pack_rows(t.data_ptr(), kind, stride[0], stride[1])


def _ids(t, what, n=None):
    """A contiguous int32 device tensor (a list or array is copied to the device)."""
    if not isinstance(t, torch.Tensor):
        t = torch.as_tensor(np.asarray(t, dtype=np.int32), device="cuda")
    if t.dtype != torch.int32 or not t.is_cuda or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous one-dimensional int32 CUDA tensor")
    if n is not None and t.shape[0] != n:
        raise ValueError(f"{what}: {n} entries expected, got {t.shape[0]}")
    return t


def _here(index, *tensors):
    """The library launches on the current device: a cache's or a table's (`index`) and the tensors (None: not given) have to be on it."""
    device = torch.cuda.current_device()
    if index == device:
        for t in tensors:
            if t is not None and t.get_device() != device:
                index = t.get_device()
                break
        else:
            return
    raise ValueError(f"all tensors of a call live on the current CUDA device ({device}), got one on {index}")


def _u32(x, what):
    """ctypes takes the low 32 bits of a number: 2^32 + 5 would become the call with 5."""
    if not 0 <= x < 1 << 32:
        raise ValueError(f"{what}: a number of at most 32 bits, not negative, got {x}")
    return x


def _on_stream(call):
    """With stream= given, what the binding itself allocates or copies is ordered on that stream too."""
    @functools.wraps(call)
    def wrapped(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, **kw)
    return wrapped


def _stream(t):
    return _raw_stream(t.get_device())


def rope_frequencies(rotary_dim, base=10000.0, factor=1.0, context=0, low_turns=1.0, high_turns=4.0):
    """roomie_rope_frequencies: turns per position in units of 2^-64, a host array uint64 [rotary_dim / 2]."""
    rotary_dim = _u32(max(int(rotary_dim), 0), "rotary_dim")
    out = np.empty(max(rotary_dim // 2, 1), dtype=np.uint64)
    _check(_dll.roomie_rope_frequencies(rotary_dim, float(base), float(factor), float(context), float(low_turns),
                                        float(high_turns), out.ctypes.data), "roomie_rope_frequencies")
    return out


class RopeTable:
    """Rotary frequencies on the device with the pair layout and the amplitude (roomie_rope_table)."""

    def __init__(self, rotary_dim, base=10000.0, *, interleaved=False, amplitude=1.0, factor=1.0, context=0, low_turns=1.0,
                 high_turns=4.0, device="cuda"):
        f = rope_frequencies(rotary_dim, base, factor, context, low_turns, high_turns)
        self._set(torch.from_numpy(f.view(np.int64).copy()).to(device), interleaved, amplitude)

    @classmethod
    def from_tensor(cls, frequency, *, interleaved=False, amplitude=1.0):
        """Wraps an int64 device tensor [rotary_dim / 2] that holds the fixed-point frequencies' bits."""
        self = cls.__new__(cls)
        if frequency.dtype != torch.int64 or frequency.dim() != 1 or not frequency.is_contiguous() or not frequency.is_cuda:
            raise ValueError("frequency: a contiguous one-dimensional int64 CUDA tensor")
        self._set(frequency, interleaved, amplitude)
        return self

    def _set(self, frequency, interleaved, amplitude):
        self.frequency, self.interleaved, self.amplitude = frequency, bool(interleaved), float(amplitude)
        self.rotary_dim, self.index = 2 * frequency.numel(), frequency.get_device()
        self.c = _RopeTable(self.rotary_dim, int(self.interleaved), self.amplitude, frequency.data_ptr())
        self.ref = C.byref(self.c)


def _no_tangent(call, *tensors):
    """There are gradients, but no forward-mode derivatives: a result without the tangent that its inputs have would be a wrong one."""
    # (outside of every level, which is as good as always, this is all: the number of the level is not public, without it every call asks)
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise RuntimeError(f"{call}: no forward-mode derivative")


@_on_stream
def rope(x, positions, table: RopeTable, *, inverse=False, out=None):
    """roomie_rope: x [tokens, heads, head_dim] turned to `positions` (int32 [tokens]); `inverse` is the gradient.
    `out` may be x itself.  Returns out.  Without `out` the call is differentiable in x."""
    _no_tangent("rope", x)
    if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
        if out is not None:
            raise ValueError("out: not where a gradient is wanted")
        return _Turn.apply(x, _ids(positions, "positions"), table, inverse)
    cx = _rows(x, "x")
    n, h, d = x.shape
    positions = _ids(positions, "positions", n)
    _here(table.index, x, out, positions)
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out: the shape and type of x")
    _check(_dll.roomie_rope(table.ref, cx, _rows(out, "out"), n, h, d, positions.data_ptr(), inverse, _stream(x)), "roomie_rope")
    return out


class _Turn(torch.autograd.Function):
    """The rotation where a gradient is wanted: the gradient is the turn back, which can be differentiated again."""

    @staticmethod
    def forward(ctx, x, positions, table, inverse):
        ctx.save_for_backward(positions)
        ctx.table, ctx.inverse = table, inverse
        return rope(x, positions, table, inverse=inverse)

    @staticmethod
    def backward(ctx, grad):
        positions, = ctx.saved_tensors
        return rope(grad if grad.stride(2) == 1 else grad.contiguous(), positions, ctx.table, inverse=not ctx.inverse), None, None, None


def _head_weight(w, dim, like, what):
    """(pointer, type) of a weight [head_dim]; like: the type of the other one."""
    kind = _TYPES.get(w.dtype)
    if kind is None or tuple(w.shape) != (dim,) or not w.is_contiguous() or not w.is_cuda or (like is not None and kind != like):
        raise ValueError(f"{what}: contiguous CUDA tensors [head_dim] of one type, float32, float16 or bfloat16")
    return w.data_ptr(), kind


def _norm_out(x, out, what):
    if out is None:
        return torch.empty_like(x, memory_format=torch.contiguous_format)
    if out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError(f"{what}: the shape and type of its input")
    return out


@_on_stream
def qk_norm_rope(q, k, positions, table: RopeTable | None, q_weight=None, k_weight=None, *, eps=1e-6, q_out=None, k_out=None):
    """roomie_qk_norm_rope: q and k [tokens, heads, head_dim] (k may be None), each head divided by its root mean square, times its weight
    [head_dim] (None: ones), turned to `positions` (int32 [tokens]; table None: not turned).  Outputs may be the inputs.  Returns
    (q_out, k_out).  Without outputs given the call is differentiable, once, in q, k and the weights."""
    _no_tangent("qk_norm_rope", q, k, q_weight, k_weight)
    if torch.is_grad_enabled() and (q.requires_grad or (k is not None and k.requires_grad) or
                                    any(t is not None and t.requires_grad for t in (q_weight, k_weight, q_out, k_out))):
        if q_out is not None or k_out is not None:
            raise ValueError("q_out, k_out: not where a gradient is wanted")
        if table is not None:
            positions = _ids(positions, "positions")
        return _NormTurn.apply(q, k, positions if table is not None else None, table, q_weight, k_weight, eps)
    cq = _rows(q, "q")
    n, hq, d = q.shape
    qw = kw = kind = None
    if q_weight is not None:
        qw, kind = _head_weight(q_weight, d, None, "q_weight, k_weight")
    if k_weight is not None:
        kw, kind = _head_weight(k_weight, d, kind, "q_weight, k_weight")
    hk, ck, ko = 0, None, None
    if k is not None:
        hk = k.shape[1] if k.dim() == 3 else -1
        if k.shape != (n, hk, d) or k.dtype != q.dtype:
            raise ValueError("q, k: [tokens, heads, head_dim] of one type")
    elif k_weight is not None or k_out is not None:
        raise ValueError("k_weight, k_out: without k there is nothing to scale or to write")
    at = ref = None
    index = q.get_device()
    if table is not None:
        positions = _ids(positions, "positions", n)
        at, ref, index = positions.data_ptr(), table.ref, table.index
    _here(index, q, k, q_weight, k_weight, positions if at is not None else None, q_out, k_out)
    q_out = _norm_out(q, q_out, "q_out")
    if hk:
        k_out = _norm_out(k, k_out, "k_out")
        ck, ko = _rows(k, "k"), _rows(k_out, "k_out")
    elif k is not None:
        k_out = _norm_out(k, k_out, "k_out")
    _check(_dll.roomie_qk_norm_rope(ref, eps, n, d, at, kind or 0, hq, cq, qw, _rows(q_out, "q_out"), hk, ck, kw, ko, _stream(q)), "roomie_qk_norm_rope")
    return q_out, k_out


class _NormTurn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, table, q_weight, k_weight, eps):
        ctx.save_for_backward(q, k, positions, q_weight, k_weight)
        ctx.table, ctx.eps = table, eps
        return qk_norm_rope(q, k, positions, table, q_weight, k_weight, eps=eps)

    @staticmethod
    def backward(ctx, gq, gk):
        need = ctx.needs_input_grad
        back = _NormBack.apply if torch.is_grad_enabled() else _norm_back
        dq, dk, dqw, dkw = back(*ctx.saved_tensors, gq, gk, ctx.table, ctx.eps, need[4], need[5])
        return dq, dk, None, None, dqw, dkw, None


def _norm_back(q, k, positions, q_weight, k_weight, gq, gk, table, eps, need_qw, need_kw):
    """Gradients of q, k and the weights (None where there is none); the forward call has checked its arguments."""
    n, hq, d = q.shape
    hk = 0 if k is None else k.shape[1]
    unit = lambda g: g if g.stride(2) == 1 else g.clone(memory_format=torch.contiguous_format)
    gq, gk = unit(gq), unit(gk) if hk else None
    _here(q.get_device(), gq, gk)
    new = torch.empty_like
    dq, dk = new(q, memory_format=torch.contiguous_format), None if k is None else new(k, memory_format=torch.contiguous_format)
    dqw, dkw = new(q_weight) if need_qw else None, new(k_weight) if need_kw else None
    kind = 0 if q_weight is None and k_weight is None else _TYPES[(k_weight if q_weight is None else q_weight).dtype]
    scratch = torch.empty(int(_dll.roomie_qk_norm_rope_workspace_bytes(d)), dtype=torch.uint8, device=q.device)
    at = lambda t: None if t is None else t.data_ptr()
    _check(_dll.roomie_qk_norm_rope_grad(table.ref if table is not None else None, eps, n, d, at(positions), kind, hq, _rows(q, "q"), at(q_weight), _rows(gq, "gq"),
                                         _rows(dq, "dq"), at(dqw), hk, _rows(k, "k") if hk else None, at(k_weight), _rows(gk, "gk") if hk else None,
                                         _rows(dk, "dk") if hk else None, at(dkw), scratch.data_ptr(), scratch.numel(), _stream(q)), "roomie_qk_norm_rope_grad")
    return dq, dk, dqw, dkw


class _NormBack(torch.autograd.Function):
    """The gradients where they are recorded for a second derivative, which there is not."""

    @staticmethod
    def forward(ctx, *args):
        return _norm_back(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("qk_norm_rope can be differentiated once")


class KVCache:
    """A paged cache of 8-bit keys and values (roomie_kv_cache): codes k, v [layers, num_pages, ...], a float32 scale for each
    page and head, reference counts, the page table and the sequences' lengths, all device tensors."""

    def __init__(self, num_pages, page_tokens, kv_heads, head_dim, max_seqs, max_pages, *, layers=1, fmt="e4m3", layout="hnd",
                 device="cuda"):
        page = (kv_heads, page_tokens, head_dim) if layout == "hnd" else (page_tokens, kv_heads, head_dim)
        codes = lambda: torch.zeros((layers, num_pages) + page, dtype=torch.uint8, device=device)
        scales = lambda: torch.ones((layers, num_pages, kv_heads), dtype=torch.float32, device=device)
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)
        self._set(codes(), codes(), scales(), scales(), ints(num_pages), ints(max_seqs, max_pages).fill_(-1), ints(max_seqs), fmt, layout)

    @classmethod
    def from_tensors(cls, k, v, k_scale, v_scale, refs, pages, length, *, fmt="e4m3", layout="hnd"):
        """Wraps tensors without copying.  k and v may be strided over layers and pages (alike), not inside a page."""
        self = cls.__new__(cls)
        self._set(k, v, k_scale, v_scale, refs, pages, length, fmt, layout)
        return self

    def _set(self, k, v, k_scale, v_scale, refs, pages, length, fmt, layout):
        if fmt not in _FORMATS or layout not in _LAYOUTS:
            raise ValueError("fmt is 'e4m3' or 'int8', layout 'hnd' or 'nhd'")
        if k.dim() != 5 or k.shape != v.shape or k.dtype.itemsize != 1 or v.dtype.itemsize != 1:
            raise ValueError("k, v: 8-bit tensors [layers, pages, heads, tokens, dim] (hnd) or [layers, pages, tokens, heads, dim] (nhd)")
        layers, num_pages, a, b, dim = k.shape
        heads, tokens = (a, b) if layout == "hnd" else (b, a)
        for t in (k, v):
            if t.stride()[2:] != (b * dim, dim, 1) or t.stride()[:2] != k.stride()[:2]:
                raise ValueError("k, v: contiguous pages, and the same strides over layers and pages")
        for t, shape, kind in ((k_scale, (layers, num_pages, heads), torch.float32), (v_scale, (layers, num_pages, heads), torch.float32),
                               (refs, (num_pages,), torch.int32), (length, (pages.shape[0],), torch.int32),
                               (pages, tuple(pages.shape), torch.int32)):
            if tuple(t.shape) != shape or t.dtype != kind or not t.is_contiguous():
                raise ValueError(f"a contiguous {kind} tensor of shape {shape} expected, got {t.dtype} {tuple(t.shape)}")
        if not all(t.is_cuda and t.device == k.device for t in (k, v, k_scale, v_scale, refs, pages, length)):
            raise ValueError("the cache's tensors live on one CUDA device")
        self.k, self.v, self.k_scale, self.v_scale, self.refs, self.pages, self.length = k, v, k_scale, v_scale, refs, pages, length
        self.fmt, self.layout = fmt, layout
        self.layers, self.num_pages, self.page_tokens, self.kv_heads, self.head_dim = layers, num_pages, tokens, heads, dim
        self.max_seqs, self.max_pages = pages.shape
        self.index = k.get_device()
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.c = _KVCache(layers, num_pages, tokens, heads, dim, _FORMATS[fmt], _LAYOUTS[layout], self.max_seqs, self.max_pages,
                          k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k_scale.data_ptr(), v_scale.data_ptr(),
                          refs.data_ptr(), pages.data_ptr(), length.data_ptr(), self.status.data_ptr())
        self.ref = C.byref(self.c)
        with torch.cuda.device(k.device):                # the size follows the device's number of SMs
            self._bytes = int(_dll.roomie_kv_workspace_bytes(self.ref))
        if self._bytes == 0:
            raise ValueError("cache shape outside the library's limits (page_tokens 16..128, head_dim a multiple of 16 up to 256)")

    def workspace(self):
        """Device scratch for the calls that take one; keep it and pass it to each of them."""
        scratch = torch.empty(self._bytes, dtype=torch.uint8, device=self.k.device)
        scratch[:16384].zero_()                          # ROOMIE_KV_WORKSPACE_ZEROED
        return scratch

    def key_weights(self):
        """Zeros for the weights that kv_weights gathers: float32 [layers, max_seqs, kv_heads, max_pages * page_tokens]."""
        return torch.zeros((self.layers, self.max_seqs, self.kv_heads, self.max_pages * self.page_tokens), dtype=torch.float32, device=self.k.device)

    def status_flags(self) -> int:
        """Synchronises and returns the sticky ROOMIE_FLAG_KV_* bits."""
        return int(self.status.item()) & 0xFFFFFFFF

    def check(self):
        f = self.status_flags()
        if f:
            names = [n for b, n in ((8, "WAIT_TIMEOUT"), (16, "KV_PAGE"), (32, "KV_SEQUENCE"), (64, "KV_NONFINITE"), (128, "KV_FULL")) if f & b]
            raise RoomieError("cache status flags set: " + "|".join(names))


def _key_weights(cache, t, what):
    if tuple(t.shape) != (cache.layers, cache.max_seqs, cache.kv_heads, cache.max_pages * cache.page_tokens) or t.dtype != torch.float32 or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous float32 tensor [layers, max_seqs, kv_heads, max_pages * page_tokens] (cache.key_weights())")


def _scratch(cache, workspace):
    return cache.workspace() if workspace is None else workspace


@_on_stream
def kv_append(cache: KVCache, seqs, k, v, q_offset=None, *, layer=0, rope: RopeTable | None = None, q=None, q_out=None):
    """roomie_kv_append: rows of k, v [rows, kv_heads, head_dim] become the last tokens of sequences `seqs` (rows
    q_offset[i]..q_offset[i+1] of sequence i; None: one row each), rotated when `rope` is given.  With `q` its rotated rows are
    returned in q_out (q itself, or its copy in q_out, without `rope`).  For serving: no gradient passes through."""
    rows, d, layer = k.shape[0], cache.head_dim, _u32(layer, "layer")
    if k.shape[1:] != (cache.kv_heads, d) or k.shape != v.shape or k.dtype != v.dtype:
        raise ValueError("k, v: [rows, kv_heads, head_dim] of one type")
    seqs = _ids(seqs, "seqs")
    n = seqs.shape[0]
    if q_offset is not None:
        q_offset = _ids(q_offset, "q_offset", n + 1)
    elif rows != n:
        raise ValueError("without q_offset every sequence brings one row")
    _here(cache.index, seqs, q_offset, k, v, q, q_out)
    if rope is not None and rope.index != cache.index:
        raise ValueError("rope: a table on the cache's device")
    ck, cv = _rows(k, "k"), _rows(v, "v")
    turn = rope is not None and q is not None
    if q is None:
        if q_out is not None:
            raise ValueError("q_out: without q there is nothing to write")
    elif turn or q_out is not None:
        if q.dim() != 3 or q.shape[0] != rows or q.shape[2] != d or q.dtype != k.dtype:
            raise ValueError("q: [rows, q_heads, head_dim] of k's type")
        if q_out is not None and (q_out.shape != q.shape or q_out.dtype != q.dtype):
            raise ValueError("q_out: the shape and type of q")
    if turn:
        if q_out is None:
            q_out = torch.empty_like(q)
        cq, co = _rows(q, "q"), _rows(q_out, "q_out")
    _check(_dll.roomie_kv_append(cache.ref, layer, seqs.data_ptr(), n, None if q_offset is None else q_offset.data_ptr(), rows, ck, cv,
                                 rope.ref if rope is not None else None, q.shape[1] if turn else 0, cq if turn else None,
                                 co if turn else None, _stream(k)), "roomie_kv_append")
    if not turn and q_out is not None:
        return q_out.copy_(q)
    return q_out if turn else q


@_on_stream
def kv_attention(cache: KVCache, seqs, q, q_offset=None, *, layer=0, scale=None, window=0, out=None, lse=None, workspace=None):
    """roomie_kv_attention: q [rows, q_heads, head_dim] over the cached tokens of `seqs`.  Returns (out, lse); rows of no sequence are
    not written.  For serving: no gradient passes through."""
    rows, heads, d = q.shape
    layer, window = _u32(layer, "layer"), _u32(window, "window")
    if d != cache.head_dim or heads % cache.kv_heads:
        raise ValueError("q: [rows, q_heads, head_dim] with q_heads a multiple of the cache's kv_heads")
    seqs = _ids(seqs, "seqs")
    n = seqs.shape[0]
    if q_offset is not None:
        q_offset = _ids(q_offset, "q_offset", n + 1)
    elif rows != n:
        raise ValueError("without q_offset every sequence brings one row")
    _here(cache.index, seqs, q_offset, q, out, lse, workspace)
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out: the shape and type of q")
    if lse is None:
        lse = cache.k_scale.new_empty((rows, heads))
    elif tuple(lse.shape) != (rows, heads) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse: a contiguous float32 tensor [rows, q_heads]")
    workspace = _scratch(cache, workspace)
    _check(_dll.roomie_kv_attention(cache.ref, layer, seqs.data_ptr(), n, None if q_offset is None else q_offset.data_ptr(), rows, heads,
                                    _rows(q, "q"), d ** -0.5 if scale is None else scale, window, _rows(out, "out"), lse.data_ptr(),
                                    workspace.data_ptr(), workspace.shape[0], _stream(q)), "roomie_kv_attention")
    return out, lse


@_on_stream
def kv_reserve(cache: KVCache, seqs, want, *, workspace=None):
    """roomie_kv_reserve: sequences get pages for `want` tokens and that length."""
    seqs = _ids(seqs, "seqs")
    want = _ids(want, "want", seqs.numel())
    _here(cache.index, seqs, want, workspace)
    workspace = _scratch(cache, workspace)
    _check(_dll.roomie_kv_reserve(cache.ref, seqs.data_ptr(), want.data_ptr(), seqs.numel(), workspace.data_ptr(), workspace.numel(),
                                  _stream(cache.k)), "roomie_kv_reserve")


@_on_stream
def kv_fork(cache: KVCache, parents, children, *, workspace=None):
    """roomie_kv_fork: children become copies of parents; whole pages shared, part-filled last pages copied."""
    parents = _ids(parents, "parents")
    children = _ids(children, "children", parents.numel())
    _here(cache.index, parents, children, workspace)
    workspace = _scratch(cache, workspace)
    _check(_dll.roomie_kv_fork(cache.ref, parents.data_ptr(), children.data_ptr(), parents.numel(), workspace.data_ptr(),
                               workspace.numel(), _stream(cache.k)), "roomie_kv_fork")


@_on_stream
def kv_free(cache: KVCache, seqs):
    """roomie_kv_free: the sequences become empty, their pages lose a reference."""
    seqs = _ids(seqs, "seqs")
    _here(cache.index, seqs)
    _check(_dll.roomie_kv_free(cache.ref, seqs.data_ptr(), seqs.numel(), _stream(cache.k)), "roomie_kv_free")


@_on_stream
def kv_reorder(cache: KVCache, seqs, parents, *, workspace=None):
    """roomie_kv_reorder: sequence seqs[i] becomes what seqs[parents[i]] was (parents: indexes into seqs, as beam_select returns them; -1: empty)."""
    seqs = _ids(seqs, "seqs")
    parents = _ids(parents.reshape(-1) if isinstance(parents, torch.Tensor) else np.reshape(parents, -1), "parents", seqs.numel())
    _here(cache.index, seqs, parents, workspace)
    workspace = _scratch(cache, workspace)
    _check(_dll.roomie_kv_reorder(cache.ref, seqs.data_ptr(), parents.data_ptr(), seqs.numel(), workspace.data_ptr(), workspace.numel(),
                                  _stream(cache.k)), "roomie_kv_reorder")


@_on_stream
def kv_weights(cache: KVCache, seqs, q, lse, weight, q_offset=None, *, layer=0, scale=None, window=0, fresh=False):
    """roomie_kv_weights: adds to `weight` (cache.key_weights()) what the rows of q give to the keys of their sequences: q, q_offset, scale and window as in
    kv_attention, lse what it returned.  The call's own tokens start from nothing; with `fresh` all of the sequences' do.  A sequence named again is reported.
    Returns weight."""
    rows, heads, d = q.shape
    layer, window = _u32(layer, "layer"), _u32(window, "window")
    if d != cache.head_dim or heads % cache.kv_heads:
        raise ValueError("q: [rows, q_heads, head_dim] with q_heads a multiple of the cache's kv_heads")
    if tuple(lse.shape) != (rows, heads) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse: a contiguous float32 tensor [rows, q_heads]")
    _key_weights(cache, weight, "weight")
    seqs = _ids(seqs, "seqs")
    n = seqs.shape[0]
    if q_offset is not None:
        q_offset = _ids(q_offset, "q_offset", n + 1)
    elif rows != n:
        raise ValueError("without q_offset every sequence brings one row")
    _here(cache.index, seqs, q_offset, q, lse, weight)
    _check(_dll.roomie_kv_weights(cache.ref, layer, seqs.data_ptr(), n, None if q_offset is None else q_offset.data_ptr(), rows, heads, _rows(q, "q"),
                                  lse.data_ptr(), d ** -0.5 if scale is None else scale, window, fresh, weight.data_ptr(), _stream(q)), "roomie_kv_weights")
    return weight


@_on_stream
def kv_evict(cache: KVCache, seqs, weight, keep, *, first=0, recent=0, weight_out=None, workspace=None):
    """roomie_kv_evict: sequences longer than `keep` tokens keep, for each layer and head, their `first` first and `recent` last tokens and the heaviest
    of the others by `weight` (float32 [layers, max_seqs, kv_heads, max_pages * page_tokens]).  weight_out None: weight itself is updated.  Returns it."""
    seqs = _ids(seqs, "seqs")
    weight_out = weight if weight_out is None else weight_out
    _key_weights(cache, weight, "weight")
    _key_weights(cache, weight_out, "weight_out")
    keep, first, recent = _u32(keep, "keep"), _u32(first, "first"), _u32(recent, "recent")
    _here(cache.index, seqs, weight, weight_out, workspace)
    workspace = _scratch(cache, workspace)
    _check(_dll.roomie_kv_evict(cache.ref, seqs.data_ptr(), seqs.numel(), weight.data_ptr(), keep, first, recent, weight_out.data_ptr(), workspace.data_ptr(),
                                workspace.numel(), _stream(cache.k)), "roomie_kv_evict")
    return weight_out


@_on_stream
def kv_copy(src: KVCache, src_pages, dst: KVCache, dst_pages):
    """roomie_kv_copy: page src_pages[i] of src to page dst_pages[i] of dst, all layers, codes and scales."""
    src_pages = _ids(src_pages, "src_pages")
    dst_pages = _ids(dst_pages, "dst_pages", src_pages.numel())
    _here(src.index, dst.k, src_pages, dst_pages)
    _check(_dll.roomie_kv_copy(src.ref, src_pages.data_ptr(), dst.ref, dst_pages.data_ptr(), src_pages.numel(), _stream(src.k)),
           "roomie_kv_copy")


@_on_stream
def kv_compact(cache: KVCache, *, refs_out=None, pages_out=None, used_out=None, workspace=None):
    """roomie_kv_compact: the used pages move to the pool's lower end.  refs_out / pages_out None: the cache's own tensors are
    updated.  used_out: int32 [1] for the number of used pages."""
    refs_out = cache.refs if refs_out is None else refs_out
    pages_out = cache.pages if pages_out is None else pages_out
    for t, like in ((refs_out, cache.refs), (pages_out, cache.pages)):
        if t.shape != like.shape or t.dtype != like.dtype or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("refs_out, pages_out: the shape and type of the cache's refs and pages")
    if used_out is not None:
        _ids(used_out, "used_out", 1)
    _here(cache.index, refs_out, pages_out, used_out, workspace)
    workspace = _scratch(cache, workspace)
    _check(_dll.roomie_kv_compact(cache.ref, refs_out.data_ptr(), pages_out.data_ptr(), _ptr(used_out), workspace.data_ptr(),
                                  workspace.numel(), _stream(cache.k)), "roomie_kv_compact")


def beam_workspace(requests, beams, vocab, num, dtype=torch.float32, device="cuda"):
    """Device scratch for beam_select calls of this shape; keep it and pass it to each of them."""
    kind, sizes = _TYPES.get(dtype), [int(x) for x in (requests, beams, vocab, num)]
    size = 0 if kind is None or not all(0 <= x < 1 << 32 for x in sizes) else int(_dll.roomie_beam_workspace_bytes(*sizes, kind))
    if size == 0:
        raise ValueError("beam shape outside the library's limits (requests * beams up to 65535, beams up to 256, vocab up to 2^24, num up to 128)")
    return torch.empty(size, dtype=torch.uint8, device=device)


@_on_stream
def beam_select(logits, scores, num, *, ended=None, pad=0, out=None, workspace=None):
    """roomie_beam_select: logits [requests, beams, vocab] and the beams' scores (float32 [requests, beams]) to the `num` best continuations of
    each request: (scores float32, parent int32, token int32), each [requests, num].  parent is the row r * beams + b that a continuation comes
    from: what kv_reorder takes.  `ended` (bool [requests, beams]): beams that go on as they are, with the token `pad`.  `out`: tensors for the three
    results.  For serving: no gradient passes through."""
    kind, stride = _TYPES.get(logits.dtype), logits.stride()
    if kind is None or len(stride) != 3 or not logits.is_cuda or (stride[2] != 1 and logits.shape[2] > 1):
        raise ValueError("logits: a [requests, beams, vocab] CUDA tensor of float32, float16 or bfloat16 whose last dimension is contiguous")
    requests, beams, vocab = logits.shape
    shape, num, pad = (requests, beams), _u32(num, "num"), _u32(pad, "pad")
    if tuple(scores.shape) != shape or scores.dtype != torch.float32 or not scores.is_contiguous():
        raise ValueError("scores: a contiguous float32 tensor [requests, beams]")
    if ended is not None and (tuple(ended.shape) != shape or ended.dtype not in (torch.bool, torch.uint8) or not ended.is_contiguous()):
        raise ValueError("ended: a contiguous bool tensor [requests, beams]")
    if out is None:
        new = scores.new_empty
        out = (new((requests, num)), new((requests, num), dtype=torch.int32), new((requests, num), dtype=torch.int32))
    elif len(out) != 3 or any(tuple(t.shape) != (requests, num) or not t.is_contiguous() or t.dtype != k
                              for t, k in zip(out, (torch.float32, torch.int32, torch.int32))):
        raise ValueError("out: contiguous tensors [requests, num] of float32, int32 and int32")
    if workspace is None and requests:
        workspace = beam_workspace(requests, beams, vocab, num, logits.dtype, logits.device)
    _here(logits.get_device(), scores, ended, workspace, *out)
    _check(_dll.roomie_beam_select(logits.data_ptr(), kind, stride[0], stride[1], requests, beams, vocab, scores.data_ptr(), _ptr(ended), pad, num,
                                   out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                   _stream(logits)), "roomie_beam_select")
    return out


@contextmanager
def record_launches(capacity=4096):
    """Notes the serving operators' launches inside the block (roomie_record_*).  Yields a list that is filled when the block
    ends: dicts with name, grid_blocks, block_threads, regs_per_thread, smem_per_block, dur_us, gap_us, in launch order."""
    launches = []
    _check(_dll.roomie_record_enable(int(capacity)), "roomie_record_enable")
    try:
        yield launches
        got, n = (_Launch * max(int(capacity), 1))(), C.c_uint32(0)
        _check(_dll.roomie_record_read(got, int(capacity), C.byref(n)), "roomie_record_read")
        for r in got[:n.value]:
            d = {f: getattr(r, f) for f, _ in _Launch._fields_}
            launches.append(dict(d, name=d["name"].decode()))
    finally:
        _dll.roomie_record_enable(0)


def profile_columns(launches):
    """(grid, threads, regs, smem, dur_us, gap_us) arrays of recorded launches: the columns library_build takes."""
    col = lambda f, t: np.array([r[f] for r in launches], dtype=t)
    return tuple(col(f, np.uint32) for f in ("grid_blocks", "block_threads", "regs_per_thread", "smem_per_block")) + \
        tuple(col(f, np.float32) for f in ("dur_us", "gap_us"))
