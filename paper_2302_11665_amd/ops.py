"""Thin ctypes binding of the operators of a served model's step (see
include/alpaserve_ops.h): linear layers with 8-bit weights, a paged cache of 4
bits with attention over it, and the cache's eviction by accumulated weight.

Argument marshalling only, as in `sim`: arrays are torch CUDA tensors, outputs
and scratch memory are torch allocations, calls run on torch's current stream of
the tensors' device, and errors raise `sim.SimError`.  None of the operators has
a gradient.
"""
from __future__ import annotations

import ctypes
import dataclasses

import torch

from . import sim

AS_BF16, AS_F16, AS_F32 = 0, 1, 2
AS_I8_MAX_INPUTS = 131072
_TYPES = {torch.bfloat16: AS_BF16, torch.float16: AS_F16, torch.float32: AS_F32}

_P, _I32, _I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class as_cache_t(ctypes.Structure):
    _fields_ = [("n_pages", _I32), ("n_heads", _I32), ("dim", _I32), ("group", _I32), ("page", _I32),
                ("n_seqs", _I32), ("max_pages", _I32), ("reserved", _I32), ("k", _P), ("v", _P),
                ("k_par", _P), ("v_par", _P), ("pos", _P), ("acc", _P), ("page_table", _P)]


_lib = None


def lib():
    global _lib
    if _lib is None:
        L = sim.lib()
        C = ctypes.POINTER(as_cache_t)
        for name, res, args in (
                ("as_i8_bytes", _I64, [_I64, _I64]),
                ("as_quantize_i8", ctypes.c_int, [_P, _I32, _I64, _I64, _I64, _P, _P, _P]),
                ("as_linear_i8_workspace", _I64, [_I64, _I64, _I64]),
                ("as_linear_i8", ctypes.c_int, [_P, _I32, _I64, _I64, _I64, _P, _P, _P, _I64, _P, _I32, _I64, _P,
                                                _I64, _P]),
                ("as_cache_append", ctypes.c_int, [C, _P, _P, _I32, _I32, _I64, _I64, _I64, _I64, _P, _P, _P, _P,
                                                   _P]),
                ("as_attention_kv4_workspace", _I64, [C, _I32, _I32, _I32]),
                ("as_attention_kv4", ctypes.c_int, [C, _P, _I32, _I32, _I32, _I64, _I64, _P, ctypes.c_float, _P, _P,
                                                    _P, _P, _I64, _P]),
                ("as_cache_evict_workspace", _I64, [C, _I32]),
                ("as_cache_evict", ctypes.c_int, [C, C, _P, _P, _I32, _I32, _P, _P, _I64, _P])):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _bad(msg):
    raise sim.SimError(sim.AS_E_INVALID_ARG, msg)


def _need(x, name, dtypes, dim=None, device=None, contiguous=True):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        _bad(f"{name}: a CUDA tensor is needed")
    if x.dtype not in dtypes:
        _bad(f"{name}: type {x.dtype}")
    if dim is not None and x.dim() != dim:
        _bad(f"{name}: {x.dim()} dimensions, {dim} needed")
    if device is not None and x.device != device:
        _bad(f"{name}: on {x.device}, not {device}")
    if contiguous and not x.is_contiguous():
        _bad(f"{name}: not contiguous")
    return x


def _on(fn, device, *args):
    """fn(*args) with the tensors' device current meanwhile."""
    index = device.index
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return fn(*args)
    return fn(*args)


def _call(fn, device, *args):
    """fn(*args, stream) on the current stream of the tensors' device, that device current meanwhile."""
    rc = _on(fn, device, *args, torch._C._cuda_getCurrentRawStream(device.index))
    if rc != sim.AS_OK:
        sim._check(rc)


def _workspace(n, device):
    """Scratch memory of one call (torch's allocator keeps it stream-ordered), and its address."""
    if n == 0:
        return None, None
    w = torch.empty(n, dtype=torch.uint8, device=device)
    return w, w.data_ptr()


def _rows(x):
    """x [rows, columns] as rows that lie apart, and their stride: a broadcast row or overlapping windows are copied."""
    (t, n), (stride, step) = x.shape, x.stride()
    if (n > 1 and step != 1) or (t > 1 and stride < n):
        x, stride = x.contiguous(), n
    return x, stride if t > 1 else n


_16 = (torch.bfloat16, torch.float16)
_FLOATS = (torch.bfloat16, torch.float16, torch.float32)


# ------------------------------------------------------------------- 8 bits

@dataclasses.dataclass
class PackedWeight:
    """A linear layer's weights of 8 bits: codes in the tiles that
    `as_quantize_i8` writes (int8, as_i8_bytes(n_out, n_in) of them), one fp32
    scale per output."""
    codes: torch.Tensor
    scale: torch.Tensor
    n_out: int
    n_in: int

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.scale.numel() * 4


def pack_weight(w) -> PackedWeight:
    """Quantise weights [n_out, n_in] (bf16, fp16 or fp32) per output, once."""
    _need(w, "weight", _FLOATS, 2, contiguous=False)
    w, stride = _rows(w)
    n, k = w.shape
    codes = torch.empty(lib().as_i8_bytes(n, k), dtype=torch.int8, device=w.device)
    scale = torch.empty(n, dtype=torch.float32, device=w.device)
    _call(lib().as_quantize_i8, w.device, w.data_ptr(), _TYPES[w.dtype], n, k, stride,
          codes.data_ptr(), scale.data_ptr())
    return PackedWeight(codes, scale, n, k)


def linear_i8(x, w: PackedWeight, bias=None, dtype=None, out=None):
    """x [..., n_in] (bf16 or fp16) quantised per token, times the packed
    weights: [..., n_out] of `dtype` (default: x's; fp32 allowed).  `out`, if
    given, is [tokens, n_out] with contiguous rows that do not overlap."""
    L = lib()
    _need(x, "x", _16, contiguous=False)
    dev = x.device
    if x.dim() < 1 or x.shape[-1] != w.n_in:
        _bad(f"linear_i8: x has {tuple(x.shape)}, the weights take {w.n_in} inputs")
    x2, x_stride = _rows(x if x.dim() == 2 else x.reshape(-1, w.n_in))
    t = x2.shape[0]
    codes, scale = w.codes, w.scale
    if not (codes.device == scale.device == dev and codes.dtype in (torch.int8, torch.uint8)
            and scale.dtype is torch.float32 and codes.is_contiguous() and scale.is_contiguous()
            and codes.numel() == L.as_i8_bytes(w.n_out, w.n_in) and scale.numel() == w.n_out):
        _bad(f"linear_i8: {codes.numel()} codes {codes.dtype} on {codes.device} and {scale.numel()} scales for "
             f"{w.n_out} x {w.n_in} weights")
    if bias is not None and _need(bias, "bias", (torch.float32,), device=dev).numel() != w.n_out:
        _bad(f"linear_i8: {bias.numel()} biases for {w.n_out} outputs")
    if out is None:
        y = torch.empty((t, w.n_out), dtype=dtype or x.dtype, device=dev)
    else:
        y = _need(out, "out", _FLOATS, 2, dev, contiguous=False)
        if tuple(y.shape) != (t, w.n_out) or (w.n_out > 1 and y.stride(1) != 1) or (
                t > 1 and y.stride(0) < w.n_out) or (dtype and y.dtype != dtype):
            _bad(f"linear_i8: out has {tuple(y.shape)} with strides {y.stride()}, {y.dtype}")
    if y.dtype not in _TYPES:
        _bad(f"linear_i8: type {y.dtype}")
    n = L.as_linear_i8_workspace(t, w.n_in, w.n_out)
    _keep, ws = _workspace(n, dev)
    _call(L.as_linear_i8, dev, x2.data_ptr(), _TYPES[x.dtype], t, w.n_in, x_stride,
          w.codes.data_ptr(), w.scale.data_ptr(), None if bias is None else bias.data_ptr(), w.n_out, y.data_ptr(),
          _TYPES[y.dtype], y.stride(0) if t > 1 else w.n_out, ws, n)
    return y if out is not None or x.dim() == 2 else y.view(*x.shape[:-1], w.n_out)


# -------------------------------------------------------------------- cache

@dataclasses.dataclass(frozen=True, eq=False, init=False)
class Cache:
    """A paged cache of 4 bits; the arrays are those of as_cache_t:
    k int32 [pages, heads, page, 4, dim/32], v int32 [pages, heads, page/32, 4,
    16, dim/16], k_par and v_par float16 [pages, heads, dim/group, page, 2], pos
    int32 and acc float32 [pages, heads, page] (either may be None where no
    weights are kept), page_table int32 [seqs, max_pages].  Sequences may share
    pages that a call only reads; a page that it writes (tokens appended,
    weights accumulated, an eviction's destination) is one sequence's.  Calls use the
    addresses that these had when the cache was made, so none can be replaced:
    `dataclasses.replace(cache, page_table=..)` makes a cache with another one."""
    k: torch.Tensor
    v: torch.Tensor
    k_par: torch.Tensor
    v_par: torch.Tensor
    pos: torch.Tensor
    acc: torch.Tensor
    page_table: torch.Tensor

    def __init__(self, k, v, k_par, v_par, pos, acc, page_table):
        # one cheap look at everything first: a step may make its handles anew
        kp, vp, table = k_par, v_par, page_table
        try:
            pages, heads, page, four, words = k.shape
            groups = kp.shape[2]
            rows, par = (pages, heads, page), (pages, heads, groups, page, 2)
            dev, i32 = k.device, torch.int32
            dim = words * 32
            fine = (k.is_cuda and k.dtype is i32 and v.dtype is i32 and kp.dtype is vp.dtype is torch.float16
                    and table.dtype is i32 and four == 4 and kp.shape == par and vp.shape == par
                    and v.shape == (pages, heads, page // 32, 4, 16, words * 2) and page % 32 == 0
                    and dim % groups == 0 and table.dim() == 2 and k.is_contiguous() and v.is_contiguous()
                    and kp.is_contiguous() and vp.is_contiguous() and table.is_contiguous()
                    and v.device == kp.device == vp.device == table.device == dev
                    and (pos is None or (pos.shape == rows and pos.dtype is i32 and pos.is_contiguous()
                                         and pos.device == dev))
                    and (acc is None or (acc.shape == rows and acc.dtype is torch.float32 and acc.is_contiguous()
                                         and acc.device == dev)))
        except (AttributeError, ValueError, IndexError, ZeroDivisionError):
            fine = False
        if not fine:
            what = [None if x is None else (tuple(x.shape), x.dtype, str(x.device)) if isinstance(x, torch.Tensor)
                    else type(x) for x in (k, v, kp, vp, pos, acc, table)]
            _bad(f"cache: contiguous CUDA arrays of one cache are needed, not {what}")
        self.__dict__.update(k=k, v=v, k_par=kp, v_par=vp, pos=pos, acc=acc, page_table=table, _c=as_cache_t(
            pages, heads, dim, dim // groups, page, table.shape[0], table.shape[1], 0, k.data_ptr(), v.data_ptr(),
            kp.data_ptr(), vp.data_ptr(), None if pos is None else pos.data_ptr(),
            None if acc is None else acc.data_ptr(), table.data_ptr()))

    @staticmethod
    def empty(n_pages, n_heads, dim, page_table, group=64, page=64, device="cuda") -> "Cache":
        """A cache of zeros."""
        if dim < 1 or group < 1 or page < 1 or dim % 32 or dim % group or page % 32:
            _bad(f"cache: heads of {dim} channels, {group} channels to a scale, pages of {page} slots (whole scales a "
                 "head; multiples of 32)")
        z = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        par = (n_pages, n_heads, dim // group, page, 2)
        return Cache(k=z((n_pages, n_heads, page, 4, dim // 32), torch.int32),
                     v=z((n_pages, n_heads, page // 32, 4, 16, dim // 16), torch.int32),
                     k_par=z(par, torch.float16), v_par=z(par, torch.float16),
                     pos=z((n_pages, n_heads, page), torch.int32), acc=z((n_pages, n_heads, page), torch.float32),
                     page_table=page_table)

    @property
    def bytes_per_slot(self) -> int:
        """Bytes of one slot of all heads: codes, scales, position and weight."""
        c = self._c
        return c.n_heads * (c.dim + 8 * (c.dim // c.group) + (self.pos is not None) * 4 + (self.acc is not None) * 4)


def _counts(x, name, cache):
    if not (x.dtype is torch.int32 and x.shape == (cache._c.n_seqs,) and x.device == cache.k.device
            and x.is_contiguous()):
        _bad(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device} for {cache._c.n_seqs} sequences (int32)")
    return x.data_ptr()


def _tokens(x, name, cache, heads):
    """x [seqs, tokens, heads, dim] with its last two dimensions contiguous."""
    c = cache._c
    if x.dim() != 4 or x.dtype not in _16 or x.device != cache.k.device or x.shape[0] != c.n_seqs or x.shape[
            3] != c.dim or (heads and x.shape[2] != heads):
        _bad(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}")
    if not x.is_contiguous() and (x.stride(3) != 1 or (x.shape[2] > 1 and x.stride(2) != c.dim)):
        x = x.contiguous()
    return x


def cache_append(cache: Cache, k, v, start, first_pos=None, held=False):
    """Put k, v [seqs, tokens, heads, dim] into slots start[b].. of every
    sequence (start: int32 [seqs]); positions count from first_pos[b] (default:
    start).  With `held`, returns the values that the cache holds for them now
    (two fp32 tensors of k's shape)."""
    heads = cache._c.n_heads
    k, v = _tokens(k, "k", cache, heads), _tokens(v, "v", cache, heads)
    if k.shape != v.shape or k.dtype != v.dtype:
        _bad(f"cache_append: k has {tuple(k.shape)} {k.dtype}, v {tuple(v.shape)} {v.dtype}")
    at = _counts(start, "start", cache)
    pos = None if first_pos is None else _counts(first_pos, "first_pos", cache)
    hk = hv = None
    if held:
        hk = torch.empty_like(k, dtype=torch.float32, memory_format=torch.contiguous_format)
        hv = torch.empty_like(hk)
    _call(lib().as_cache_append, k.device, cache._c, k.data_ptr(), v.data_ptr(), _TYPES[k.dtype], k.shape[1],
          k.stride(0), k.stride(1), v.stride(0), v.stride(1), at, pos, hk.data_ptr() if held else None,
          hv.data_ptr() if held else None)
    return (hk, hv) if held else None


def attention_kv4(q, cache: Cache, length, scale=None, acc_in=None, acc_out=None):
    """Attention of q [seqs, queries, q_heads, dim] (bf16 or fp16) over the
    first length[b] slots of every sequence, the queries being the last of them:
    query i sees slots below length - queries + i + 1.  `scale` defaults to
    dim ** -0.5.  With acc_out (fp32, laid out as cache.acc), acc_out = acc_in +
    the attention weight that every slot got from the queries of its head; the
    sequences then may not share pages."""
    q = _tokens(q, "q", cache, 0)
    # (the stride of a dimension of one entry may be anything, and is not used)
    seqs, queries, heads, _ = q.shape
    q_seq, q_token, _, _ = q.stride()
    q_seq, q_token = q_seq if seqs > 1 else 0, q_token if queries > 1 else 0
    if q.data_ptr() % 16 or q_seq % 8 or q_token % 8:
        q = q.clone(memory_format=torch.contiguous_format)
        q_seq, q_token, _, _ = q.stride()
    n = _counts(length, "length", cache)
    c = cache._c
    if acc_out is not None:
        rows = (c.n_pages, c.n_heads, c.page)
        for name, x in (("acc_in", acc_in), ("acc_out", acc_out)):
            if x is not None and (x.shape != rows or x.dtype is not torch.float32 or x.device != q.device
                                  or not x.is_contiguous()):
                _bad(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}")
    elif acc_in is not None:
        _bad("attention_kv4: acc_in without acc_out")
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    L = lib()
    # (its size depends on the device's compute units)
    dev = q.device
    need = _on(L.as_attention_kv4_workspace, dev, c, queries, heads, 0 if acc_out is None else 1)
    _keep, ws = _workspace(need, dev)
    _call(L.as_attention_kv4, dev, c, q.data_ptr(), _TYPES[q.dtype], queries, heads, q_seq, q_token, n,
          c.dim ** -0.5 if scale is None else scale, out.data_ptr(), None if acc_in is None else acc_in.data_ptr(),
          None if acc_out is None else acc_out.data_ptr(), ws, need)
    return out


def cache_evict(src: Cache, dst: Cache, length, total, keep, recent):
    """Copy to `dst` what a budget of `keep` tokens keeps of every sequence and
    head of `src`: the `recent` newest positions (total[b] tokens were there in
    all) and, of the others, those of the largest accumulated weight, in slot
    order.  Returns the new lengths, int32 [seqs]."""
    n, t = _counts(length, "length", src), _counts(total, "total", src)
    if src.k.device != dst.k.device:
        _bad("cache_evict: caches on different devices")
    if not 0 <= recent <= keep < 1 << 31:  # (ctypes passes the lowest 32 bits of others)
        _bad(f"cache_evict: keep {keep}, recent {recent}")
    new = torch.empty(length.shape[0], dtype=torch.int32, device=length.device)
    L = lib()
    need = L.as_cache_evict_workspace(src._c, keep)
    _keep, ws = _workspace(need, length.device)
    _call(L.as_cache_evict, length.device, src._c, dst._c, n, t, keep, recent, new.data_ptr(), ws, need)
    return new
