"""Thin ctypes binding of the operators of a served model's step (see
include/alpaserve_ops.h): linear layers with 8-bit weights, a paged cache of 4
bits with attention over it, and the cache's eviction by accumulated weight; and
of those that take prompts in: norms in 8 bits, attention over packed prompts,
pages from a pool, packed appends.

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
                ("as_linear_i8_codes", ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _P, _I64, _P, _I32, _I64, _P]),
                ("as_norm_i8", ctypes.c_int, [_P, _P, _I32, _I64, _I64, _I64, _I64, _P, ctypes.c_float, _P, _I64, _P,
                                              _P, _P, _P]),
                ("as_attention_prompt", ctypes.c_int, [_P, _P, _P, _I32, _I64, _I32, _I32, _I32, _I64, _I64, _I64, _P,
                                                       _I32, ctypes.c_float, _P, _P, _I64, _P]),
                ("as_attention_prompt_workspace", _I64, [_I64, _I32, _I32, _I32]),
                ("as_pages_reserve_workspace", _I64, [_I32]),
                ("as_pages_reserve", ctypes.c_int, [_P, _P, _I32, _P, _I32, _I32, _I32, _P, _P, _I64, _P, _P, _P, _P,
                                                    _P, _P, _I64, _P]),
                ("as_pages_release", ctypes.c_int, [_P, _P, _I32, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P]),
                ("as_cache_append_packed", ctypes.c_int, [C, _P, _P, _I32, _I64, _I64, _I64, _P, _P, _P, _P, _P, _P]),
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


@dataclasses.dataclass
class Codes:
    """Activations of 8 bits: the codes of n_rows rows of n_cols columns in the
    tiles of as_quantize_i8 (int8), one fp32 scale per row, and the type of the
    rows that they were made from."""
    codes: torch.Tensor
    scale: torch.Tensor
    n_rows: int
    n_cols: int
    dtype: torch.dtype


def _norm_args(x, residual, gain, out):
    """x and the residual as rows, their strides, and the sum: `norm_i8`'s checks."""
    _need(x, "x", _16, contiguous=False)
    dev = x.device
    if x.dim() < 1 or x.shape[-1] < 1:
        _bad(f"norm_i8: x has {tuple(x.shape)}")
    cols = x.shape[-1]
    x2, x_stride = _rows(x if x.dim() == 2 else x.reshape(-1, cols))
    t = x2.shape[0]
    r2, r_stride, s, s_stride = None, 0, None, 0
    if residual is not None:
        _need(residual, "residual", (x.dtype,), device=dev, contiguous=False)
        if residual.shape != x.shape:
            _bad(f"norm_i8: x has {tuple(x.shape)}, the residual {tuple(residual.shape)}")
        r2, r_stride = _rows(residual if x.dim() == 2 else residual.reshape(-1, cols))
        s = torch.empty_like(x2, memory_format=torch.contiguous_format) if out is None else _need(
            out, "out", (x.dtype,), 2, dev, contiguous=False)
        s_stride = s.stride(0) if t > 1 else cols
        if tuple(s.shape) != (t, cols) or (cols > 1 and s.stride(1) != 1) or s_stride < cols:
            _bad(f"norm_i8: out has {tuple(s.shape)} with strides {s.stride()}")
    elif out is not None:
        _bad("norm_i8: out without a residual")
    if gain is not None and _need(gain, "gain", (torch.float32,), 1, dev).numel() != cols:
        _bad(f"norm_i8: {gain.numel()} gains for {cols} columns")
    return x2, x_stride, r2, r_stride, s, s_stride


def norm_i8(x, residual=None, gain=None, eps=1e-6, out=None, held=False):
    """Rows of x [..., columns] (bf16 or fp16), or of x + residual rounded to
    their type, brought to mean square 1, times gain [columns] (fp32), in 8 bits
    for `linear_i8`: (Codes, the sum, which is x without a residual), with
    `held` also the values that the codes stand for (fp32, x's shape).  `out`, if
    given, gets the sum: [rows, columns] with contiguous rows that do not
    overlap; it may be x or the residual."""
    L = lib()
    try:  # one cheap look at everything first: most calls need no more
        dev, dtype, (t, cols), x_stride = x.device, x.dtype, x.shape, x.stride(0)
        plain = (x.is_cuda and dtype in _16 and t > 0 and cols > 1 and x.stride(1) == 1 and x_stride >= cols and out is None
                 and (residual is None or (residual.dtype is dtype and residual.shape == x.shape and residual.device == dev
                                           and residual.stride(1) == 1 and residual.stride(0) >= cols))
                 and (gain is None or (gain.dtype is torch.float32 and gain.shape == (cols,) and gain.device == dev
                                       and gain.is_contiguous())))
    except (AttributeError, ValueError, TypeError, IndexError):
        plain = False
    if plain:
        x2, r2, r_stride, s, s_stride = x, residual, 0, None, 0
        if residual is not None:
            r_stride, s, s_stride = residual.stride(0), torch.empty_like(x, memory_format=torch.contiguous_format), cols
    else:
        x2, x_stride, r2, r_stride, s, s_stride = _norm_args(x, residual, gain, out)
        dev, (t, cols) = x.device, x2.shape
    codes = torch.empty(L.as_i8_bytes(t, cols), dtype=torch.int8, device=dev)
    scale = torch.empty(t, dtype=torch.float32, device=dev)
    values = torch.empty(x.shape, dtype=torch.float32, device=dev) if held else None
    _call(L.as_norm_i8, dev, x2.data_ptr(), None if r2 is None else r2.data_ptr(), _TYPES[x.dtype], t, cols, x_stride,
          r_stride, None if gain is None else gain.data_ptr(), eps, None if s is None else s.data_ptr(), s_stride,
          codes.data_ptr(), scale.data_ptr(), values.data_ptr() if held else None)
    total = x if s is None else s if out is not None or x.dim() == 2 else s.view(x.shape)
    c = Codes(codes, scale, t, cols, x.dtype)
    return (c, total, values) if held else (c, total)


def linear_i8(x, w: PackedWeight, bias=None, dtype=None, out=None):
    """x [..., n_in] (bf16 or fp16) quantised per token, times the packed
    weights: [..., n_out] of `dtype` (default: x's; fp32 allowed).  x may be
    `Codes`: [rows, n_out].  `out`, if given, is [tokens, n_out] with contiguous
    rows that do not overlap."""
    L = lib()
    held = isinstance(x, Codes)
    if held:
        dev, t = x.codes.device, x.n_rows
        if not (x.codes.is_cuda and x.codes.dtype is torch.int8 and x.scale.dtype is torch.float32
                and x.scale.device == dev and x.codes.is_contiguous() and x.scale.is_contiguous()
                and x.n_cols == w.n_in and x.codes.numel() == L.as_i8_bytes(t, w.n_in) and x.scale.numel() == t):
            _bad(f"linear_i8: {x.codes.numel()} codes {x.codes.dtype} on {dev} and {x.scale.numel()} scales of "
                 f"{t} x {x.n_cols}, the weights take {w.n_in} inputs")
    else:
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
    y_stride = y.stride(0) if t > 1 else w.n_out
    bias_at = None if bias is None else bias.data_ptr()
    if held:
        _call(L.as_linear_i8_codes, dev, x.codes.data_ptr(), x.scale.data_ptr(), t, w.n_in, codes.data_ptr(),
              scale.data_ptr(), bias_at, w.n_out, y.data_ptr(), _TYPES[y.dtype], y_stride)
        return y
    n = L.as_linear_i8_workspace(t, w.n_in, w.n_out)
    _keep, ws = _workspace(n, dev)
    _call(L.as_linear_i8, dev, x2.data_ptr(), _TYPES[x.dtype], t, w.n_in, x_stride, codes.data_ptr(),
          scale.data_ptr(), bias_at, w.n_out, y.data_ptr(), _TYPES[y.dtype], y_stride, ws, n)
    return y if out is not None or x.dim() == 2 else y.view(*x.shape[:-1], w.n_out)


# ------------------------------------------------------------------ prompts

def _packed(x, name, dtype=None, device=None, dim=None):
    """x [tokens, heads, dim] with its last two dimensions contiguous, and its
    row stride (0 for one row, where it is not used)."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 3 and x.dtype in _16 and x.shape[1] >= 1
            and (dtype is None or (x.dtype == dtype and x.device == device and x.shape[2] == dim))):
        what = f"{tuple(x.shape)} {x.dtype} on {x.device}" if isinstance(x, torch.Tensor) else type(x)
        _bad(f"{name}: {what}, not [tokens, heads, channels] in 16 bits on one device")
    token, head, step = x.stride()
    if step != 1 or (x.shape[1] > 1 and head != x.shape[2]):
        x = x.contiguous()
        token = x.stride(0)
    return x, token if x.shape[0] > 1 else 0


def _aligned_rows(x, stride):
    """Rows at addresses that are multiples of 16 bytes."""
    if x.data_ptr() % 16 or stride % 8:
        x = x.clone(memory_format=torch.contiguous_format)
        stride = x.stride(0) if x.shape[0] > 1 else 0
    return x, stride


def attention_prompt(q, k, v, offsets, scale=None, out=None):
    """Causal attention of packed sequences: q [tokens, q_heads, dim], k and v
    [tokens, kv_heads, dim] (bf16 or fp16; parts of one projection's output are
    fine), rows offsets[b]..offsets[b + 1] - 1 being sequence b's (int32 [seqs +
    1], rising from 0).  Every token attends to its sequence's tokens up to
    itself, head j to key/value head j / (q_heads / kv_heads).  `scale` defaults
    to dim ** -0.5.  Rows of no sequence are not written: give `out` (contiguous,
    q's shape) where what they hold matters."""
    try:  # one cheap look at everything first: most calls need no more
        dev, dtype, (t, heads, dim) = q.device, q.dtype, q.shape
        (q_token, q_head, q_step), (k_token, k_head, k_step), (v_token, v_head, v_step) = q.stride(), k.stride(), v.stride()
        at = q.data_ptr(), k.data_ptr(), v.data_ptr()
        plain = (q.is_cuda and dtype in _16 and k.dtype is dtype and v.dtype is dtype and k.device == v.device == dev
                 and t > 1 and k.shape == v.shape == (t, k.shape[1], dim) and q_step == k_step == v_step == 1
                 and q_head == k_head == v_head == dim and not (at[0] | at[1] | at[2]) & 15
                 and not (q_token | k_token | v_token) & 7)
    except (AttributeError, ValueError, TypeError, IndexError):
        plain = False
    if not plain:
        q, q_token = _packed(q, "q")
        dev, (t, heads, dim) = q.device, q.shape
        k, k_token = _packed(k, "k", q.dtype, dev, dim)
        v, v_token = _packed(v, "v", q.dtype, dev, dim)
        if k.shape != v.shape or k.shape[0] != t:
            _bad(f"attention_prompt: q has {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
        q, q_token = _aligned_rows(q, q_token)
        k, k_token = _aligned_rows(k, k_token)
        v, v_token = _aligned_rows(v, v_token)
        at = q.data_ptr(), k.data_ptr(), v.data_ptr()
    if not (isinstance(offsets, torch.Tensor) and offsets.dtype is torch.int32 and offsets.dim() == 1
            and offsets.shape[0] >= 1 and offsets.device == dev and offsets.is_contiguous()):
        _bad("attention_prompt: offsets are int32 [sequences + 1] on the device of q")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif not (isinstance(out, torch.Tensor) and out.dtype == q.dtype and out.shape == q.shape and out.device == dev
              and out.is_contiguous()):
        _bad("attention_prompt: out is contiguous and of q's shape, type and device")
    L = lib()
    seqs, kv_heads = offsets.shape[0] - 1, k.shape[1]
    need = _on(L.as_attention_prompt_workspace, dev, t, heads, kv_heads, seqs)
    _keep, ws = _workspace(need, dev)
    _call(L.as_attention_prompt, dev, *at, _TYPES[q.dtype], t, heads, kv_heads, dim, q_token, k_token, v_token, offsets.data_ptr(), seqs, dim ** -0.5 if scale is None else scale,
          out.data_ptr(), ws, need)
    return out


@dataclasses.dataclass
class PagePool:
    """Free pages: a stack of page numbers, int32 [pages], of which the first
    count[0] (int32 [1]) are free; the last one is taken first."""
    stack: torch.Tensor
    count: torch.Tensor

    @staticmethod
    def full(n_pages, device="cuda") -> "PagePool":
        """All of n_pages pages, page 0 taken first."""
        return PagePool(torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device),
                        torch.full((1,), n_pages, dtype=torch.int32, device=device))


@dataclasses.dataclass
class Places:
    """Where packed tokens go: offsets int32 [seqs + 1] (first row of every
    sequence, and the number of rows), sequence and slot of every row (int32
    [tokens]; -1 where a sequence was refused)."""
    offsets: torch.Tensor
    seq: torch.Tensor
    slot: torch.Tensor


def _pool_args(name, pool, page_table, length, other, other_types, new_length, new_count):
    """Checks of what a pool's calls take: addresses of the stack, its count, the
    table, the lengths, the other array and the new lengths and count."""
    stack, count, i32, one = pool.stack, pool.count, torch.int32, (1,)
    try:
        dev, row = page_table.device, page_table.shape[:1]
        fine = (page_table.is_cuda and page_table.dim() == 2 and len(stack.shape) == 1
                and page_table.dtype is stack.dtype is count.dtype is length.dtype is i32
                and new_length.dtype is new_count.dtype is i32 and other.dtype in other_types
                and count.shape == new_count.shape == one and length.shape == other.shape == new_length.shape == row
                and stack.device == count.device == length.device == other.device == dev
                and new_length.device == new_count.device == dev and page_table.is_contiguous()
                and stack.is_contiguous() and length.is_contiguous() and other.is_contiguous()
                and new_length.is_contiguous())
    except AttributeError:
        fine = False
    if not fine:
        what = [(tuple(x.shape), x.dtype, str(x.device)) if isinstance(x, torch.Tensor) else type(x)
                for x in (stack, count, page_table, length, other, new_length, new_count)]
        _bad(f"{name}: contiguous CUDA arrays of one pool and its sequences are needed, not {what}")
    return [x.data_ptr() for x in (stack, count, page_table, length, other, new_length, new_count)]


def pages_reserve(pool: PagePool, page_table, page, length, add, n_tokens, new_length=None, new_count=None) -> Places:
    """Pages for add[b] more tokens of every sequence b, which holds length[b]
    (int32 [seqs]), and where the n_tokens packed rows go.  In order, sequences get
    their pages as long as the pool has them for all up to them; a refused one
    keeps its length.  `length` and the pool's count are brought up to date in
    place, or left alone and written to `new_length` and `new_count` where given."""
    new_length = length if new_length is None else new_length
    new_count = pool.count if new_count is None else new_count
    stack, count, table, held, more, after, left = _pool_args("pages_reserve", pool, page_table, length, add, (torch.int32,),
                                                              new_length, new_count)
    dev, (seqs, max_pages) = page_table.device, page_table.shape
    if not 0 <= n_tokens <= 1 << 30 or not 0 < page <= 4096:  # (ctypes passes the lowest 32 bits of others)
        _bad(f"pages_reserve: {n_tokens} tokens, pages of {page} slots")
    L = lib()
    # one allocation: scratch memory, then the three results
    need = L.as_pages_reserve_workspace(seqs)
    ints = torch.empty(need // 4 + seqs + 1 + 2 * n_tokens, dtype=torch.int32, device=dev)
    at = ints.data_ptr()
    first = at + need
    seq = first + 4 * (seqs + 1)
    _call(L.as_pages_reserve, dev, stack, count, pool.stack.numel(), table, seqs, max_pages, page, held, more,
          n_tokens, left, after, first, seq, seq + 4 * n_tokens, at, need)
    return Places(*ints.split_with_sizes((need // 4, seqs + 1, n_tokens, n_tokens))[1:])


def pages_release(pool: PagePool, page_table, page, length, which, new_length=None, new_count=None):
    """Give back the pages of the sequences that `which` marks (bool [seqs]);
    their lengths become 0.  In place, or into `new_length` and `new_count`, as
    for `pages_reserve`; the stack of free pages is written in either case."""
    new_length = length if new_length is None else new_length
    new_count = pool.count if new_count is None else new_count
    stack, count, table, held, marks, after, left = _pool_args("pages_release", pool, page_table, length, which,
                                                               (torch.bool, torch.uint8), new_length, new_count)
    if not 0 < page <= 4096:
        _bad(f"pages_release: pages of {page} slots")
    seqs, max_pages = page_table.shape
    _call(lib().as_pages_release, page_table.device, stack, count, pool.stack.numel(), table, seqs, max_pages, page,
          held, marks, left, after)


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


def cache_append_packed(cache: Cache, k, v, seq, slot, pos=None, held=False):
    """Put packed k, v [tokens, heads, dim] into slot slot[t] of sequence seq[t]
    (int32 [tokens]; -1: passed over), as `pages_reserve` gives them.  Positions are
    pos[t] (default: slot).  With `held`, returns the values that the cache holds for them now (two
    fp32 tensors of k's shape, not written for tokens passed over)."""
    c = cache._c
    dev = cache.k.device
    try:  # one cheap look at everything first: most calls need no more
        dtype, (t, heads, dim), (k_token, k_head, k_step), (v_token, v_head, v_step) = k.dtype, k.shape, k.stride(), v.stride()
        i32, rows = torch.int32, (t,)
        plain = (dtype in _16 and v.dtype is dtype and k.device == v.device == seq.device == slot.device == dev and t > 1
                 and v.shape == k.shape and heads == c.n_heads and dim == c.dim and k_step == v_step == 1
                 and k_head == v_head == dim and seq.dtype is slot.dtype is i32 and seq.shape == slot.shape == rows
                 and seq.is_contiguous() and slot.is_contiguous()
                 and (pos is None or (pos.dtype is i32 and pos.shape == rows and pos.device == dev
                                      and pos.is_contiguous())))
    except (AttributeError, ValueError, TypeError, IndexError):
        plain = False
    if not plain:
        if not (isinstance(k, torch.Tensor) and k.dtype in _16):
            _bad("cache_append_packed: k in 16 bits is needed")
        k, k_token = _packed(k, "k", k.dtype, dev, c.dim)
        v, v_token = _packed(v, "v", k.dtype, dev, c.dim)
        t = k.shape[0]
        if k.shape != v.shape or k.shape[1] != c.n_heads:
            _bad(f"cache_append_packed: k has {tuple(k.shape)}, v {tuple(v.shape)}, the cache {c.n_heads} heads")
        for name, x in (("seq", seq), ("slot", slot), ("pos", pos)):
            if x is not None and _need(x, name, (torch.int32,), 1, dev).numel() != t:
                _bad(f"{name}: {x.numel()} numbers for {t} tokens")
    hk = hv = None
    if held:
        hk = torch.empty(k.shape, dtype=torch.float32, device=dev)
        hv = torch.empty_like(hk)
    _call(lib().as_cache_append_packed, dev, c, k.data_ptr(), v.data_ptr(), _TYPES[k.dtype], t, k_token, v_token,
          seq.data_ptr(), slot.data_ptr(), None if pos is None else pos.data_ptr(), hk.data_ptr() if held else None,
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
