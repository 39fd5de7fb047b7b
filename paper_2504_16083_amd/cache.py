"""ctypes binding of include/mmi_cache.h: rotary positions, the paged cache and
the attention of drafted tokens over it.

As in mmi.py the functions have the C names and marshal arguments only; what
the C side cannot see (types, shapes and devices of the tensors) is checked
here with ValueError, the rest by the library (MMIError). Tensors are torch
device tensors on the context's device; their strides are passed on, the last
dimension must be contiguous, the others not broadcast. Work goes to `stream`, or to the device's
current stream."""
from __future__ import annotations

import ctypes as ct
import math

import torch

from . import mmi
from .mmi import _check

D = 128
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}
TYPES = {"bf16": 0, "fp8": 1, "int8": 2, "fp4": 3}
ROW_BYTES = {"bf16": 256, "fp8": 128, "int8": 128, "fp4": 64}


class mmi_rope_cfg(ct.Structure):
    _fields_ = [("rot_dim", ct.c_int32), ("layout", ct.c_int32), ("scaling", ct.c_int32), ("inverse", ct.c_int32),
                ("sections", ct.c_int32 * 3), ("reserved", ct.c_int32),
                ("theta", ct.c_double), ("factor", ct.c_double), ("orig_len", ct.c_double),
                ("beta_fast", ct.c_double), ("beta_slow", ct.c_double), ("attn_factor", ct.c_double),
                ("inv_freq", ct.POINTER(ct.c_double))]


class mmi_cache(ct.Structure):
    _fields_ = [("type", ct.c_int32), ("page", ct.c_int32), ("Hkv", ct.c_int32), ("D", ct.c_int32),
                ("n_pages", ct.c_int64), ("k", ct.c_void_p), ("v", ct.c_void_p),
                ("k_scale", ct.c_void_p), ("v_scale", ct.c_void_p),
                ("page_stride", ct.c_int64), ("scale_stride", ct.c_int64)]


class mmi_tree(ct.Structure):
    _fields_ = [("n_seq", ct.c_int32), ("n_rows", ct.c_int32), ("Hq", ct.c_int32), ("max_rows", ct.c_int32),
                ("max_len", ct.c_int64), ("max_pages", ct.c_int32), ("mask_words", ct.c_int32),
                ("row_start", ct.c_void_p), ("length", ct.c_void_p), ("pages", ct.c_void_p), ("mask", ct.c_void_p),
                ("q_stride_s", ct.c_int64), ("q_stride_h", ct.c_int64),
                ("k_stride_s", ct.c_int64), ("k_stride_h", ct.c_int64),
                ("v_stride_s", ct.c_int64), ("v_stride_h", ct.c_int64),
                ("o_stride_s", ct.c_int64), ("o_stride_h", ct.c_int64),
                ("scale", ct.c_float), ("reserved", ct.c_int32)]


SYMBOLS = ["mmi_rope_freq", "mmi_rope", "mmi_cache_write", "mmi_cache_read", "mmi_tree_workspace", "mmi_tree_attention"]

_lib = None


def lib():
    global _lib
    if _lib is None:
        L = mmi.lib()
        vp, i64, sz, P = ct.c_void_p, ct.c_int64, ct.c_size_t, ct.POINTER
        sig = {
            "mmi_rope_freq": [P(mmi_rope_cfg), P(ct.c_double)],
            "mmi_rope": [vp, P(mmi.mmi_problem), P(mmi_rope_cfg), vp, vp, vp, vp, vp, vp],
            "mmi_cache_write": [vp, P(mmi_cache), vp, i64, i64, vp, i64, i64, vp, i64, vp],
            "mmi_cache_read": [vp, P(mmi_cache), vp, i64, vp, i64, i64, vp, i64, i64, vp],
            "mmi_tree_workspace": [vp, P(mmi_cache), P(mmi_tree), P(sz)],
            "mmi_tree_attention": [vp, P(mmi_cache), P(mmi_tree), vp, vp, vp, vp, vp, vp, sz, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes, f.restype = args, ct.c_int
        _lib = L
    return _lib


def _stream(ctx, stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(ctx.device)    # current_stream() without its object
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_BF16 = torch.bfloat16


def _rows(ctx, name, t, n, heads):
    """Strides of a [n, heads, 128] bfloat16 tensor on the context's device."""
    # one pass over what is right; the reasons are looked for only where something is wrong
    if t.dtype is _BF16 and t.get_device() == ctx.device and t.dim() == 3:
        rows, h, d = t.shape
        if d == D and (n is None or rows == n) and (heads is None or h == heads):
            ss, sh, sd = t.stride()
            if sd == 1:
                # torch leaves the stride of a dimension of one entry open
                if h == 1:
                    sh = D
                if rows <= 1:
                    ss = max(sh * h, D)
                if ss <= 0 or sh <= 0:             # two zeros would be read as packed
                    raise ValueError(f"{name} is broadcast over tokens or heads")
                return ss, sh
            raise ValueError(f"the last dimension of {name} must be contiguous")
    if t.dtype != _BF16 or t.dim() != 3 or t.shape[2] != D:
        raise ValueError(f"{name} must be a bfloat16 tensor [tokens, heads, {D}]")
    _here(ctx, name, t)
    raise ValueError(f"{name} has shape {tuple(t.shape)}, [{n}, {heads}, {D}] expected")


def _here(ctx, name, t):
    if t.get_device() != ctx.device:
        raise ValueError(f"{name} is on {t.device}, the context on device {ctx.device}")


def _array(ctx, name, t, dtype, shape):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    _here(ctx, name, t)
    return t.data_ptr()


def _kept(i, what):
    """Property: tensor i of what the object was made of, of which it has handed the address on."""
    def same(self, t):                             # x.t += 1 ends here with the tensor itself
        if t is not self._tensors[i]:
            raise AttributeError(f"a {what} keeps its tensors; make another one for others")
    return property(lambda self: self._tensors[i], same)


_data_ptr = torch.Tensor.data_ptr


def _ptr(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ rotary positions
class RopeCfg:
    """Rotation of the first rot_dim channels (mmi_rope_cfg). layout: "half"
    (pair i = channels i, i + rot_dim / 2) or "interleaved" (2i, 2i + 1);
    scaling: "none", "linear", "ntk" or "parts"; sections: pairs that take
    their position from the t, h and w axis; attn_factor 0: the default of the
    scaling; inv_freq: radians a position of every pair, in place of theta and
    the scaling."""

    def __init__(self, rot_dim=128, layout="half", theta=10000.0, scaling="none", factor=1.0, orig_len=0.0,
                 beta_fast=32.0, beta_slow=1.0, attn_factor=0.0, sections=(0, 0, 0), inv_freq=None):
        if layout not in LAYOUTS or scaling not in SCALINGS:
            raise ValueError(f"layout {layout!r} or scaling {scaling!r} is unknown")
        if len(sections) != 3:
            raise ValueError("sections are three numbers of pairs")
        self.axes = 3 if any(sections) else 1
        table = (ct.c_double * 64)()
        if inv_freq is not None:
            if len(inv_freq) != rot_dim // 2 or len(inv_freq) > 64:
                raise ValueError(f"{len(inv_freq)} frequencies for {rot_dim // 2} pairs")
            table[:len(inv_freq)] = [float(f) for f in inv_freq]
        self._table = table
        self.c = [mmi_rope_cfg(rot_dim, LAYOUTS[layout], SCALINGS[scaling], inverse, (ct.c_int32 * 3)(*sections), 0,
                               theta, factor, orig_len, beta_fast, beta_slow, attn_factor,
                               None if inv_freq is None else table)
                  for inverse in (0, 1)]
        if inv_freq is None:                       # once, not with every call
            _check(lib().mmi_rope_freq(ct.byref(self.c[0]), table))
            for c in self.c:
                c.inv_freq = ct.cast(table, ct.POINTER(ct.c_double))
        self.ref = [ct.byref(c) for c in self.c]


def mmi_rope(ctx, cfg, q=None, k=None, pos=None, q_out=None, k_out=None, inverse=False, stream=None):
    """Rotates q [S, Hq, 128] and k [S, Hkv, 128] (either may be None), in place
    unless q_out / k_out are given (strides as the inputs'). pos: int32 [S], or
    [3, S] with sections; None: 0 .. S-1. inverse: the gradient's rotation."""
    if q is None and k is None:
        raise ValueError("neither q nor k")
    S = (k if q is None else q).shape[0]
    Hq = Hkv = 1
    qs = ks = (0, 0)
    qp = kp = qo = ko = None
    if k is not None:
        ks, Hkv = _rows(ctx, "k", k, S, None), k.shape[1]
        Hq = Hkv
        kp = ko = k.data_ptr()
        if k_out is not None:
            if _rows(ctx, "k_out", k_out, S, Hkv) != ks:
                raise ValueError("k_out must have the strides of k")
            ko = k_out.data_ptr()
    if q is not None:
        qs, Hq = _rows(ctx, "q", q, S, None), q.shape[1]
        qp = qo = q.data_ptr()
        if q_out is not None:
            if _rows(ctx, "q_out", q_out, S, Hq) != qs:
                raise ValueError("q_out must have the strides of q")
            qo = q_out.data_ptr()
    pp = None
    if pos is not None:
        pp = _array(ctx, "pos", pos, torch.int32, (S,) if cfg.axes == 1 else (3, S))
    p = mmi.mmi_problem(S, Hq, Hkv, D, 64, *qs, *ks)
    _check(lib().mmi_rope(ctx.h, ct.byref(p), cfg.ref[1 if inverse else 0], pp, qp, kp, qo, ko, _stream(ctx, stream)))


# ------------------------------------------------------------------ the cache
class Cache:
    """The memory of a paged cache (mmi_cache). k, v: [n_pages, Hkv, page, 128]
    bfloat16 for type "bf16", else uint8 [n_pages, Hkv, page, bytes a row]
    (128 for "fp8" and "int8", 64 for "fp4") with k_scale, v_scale uint8
    [n_pages, Hkv, page, 4]; only the first dimension may be strided. The
    tensors stay the cache's, with the memory that they had when it was made."""

    def __init__(self, type, k, v, k_scale=None, v_scale=None):
        if type not in TYPES:
            raise ValueError(f"cache type {type!r} is unknown")
        bf16 = type == "bf16"
        self.type = type
        self._tensors = (k, v, None, None) if bf16 else (k, v, k_scale, v_scale)
        self.n_pages, self.Hkv, self.page = k.shape[:3]
        want = (self.n_pages, self.Hkv, self.page)
        self.device, self.index = k.device, k.get_device()
        row = D if bf16 else ROW_BYTES[type]
        stride = self._pool("k", k, torch.bfloat16 if bf16 else torch.uint8, want + (row,))
        if self._pool("v", v, torch.bfloat16 if bf16 else torch.uint8, want + (row,)) != stride:
            raise ValueError("k and v must have the same strides")
        scale = 0
        if not bf16:
            if k_scale is None or v_scale is None:
                raise ValueError(f"a cache of type {type!r} has scales")
            scale = self._pool("k_scale", k_scale, torch.uint8, want + (4,))
            if self._pool("v_scale", v_scale, torch.uint8, want + (4,)) != scale:
                raise ValueError("k_scale and v_scale must have the same strides")
        self.c = mmi_cache(TYPES[type], self.page, self.Hkv, D, self.n_pages, *map(_ptr, self._tensors),
                           stride * (2 if bf16 else 1), scale)
        self._used = [t for t in self._tensors if t is not None]
        self._at = [*map(_data_ptr, self._used)]
        self.ref = ct.byref(self.c)

    k, v, k_scale, v_scale = (_kept(i, "cache") for i in range(4))

    def _pool(self, name, t, dtype, shape):
        if t.dtype != dtype or tuple(t.shape) != shape:
            raise ValueError(f"{name} must be a {dtype} tensor of shape {shape}")
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, k on {self.device}")
        if math.prod(shape) and not t[0].is_contiguous():
            raise ValueError(f"the pages of {name} must be contiguous")
        if shape[0] <= 1:
            return 0
        if t.stride(0) < math.prod(shape[1:]):
            raise ValueError(f"the pages of {name} overlap")
        return t.stride(0)

    @classmethod
    def empty(cls, type, n_pages, Hkv, page, device=0):
        """A cache of this size, its memory zeroed."""
        if type not in TYPES:
            raise ValueError(f"cache type {type!r} is unknown")
        dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        if type == "bf16":
            return cls(type, *(torch.zeros(n_pages, Hkv, page, D, dtype=torch.bfloat16, device=dev) for _ in "kv"))
        return cls(type, *(torch.zeros(n_pages, Hkv, page, n, dtype=torch.uint8, device=dev)
                           for n in (ROW_BYTES[type], ROW_BYTES[type], 4, 4)))


def _on(ctx, cache):
    if cache.index != ctx.device:
        raise ValueError(f"the cache is on {cache.device}, the context on device {ctx.device}")
    if [*map(_data_ptr, cache._used)] != cache._at:
        raise ValueError("the cache's tensors have been given other memory")


def mmi_cache_write(ctx, cache, k, v, slot, stream=None):
    """Rows i of k and v [n, Hkv, 128] into slot[i] (int64 [n], page number *
    page + place; outside the cache: nowhere)."""
    _on(ctx, cache)
    n = k.shape[0]
    ks, vs = _rows(ctx, "k", k, n, cache.Hkv), _rows(ctx, "v", v, n, cache.Hkv)
    _check(lib().mmi_cache_write(ctx.h, cache.ref, k.data_ptr(), *ks, v.data_ptr(), *vs,
                                 _array(ctx, "slot", slot, torch.int64, (n,)), n, _stream(ctx, stream)))


def mmi_cache_read(ctx, cache, slot, k, v, stream=None):
    """Rows i of k and v [n, Hkv, 128] = what slot[i] holds (outside: zeros)."""
    _on(ctx, cache)
    n = k.shape[0]
    ks, vs = _rows(ctx, "k", k, n, cache.Hkv), _rows(ctx, "v", v, n, cache.Hkv)
    _check(lib().mmi_cache_read(ctx.h, cache.ref, _array(ctx, "slot", slot, torch.int64, (n,)), n,
                                k.data_ptr(), *ks, v.data_ptr(), *vs, _stream(ctx, stream)))


# ------------------------------------------------------------------ drafted tokens
class Tree:
    """A batch of sequences with drafted tokens (mmi_tree): row_start int32
    [n_seq + 1], length int32 [n_seq] (cached tokens), pages int32 [n_seq,
    max_pages], mask int64 [n_rows, words] (bit j of a row: it sees drafted
    token j; None: token i sees 0 .. i), max_rows and max_len the most drafted
    and cached tokens of a sequence. The tensors are checked once, here, and
    stay the batch's, with the memory that they have; their contents may change between calls, within these
    bounds, and so may max_rows, max_len and scale."""

    def __init__(self, row_start, length, pages, mask=None, max_rows=1, max_len=0, scale=0.0):
        self.max_rows, self.max_len, self.scale = max_rows, max_len, scale
        self._tensors = row_start, length, pages, mask
        self._n_seq, self.index = length.shape[0], length.get_device()
        # a mask of no words has no address and would be taken for none
        if pages.dim() != 2 or mask is not None and (mask.dim() != 2 or mask.shape[1] < 1):
            raise ValueError("pages must be a tensor [n_seq, max_pages], mask one [n_rows, words], words >= 1")
        self._max_pages = pages.shape[1]
        self._mask_rows, self._words = (None, 0) if mask is None else mask.shape
        self._check("row_start", row_start, torch.int32, (self._n_seq + 1,))
        self._check("length", length, torch.int32, (self._n_seq,))
        self._check("pages", pages, torch.int32, (self._n_seq, self._max_pages))
        if mask is not None:
            self._check("mask", mask, torch.int64, tuple(mask.shape))
        self._ptr = tuple(map(_ptr, self._tensors))
        self._used = [t for t in self._tensors if t is not None]
        self._at = [*map(_data_ptr, self._used)]

    row_start, length, pages, mask = (_kept(i, "batch") for i in range(4))

    def _check(self, name, t, dtype, shape):
        if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape}")
        if t.get_device() != self.index:
            raise ValueError(f"{name} is on {t.device}, length on {self.length.device}")

    def _struct(self, ctx, Hq, n_rows, *strides):
        if self.index != ctx.device:
            raise ValueError(f"the tree is on {self.length.device}, the context on device {ctx.device}")
        if [*map(_data_ptr, self._used)] != self._at:
            raise ValueError("the batch's tensors have been given other memory")
        if self._mask_rows is not None and self._mask_rows != n_rows:
            raise ValueError(f"mask has {self._mask_rows} rows for {n_rows} of q")
        if not strides:
            strides = (0,) * 8
        return mmi_tree(self._n_seq, n_rows, Hq, self.max_rows, self.max_len, self._max_pages, self._words, *self._ptr,
                        *strides, self.scale)


def mmi_tree_workspace(ctx, cache, tree, Hq, n_rows) -> int:
    """Bytes of workspace of a batch with these bounds."""
    need = ct.c_size_t()
    _check(lib().mmi_tree_workspace(ctx.h, cache.ref, ct.byref(tree._struct(ctx, Hq, n_rows)),
                                    ct.byref(need)))
    return need.value


def mmi_tree_attention(ctx, cache, tree, q, k, v, o, workspace, lse=None, stream=None):
    """o [n_rows, Hq, 128] = attention of the drafted tokens' rows q over their
    sequences' cached tokens and the drafted k, v [n_rows, Hkv, 128]; lse:
    float32 [Hq, n_rows] or None; workspace: uint8 of mmi_tree_workspace bytes,
    not shared with a call that may run at the same time."""
    _on(ctx, cache)
    n = q.shape[0]
    qs = _rows(ctx, "q", q, None, None)
    Hq = q.shape[1]
    t = tree._struct(ctx, Hq, n, *qs, *_rows(ctx, "k", k, n, cache.Hkv), *_rows(ctx, "v", v, n, cache.Hkv),
                     *_rows(ctx, "o", o, n, Hq))
    lp = None if lse is None else _array(ctx, "lse", lse, torch.float32, (Hq, n))
    wp = _array(ctx, "workspace", workspace, torch.uint8, (workspace.numel(),))
    _check(lib().mmi_tree_attention(ctx.h, cache.ref, ct.byref(t), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                    o.data_ptr(), lp, wp, workspace.numel(), _stream(ctx, stream)))
