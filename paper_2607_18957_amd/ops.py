"""Python binding of the operators in libii.so (include/ii_ops.h): products
with a model's matrices, its paged key/value cache, attention over that cache.

As in ``ii``, every function has the name of the C entry point it calls and
turns its arguments into addresses, sizes and strides; the library checks and
runs them. Tensors are torch tensors on the GPU (any object with data_ptr,
shape, stride and dtype), their last axis contiguous; outputs are the
caller's. Shapes that do not fit each other raise ValueError here, what the
library refuses raises ii.IIError.

  work    None, or a uint8 tensor that was zero-filled once before its first
          use (work_buffer makes one): scratch for work split over a long
          axis. Calls that may overlap on different streams need one each.
  stream  as in ``ii``: None (null stream), an int handle, a torch stream
"""
from __future__ import annotations

import struct

import torch

from . import ii

__all__ = ["Cache", "ii_attend", "ii_cache_read", "ii_cache_write", "ii_linear", "work_buffer",
           "WORK_BYTES"]

WORK_BYTES = 64 << 20
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}

_c = ii._c
_lib = ii._lib
for _n, _k in (("ii_linear", 1), ("ii_cache_write", 2), ("ii_cache_read", 2), ("ii_attend", 2)):
    ii._sig(_n, _c.c_int, *[_c.c_char_p] * _k, _c.c_void_p)
_call_linear, _call_attend = _lib.ii_linear, _lib.ii_attend
_call_write, _call_read = _lib.ii_cache_write, _lib.ii_cache_read

_CODES = {getattr(torch, n): c for c, n in ii._TORCH_DTYPES.items()}
_LINEAR = struct.Struct("=4i3qPqPqPqPPPqPqPQ".replace("P", "Q"))  # struct ii_linear_args
_CACHE = struct.Struct("=4iq4Q6q")                                # struct ii_cache
_TOKENS = struct.Struct("=2iqQ2qQ2qQ")                            # struct ii_tokens
_ATTEND = struct.Struct("=2i2qQ2qQ2qQ2q2Q3qfiQQ")                 # struct ii_attend_args


def work_buffer(nbytes: int = WORK_BYTES, device="cuda"):
    """Zero-filled scratch for ``work`` (filled on torch's current stream)."""
    return torch.zeros(nbytes, dtype=torch.uint8, device=device)


def _fits(ok, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _code(names, key) -> int:
    try:
        return names[key]
    except KeyError:
        raise ValueError(f"{key} is none of {', '.join(map(str, names))}") from None


def _rows(t, what: str) -> tuple[int, int]:
    """(address, row stride) of a matrix."""
    s, last = t.stride()
    if last != 1 and t.shape[1] > 1:
        raise ValueError(f"{what}: the last axis is not contiguous")
    return t.data_ptr(), s


def _vector(t, n: int, dt, what: str) -> int:
    if t is None:
        return 0
    if t.dtype != dt or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what} is not a contiguous {dt} vector of {n}")
    return t.data_ptr()


def _work(t) -> tuple[int, int]:
    if t is None:
        return 0, 0
    _fits(t.is_contiguous(), "work is not contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def ii_linear(out, x, w, *, bias=None, w2=None, bias2=None, residual=None, act: str = "none",
              work=None, stream=None) -> None:
    """out = act(x w^T + bias) * (x w2^T + bias2) + residual; x [m, k], w and
    w2 [n, k] as a load leaves them, out and residual [m, n]."""
    (m, k), (n, kw), dt = x.shape, w.shape, x.dtype
    _fits(kw == k and w.dtype == dt and out.shape == (m, n), "shapes or types of out, x, w differ")
    xp, xs = _rows(x, "x")
    wp, ws = _rows(w, "w")
    op, os_ = _rows(out, "out")
    w2p = w2s = rp = rs = 0
    if w2 is not None:
        _fits(w2.shape == (n, k) and w2.dtype == dt, "w2 is not like w")
        w2p, w2s = _rows(w2, "w2")
    if residual is not None:
        _fits(residual.shape == (m, n) and residual.dtype == dt, "residual is not [m, n] of x's type")
        rp, rs = _rows(residual, "residual")
    args = _LINEAR.pack(_code(_CODES, dt), _code(_CODES, out.dtype), _code(ACTS, act), 0, m, n, k, xp,
                        xs, wp, ws, w2p, w2s, _vector(bias, n, dt, "bias"),
                        _vector(bias2, n, dt, "bias2"), rp, rs, op, os_, *_work(work))
    rc = _call_linear(args, ii._stream(stream))
    if rc:
        ii._check(rc, "ii_linear")


class Cache:
    """A paged key/value cache: k and v [pages, heads, page, dim] (any strides
    but the last axis'), in the activations' type or torch.float8_e4m3fn with
    k_scale and v_scale [pages, heads, page, dim / 32] of torch.uint8."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "heads", "dim", "page", "args")

    def __init__(self, k, v, k_scale=None, v_scale=None):
        pages, self.heads, self.page, self.dim = shape = k.shape
        ps, hs, ts, last = strides = k.stride()
        _fits(v.shape == shape and v.dtype == k.dtype and v.stride() == strides and last == 1,
              "k and v differ in shape, type or strides, or their last axis is not contiguous")
        ks = vs = sps = shs = sts = 0
        if k_scale is not None:
            _fits(v_scale is not None and k_scale.shape == v_scale.shape == (*shape[:3], self.dim // 32)
                  and k_scale.dtype == v_scale.dtype == torch.uint8
                  and k_scale.stride() == v_scale.stride() and k_scale.stride(3) == 1,
                  "scales are not uint8 [pages, heads, page, dim / 32] at the same strides")
            sps, shs, sts, _ = k_scale.stride()
            ks, vs = k_scale.data_ptr(), v_scale.data_ptr()
        _fits((k.dtype == torch.float8_e4m3fn) == (k_scale is not None),
              "scales go with float8_e4m3fn, and only with it")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.args = _CACHE.pack(_code(_CODES, k.dtype), self.heads, self.dim, self.page, pages,
                                k.data_ptr(), v.data_ptr(), ks, vs, ps, hs, ts, sps, shs, sts)

    @classmethod
    def empty(cls, pages: int, heads: int, page: int, dim: int, dtype=torch.float8_e4m3fn,
              device="cuda") -> "Cache":
        """A cache of zeros."""
        make = lambda last, dt: torch.zeros(pages, heads, page, last, dtype=dt, device=device)  # noqa: E731
        scales = [make(dim // 32, torch.uint8) for _ in range(2 * (dtype == torch.float8_e4m3fn))]
        return cls(make(dim, dtype), make(dim, dtype), *scales)


def _tokens(cache: Cache, k, v, slots) -> bytes:
    t, dt = k.shape[0], k.dtype
    _fits(k.shape == v.shape == (t, cache.heads, cache.dim) and v.dtype == dt,
          "k and v are not [tokens, heads, dim] of one type")
    _fits(slots.shape == (t,) and slots.dtype == torch.int64 and (t < 2 or slots.stride(0) == 1),
          "slots is not a contiguous int64 vector of a slot a token")
    ka, kb, kl = k.stride()
    va, vb, vl = v.stride()
    _fits(kl == vl == 1, "the last axis of k or v is not contiguous")
    return _TOKENS.pack(_code(_CODES, dt), 0, t, k.data_ptr(), ka, kb, v.data_ptr(), va, vb,
                        slots.data_ptr())


def ii_cache_write(cache: Cache, k, v, slots, *, stream=None) -> None:
    """Put k and v [tokens, heads, dim] into the cache at slots [tokens]
    (page * cache.page + token; negative: left out)."""
    rc = _call_write(cache.args, _tokens(cache, k, v, slots), ii._stream(stream))
    if rc:
        ii._check(rc, "ii_cache_write")


def ii_cache_read(cache: Cache, slots, k, v, *, stream=None) -> None:
    """Take the tokens at slots out of the cache into k and v [tokens, heads,
    dim] (slots that hold nothing give zeros)."""
    rc = _call_read(cache.args, _tokens(cache, k, v, slots), ii._stream(stream))
    if rc:
        ii._check(rc, "ii_cache_read")


def ii_attend(out, q, cache: Cache, pages, lengths, q_start=None, *, max_q: int = 1,
              max_len: int = 0, window: int = 0, scale: float | None = None, work=None,
              stream=None) -> None:
    """Attention of q [rows, heads, dim] over the cache into out, through the
    page table [seqs, columns]; scale defaults to dim ** -0.5."""
    (rows, heads, dim), dt = q.shape, q.dtype
    _fits(out.shape == q.shape and out.dtype == dt and dim == cache.dim,
          "out, q and the cache differ in shape or type")
    seqs, columns = pages.shape
    _fits(pages.dtype == lengths.dtype == torch.int32 and lengths.shape == (seqs,)
          and (seqs < 2 or lengths.stride(0) == 1), "pages or lengths are not int32 [seqs, ...]")
    starts = 0
    if q_start is not None:
        _fits(q_start.dtype == torch.int32 and q_start.shape == (seqs + 1,)
              and q_start.stride(0) == 1, "q_start is not a contiguous int32 vector of seqs + 1")
        starts = q_start.data_ptr()
    qr, qh, ql = q.stride()
    outr, outh, outl = out.stride()
    _fits(ql == outl == 1, "the last axis of q or out is not contiguous")
    at, table = _rows(pages, "pages")
    args = _ATTEND.pack(_code(_CODES, dt), heads, rows, seqs, q.data_ptr(), qr, qh, out.data_ptr(), outr,
                        outh, at, table, columns, lengths.data_ptr(), starts, max_q, max_len,
                        window, dim ** -0.5 if scale is None else scale, 0, *_work(work))
    rc = _call_attend(args, cache.args, ii._stream(stream))
    if rc:
        ii._check(rc, "ii_attend")
