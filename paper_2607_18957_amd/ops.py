"""Python binding of the operators in libii.so (include/ii_ops.h): products
with a model's matrices, its paged key/value cache, attention over that cache,
norms at the borders of blocks, rotary positions, low-rank adapters, log-probabilities
of tokens.

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

__all__ = ["Cache", "ii_adapt", "ii_attend", "ii_cache_append", "ii_cache_read", "ii_cache_write",
           "ii_linear", "ii_logprobs", "ii_norm", "ii_rotary_freqs", "ii_rotate", "work_buffer", "MAX_TOP", "WORK_BYTES"]

WORK_BYTES = 64 << 20
MAX_TOP = 64
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
NORMS = {"rms": 0, "layer": 1}
LAYOUTS = {"half": 0, "interleaved": 1}

_c = ii._c
_lib = ii._lib
for _n, _k in (("ii_linear", 1), ("ii_cache_write", 2), ("ii_cache_read", 2), ("ii_attend", 2),
               ("ii_norm", 1), ("ii_rotate", 2), ("ii_cache_append", 4), ("ii_logprobs", 1),
               ("ii_adapt", 1)):
    ii._sig(_n, _c.c_int, *[_c.c_char_p] * _k, _c.c_void_p)
_call_linear, _call_attend = _lib.ii_linear, _lib.ii_attend
_call_write, _call_read = _lib.ii_cache_write, _lib.ii_cache_read
_call_norm, _call_rotate = _lib.ii_norm, _lib.ii_rotate
_call_append, _call_logprobs = _lib.ii_cache_append, _lib.ii_logprobs
_call_adapt = _lib.ii_adapt
ii._sig("ii_rotary_freqs", _c.c_int, _c.c_int32, *[_c.c_double] * 4, _c.c_int64, _c.POINTER(_c.c_double))

_CODES = {getattr(torch, n): c for c, n in ii._TORCH_DTYPES.items()}
_LINEAR = struct.Struct("=4i3qPqPqPqPPPqPqPQ".replace("P", "Q"))  # struct ii_linear_args
_CACHE = struct.Struct("=4iq4Q6q")                                # struct ii_cache
_TOKENS = struct.Struct("=2iqQ2qQ2qQ")                            # struct ii_tokens
_ATTEND = struct.Struct("=2i2qQ2qQ2qQ2q2Q3qfiQQ")                 # struct ii_attend_args
_NORM = struct.Struct("=4i2qQqQqQq4QQqQq3fi")                     # struct ii_norm_args
_ROTARY = struct.Struct("=2Q2ifi")                                # struct ii_rotary
_TURN = struct.Struct("=4iqQ2qQ2q")                               # struct ii_turn
_LOGPROBS = struct.Struct("=2i2qQq5Qfi2Q")                        # struct ii_logprobs_args
_ADAPT = struct.Struct("=4i4qQqQ2qQ2q3QQqQqQQ")                  # struct ii_adapt_args


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


def _matrix(t, shape, dt, what: str) -> tuple[int, int]:
    """(address, row stride) of a matrix that may be missing."""
    if t is None:
        return 0, 0
    if t.shape != shape or t.dtype != dt:
        raise ValueError(f"{what} is not {list(shape)} of {dt}")
    return _rows(t, what)


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
    (t, _, _), dt = k.shape, k.dtype
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


def ii_norm(out, x, weight=None, *, bias=None, post: bool = False, post_weight=None, post_bias=None,
            gate=None, residual=None, sum=None, scale: float = 1.0, kind: str = "rms",
            eps: float = 1e-5, offset: float = 0.0, stream=None) -> None:
    """sum = scale * gate * y + residual, y = x or (post) x normalised; out = sum
    normalised. A norm is of kind "rms" or "layer", times (weight + offset), plus
    bias. out or sum may be None; sum may be residual, and out x."""
    shape, dt = x.shape, x.dtype
    m, n = shape
    xp, xs = _rows(x, "x")
    held = dt if residual is None and sum is None else (sum if residual is None else residual).dtype
    gp, gs = _matrix(gate, shape, dt, "gate")
    rp, rs = _matrix(residual, shape, held, "residual")
    sp, ss = _matrix(sum, shape, held, "sum")
    op, os_ = _matrix(out, shape, dt, "out")
    pw = pb = wp = bp = 0
    if post_weight is not None:
        pw = _vector(post_weight, n, dt, "post_weight")
    if post_bias is not None:
        pb = _vector(post_bias, n, dt, "post_bias")
    if weight is not None:
        wp = _vector(weight, n, dt, "weight")
    if bias is not None:
        bp = _vector(bias, n, dt, "bias")
    args = _NORM.pack(_code(_CODES, dt), _code(_CODES, held), _code(NORMS, kind), bool(post), m, n, xp, xs,
                      gp, gs, rp, rs, pw, pb, wp, bp, sp, ss, op, os_, scale, eps, offset, 0)
    rc = _call_norm(args, ii._stream(stream))
    if rc:
        ii._check(rc, "ii_norm")


def ii_rotary_freqs(rot_dim: int, *, base: float = 10000.0, factor: float = 1.0, low: float = 1.0,
                    high: float = 4.0, original: int = 0, device="cuda"):
    """Radians a position of each of rot_dim / 2 pairs: base^(-2 i / rot_dim),
    divided by factor where a pair turns less than `low` times over the
    `original` context, kept where it turns more than `high` times, in proportion
    between (original 0: all are divided)."""
    freqs = torch.empty(max(rot_dim // 2, 0), dtype=torch.float64)
    rc = _lib.ii_rotary_freqs(rot_dim, base, factor, low, high, original,
                              _c.cast(freqs.data_ptr(), _c.POINTER(_c.c_double)))
    if rc:
        ii._check(rc, "ii_rotary_freqs")
    return freqs.to(device)


def _rotary(tokens: int, positions, freqs, layout: str, magnitude: float) -> bytes:
    _fits(freqs.dim() == 1, "freqs is not a vector")
    return _ROTARY.pack(_vector(positions, tokens, torch.int64, "positions"),
                        _vector(freqs, freqs.shape[0], torch.float64, "freqs"), 2 * freqs.shape[0],
                        _code(LAYOUTS, layout), magnitude, 0)


def _turn(out, x) -> bytes:
    tokens, heads, dim = x.shape
    _fits(out.shape == x.shape and out.dtype == x.dtype, "out and x differ in shape or type")
    xt, xh, xl = x.stride()
    ot, oh, ol = out.stride()
    _fits(xl == ol == 1, "the last axis of x or out is not contiguous")
    return _TURN.pack(_code(_CODES, x.dtype), heads, dim, 0, tokens, x.data_ptr(), xt, xh, out.data_ptr(),
                      ot, oh)


def ii_rotate(out, x, positions, freqs, *, layout: str = "half", magnitude: float = 1.0,
              stream=None) -> None:
    """Turn heads x [tokens, heads, dim] by their tokens' positions [tokens] into
    out, which may be x: pair i of the first 2 * len(freqs) elements by position *
    freqs[i], pairs (i, i + len(freqs)) or, "interleaved", (2 i, 2 i + 1)."""
    rc = _call_rotate(_turn(out, x), _rotary(x.shape[0], positions, freqs, layout, magnitude),
                      ii._stream(stream))
    if rc:
        ii._check(rc, "ii_rotate")


def ii_cache_append(cache: Cache, k, v, slots, positions, freqs, *, q=None, q_out=None,
                    layout: str = "half", magnitude: float = 1.0, stream=None) -> None:
    """ii_cache_write with the keys turned by their tokens' positions on the way;
    queries q [tokens, heads, dim] of the same tokens are turned into q_out, which
    may be q."""
    _fits((q is None) == (q_out is None), "q and q_out go together")
    turn = None
    tokens, _, _ = k.shape
    if q is not None:
        rows, _, dim = q.shape
        _fits(rows == tokens and dim == cache.dim and q.dtype == k.dtype,
              "q is not [tokens, heads, dim] of the keys' type")
        turn = _turn(q_out, q)
    rc = _call_append(cache.args, _tokens(cache, k, v, slots),
                      _rotary(tokens, positions, freqs, layout, magnitude), turn, ii._stream(stream))
    if rc:
        ii._check(rc, "ii_cache_append")


def ii_logprobs(logits, *, targets=None, logprob=None, entropy=None, top_ids=None, top_logprobs=None,
                scale: float = 1.0, work=None, stream=None) -> None:
    """From logits [rows, vocab], times scale: log-probabilities of targets [rows]
    into logprob [rows], the entropy of each row into entropy [rows], the largest
    logits' tokens, equal ones in their order and NaN as -infinity, into top_ids
    [rows, top] and their log-probabilities into top_logprobs."""
    rows, vocab = logits.shape
    at, stride = _rows(logits, "logits")
    f32, i64 = torch.float32, torch.int64
    top = 0
    _fits((top_ids is None) == (top_logprobs is None), "top_ids and top_logprobs go together")
    _fits((targets is None) == (logprob is None), "targets and logprob go together")
    ids = values = 0
    if top_ids is not None:
        _, top = top_ids.shape
        _fits(top_ids.shape == top_logprobs.shape == (rows, top) and top_ids.is_contiguous()
              and top_logprobs.is_contiguous() and top_ids.dtype == i64 and top_logprobs.dtype == f32,
              "top_ids and top_logprobs are not contiguous [rows, top] of int64 and float32")
        if top:
            ids, values = top_ids.data_ptr(), top_logprobs.data_ptr()
    args = _LOGPROBS.pack(_code(_CODES, logits.dtype), top, rows, vocab, at, stride,
                          _vector(targets, rows, i64, "targets"), _vector(logprob, rows, f32, "logprob"),
                          _vector(entropy, rows, f32, "entropy"), ids, values, scale, 0, *_work(work))
    rc = _call_logprobs(args, ii._stream(stream))
    if rc:
        ii._check(rc, "ii_logprobs")


def ii_adapt(out, x, a, b, adapters, *, scales=None, ranks=None, base=None, work=None,
             stream=None) -> None:
    """out = base + scales[c] * B_c (A_c x) for each row of x [m, k], c its adapter
    in adapters [m] (int32; none where it is negative or past the last): a [count,
    rank, k], b [count, n, rank], of which adapter c uses the first ranks[c] rows
    and columns. base [m, n] may be out; either may be float32."""
    (m, k), (count, rank, ka), dt = x.shape, a.shape, x.dtype
    _, n, _ = b.shape
    _fits(ka == k and b.shape == (count, n, rank) and a.dtype == b.dtype == dt and out.shape == (m, n),
          "shapes or types of out, x, a, b differ")
    ac, ar, al = a.stride()
    bc, br, bl = b.stride()
    _fits((al == 1 or k < 2) and (bl == 1 or rank < 2), "the last axis of a or b is not contiguous")
    xp, xs = _rows(x, "x")
    op, os_ = _rows(out, "out")
    bp = bs = 0
    base_dt = dt
    if base is not None:
        _fits(base.shape == (m, n), "base is not [m, n]")
        bp, bs = _rows(base, "base")
        base_dt = base.dtype
    args = _ADAPT.pack(_code(_CODES, dt), _code(_CODES, out.dtype), _code(_CODES, base_dt), rank, m, n, k,
                       count, xp, xs, a.data_ptr(), ac, ar, b.data_ptr(), bc, br,
                       _vector(adapters, m, torch.int32, "adapters"),
                       _vector(scales, count, torch.float32, "scales"),
                       _vector(ranks, count, torch.int32, "ranks"), bp, bs, op, os_, *_work(work))
    rc = _call_adapt(args, ii._stream(stream))
    if rc:
        ii._check(rc, "ii_adapt")
