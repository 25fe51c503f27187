"""The operators' definitions in 64 bits, element by element as their header
states them, and bounds of what float arithmetic may differ by."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# half a unit in the last place, of 1 and of the least value
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
# one rounding of a 32-bit sum (matrix instructions may truncate)
STEP = 2.0 ** -23


def act64(y, act):
    if act == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == "silu":
        return y / (1 + torch.exp(-y))
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y / math.sqrt(2)))
    return y


def linear(x, w, out_dtype, bias=None, w2=None, bias2=None, residual=None, act="none"):
    """(result, bound of the error) in 64 bits.

    Sums: blocks of 32 products added one after another, then at most 40 more
    additions (inside a block, across waves and splits), each off by STEP of the
    sum of magnitudes. Activations have slopes up to 1.13 and are off by less
    than 8 STEP themselves. The result is rounded once."""
    d = lambda t: None if t is None else t.double()  # noqa: E731
    x, w, bias, w2, bias2, residual = map(d, (x, w, bias, w2, bias2, residual))
    steps = (x.shape[1] / 32 + 40) * STEP

    def product(m, b):
        y, size = x @ m.t(), x.abs() @ m.abs().t()
        if b is not None:
            y, size = y + b, size + b.abs()
        return y, steps * size

    y, ey = product(w, bias)
    a = act64(y, act)
    ea = 1.13 * ey + (8 * STEP * a.abs() if act != "none" else 0)
    if w2 is not None:
        z, ez = product(w2, bias2)
        a, ea = a * z, ea * z.abs() + a.abs() * ez + ea * ez + STEP * (a * z).abs()
    if residual is not None:
        a = a + residual
        ea = ea + STEP * a.abs()
    return a, ea + (a.abs() + ea) * U[out_dtype] + TINY[out_dtype]


def two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def kept(x):
    """(value the 8-bit cache stands for, exponent byte) of [..., dim]: NaN
    where x is not finite."""
    y = x.double().unflatten(-1, (-1, 32))
    known = torch.isfinite(y)
    top = torch.where(known, y.abs(), 0.0).amax(-1, keepdim=True)
    m, e = torch.frexp(top / 448)               # top / 448 = m 2^e, 0.5 <= m < 1
    e = torch.where(m > 0.5, e, e - 1)          # least e with top / 448 <= 2^e
    e = torch.where(top > 0, e, torch.full_like(e, -126)).clamp(-126, 120)
    z = torch.where(known, y, 0.0) / two_to(e)
    _, f = torch.frexp(z)
    step = two_to((f - 1).clamp(min=-6) - 3)
    z = torch.round(z / step) * step * two_to(e)
    if x.dtype == torch.float16:
        z = z.clamp(-61440, 61440)
    return torch.where(known, z, math.nan).flatten(-2), (e.squeeze(-1) + 127).to(torch.uint8)


def cache_values(cache):
    """k and v of a cache in 64 bits, [pages, heads, page, dim]."""
    out = []
    for codes, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = codes.double()
        if scales is not None:
            x = x * two_to(scales.long() - 127).repeat_interleave(32, -1)
        out.append(x)
    return out


def attend(q, cache, pages, lengths, q_start=None, window=0, scale=None):
    """(result, bound of the error) in 64 bits; pages, lengths, q_start lists.

    The weights of the product with the values are rounded to the type of q
    (U of each, weights of a type's least normal and below lost), the result
    too; scores are off by some STEP of the sums of magnitudes, which the
    exponential turns into relative errors of the weights."""
    dt, dim = q.dtype, q.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    group = q.shape[1] // cache.heads
    kv = cache_values(cache)
    seqs = len(lengths)
    if q_start is None:
        q_start = list(range(seqs + 1))
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    far = torch.zeros_like(out)
    covered = torch.zeros(q.shape[0], dtype=torch.bool)
    for b in range(seqs):
        n, first = q_start[b + 1] - q_start[b], q_start[b]
        if n <= 0:
            continue
        covered[first:first + n] = True
        reach = min(max(lengths[b], 0), len(pages[b]) * cache.page)
        held = [j for j in range(reach) if 0 <= pages[b][j // cache.page] < cache.k.shape[0]]
        if not held:
            continue
        j = torch.tensor(held, device=q.device)
        table = torch.tensor(pages[b], device=q.device)
        k, v = (x[table[j // cache.page], :, j % cache.page] for x in kv)     # [keys, heads, dim]
        k, v = (x.repeat_interleave(group, 1).transpose(0, 1) for x in (k, v))
        qb = q[first:first + n].double().transpose(0, 1)                       # [heads, n, dim]
        s = torch.matmul(qb, k.transpose(1, 2).contiguous()) * scale
        size = torch.matmul(qb.abs(), k.abs().transpose(1, 2).contiguous()) * abs(scale)
        p = lengths[b] - n + torch.arange(n, device=q.device)[:, None]
        seen = j <= p
        if window:
            seen = seen & (j > p - window)
        s = torch.where(seen, s, -math.inf)
        top = s.amax(-1, keepdim=True)
        e = torch.where(seen, torch.exp(s - torch.where(top > -math.inf, top, 0.0)), 0.0)
        w = e / e.sum(-1, keepdim=True).clamp(min=1e-300)
        # masked values do not count, whatever they are
        v0 = torch.where(torch.isfinite(v), v, 0.0)
        r = torch.matmul(w, v0)
        for h, key in torch.nonzero(~torch.isfinite(v).all(-1)).tolist():
            hit = w[h, :, key] > 0
            r[h, hit] = r[h, hit] + w[h, hit, key, None] * (v[h, key] - v0[h, key])
        spread = torch.where(seen, torch.nan_to_num(size), 0.0).amax(-1, keepdim=True)
        rel = 2 * (dim / 16 + 8) * STEP * spread + 16 * STEP + (len(held) / 16 + 40) * STEP
        mass = torch.matmul(w, v0.abs())
        bound = (U[dt] + rel) * mass + U[dt] * (r.abs() + mass * rel)
        lost = 2.0 ** -24 if dt == torch.float16 else 0.0
        bound = bound + lost * v0.abs().sum(1, keepdim=True) + TINY[dt]
        out[first:first + n] = r.transpose(0, 1)
        far[first:first + n] = bound.transpose(0, 1)
    return out, far, covered
