"""Definitions in 64 bits of the operators between a decoder's products and its
answer, as their header states them, and bounds of what 32-bit arithmetic may
differ by. U is half a step of a type, E half a step of float."""
import math

import torch

from ops_ref import TINY, U, two_to

E = 2.0 ** -24


def norm(x, weight=None, bias=None, post=False, post_weight=None, post_bias=None, gate=None,
         residual=None, scale=1.0, kind="rms", eps=1e-5, offset=0.0, stream=None):
    """((sum, its bound), (out, its bound))."""
    d = lambda t: None if t is None else t.double()  # noqa: E731
    dt = x.dtype
    eps, offset = float(torch.tensor(eps)), float(torch.tensor(offset))  # as floats

    def one(y, off, w, b):
        """Normalised values; `off` is how far y may be off.

        The root is off by E, and by as much as y is in all; y - mean by E of
        either and what the mean is off; three products and a sum by E each."""
        mean = y.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(y[..., :1])
        var = ((y - mean) ** 2).mean(-1, keepdim=True)
        r = (var + eps) ** -0.5
        z = (y - mean) * r
        shift = off.mean(-1, keepdim=True) if kind == "layer" else 0
        far = (off + shift + 2 * E * (y.abs() + mean.abs())) * r
        root = (((off + shift) ** 2).mean(-1, keepdim=True) ** 0.5) * r + 4 * E
        far = far + z.abs() * (root + 4 * E)
        if w is not None:
            w = d(w) + offset
            z, far = z * w, far * w.abs() + (z * w).abs() * 3 * E
        if b is not None:
            z = z + d(b)
            far = far + z.abs() * 2 * E
        return z, far

    y, off = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    if post:
        y, off = one(y, off, post_weight, post_bias)
    f = scale * (torch.ones_like(y) if gate is None else d(gate))
    y, off = y * f, off * f.abs() + (y * f).abs() * 3 * E
    if residual is not None:
        y = y + d(residual)
        off = off + y.abs() * 2 * E
    stream = stream or dt
    total = y, off + (y.abs() + off) * U[stream] + TINY[stream]
    z, far = one(y, off, weight, bias)
    return total, (z, far + (z.abs() + far) * U[dt] + TINY[dt])


def turn(x, positions, freqs, layout="half", magnitude=1.0):
    """x turned, in 64 bits."""
    half = freqs.shape[0]
    magnitude = float(torch.tensor(magnitude))
    angle = positions.double()[:, None] * freqs
    turns = torch.polar(torch.full_like(angle, magnitude), angle)[:, None]
    y = x.double().clone()
    if layout == "half":
        z = torch.complex(y[..., :half], y[..., half:2 * half]) * turns
        y[..., :half], y[..., half:2 * half] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * turns
        y[..., :2 * half] = torch.view_as_real(z).flatten(-2)
    return y


def rounded(y, dtype):
    """Bound of a turned value that is rounded to dtype once: angles of up to
    2^24 radians are off by 2^-28, sines by as much. The sines are rounded to
    float, one product is, and their sum: 3 E of |x cos| + |o sin|, which is at
    most |x| + |o| <= 2 max(|y|, |y'|) over a pair's two results."""
    size = y.abs().amax(-1, keepdim=True) * 2
    return y.abs() * U[dtype] * (1 + 2 * E) + size * (2.0 ** -27 + 3 * E) + TINY[dtype]


def kept(y, f16=False):
    """(value the 8-bit cache stands for, exponent byte) of float64 [..., dim]."""
    z = y.unflatten(-1, (-1, 32))
    known = torch.isfinite(z)
    top = torch.where(known, z.abs(), 0.0).amax(-1, keepdim=True)
    m, e = torch.frexp(top / 448)
    e = torch.where(m > 0.5, e, e - 1)
    e = torch.where(top > 0, e, torch.full_like(e, -126)).clamp(-126, 120)
    z = torch.where(known, z, 0.0) / two_to(e)
    _, f = torch.frexp(z)
    step = two_to((f - 1).clamp(min=-6) - 3)
    z = torch.round(z / step) * step * two_to(e)
    if f16:
        z = z.clamp(-61440, 61440)
    return torch.where(known, z, math.nan).flatten(-2), (e.squeeze(-1) + 127).to(torch.uint8)


def logprobs(logits, scale=1.0):
    """(log p, its bound, entropy, its bound) in 64 bits.

    An exponential of d = z - max is off by 2 E (1 + |d|) of itself and moves to
    another maximum some ten times, each as far off; a sum of 16 of them is off
    by 16 E. log s is off by what s is, in proportion; so is t / s, twice."""
    scale = float(torch.tensor(scale))
    z = logits.double() * scale
    top = z.amax(-1, keepdim=True)
    d = torch.where(z > -math.inf, z - top, 0.0)
    e = torch.where(z > -math.inf, torch.exp(z - top), 0.0)
    s = e.sum(-1, keepdim=True)
    t = (e * d).sum(-1, keepdim=True)
    mean = -t / s
    off = 2 * E * (40 + 2 * mean)
    logp = z - top - torch.log(s)
    # results are floats: what is past their range is infinite
    logp = torch.where(logp > -torch.finfo(torch.float32).max, logp, -math.inf)
    h = torch.log(s) + mean
    spread = (e * d * d).sum(-1, keepdim=True) / s     # |d| falls on t once more
    far = off * (1 + 2 * mean) + 4 * E * spread
    return logp, off + torch.where(logp > -math.inf, logp.abs(), 0.0) * 2 * E, h[:, 0], (far + h.abs() * 2 * E)[:, 0]


def adapt(x, a, b, adapters, scales=None, ranks=None, base=None, out_dtype=None):
    """(result, bound of the error) in 64 bits.

    Sums as those of ops_ref.linear: k / 32 + 40 roundings of 2 E of the sum of
    magnitudes, rank / 8 + 40 for the second. h goes into it in parts that leave
    out 2^-16 of it (bf16) or 2^-22 (f16, or three parts), then three roundings."""
    count, rank, k = a.shape
    dt = out_dtype or x.dtype
    m, n = x.shape[0], b.shape[1]
    y = torch.zeros(m, n, dtype=torch.float64, device=x.device)
    far = torch.zeros_like(y)
    left = 2.0 ** -16 if x.dtype == torch.bfloat16 and dt != torch.float32 else 2.0 ** -22
    for c in range(count):
        rows = adapters == c
        r = rank if ranks is None else min(max(int(ranks[c]), 0), rank)
        if not rows.any() or not r:
            continue
        xc, ac, bc = x[rows].double(), a[c, :r].double(), b[c, :, :r].double()
        h, size = xc @ ac.t(), xc.abs() @ ac.abs().t()
        off = (k / 32 + 40) * 2 * E * size + left * h.abs()
        if x.dtype == torch.float16:    # the parts of small ones beside the row's largest
            off = off + 2.0 ** -36 * h.abs().amax(1, keepdim=True)
        s = 1.0 if scales is None else scales[c].double()
        y[rows] = s * (h @ bc.t())
        far[rows] = abs(s) * ((off + (rank / 8 + 40) * 2 * E * (h.abs() + off)) @ bc.abs().t())
    if base is not None:
        y = y + base.double()
    far = far + (y.abs() + (0 if base is None else base.double().abs())) * 4 * E
    return y, far + (y.abs() + far) * U[dt] + TINY[dt]
