"""Norms, rotary positions, the cache they are written to and log-probabilities
against their definitions in 64 bits (decoder_ref), on the GPU."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ii, ops  # noqa: E402  (fails loudly if libii.so is missing)

import decoder_ref as ref  # noqa: E402
import ops_ref  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F16, F32, F8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def work():
    return ops.work_buffer()


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, dtype=BF16, std=1.0, pad=0, lead=0):
    """Normal values, rows `pad` elements apart, `lead` elements into a buffer."""
    row = math.prod(shape[1:])
    buf = torch.empty(shape[0] * (row + pad) + lead, device=DEV).normal_(0, std, generator=g).to(dtype)
    return buf[lead:].view(shape[0], row + pad)[:, :row].unflatten(1, shape[1:])


def _close(got, want, bound, what=""):
    got = got.double()
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~(((got - want).abs() <= bound) | same)
    if bad.any():
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} past the bound, first at {at}: "
                             f"{got[at].item()} against {want[at].item()} +- {bound[at].item()}")


def _refused(name, call, *untouched):
    before = [t.clone() for t in untouched]
    with pytest.raises(ii.IIError) as e:
        call()
    assert e.value.name == name, e.value
    torch.cuda.synchronize()
    for a, b in zip(untouched, before):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# ii_norm

SIZES = [1, 7, 8, 64, 65, 256, 504, 512, 513, 520, 1001, 2048, 2056, 4096, 4104, 5001, 8192, 8200, 9001,
         16384, 16392, 20001, 32760, 32768]


def _norm(g, m, n, dt=BF16, stream=None, post=False, gate="", residual=True, bias=False, pad=0, lead=0,
          wants=("sum", "out"), **kw):
    stream = stream or dt
    vector = lambda mean: (_normal(g, 1, n, dtype=F32, std=0.3)[0] + mean).to(dt)  # noqa: E731
    x = _normal(g, m, n, dtype=dt, pad=pad, lead=lead, std=2.0)
    a = dict(weight=vector(1.0) if "out" in wants else None,
             bias=vector(0.0) if bias and "out" in wants else None, post=post,
             post_weight=vector(1.0) if post else None, post_bias=vector(0.0) if post and bias else None,
             gate={"": None, "row": vector(0.5).expand(m, n),
                   "each": _normal(g, m, n, dtype=dt, pad=pad, lead=lead)}[gate],
             residual=_normal(g, m, n, dtype=stream, pad=pad, lead=lead, std=3.0) if residual else None, **kw)
    total = torch.full((m, n + pad), NAN, dtype=stream, device=DEV)[:, :n]
    out = torch.full((m, n + pad), NAN, dtype=dt, device=DEV)[:, :n]
    ops.ii_norm(out if "out" in wants else None, x, sum=total if "sum" in wants else None, **a)
    want = ref.norm(x, stream=stream, **a)
    for got, (value, far), what in ((total, want[0], "sum"), (out, want[1], "out")):
        if what in wants:
            _close(got, value, far, f"{what} of {m} x {n}")
        else:
            assert got.isnan().all()
    return x, a, total, out


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("m", [1, 3, 70])
def test_norm_sizes(m, n):
    g = _gen(m * 100000 + n)
    for kind in ("rms", "layer"):
        _norm(g, m, n, kind=kind)
        _norm(g, m, n, F16, F32, post=True, gate="each", bias=True, kind=kind, offset=1.0, scale=0.5)


@pytest.mark.parametrize("n", [64, 200, 1001, 4096])
@pytest.mark.parametrize("dt,stream", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_parts(n, dt, stream, kind):
    g = _gen(n)
    for post, gate, residual, bias in itertools.product((False, True), ("", "row", "each"), (False, True),
                                                        (False, True)):
        _norm(g, 5, n, dt, stream, post, gate, residual, bias, kind=kind, scale=-1.5, offset=0.25)
    for wants in (("sum",), ("out",)):
        _norm(g, 5, n, dt, stream if wants == ("sum",) else dt, True, "each", True, True, wants=wants,
              kind=kind)
    # rows further apart, and from an odd place
    _norm(g, 9, n, dt, stream, True, "each", pad=24, kind=kind)
    _norm(g, 9, n, dt, stream, True, "each", pad=3, lead=1, kind=kind)


def test_norm_without_weights():
    x = _normal(_gen(1), 4, 300)
    out = torch.empty_like(x)
    ops.ii_norm(out, x, post=True, offset=3.0)      # the offset goes with a weight
    _close(out, *ref.norm(x, post=True, offset=3.0)[1])


@pytest.mark.parametrize("n", [256, 1001, 9000])
def test_norm_in_place(n):
    g = _gen(n)
    for m, stream in ((1, BF16), (33, BF16), (33, F32)):
        x, r = _normal(g, m, n), _normal(g, m, n, dtype=stream, pad=8)
        w = _normal(g, 1, n)[0].contiguous()
        want = ref.norm(x, w, residual=r, stream=stream)
        ops.ii_norm(x, x, w, residual=r, sum=r)
        _close(r, *want[0])
        _close(x, *want[1])


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_far_values(kind):
    """Squares past float's range on both sides, rows that are all alike, rows of zeros."""
    n = 300
    base = _normal(_gen(3), 1, n, dtype=F32)
    rows = torch.cat([base * s for s in (1e-30, 1e-18, 1.0, 1e15, 1e25, 1e37)]).to(BF16)
    out = torch.empty_like(rows)
    for eps in (0.0, 1e-30, 1e-5):
        ops.ii_norm(out, rows, kind=kind, eps=eps)
        _close(out, *ref.norm(rows, kind=kind, eps=eps)[1], f"eps {eps}")
    flat = torch.full((2, n), 3.0, dtype=BF16, device=DEV)
    flat[1] = 0
    out = torch.empty_like(flat)
    ops.ii_norm(out, flat, kind=kind)
    _close(out, *ref.norm(flat, kind=kind)[1])
    # what is not finite stays in its row
    bad = torch.ones(4, n, dtype=BF16, device=DEV)
    bad[1, 5], bad[2, 299] = NAN, INF
    out = torch.empty_like(bad)
    ops.ii_norm(out, bad, kind=kind)
    assert out[[0, 3]].isfinite().all() and out[1].isnan().all() and out[2, 299].isnan()
    assert out[2].isnan().all() if kind == "layer" else (out[2, :299] == 0).all()


def test_norm_many_rows():
    """More rows than one pass of the grid takes, at a stride of zero."""
    m, n = (1 << 23) + 5, 8
    x = _normal(_gen(4), 1, n)
    out = torch.empty(m, n, dtype=BF16, device=DEV)
    ops.ii_norm(out, x.expand(m, n))
    _close(out[0], *[t[0] for t in ref.norm(x)[1]])
    assert (out == out[0]).all()


# ---------------------------------------------------------------------------
# ii_rotate, ii_cache_append


def _turn_inputs(g, tokens, heads, dim, dt, pad=0, far=100000):
    x = _normal(g, tokens, heads, dim, dtype=dt, pad=pad)
    return x, torch.randint(0, far, (tokens,), generator=g, device=DEV)


@pytest.mark.parametrize("dim,rots", [(8, (0, 2, 8)), (64, (64, 32, 20, 2)), (80, (80, 40, 34)), (96, (96, 48)),
                                      (128, (128, 64, 126, 16)), (256, (256, 64)), (200, (200, 50)),
                                      (512, (512, 258))])
@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotate(dim, rots, dt, layout):
    g = _gen(dim)
    for rot, (tokens, heads) in itertools.product(rots, ((1, 1), (3, 5), (70, 9), (2, 130))):
        x, at = _turn_inputs(g, tokens, heads, dim, dt, pad=8 if heads == 9 else 0)
        freqs = ops.ii_rotary_freqs(rot)
        out = torch.full((tokens, heads, dim), NAN, dtype=dt, device=DEV)
        ops.ii_rotate(out, x, at, freqs, layout=layout, magnitude=1.25)
        want = ref.turn(x, at, freqs, layout, 1.25)
        _close(out, want, ref.rounded(want, dt), f"{tokens} x {heads} x {dim}, {rot}")
        assert torch.equal(out[..., rot:], x[..., rot:])
        ops.ii_rotate(x, x, at, freqs, layout=layout, magnitude=1.25)
        assert torch.equal(x, out)


def test_rotate_many_tokens():
    g = _gen(5)
    x, at = _turn_inputs(g, 9001, 4, 64, BF16)
    freqs = ops.ii_rotary_freqs(64, base=500000.0, factor=8.0, original=8192)
    out = torch.empty_like(x)
    ops.ii_rotate(out, x, at, freqs)
    want = ref.turn(x, at, freqs)
    _close(out, want, ref.rounded(want, BF16))


def test_rotate_far_positions():
    """Positions past 32 bits, and before 0: whole turns do not show."""
    import decimal
    decimal.getcontext().prec = 60
    pi = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    at = [0, 1, -1, 2 ** 31, 2 ** 33 + 12345, -2 ** 40 + 3, 2 ** 45 + 1]
    freqs = torch.tensor([1.0, 0.1, 0.37, 1e-5], dtype=torch.float64)
    x = torch.zeros(len(at), 1, 8, dtype=F16, device=DEV)
    x[..., :4] = 1
    out = torch.empty_like(x)
    ops.ii_rotate(out, x, torch.tensor(at, device=DEV), freqs.to(DEV))
    for i, p in enumerate(at):
        for j, f in enumerate(freqs.tolist()):
            r = float(decimal.Decimal(p) * decimal.Decimal(f) % (2 * pi))
            for got, want in ((out[i, 0, j], math.cos(r)), (out[i, 0, 4 + j], math.sin(r))):
                assert abs(float(got) - want) <= abs(want) * 2.0 ** -11 + 2.0 ** -25 + 2.0 ** -40, (p, f)


def test_rotary_freqs():
    f = ops.ii_rotary_freqs(128, base=500000.0, factor=8.0, low=1.0, high=4.0, original=8192, device="cpu")
    for i in range(64):
        w = 500000.0 ** (-2 * i / 128)
        turns = 8192 * w / (2 * math.pi)
        want = w if turns > 4 else w / 8 if turns < 1 else w * (turns - 1) / 3 + w / 8 * (4 - turns) / 3
        assert abs(float(f[i]) - want) <= 1e-14 * want
    assert torch.equal(ops.ii_rotary_freqs(64, factor=2.0, device="cpu") * 2, ops.ii_rotary_freqs(64, device="cpu"))
    assert ops.ii_rotary_freqs(0).shape == (0,)


def _cache(pages, heads, page, dim, dt):
    """A cache of marks, heads before or behind the tokens."""
    c = ops.Cache.empty(pages, heads, page, dim, dt, device=DEV)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0x2f)
    return c


@pytest.mark.parametrize("dt,kept", [(BF16, F8), (F16, F8), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(0, 1, 64, 1), (4, 4, 64, 16), (8, 2, 128, 64), (3, 3, 128, 2),
                                                     (70, 5, 64, 8)])
def test_cache_append(dt, kept, layout, heads, kv_heads, dim, page):
    g = _gen(heads + dim)
    for tokens, rot in ((1, dim), (7, dim // 2), (150, dim), (33, 0), (20, 18)):
        pages = -(-tokens // page) + 2
        cache = _cache(pages, kv_heads, page, dim, kept)
        slots = torch.randperm(pages * page, generator=g, device=DEV)[:tokens].contiguous()
        if tokens > 5:
            slots[2], slots[5] = -1, pages * page     # left out
        k, at = _turn_inputs(g, tokens, kv_heads, dim, dt, pad=16)
        v, _ = _turn_inputs(g, tokens, kv_heads, dim, dt)
        q, _ = _turn_inputs(g, tokens, max(heads, 1), dim, dt, pad=8)
        freqs = ops.ii_rotary_freqs(rot)
        q_out = torch.full_like(q, NAN)
        before = [t.clone() for t in (cache.k, cache.v)]
        ops.ii_cache_append(cache, k, v, slots, at, freqs, layout=layout,
                            **(dict(q=q, q_out=q_out) if heads else {}))
        if heads:
            want = ref.turn(q, at, freqs, layout)
            _close(q_out, want, ref.rounded(want, dt))
        back = [torch.empty_like(k) for _ in "kv"]
        ops.ii_cache_read(cache, slots, *back)
        here = (slots >= 0) & (slots < pages * page)
        turned = ref.turn(k, at, freqs, layout)
        if kept == F8:      # not a code is off
            for got, y in zip(back, (turned, v.double())):
                assert torch.equal(got[here].double(), ref.kept(y[here], dt == F16)[0].to(dt).double())
        else:
            _close(back[0][here], turned[here], ref.rounded(turned, dt)[here])
            assert torch.equal(back[1][here], v[here])
        # nothing else was written
        used = torch.zeros(pages * page, dtype=torch.bool, device=DEV)
        used[slots[here]] = True
        rest = ~used.view(pages, page)
        for t, b in zip((cache.k, cache.v), before):
            assert torch.equal(t.view(torch.uint8).transpose(1, 2)[rest], b.view(torch.uint8).transpose(1, 2)[rest])


def test_append_is_write_and_rotate():
    """Without a turn it is ii_cache_write, bit for bit; q in place, out of one fused buffer."""
    g = _gen(9)
    fused = _normal(g, 50, 12, 128)
    q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    slots = torch.randperm(64, generator=g, device=DEV)[:50].contiguous()
    at = torch.zeros(50, dtype=torch.int64, device=DEV)
    a, b = (ops.Cache.empty(4, 2, 16, 128) for _ in "ab")
    ops.ii_cache_write(a, k, v, slots)
    before = fused.clone()
    ops.ii_cache_append(b, k, v, slots, at, ops.ii_rotary_freqs(128), q=q, q_out=q)
    for name in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8))
    assert torch.equal(fused, before)
    at += 7
    want = ref.turn(q, at, ops.ii_rotary_freqs(128))
    ops.ii_cache_append(b, k, v, slots, at, ops.ii_rotary_freqs(128), q=q, q_out=q)
    _close(q, want, ref.rounded(want, BF16))
    assert torch.equal(fused[:, 8:], before[:, 8:])


def test_append_not_finite():
    """What is not finite becomes NaN and leaves the other blocks alone."""
    k = _normal(_gen(2), 2, 1, 64)
    k[0, 0, 3], k[1, 0, 40] = NAN, INF
    cache = ops.Cache.empty(1, 1, 4, 64)
    slots, at = torch.arange(2, device=DEV), torch.tensor([3, 0], device=DEV)
    ops.ii_cache_append(cache, k, k, slots, at, ops.ii_rotary_freqs(64))
    back = [torch.empty_like(k) for _ in "kv"]
    ops.ii_cache_read(cache, slots, *back)
    assert back[0][0, 0].isnan().nonzero().flatten().tolist() == [3, 35]
    # position 0: infinity times sin 0
    assert back[0][1, 0].isnan().nonzero().flatten().tolist() == [8, 40]
    assert back[1].isnan().sum() == 2


# ---------------------------------------------------------------------------
# ii_logprobs


def _logprobs(logits, targets=None, top=0, scale=1.0, work=None):
    rows, vocab = logits.shape
    if targets is None:
        targets = torch.arange(rows, device=DEV) * 7919 % vocab
    f32 = lambda *s: torch.full(s, 7.0, device=DEV)  # noqa: E731
    logprob, entropy = f32(rows), f32(rows)
    ids = torch.full((rows, top), -7, dtype=torch.int64, device=DEV) if top else None
    values = f32(rows, top) if top else None
    ops.ii_logprobs(logits, targets=targets, logprob=logprob, entropy=entropy, top_ids=ids,
                    top_logprobs=values, scale=scale, work=work)
    return targets, logprob, entropy, ids, values


def _check_logprobs(logits, top=0, scale=1.0, work=None, targets=None):
    targets, logprob, entropy, ids, values = _logprobs(logits, targets, top, scale, work)
    vocab = logits.shape[1]
    logp, off, h, far = ref.logprobs(logits, scale)
    _close(logprob, logp.gather(1, targets[:, None])[:, 0], off.gather(1, targets[:, None])[:, 0], "logprob")
    _close(entropy, h, far, "entropy")
    if top:
        n = min(top, vocab)
        want = torch.sort(logits.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :n]
        assert torch.equal(ids[:, :n], want)
        _close(values[:, :n], logp.gather(1, want), off.gather(1, want), "top_logprobs")
        assert (ids[:, n:] == -1).all() and (values[:, n:] == -INF).all()


@pytest.mark.parametrize("vocab", [1, 2, 5, 63, 64, 65, 1000, 4095, 4096, 4097, 8192, 12289, 32000, 50257, 128256])
@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("split", [False, True])
def test_logprobs_sizes(vocab, dt, split, work):
    g = _gen(vocab)
    for rows, top in ((1, 0), (1, 5), (3, 64), (9, 20), (2, 1)):
        for pad in (0, 3):
            _check_logprobs(_normal(g, rows, vocab, dtype=dt, std=3.0, pad=pad), top, 0.8, work if split else None)


@pytest.mark.parametrize("rows", [300, 1025, 2000])
def test_logprobs_many_rows(rows, work):
    g = _gen(rows)
    for top in (0, 7):
        _check_logprobs(_normal(g, rows, 9001, dtype=F32, std=4.0), top, 1.0, work)


@pytest.mark.parametrize("split", [False, True])
def test_logprobs_orders(split, work):
    """Rows that rise, fall, are all alike, or tie at many places."""
    n = 30011
    up = torch.arange(n, device=DEV, dtype=F32) / 1000
    rows = torch.stack([up, -up, torch.zeros(n, device=DEV), (up * 10).floor() % 7, -(up * 300).floor() % 3,
                        torch.where(torch.arange(n, device=DEV) % 2 == 0, 0.0, -0.0)])
    for top in (1, 20, 64):
        for dt in (F32, BF16):
            _check_logprobs(rows.to(dt), top, 1.0, work if split else None)


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_logprobs_masked(dt, split, work):
    n = 20000
    x = _normal(_gen(6), 5, n, dtype=dt, std=2.0)
    x[0, ::2] = -INF
    x[1] = -INF
    x[1, 12345] = 3.0
    x[2, :19990] = -INF
    x[3, 8000:] = -INF
    x[4] = -INF
    x[4, [5, 19999]] = torch.finfo(dt).min
    for top in (3, 64):
        _check_logprobs(x, top, 1.0, work if split else None,
                        torch.tensor([4, 12345, 19995, 9000, 5], device=DEV))


@pytest.mark.parametrize("split", [False, True])
def test_logprobs_nothing_left_and_not_finite(split, work):
    n, w = 10000, work if split else None
    x = _normal(_gen(8), 4, n, dtype=F32)
    x[0] = -INF
    x[1, 777] = NAN
    x[2, 9999] = INF
    targets, logprob, entropy, ids, values = _logprobs(x, None, 4, 1.0, w)
    assert logprob[0] == -INF and entropy[0] == 0
    assert ids[0].tolist() == [0, 1, 2, 3] and (values[0] == -INF).all()
    for row in (1, 2):
        assert logprob[row].isnan() and entropy[row].isnan() and values[row].isnan().all()
    order = torch.sort(torch.where(x.isnan(), -INF, x), dim=1, descending=True, stable=True).indices
    assert torch.equal(ids, order[:, :4])
    assert logprob[3].isfinite() and entropy[3].isfinite()


def test_logprobs_targets_that_are_none(work):
    x = _normal(_gen(9), 3, 100, dtype=F32)
    logp, off, _, _ = ref.logprobs(x)
    _, logprob, *_ = _logprobs(x, torch.tensor([-1, 99, 100], device=DEV), 0, 1.0, work)
    assert logprob[0] == 0 and logprob[2] == 0
    _close(logprob[1:2], logp[1, 99:], off[1, 99:])


def test_logprobs_extreme():
    x = torch.tensor([[3e38, -3e38, 0.0], [1e30, 1e30, 1e30], [-1e30, -2e30, -INF], [80.0, -80.0, 79.0]], device=DEV)
    for scale in (1e-3, 1.0, 30.0):
        _check_logprobs(x, 3, scale)


def test_logprobs_same_bits(work):
    x = _normal(_gen(10), 7, 50000, dtype=BF16)
    first = _logprobs(x, None, 20, 1.0, work)
    for _ in range(5):
        for a, b in zip(first, _logprobs(x, None, 20, 1.0, work)):
            assert torch.equal(a, b)
    assert not work[:65536].any()


def test_logprobs_only_what_is_wanted(work):
    x = _normal(_gen(11), 3, 5000, dtype=F32)
    _, logprob, entropy, ids, values = _logprobs(x, None, 4, 1.0, work)
    h = torch.empty(3, device=DEV)
    ops.ii_logprobs(x, entropy=h, work=work)
    _close(h, entropy.double(), 8 * ref.E * entropy.double())
    i, v = torch.empty_like(ids), torch.empty_like(values)
    ops.ii_logprobs(x, top_ids=i, top_logprobs=v, work=work)
    assert torch.equal(i, ids) and torch.equal(v, values)


# ---------------------------------------------------------------------------
# refusals that need device memory (the others run without a GPU)


def test_refusals(work):
    g = _gen(12)
    x, w = _normal(g, 4, 64), _normal(g, 1, 64)[0].contiguous()
    out, total = torch.zeros_like(x), torch.zeros_like(x)
    _refused("II_EINVAL", lambda: ops.ii_norm(out, x.cpu(), w), out)
    _refused("II_EINVAL", lambda: ops.ii_norm(out.cpu(), x, w))
    _refused("II_EINVAL", lambda: ops.ii_norm(out, x, w.cpu()), out)
    _refused("II_EINVAL", lambda: ops.ii_norm(out, x, w, post_weight=w), out)
    _refused("II_EINVAL", lambda: ops.ii_norm(None, x), out)
    _refused("II_EINVAL", lambda: ops.ii_norm(None, x, w, sum=total), total)
    _refused("II_EOVERLAP", lambda: ops.ii_norm(out, x, w, sum=out), out)
    _refused("II_EOVERLAP", lambda: ops.ii_norm(out, x, w, sum=x), x)
    _refused("II_EOVERLAP", lambda: ops.ii_norm(x, x, x[0]), x)
    _refused("II_EOVERLAP", lambda: ops.ii_norm(out, x, w, gate=out), out)
    wide = torch.zeros(5, 64, dtype=BF16, device=DEV)
    _refused("II_EOVERLAP", lambda: ops.ii_norm(None, x, residual=wide[:4], sum=wide[1:]), wide)
    _refused("II_EINVAL", lambda: ops.ii_norm(torch.as_strided(wide, (4, 64), (32, 1)), x), wide)

    q, at = _turn_inputs(g, 3, 2, 64, BF16)
    freqs, turned = ops.ii_rotary_freqs(64), torch.zeros_like(q)
    _refused("II_EINVAL", lambda: ops.ii_rotate(turned, q, at.cpu(), freqs), turned)
    _refused("II_EINVAL", lambda: ops.ii_rotate(turned, q, at, freqs.cpu()), turned)
    _refused("II_EINVAL", lambda: ops.ii_rotate(turned, q.cpu(), at, freqs), turned)
    _refused("II_EINVAL", lambda: ops.ii_rotate(turned, q, at, ops.ii_rotary_freqs(66)), turned)
    flat = torch.zeros(4 * 128, dtype=BF16, device=DEV)
    _refused("II_EOVERLAP", lambda: ops.ii_rotate(flat[64:448].view(3, 2, 64), flat[:384].view(3, 2, 64), at, freqs),
             flat)
    _refused("II_EALIGN", lambda: ops.ii_rotate(flat[4:388].view(3, 2, 64), q, at, freqs), flat)
    pos = torch.zeros(24 * 64, dtype=torch.int64, device=DEV)
    _refused("II_EOVERLAP", lambda: ops.ii_rotate(pos.view(BF16)[:384].view(3, 2, 64), q, pos[:3], freqs), pos)

    cache = ops.Cache.empty(2, 2, 16, 64, BF16)
    slots = torch.arange(3, device=DEV)
    args = (slots, at, freqs)
    _refused("II_EOVERLAP", lambda: ops.ii_cache_append(cache, q, q, *args, q=q, q_out=cache.k[0, :, :3].transpose(0, 1)),
             cache.k)
    _refused("II_EOVERLAP", lambda: ops.ii_cache_append(cache, q, turned, *args, q=turned.clone(), q_out=q), q)
    _refused("II_EOVERLAP", lambda: ops.ii_cache_append(cache, cache.v[0, :, :3].transpose(0, 1), q, *args), cache.k)
    _refused("II_EOVERLAP", lambda: ops.ii_cache_append(cache, q, q, slots, cache.k.view(torch.int64).flatten()[:3],
                                                        freqs), cache.k)
    _refused("II_EINVAL", lambda: ops.ii_cache_append(cache, q, q, slots.cpu(), at, freqs), cache.k)

    z, p = _normal(g, 4, 64, dtype=F32), torch.zeros(4, device=DEV)
    t = torch.arange(4, device=DEV)
    _refused("II_EINVAL", lambda: ops.ii_logprobs(z.cpu(), entropy=p), p)
    _refused("II_EINVAL", lambda: ops.ii_logprobs(z, targets=t.cpu(), logprob=p), p)
    _refused("II_EINVAL", lambda: ops.ii_logprobs(z, entropy=p.cpu()))
    _refused("II_EINVAL", lambda: ops.ii_logprobs(z))
    _refused("II_EINVAL", lambda: ops.ii_logprobs(z, entropy=p, scale=0.0), p)
    _refused("II_EOVERLAP", lambda: ops.ii_logprobs(z, entropy=z.flatten()[:4]), z)
    _refused("II_EOVERLAP", lambda: ops.ii_logprobs(z, entropy=p, targets=t, logprob=p), p)
    _refused("II_EOVERLAP", lambda: ops.ii_logprobs(z, entropy=p, targets=t, logprob=t.view(F32)[:4]), t)
    _refused("II_EOVERLAP", lambda: ops.ii_logprobs(z, entropy=work.view(F32)[:4], work=work))
    many = torch.zeros(4, 65, dtype=torch.int64, device=DEV)
    _refused("II_EINVAL", lambda: ops.ii_logprobs(z, top_ids=many, top_logprobs=many.float()))


@pytest.mark.parametrize("nbytes", [16, 65536, 65536 + 64, 65536 + 4096, 1 << 20])
def test_logprobs_scratch(nbytes):
    """Any size of scratch will do; its counters are left at zero."""
    scratch = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)
    x = _normal(_gen(13), 5, 70001, dtype=F32, std=3.0)
    for top in (0, 9, 64):
        _check_logprobs(x, top, 1.0, scratch)
    assert not scratch[:65536].any()


def test_rows_of_no_elements():
    """Nothing to write, nothing to read: no address is looked at."""
    none = torch.empty(3, 0, dtype=BF16, device=DEV)
    ops.ii_norm(none, none, residual=none.float(), sum=none.float())
    ops.ii_rotate(*[torch.empty(0, 4, 64, dtype=BF16, device=DEV)] * 2, torch.empty(0, dtype=torch.int64, device=DEV),
                  ops.ii_rotary_freqs(64))
    ops.ii_logprobs(torch.empty(0, 100, device=DEV), entropy=torch.empty(0, device=DEV))
