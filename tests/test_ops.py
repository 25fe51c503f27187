"""The operators against their definitions in 64 bits (ops_ref), on the GPU:
sizes and masks where they can go wrong, strides, streams, graphs, refusals."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ii, ops  # noqa: E402  (fails loudly if libii.so is missing)

import ops_ref  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F16, F32, F8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


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
    assert torch.isfinite(got).all() or not torch.isfinite(want).all(), what
    off = (got.double() - want).abs()
    bad = ~((off <= bound) | (got.double() == want))
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} past the bound, first at {at}: "
                             f"{got[tuple(at)].item()} against {want[tuple(at)].item()} "
                             f"+- {bound[tuple(at)].item()}")


# ---------------------------------------------------------------------------
# ii_linear


def _linear(g, m, n, k, dt=BF16, out=None, act="none", gated=False, bias=False, residual=False,
            pad=0, lead=0, work=None, whole=False):
    """One product against its definition; `whole`: small whole numbers, whose
    sums are exact, so the result has to be the definition's rounded."""
    out = out or dt
    if whole:
        make = lambda *s, **kw: torch.randint(-3, 4, s, generator=g, device=DEV).to(dt)  # noqa: E731
    else:
        make = lambda *s, **kw: _normal(g, *s, dtype=dt, **kw)  # noqa: E731
    kw = dict(std=max(k, 1) ** -0.5) if not whole else {}
    x, w = make(m, k, pad=pad, lead=lead), make(n, k, pad=pad, lead=lead, **kw)
    w2 = make(n, k, pad=pad, lead=lead, **kw) if gated else None
    b = make(1, n)[0].contiguous() if bias else None
    b2 = make(1, n)[0].contiguous() if bias and gated else None
    r = make(m, n, pad=pad, lead=lead) if residual else None
    guard = torch.full((m + 2, n + 7), 77.0, dtype=out, device=DEV)
    got = guard[1:m + 1, 3:n + 3]
    ops.ii_linear(got, x, w, bias=b, w2=w2, bias2=b2, residual=r, act=act, work=work)
    want, bound = ops_ref.linear(x, w, out, b, w2, b2, r, act)
    what = f"m={m} n={n} k={k} {dt} -> {out} {act} gated={gated} bias={bias} residual={residual} " \
           f"pad={pad} lead={lead} work={work is not None} whole={whole}"
    if whole and act in ("none", "relu") and not gated:
        assert torch.equal(got, want.to(out)), what
    else:
        _close(got, want, bound, what)
    assert bool((guard[0] == 77).all() and (guard[-1] == 77).all() and (guard[:, :3] == 77).all()
                and (guard[:, n + 3:] == 77).all()), "written outside: " + what
    if work is not None:
        assert not work[:65536].any(), "counters left: " + what


SIZES = [(1, 1, 1), (1, 16, 8), (1, 1024, 256), (2, 17, 33), (3, 100, 64), (15, 64, 72), (16, 48, 96),
         (17, 130, 40), (31, 257, 129), (33, 64, 1000), (64, 192, 520), (65, 65, 65), (100, 300, 200),
         (129, 127, 256), (200, 256, 512), (256, 256, 64), (257, 513, 136), (300, 1000, 328)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dt", [BF16, F16])
def test_linear_sizes(m, n, k, dt, work):
    for i, (w, whole) in enumerate(itertools.product([None, work], [False, True])):
        _linear(_gen(i), m, n, k, dt, work=w, whole=whole)
    _linear(_gen(9), m, n, k, dt, out=F32, bias=True, act="gelu", residual=True, work=work)
    _linear(_gen(10), m, n, k, dt, gated=True, bias=True, act="silu", work=work)
    _linear(_gen(11), m, n, k, dt, gated=True, act="relu", residual=True, pad=5, lead=1)
    _linear(_gen(12), m, n, k, dt, bias=True, pad=24, lead=8, work=work, whole=True)


@pytest.mark.parametrize("m", [1, 4, 13, 24, 40, 64, 90, 128, 250, 600])
@pytest.mark.parametrize("n,k", [(256, 8192), (96, 14336), (5000, 1024), (2048, 2048)])
def test_linear_long_and_wide(m, n, k, work):
    """Few rows of a long axis (split, joined), many rows of a short one."""
    _linear(_gen(1), m, n, k, work=work)
    _linear(_gen(2), m, n, k, work=work, whole=True, bias=True, residual=True)
    _linear(_gen(3), m, n, k, F16, gated=True, act="silu", work=work[:1 << 20])


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_linear_special_values(act):
    """Infinities and NaN stay in their row and column, as in the definition."""
    x = torch.zeros(5, 64, dtype=BF16, device=DEV)
    w = torch.eye(64, dtype=BF16, device=DEV)[:20].contiguous()
    x[0, :4] = torch.tensor([1.0, -2.0, 300.0, -300.0])
    x[1, 0] = math.inf
    x[2, 1] = math.nan
    x[3, :3] = torch.tensor([-80.0, 80.0, 1e30])
    out = torch.empty(5, 20, dtype=F32, device=DEV)
    ops.ii_linear(out, x, w, act=act)
    y = torch.zeros(5, 20, dtype=torch.float64)
    xs, ws = x.double().cpu(), w.double().cpu()
    for i in range(5):  # inf * 0 = NaN, so products are summed as the definition has them
        y[i] = (xs[i] * ws).sum(1)
    want = ops_ref.act64(y, act)
    got = out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    near = (got == want) | ((got - want).abs() <= 1e-5 * want.abs() + 1e-30)
    assert near[ok].all()


def test_linear_no_sums(work):
    """k = 0: the epilogue alone; m = 0 or n = 0: nothing."""
    g = _gen(3)
    b, r = _normal(g, 1, 40)[0].contiguous(), _normal(g, 7, 40)
    x, w, out = (torch.empty(s, dtype=BF16, device=DEV) for s in ((7, 0), (40, 0), (7, 40)))
    ops.ii_linear(out, x, w, bias=b, residual=r, act="gelu", work=work)
    want, bound = ops_ref.linear(x, w, BF16, b, None, None, r, "gelu")
    _close(out, want, bound)
    for m, n in ((0, 40), (7, 0), (0, 0)):
        ops.ii_linear(out[:m, :n], _normal(g, max(m, 1), 16)[:m], _normal(g, max(n, 1), 16)[:n])


@pytest.mark.parametrize("m,n,k", [(4, 512, 512), (300, 512, 256), (24, 64, 9000)])
def test_linear_in_place_residual(m, n, k, work):
    g = _gen(4)
    x, w, r = _normal(g, m, k), _normal(g, n, k, std=k ** -0.5), _normal(g, m, n)
    want, bound = ops_ref.linear(x, w, BF16, residual=r)
    ops.ii_linear(r, x, w, residual=r, work=work)
    _close(r, want, bound)


def test_linear_broadcast_rows():
    """Rows at stride 0."""
    g = _gen(5)
    x, r = _normal(g, 1, 128).expand(20, 128), _normal(g, 1, 64).expand(20, 64)
    w = _normal(g, 64, 128, std=0.1)
    out = torch.empty(20, 64, dtype=BF16, device=DEV)
    ops.ii_linear(out, x, w, residual=r)
    _close(out, *ops_ref.linear(x, w, BF16, residual=r))


def test_linear_same_bits(work):
    """Split sums are joined in one order."""
    g = _gen(6)
    for m, n, k in ((1, 128, 16384), (24, 512, 14336), (100, 256, 8192), (700, 512, 4096)):
        x, w = _normal(g, m, k), _normal(g, n, k, std=k ** -0.5)
        a, b = (torch.empty(m, n, dtype=F32, device=DEV) for _ in "ab")
        ops.ii_linear(a, x, w, work=work)
        for _ in range(5):
            ops.ii_linear(b, x, w, work=work)
            assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# the cache


def _cache(pages, heads, page, dim, dt, layout="heads"):
    """An empty cache, contiguous or with tokens outside heads, or with keys
    and values in one buffer."""
    if layout == "heads":
        return ops.Cache.empty(pages, heads, page, dim, dt)
    scales = []
    if layout == "tokens":
        make = lambda d, t: torch.zeros(pages, page, heads, d, dtype=t, device=DEV).transpose(1, 2)  # noqa: E731
        if dt == F8:
            scales = [make(dim // 32, torch.uint8) for _ in "kv"]
        return ops.Cache(make(dim, dt), make(dim, dt), *scales)
    both = torch.zeros(pages, 2, heads, page, dim, dtype=dt, device=DEV)
    if dt == F8:
        s = torch.zeros(pages, 2, heads, page, dim // 32, dtype=torch.uint8, device=DEV)
        scales = [s[:, 0], s[:, 1]]
    return ops.Cache(both[:, 0], both[:, 1], *scales)


@pytest.mark.parametrize("dt,kept", [(BF16, F8), (F16, F8), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("heads,dim,page", [(1, 64, 1), (3, 64, 16), (8, 128, 64), (5, 128, 2)])
@pytest.mark.parametrize("layout", ["heads", "tokens", "both"])
def test_cache_write_and_read(dt, kept, heads, dim, page, layout):
    g = _gen(heads + dim)
    pages = 40 // page + 3
    cache = _cache(pages, heads, page, dim, kept, layout)
    for n in (0, 1, 2, 33, 40):
        slots = torch.randperm(pages * page, generator=g, device=DEV)[:n].contiguous()
        if n > 30:
            slots[3], slots[8], slots[n - 1] = -1, pages * page, -2 ** 40
        before = [x.view(torch.uint8).clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)
                  if x is not None]
        # magnitudes over many powers of two, blocks of zeros among them
        k, v = (_normal(g, n, heads, dim, dtype=dt, pad=8 * i) *
                torch.exp2(torch.randint(-14, 12, (n, heads, 1), generator=g, device=DEV)).to(dt)
                for i in (0, 3))
        k[:n // 2, :, :32] = 0
        ops.ii_cache_write(cache, k, v, slots)
        kb, vb = (torch.full((n, heads, dim), 5.0, dtype=dt, device=DEV) for _ in "kv")
        ops.ii_cache_read(cache, slots, kb, vb)
        held = (slots >= 0) & (slots < pages * page)
        for x, got in ((k, kb), (v, vb)):
            want = ops_ref.kept(x)[0] if kept == F8 else x.double()
            assert torch.equal(got[held].double(), want[held].to(dt).double())
            assert not got[~held].any()
        # nothing else was touched
        rest = torch.ones(pages * page, dtype=torch.bool, device=DEV)
        rest[slots[held]] = False
        rest = rest.view(pages, page)
        after = [x.view(torch.uint8) for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)
                 if x is not None]
        for a, b in zip(before, after):
            assert torch.equal(a.transpose(1, 2)[rest], b.transpose(1, 2)[rest])


@pytest.mark.parametrize("dt", [BF16, F16])
def test_cache_codes(dt):
    """Every finite value of the type as a block's largest element, and every
    pattern beside it: codes and exponents are the definition's."""
    bits = torch.arange(65536, device=DEV, dtype=torch.int32).to(torch.int16).view(dt)
    x = bits[torch.isfinite(bits)]
    n = x.numel() // 64 * 64
    for rows in (x[:n].view(-1, 1, 64), x[torch.randperm(n, device=DEV, generator=_gen(0))].view(-1, 1, 64)):
        t = rows.shape[0]
        cache = ops.Cache.empty(-(-t // 64), 1, 64, 64)
        slots = torch.arange(t, device=DEV)
        ops.ii_cache_write(cache, rows.contiguous(), rows.contiguous(), slots)
        want, e = ops_ref.kept(rows)
        codes = cache.k.view(-1, 64)[:t].double()
        scale = cache.k_scale.view(-1, 2)[:t]
        assert torch.equal(scale, e[:, 0])
        got = codes * ops_ref.two_to(scale.long() - 127).repeat_interleave(32, -1)
        assert torch.equal(got, want[:, 0])
        kb, vb = torch.empty_like(rows), torch.empty_like(rows)
        ops.ii_cache_read(cache, slots, kb, vb)
        assert torch.equal(kb.double(), want.to(dt).double()) and torch.equal(kb, vb)


def test_cache_not_finite():
    x = torch.ones(2, 1, 64, dtype=BF16, device=DEV)
    x[0, 0, 3], x[0, 0, 40], x[1, 0, :32] = math.nan, -math.inf, math.inf
    cache = ops.Cache.empty(1, 1, 2, 64)
    ops.ii_cache_write(cache, x, x, torch.arange(2, device=DEV))
    back, again = torch.empty_like(x), torch.empty_like(x)
    ops.ii_cache_read(cache, torch.arange(2, device=DEV), back, again)
    want = torch.where(torch.isfinite(x), x, math.nan)
    assert torch.equal(torch.isnan(back), torch.isnan(want))
    assert torch.equal(back.nan_to_num(7.0), want.nan_to_num(7.0))


def test_cache_past_32_bits():
    """Pages whose byte offsets need more than 32 bits."""
    pages, heads, page, dim = 40000, 8, 128, 128   # 5.2 GB of keys
    cache = ops.Cache.empty(pages, heads, page, dim)
    slots = torch.tensor([0, pages * page - 1, 33000 * page + 5, 17], device=DEV)
    k, v = (_normal(_gen(i), 4, heads, dim) for i in (1, 2))
    ops.ii_cache_write(cache, k, v, slots)
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    ops.ii_cache_read(cache, slots, kb, vb)
    assert torch.equal(kb.double(), ops_ref.kept(k)[0]) and torch.equal(vb.double(), ops_ref.kept(v)[0])
    # and attention over them
    q = _normal(_gen(3), 1, 16, dim)
    out = torch.empty_like(q)
    table = [33000, pages - 1]
    ops.ii_attend(out, q, cache, torch.tensor([table], dtype=torch.int32, device=DEV),
                  torch.tensor([2 * page], dtype=torch.int32, device=DEV))
    small = ops.Cache(cache.k[table], cache.v[table], cache.k_scale[table], cache.v_scale[table])
    want, far, _ = ops_ref.attend(q, small, [[0, 1]], [2 * page])
    _close(out, want, far)


# ---------------------------------------------------------------------------
# ii_attend


def _batch(g, keys, queries, heads, kv_heads, dim, page, dt=BF16, kept=F8, layout="heads",
           spare=1, pad=0):
    """A ragged batch over a cache full of values, its page tables shuffled."""
    used = [-(-n // page) for n in keys]
    pages = sum(used) + spare
    order = torch.randperm(pages, generator=g, device=DEV).tolist()
    columns = max(max(used), 1)
    tables, at = [], 0
    for u in used:
        tables.append(order[at:at + u] + [-1] * (columns - u))
        at += u
    cache = _cache(pages, kv_heads, page, dim, kept, layout)
    t = pages * page
    k, v = (_normal(g, t, kv_heads, dim, dtype=dt) for _ in "kv")
    ops.ii_cache_write(cache, k, v, torch.arange(t, device=DEV))
    starts = list(itertools.accumulate(queries, initial=0))
    q = _normal(g, max(starts[-1], 1), heads, dim, dtype=dt, pad=pad)[:starts[-1]]
    return cache, q, tables, list(keys), starts


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _attend(cache, q, tables, keys, starts, window=0, scale=None, work=None, max_q=None, max_len=0):
    if max_q is None:
        max_q = max(b - a for a, b in zip(starts, starts[1:]))
    guard = torch.full((q.shape[0] + 2, q.shape[1], q.shape[2]), 77.0, dtype=q.dtype, device=DEV)
    out = guard[1:-1]
    ops.ii_attend(out, q, cache, _i32(tables), _i32(keys), _i32(starts), max_q=max_q, max_len=max_len,
                  window=window, scale=scale, work=work)
    want, far, covered = ops_ref.attend(q, cache, tables, keys, starts, window, scale)
    what = f"keys={keys[:8]} starts={starts[:8]} q={tuple(q.shape)} {q.dtype} kv={cache.heads} " \
           f"page={cache.page} {cache.k.dtype} window={window} work={work is not None} max_q={max_q}"
    _close(out[covered], want[covered], far[covered], what)
    assert bool((out[~covered] == 77).all()), "rows of no sequence written: " + what
    assert bool((guard[0] == 77).all() and (guard[-1] == 77).all()), "written outside: " + what
    if work is not None:
        assert not work[:65536].any(), "counters left: " + what
    return out


HEADS = [(4, 4, 64), (8, 2, 128), (16, 1, 64), (6, 2, 128), (17, 1, 128), (64, 4, 64)]


@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("dt,kept", [(BF16, F8), (F16, F8), (BF16, BF16), (F16, F16)])
def test_attend_tokens(heads, kv_heads, dim, dt, kept, work):
    """One query a sequence: lengths from none to some pages, odd ones."""
    keys = [1, 0, 15, 16, 17, 63, 64, 65, 127, 129, 300, 31]
    for page, layout, w in ((16, "heads", None), (64, "tokens", work), (1, "both", work)):
        b = _batch(_gen(page), keys, [1] * len(keys), heads, kv_heads, dim, page, dt, kept, layout)
        _attend(*b, work=w)
        _attend(*b, work=w, window=20)
        _attend(*b, work=w, max_len=40)     # too small a hint
    out = torch.empty_like(b[1])            # without q_start: a row a sequence
    ops.ii_attend(out, b[1], b[0], _i32(b[2]), _i32(keys), work=work)
    want, far, _ = ops_ref.attend(b[1], b[0], b[2], keys)
    _close(out, want, far)


@pytest.mark.parametrize("n", [1000, 4097, 20000])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (4, 4, 64), (16, 1, 128)])
def test_attend_long(n, heads, kv_heads, dim, work):
    """Long contexts, split and joined: alike with and without scratch."""
    b = _batch(_gen(n), [n, 3, n // 2 + 1], [1, 1, 1], heads, kv_heads, dim, 32)
    for w in (work, None, work[:200000]):
        _attend(*b, work=w, max_len=n)
    _attend(*b, work=work, window=n // 3)


@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("dt,kept", [(BF16, F8), (F16, F8), (BF16, BF16), (F16, F16)])
def test_attend_chunks(heads, kv_heads, dim, dt, kept, work):
    """Several queries a sequence: whole prompts, chunks, single tokens, more
    queries than keys (rows that see nothing), none at all."""
    keys = [1, 33, 64, 100, 130, 200, 5, 0, 77]
    queries = [1, 33, 17, 100, 3, 64, 9, 2, 0]
    for page, layout in ((16, "heads"), (4, "tokens")):
        b = _batch(_gen(page), keys, queries, heads, kv_heads, dim, page, dt, kept, layout, pad=8)
        _attend(*b, work=work)
        _attend(*b, window=1)
        _attend(*b, work=work, window=37)
        _attend(*b, max_q=2, work=work)     # too small a hint
        _attend(*b, scale=-0.3, work=work)


@pytest.mark.parametrize("n,nq", [(513, 513), (900, 300), (2000, 129), (260, 260)])
@pytest.mark.parametrize("dim,dt,kept", [(128, BF16, F8), (128, BF16, BF16), (64, F16, F16), (64, BF16, F8)])
def test_attend_prompts(n, nq, dim, dt, kept, work):
    b = _batch(_gen(n), [n, 40], [nq, 7], 8, 2, dim, 64, dt, kept)
    _attend(*b, work=work)
    _attend(*b, work=work, window=100)


def test_attend_pages_that_are_not_there(work):
    """Pages past the cache or negative hold no key; lengths past the table end there."""
    keys, queries = [200, 150, 90, 64], [1, 40, 1, 2]
    cache, q, tables, keys, starts = _batch(_gen(1), keys, queries, 8, 2, 128, 16)
    tables[0][3] = -7
    tables[1][2] = cache.k.shape[0]
    tables[1][9] = 2 ** 31 - 1
    tables[2] = [-1] * len(tables[2])
    keys[3] = 10 ** 6
    _attend(cache, q, tables, keys, starts, work=work)
    keys[2] = -5
    _attend(cache, q, tables, keys, starts, work=work, window=30)


@pytest.mark.parametrize("kept,dt", [(F8, BF16), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("queries", [[1, 1, 1], [60, 3, 20]])
def test_attend_nothing_leaks_from_masked_places(kept, dt, queries, work):
    """NaN and infinities in keys and values that a query does not see."""
    keys = [100, 37, 50]
    cache, q, tables, keys, starts = _batch(_gen(2), keys, queries, 8, 2, 128, 16, dt, kept, spare=3)
    # everything that no sequence holds
    held = torch.zeros(cache.k.shape[0], cache.page, dtype=torch.bool, device=DEV)
    for t, n in zip(tables, keys):
        for j in range(n):
            held[t[j // 16], j % 16] = True
    bad = torch.tensor(math.nan if kept == F8 else math.inf, device=DEV).to(kept)
    for x in (cache.k, cache.v):
        y = x.view(torch.uint8) if kept == F8 else x
        y.transpose(1, 2)[~held] = bad.view(torch.uint8) if kept == F8 else bad
    _attend(cache, q, tables, keys, starts, work=work)
    # a key in the middle of each: queries before it, or past its window, stay clean
    for t, j in zip(tables, (70, 30, 45)):
        for x in (cache.k, cache.v):
            y = x.view(torch.uint8) if kept == F8 else x
            y[t[j // 16], :, j % 16, 5] = bad.view(torch.uint8) if kept == F8 else bad
    for window in (0, 4, 13):
        out = torch.zeros_like(q)
        ops.ii_attend(out, q, cache, _i32(tables), _i32(keys), _i32(starts), max_q=max(queries),
                      window=window, work=work)
        clean = torch.ones(q.shape[0], dtype=torch.bool)
        for b, j in enumerate((70, 30, 45)):
            for i in range(queries[b]):
                p = keys[b] - queries[b] + i
                if p >= j and not (window and p - window >= j):
                    clean[starts[b] + i] = False
        zeroed = ops.Cache(*(x.clone() for x in (cache.k, cache.v)),
                           *(x for x in (cache.k_scale, cache.v_scale) if x is not None))
        for x in (zeroed.k, zeroed.v):
            y = x.float()
            x.copy_(torch.where(torch.isfinite(y), y, 0.0).to(kept))
        want, far, _ = ops_ref.attend(q, zeroed, tables, keys, starts, window)
        _close(out[clean], want[clean], far[clean])
        if (~clean).any():
            assert torch.isnan(out[~clean]).any(-1).all()


def test_attend_extreme_scores(work):
    """Scores far apart, and equal ones, large and small; scale 0."""
    cache, q, tables, keys, starts = _batch(_gen(3), [300, 64], [1, 30], 8, 2, 128, 16, BF16, BF16)
    q.mul_(60)
    _attend(cache, q, tables, keys, starts, work=work)
    _attend(cache, q, tables, keys, starts, work=work, scale=0.0)
    cache.k.fill_(3.0)
    _attend(cache, q, tables, keys, starts, work=work, scale=1.0)
    _attend(cache, q, tables, keys, starts, work=work, scale=-1.0)


def test_attend_same_bits(work):
    for keys, queries, heads in (([9000, 40], [1, 1], 8), ([700], [700], 8), ([50000], [3], 8)):
        b = _batch(_gen(4), keys, queries, heads, 2, 128, 64)
        a = _attend(*b, work=work).clone()
        for _ in range(4):
            assert torch.equal(_attend(*b, work=work), a)


def test_attend_queries_outside_the_rows(work):
    """q_start that points past the rows, or runs backwards, is not followed."""
    cache, q, tables, keys, starts = _batch(_gen(5), [64, 64], [5, 6], 8, 2, 128, 16)
    want, far, _ = ops_ref.attend(q, cache, tables, keys, starts)
    big = torch.full((20, 8, 128), 77.0, dtype=BF16, device=DEV)
    out = big[:11]
    ops.ii_attend(out, q, cache, _i32(tables), _i32(keys), _i32([0, 5, 11]), max_q=6, work=work)
    _close(out, want, far)
    for bad in ([0, 5, 2000], [-3, 5, 11], [0, 12, 11], [5, 3, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, 0]):
        ops.ii_attend(out, q, cache, _i32(tables), _i32(keys), _i32(bad), max_q=6, work=work)
        torch.cuda.synchronize()
        assert bool((big[11:] == 77).all())
    assert not work[:65536].any()


# ---------------------------------------------------------------------------
# streams and graphs


def test_other_stream_and_graph(work):
    """Calls on a stream of their own, then captured and replayed with new
    inputs between eager work."""
    g = _gen(7)
    m, n, k = 3, 96, 9000
    x, w = _normal(g, m, k), _normal(g, n, k, std=k ** -0.5)
    y = torch.empty(m, n, dtype=BF16, device=DEV)
    cache, q, tables, keys, starts = _batch(g, [3000, 100], [1, 1], 8, 2, 128, 64)
    t, l = _i32(tables), _i32(keys)
    out = torch.empty_like(q)
    new = _normal(g, 2, 2, 128)
    slots = torch.tensor([tables[0][2999 // 64] * 64 + 2999 % 64, tables[1][99 // 64] * 64 + 99 % 64],
                         device=DEV)
    back = [torch.empty_like(new) for _ in "kv"]
    side = torch.cuda.Stream()

    def step(stream):
        ops.ii_linear(y, x, w, work=work, stream=stream)
        ops.ii_cache_write(cache, new, new, slots, stream=stream)
        ops.ii_attend(out, q, cache, t, l, work=work, stream=stream)
        ops.ii_cache_read(cache, slots, *back, stream=stream)

    def check():
        _close(y, *ops_ref.linear(x, w, BF16))
        want, far, _ = ops_ref.attend(q, cache, tables, keys)
        _close(out, want, far)
        assert torch.equal(back[0].double(), ops_ref.kept(new)[0])

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(side)
    side.synchronize()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    for i in range(4):
        for a in (x, q, new):
            a.normal_(generator=g)
        for a in (y, out, *back):
            a.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check()


# ---------------------------------------------------------------------------
# refusals that need device memory (the others run without a GPU)


def test_refusals(work):
    x, w = _normal(_gen(0), 4, 64), _normal(_gen(1), 32, 64)
    out = torch.zeros(4, 32, dtype=BF16, device=DEV)

    def refused(name, call):
        with pytest.raises(ii.IIError) as e:
            call()
        assert e.value.name == name, e.value
        assert not out.any()

    host = torch.zeros(4, 64, dtype=BF16)
    refused("II_EINVAL", lambda: ops.ii_linear(out, host, w))
    refused("II_EINVAL", lambda: ops.ii_linear(torch.empty(4, 32, dtype=BF16), x, w))
    refused("II_EINVAL", lambda: ops.ii_linear(out, x, w, work=torch.zeros(64, dtype=torch.uint8)))
    buf = torch.zeros(4 * 96, dtype=BF16, device=DEV).view(4, 96)
    refused("II_EOVERLAP", lambda: ops.ii_linear(buf[:, 40:72], buf[:, :64], w))
    ops.ii_linear(buf[:, 64:], buf[:, :64], w)      # columns that are apart
    refused("II_EOVERLAP", lambda: ops.ii_linear(out, x, w, residual=torch.as_strided(out, (4, 32), (0, 1))))
    cache = ops.Cache.empty(4, 2, 16, 64)
    k = _normal(_gen(2), 3, 2, 64)
    slots = torch.arange(3, device=DEV)
    refused("II_EINVAL", lambda: ops.ii_cache_write(cache, k.cpu(), k, slots))
    refused("II_EINVAL", lambda: ops.ii_cache_write(cache, k, k, slots.cpu()))
    refused("II_EOVERLAP", lambda: ops.ii_cache_read(cache, slots, k, k))
    shifted = torch.zeros(3 * 128 + 4, dtype=BF16, device=DEV)[4:].view(3, 2, 64)
    refused("II_EALIGN", lambda: ops.ii_cache_write(cache, shifted, k, slots))
    q = _normal(_gen(3), 1, 4, 64)
    t, n = _i32([[0, 1]]), _i32([20])
    refused("II_EOVERLAP", lambda: ops.ii_attend(q, q, cache, t, n))
    refused("II_EINVAL", lambda: ops.ii_attend(torch.empty_like(q), q, cache, t.cpu(), n))
    refused("II_EINVAL", lambda: ops.ii_attend(torch.empty_like(q), q, cache, t, n, scale=math.inf))
    refused("II_EINVAL", lambda: ops.ii_attend(torch.empty_like(q), q, cache, t, n, window=-1))
    wide = torch.as_strided(cache.k, (4, 2, 16, 64), (2048, 512, 64, 1))
    refused("II_EINVAL", lambda: ops.ii_cache_write(
        ops.Cache(wide, wide, cache.k_scale, cache.v_scale), k, k, slots))


def test_refusal_of_x_as_residual_and_out():
    """out may be the residual, but not x or w too, though their shapes agree."""
    a = torch.zeros(64, 64, dtype=BF16, device=DEV)
    w = _normal(_gen(0), 64, 64)
    for args in ((a, a, w), (a, w, a)):
        with pytest.raises(ii.IIError) as e:
            ops.ii_linear(*args, residual=a)
        assert e.value.name == "II_EOVERLAP"
    ops.ii_linear(a, w, w, residual=a)


@pytest.mark.parametrize("m", [5, 40])
def test_linear_long_rows_at_stride_0(m, work):
    """Rows that broadcast, k past what 32-bit offsets of a tile reach: exact sums."""
    k = (1 << 21) + 64
    x = torch.ones(1, k, dtype=BF16, device=DEV)
    x[0, ::2] = -1
    x[0, -3:] = 2
    out = torch.empty(m, 3, dtype=F32, device=DEV)
    ops.ii_linear(out, x.expand(m, k), torch.ones(1, k, dtype=BF16, device=DEV).expand(3, k), work=work)
    assert bool((out == x.double().sum().item()).all())


def test_attend_a_few_queries_of_long_contexts(work):
    """Some hundred rows over long contexts, split over keys and joined; decoding
    requests beside them."""
    for keys, queries in (([9000], [40]), ([20000, 7000], [33, 90]), ([12000, 5, 300, 0], [70, 1, 2, 1])):
        b = _batch(_gen(len(keys)), keys, queries, 16, 4, 128, 64)
        for w in (work, None, work[:3 << 20]):
            _attend(*b, work=w, max_len=max(keys))
        _attend(*b, work=work, window=3000)


def test_attend_many_queries_of_extreme_scores(work):
    """Maxima that grow by little and by much, a falling and a rising row."""
    cache, q, tables, keys, starts = _batch(_gen(3), [600], [300], 8, 2, 128, 16, BF16, BF16)
    ramp = torch.linspace(-4, 4, 600, device=DEV).to(BF16)
    for j in range(600):
        cache.k[tables[0][j // 16], :, j % 16] = ramp[j]
    for by in (0.02, 0.1, -0.1, 3.0):
        q.fill_(by)
        _attend(cache, q, tables, keys, starts, work=work, scale=1.0)
        _attend(cache, q, tables, keys, starts, work=work, scale=-1.0, window=77)


@pytest.mark.parametrize("dt,kept", [(F16, F16), (F16, F8), (BF16, BF16)])
@pytest.mark.parametrize("gap", [14.0, 18.0])
@pytest.mark.parametrize("queries", [1, 200])
def test_attend_weights_far_below_the_largest(dt, kept, gap, queries, work):
    """Many keys whose weights are e^-gap of the largest: alone each is nothing,
    together they are the result. Four keys (one of each wave's first step of 32)
    have the largest score and values of zero, all others values of one.

    Scores are exact. The result is off by the rounding of a weight and its own
    (U each); the exponent's argument, up to 26 in 24 bits, is off by 2^-19, the
    exponential and the sums by some 2^-19 more (64 additions of 32 keys' sums
    grow by a power of two at most six times)."""
    n, dim, page = 65536, 64, 256
    cache = ops.Cache.empty(n // page, 1, page, dim, kept)
    k = torch.zeros(n, 1, dim, dtype=dt, device=DEV)
    v = torch.ones_like(k)
    k[:128:32, :, 0], v[:128:32] = 1, 0
    ops.ii_cache_write(cache, k, v, torch.arange(n, device=DEV))
    q = torch.zeros(queries, 1, dim, dtype=dt, device=DEV)
    q[..., 0] = gap
    out = torch.empty_like(q)
    ops.ii_attend(out, q, cache, torch.arange(n // page, dtype=torch.int32, device=DEV)[None], _i32([n]),
                  _i32([0, queries]), max_q=queries, scale=1.0)
    few = (n - queries + 1 + torch.arange(queries, device=DEV) - 4) * math.exp(-gap)
    want = (few / (few + 4))[:, None, None].double().expand(out.shape)
    _close(out, want, want * (2 * ops_ref.U[dt] + 2.0 ** -17))


@pytest.mark.parametrize("m", [2, 8])
def test_linear_longest_rows(m, work):
    """k within 63 of 2^31, rows that broadcast: x is -1, 1, -1, 1, .., but 2 in
    its last three places, against ones: 5, exactly, in any order of pairs."""
    k = (1 << 31) - 8
    x = torch.ones(1, k, dtype=BF16, device=DEV)
    x[0, ::2] = -1
    x[0, -3:] = 2
    w = torch.ones(1, k, dtype=BF16, device=DEV)
    for n, out_work in ((3, work), (130, None)):
        out = torch.empty(m, n, dtype=F32, device=DEV)
        ops.ii_linear(out, x.expand(m, k), w.expand(n, k), work=out_work)
        assert bool((out == 5).all())


def test_linear_most_columns_and_most_rows():
    """n, then m, of 2^31 - 1: whole numbers, exact."""
    most = (1 << 31) - 1
    ones = torch.ones(1, 8, dtype=BF16, device=DEV)
    add = torch.empty(most, dtype=BF16, device=DEV)
    step = 1 << 28
    for i in range(0, most, step):
        part = add[i:i + step]
        part.copy_(torch.arange(i, i + part.numel(), device=DEV) % 251 - 120)  # whole, below 2^8: exact
    out = torch.empty_like(add)
    ops.ii_linear(out[None], ones, ones.expand(most, 8), bias=add)
    assert torch.equal(out - 8, add)
    out.zero_()
    ops.ii_linear(out[:, None], ones.expand(most, 8), ones, residual=add[:, None])
    assert torch.equal(out - 8, add)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31, 2 ** 63 - 1])
@pytest.mark.parametrize("keys,queries", [([5, 300, 0], [9, 1, 3]), ([5, 200, 150], [40, 60, 150]),
                                          ([20000], [1])])
def test_attend_windows_that_hide_nothing(keys, queries, window, work):
    """Windows as long as a length can be, up to the largest number: as none, in
    both kernels, with more queries than keys too."""
    b = _batch(_gen(8), keys, queries, 8, 2, 128, 16)
    want = _attend(*b, work=work)
    out = torch.empty_like(b[1])
    ops.ii_attend(out, b[1], b[0], _i32(b[2]), _i32(keys), _i32(b[4]), max_q=max(queries), window=window,
                  work=work)
    assert torch.equal(out, want)


@pytest.mark.parametrize("queries", [1, 300])
@pytest.mark.parametrize("max_len", [0, 500])
def test_attend_without_columns(queries, max_len, work):
    """A page table of no columns: no key is seen, in both kernels."""
    cache, q, _, _, starts = _batch(_gen(9), [500, 500], [queries, 1], 8, 2, 128, 16)
    none = torch.empty(2, 0, dtype=torch.int32, device=DEV)
    for window in (0, 7):
        out = torch.full_like(q, 77.0)
        ops.ii_attend(out, q, cache, none, _i32([500, 500]), _i32(starts), max_q=queries, max_len=max_len,
                      window=window, work=work)
        assert not out.any()


def _apart_from_work(call, tensors):
    """call(work, **tensors) refuses work that meets any one of the tensors, and
    takes work that ends where the tensor starts or lies before it in one buffer."""
    for what, t in tensors.items():
        raw = t.contiguous().view(torch.uint8).flatten()
        buf = torch.zeros((1 << 20) + raw.numel() + 256, dtype=torch.uint8, device=DEV)
        for first in (0, 1 << 20):
            held = buf[first:first + raw.numel()]
            held.copy_(raw)
            moved = held.view(t.dtype).view(t.shape)
            last = first + raw.numel() - 1 & ~15          # the last aligned place inside
            for a, b in ((first, first + 4096), (last, last + (1 << 17)), (max(0, first - 4096), first + 16)):
                work = buf[a:b]
                with pytest.raises(ii.IIError) as e:
                    call(work, **{**tensors, what: moved})
                assert e.value.name == "II_EOVERLAP", (what, first, a, b)
            assert torch.equal(held, raw), what
        buf[:1 << 20] = 0
        call(buf[:1 << 20], **{**tensors, what: moved})   # ends where the tensor starts


def test_linear_work_is_apart():
    g = _gen(11)
    m, n, k = 3, 64, 9000
    x, w, w2 = _normal(g, m, k), _normal(g, n, k, std=k ** -0.5), _normal(g, n, k, std=k ** -0.5)
    b, b2, r = _normal(g, 1, n)[0].contiguous(), _normal(g, 1, n)[0].contiguous(), _normal(g, m, n)
    want, bound = ops_ref.linear(x, w, BF16, b, w2, b2, r)

    def call(work, out, x, w, w2, bias, bias2, residual):
        ops.ii_linear(out, x, w, w2=w2, bias=bias, bias2=bias2, residual=residual, work=work)
        _close(out, want, bound)

    _apart_from_work(call, dict(out=torch.zeros(m, n, dtype=BF16, device=DEV), x=x, w=w, w2=w2, bias=b,
                                bias2=b2, residual=r))


@pytest.mark.parametrize("kept", [F8, BF16])
def test_attend_work_is_apart(kept):
    cache, q, tables, keys, starts = _batch(_gen(12), [3000, 40], [1, 2], 8, 2, 128, 64, BF16, kept)
    want, far, _ = ops_ref.attend(q, cache, tables, keys, starts)
    held = dict(k=cache.k, v=cache.v)
    if kept == F8:
        held.update(k_scale=cache.k_scale, v_scale=cache.v_scale)

    def call(work, out, q, pages, lengths, q_start, **held):
        ops.ii_attend(out, q, ops.Cache(**held), pages, lengths, q_start, max_q=2, work=work)
        _close(out, want, far)

    _apart_from_work(call, dict(out=torch.zeros_like(q), q=q, pages=_i32(tables), lengths=_i32(keys),
                                q_start=_i32(starts), **held))


def test_work_past_what_a_call_uses(work):
    """Only the first WORK_BYTES of scratch are a call's: operands may follow."""
    g = _gen(13)
    x, w = _normal(g, 3, 9000), _normal(g, 64, 9000, std=9000 ** -0.5)
    arena = torch.zeros(ops.WORK_BYTES + x.numel() * 2, dtype=torch.uint8, device=DEV)
    at = arena[ops.WORK_BYTES:].view(BF16).view(3, 9000)
    at.copy_(x)
    out = torch.empty(3, 64, dtype=BF16, device=DEV)
    ops.ii_linear(out, at, w, work=arena)
    _close(out, *ops_ref.linear(x, w, BF16))


def test_cache_read_into_one_buffer():
    """k and v of one buffer, side by side in any place of an axis; not one over the other."""
    h, d, t = 3, 64, 5
    cache = ops.Cache.empty(2, h, 16, d)
    slots = torch.arange(t, device=DEV) * 3
    k, v = (_normal(_gen(i), t, h, d) for i in (1, 2))
    ops.ii_cache_write(cache, k, v, slots)
    for n in (t, 1):
        for shape, pick in (((2, n, h, d), lambda b: (b[0], b[1])), ((n, 2, h, d), lambda b: (b[:, 0], b[:, 1])),
                            ((n, h, 2, d), lambda b: (b[:, :, 0], b[:, :, 1])),
                            ((h, n, 2, d), lambda b: (b[:, :, 0].transpose(0, 1), b[:, :, 1].transpose(0, 1)))):
            kb, vb = pick(torch.zeros(shape, dtype=BF16, device=DEV))
            ops.ii_cache_read(cache, slots[:n], kb, vb)
            assert torch.equal(kb.double(), ops_ref.kept(k[:n])[0])
            assert torch.equal(vb.double(), ops_ref.kept(v[:n])[0])
            with pytest.raises(ii.IIError) as e:
                ops.ii_cache_read(cache, slots[:n], kb, kb)
            assert e.value.name == "II_EOVERLAP"


@pytest.mark.parametrize("m", [1, 3])       # 64 and 192 rows: small and large tiles
def test_linear_gelu_of_negative_values(m):
    """y from -10 to 10 through unit weights into f32, relative to the definition:
    y / sqrt(2) is off by 2^-23 (its rounding and the constant's), which erfc turns
    into at most y^2 + 1 times as much; erfc itself by 16 units, the products by 2."""
    y = torch.linspace(-10, 10, 64 * 64 * m, device=DEV).to(BF16).view(-1, 64)
    out = torch.empty(64 * m, 64, dtype=F32, device=DEV)
    ops.ii_linear(out, y, torch.eye(64, dtype=BF16, device=DEV), act="gelu")
    z = y.double().cpu()
    want = 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    _close(out.cpu(), want, want.abs() * (z * z + 19) * 2.0 ** -23)


@pytest.mark.parametrize("m", [1, 3])
@pytest.mark.parametrize("gated", [False, True])
def test_linear_silu_of_negative_values(m, gated):
    """y from -100 to 20 through unit weights into f32, relative to the definition:
    8 units (ops_ref), half a unit of the least normal value where it ends below."""
    y = torch.linspace(-100, 20, 64 * 64 * m, device=DEV).to(BF16).view(-1, 64)
    out = torch.empty(64 * m, 64, dtype=F32, device=DEV)
    eye = torch.eye(64, dtype=BF16, device=DEV)
    ops.ii_linear(out, y, eye, w2=eye if gated else None, act="silu")
    z = y.double().cpu()
    want = z / (1 + torch.exp(-z)) * (z if gated else 1)
    _close(out.cpu(), want, want.abs() * 2.0 ** -20 + 2.0 ** -127 * (z.abs() if gated else 1))


@pytest.mark.parametrize("m,n,k", [(1, 512, 9000), (1, 4096, 14336), (20, 1, 4096)])
def test_linear_stride_of_a_single_row(m, n, k, work):
    """The same kernel, so the same bits, whatever the stride of the only row is."""
    g = _gen(14)
    x, w = _normal(g, m, k), _normal(g, n, k, std=k ** -0.5)
    r = _normal(g, m, n)
    outs = []
    for stride in (k, k + 1, 1, 1 << 40):
        one = lambda t: t.as_strided(t.shape, (stride, 1)) if t.shape[0] == 1 else t  # noqa: E731
        outs.append(torch.empty(m, n, dtype=F32, device=DEV))
        ops.ii_linear(one(outs[-1]), one(x), one(w), residual=one(r), work=work)
    _close(outs[0], *ops_ref.linear(x, w, F32, residual=r))
    assert all(torch.equal(o, outs[0]) for o in outs)
