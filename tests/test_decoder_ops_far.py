"""The operators where addresses pass 32 bits, and what lies between the rows they
write: it stays as it was."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ops  # noqa: E402  (fails loudly if libii.so is missing)

import decoder_ref as ref  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, dtype=BF16, std=1.0):
    return torch.empty(*shape, device=DEV).normal_(0, std, generator=g).to(dtype)


def _close(got, want, bound):
    bad = ~(((got.double() - want).abs() <= bound) | (got.double() == want))
    assert not bad.any(), (int(bad.sum()), bad.numel())


@pytest.mark.parametrize("n", [64, 100, 256, 512, 1001, 4096, 20000])
def test_norm_leaves_the_rest(n):
    g = _gen(n)
    for lead, pad in ((8, 16), (3, 5)):
        x, r = _normal(g, 5, n), _normal(g, 5, n, dtype=F32)
        held = torch.full((5, lead + n + pad), 7.0, dtype=BF16, device=DEV)
        total = torch.full((5, lead + n + pad), 7.0, device=DEV)
        ops.ii_norm(held[:, lead:lead + n], x, residual=r, sum=total[:, lead:lead + n])
        want = ref.norm(x, residual=r, stream=F32)
        for t, (value, far) in ((total, want[0]), (held, want[1])):
            _close(t[:, lead:lead + n], value, far)
            assert (t[:, :lead] == 7).all() and (t[:, lead + n:] == 7).all()


@pytest.mark.parametrize("m", [9, 40, 1200])
@pytest.mark.parametrize("n", [8, 60, 130, 1000])
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("split", [False, True])
def test_adapt_leaves_the_rest(m, n, out, split):
    g = _gen(m + n)
    x, a, b = _normal(g, m, 96), _normal(g, 3, 16, 96), _normal(g, 3, n, 16)
    ids = torch.randint(-1, 3, (m,), generator=g, device=DEV).int()
    base = _normal(g, m, n)
    held = torch.full((m, n + 11), 7.0, dtype=out, device=DEV)
    ops.ii_adapt(held[:, 3:n + 3], x, a, b, ids, base=base, work=ops.work_buffer() if split else None)
    _close(held[:, 3:n + 3], *ref.adapt(x, a, b, ids, None, None, base, out))
    assert (held[:, :3] == 7).all() and (held[:, n + 3:] == 7).all()


def test_rotate_leaves_the_rest():
    g = _gen(1)
    held = torch.full((6, 5, 80), 7.0, dtype=BF16, device=DEV)
    x, at, freqs = _normal(g, 6, 3, 64), torch.arange(6, device=DEV) * 99, ops.ii_rotary_freqs(64)
    ops.ii_rotate(held[:, 1:4, 8:72], x, at, freqs)
    want = ref.turn(x, at, freqs)
    _close(held[:, 1:4, 8:72], want, ref.rounded(want, BF16))
    held[:, 1:4, 8:72] = 7
    assert (held == 7).all()


def test_append_past_32_bits():
    """Pages whose bytes lie past 2^32, queries too."""
    g = _gen(2)
    pages, heads, page, dim, t = 5000, 8, 1024, 128, 40
    cache = ops.Cache.empty(pages, heads, page, dim)        # 5.2 GB of keys
    slots = (torch.randint(pages - 900, pages, (t,), generator=g, device=DEV) * page
             + torch.randperm(page, generator=g, device=DEV)[:t])
    k, v, q = _normal(g, t, heads, dim), _normal(g, t, heads, dim), _normal(g, t, 4, dim)
    wide = torch.empty(t, 60_000_000, dtype=BF16, device=DEV)
    q_out = wide[:, :4 * dim].unflatten(1, (4, dim))
    at, freqs = torch.randint(0, 100000, (t,), generator=g, device=DEV), ops.ii_rotary_freqs(dim)
    ops.ii_cache_append(cache, k, v, slots, at, freqs, q=q, q_out=q_out)
    back = [torch.empty_like(k) for _ in "kv"]
    ops.ii_cache_read(cache, slots, *back)
    assert torch.equal(back[0].double(), ref.kept(ref.turn(k, at, freqs))[0])
    assert torch.equal(back[1].double(), ref.kept(v.double())[0])
    want = ref.turn(q, at, freqs)
    _close(q_out, want, ref.rounded(want, BF16))
    assert (cache.k.view(torch.uint8)[:1000] == 0).all()


def test_logprobs_past_32_bits():
    g = _gen(3)
    rows, vocab = 35000, 128257                              # 4.5e9 logits, rows that begin inside words
    x = torch.empty(rows, vocab, dtype=BF16, device=DEV).normal_(0, 3, generator=g)
    targets = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    logprob, entropy = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ids, tops = torch.empty(rows, 3, dtype=torch.int64, device=DEV), torch.empty(rows, 3, device=DEV)
    ops.ii_logprobs(x, targets=targets, logprob=logprob, entropy=entropy, top_ids=ids, top_logprobs=tops)
    some = torch.tensor([0, 1, 17000, 33488, 33489, rows - 2, rows - 1], device=DEV)
    logp, off, h, far = ref.logprobs(x[some])
    at = targets[some][:, None]
    _close(logprob[some], logp.gather(1, at)[:, 0], off.gather(1, at)[:, 0])
    _close(entropy[some], h, far)
    assert torch.equal(ids[some], torch.sort(x[some].float(), dim=1, descending=True, stable=True).indices[:, :3])
    assert logprob.isfinite().all() and (ids >= 0).all() and (ids < vocab).all()


def test_adapt_past_32_bits():
    """Adapters and results that lie past 2^32 bytes."""
    g = _gen(4)
    m, n, k, rank, count = 70001, 32000, 64, 8, 3
    x, a, b = _normal(g, m, k), _normal(g, count, rank, k), _normal(g, count, n, rank)
    far_a = torch.empty(count, 1 << 30, dtype=BF16, device=DEV)[:, -rank * k:].unflatten(1, (rank, k))
    far_a.copy_(a)
    ids = torch.randint(-1, count, (m // 100 + 1,), generator=g, device=DEV).repeat_interleave(100)[:m].int()
    out = torch.empty(m, n, dtype=BF16, device=DEV)          # 4.5 GB
    work = ops.work_buffer()
    ops.ii_adapt(out, x, far_a, b, ids, work=work)
    rows = torch.cat([torch.arange(50), torch.arange(m // 2, m // 2 + 50), torch.arange(m - 50, m)]).to(DEV)
    _close(out[rows], *ref.adapt(x[rows], a, b, ids[rows]))
    out[rows] = 0
    ops.ii_adapt(out[-300:], x[-300:], far_a, b, ids[-300:].contiguous(), work=work)
    _close(out[-50:], *ref.adapt(x[-50:], a, b, ids[-50:]))


def test_norm_past_32_bits():
    m, n = 300000, 8192                                      # 4.9 GB in, as much out
    x = torch.empty(m, n, dtype=BF16, device=DEV).normal_(0, 1, generator=_gen(5))
    out = torch.empty_like(x)
    ops.ii_norm(out, x)
    rows = torch.tensor([0, 131071, 131072, 262143, 262145, m - 1], device=DEV)
    _close(out[rows], *ref.norm(x[rows])[1])
    assert out.isfinite().all()
