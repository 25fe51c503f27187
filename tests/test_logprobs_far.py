"""Log-probabilities of the largest vocabularies."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ops  # noqa: E402  (fails loudly if libii.so is missing)

import decoder_ref as ref  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
E = 2.0 ** -24


@pytest.mark.parametrize("dt,vocab", [(BF16, (1 << 31) - 1), (F16, (1 << 31) - 16385), (F32, (1 << 31) - 16384)])
@pytest.mark.parametrize("split", [False, True])
def test_largest_vocabulary(dt, vocab, split):
    """Zeros but for three tokens, the last among them. Log p is off by what the sum of
    exponentials is, in proportion: e^-13 by 2 E (1 + 13), 31 additions of 32 bits by
    E each, at most 24 changes of the largest logit (a tile's, a wave's, a part's) by
    2 E each, and the result by its own rounding; the entropy by that and as much again
    of the mean, 13 at most, and of its terms."""
    x = torch.zeros(1, vocab, dtype=dt, device=DEV)
    x[0, 7] = x[0, vocab - 1] = 12.0
    x[0, vocab // 2] = 13.0
    f32 = lambda *s: torch.full(s, 7.0, device=DEV)  # noqa: E731
    logprob, entropy, tops = f32(1), f32(1), f32(1, 5)
    ids = torch.full((1, 5), -7, dtype=torch.int64, device=DEV)
    ops.ii_logprobs(x, targets=torch.tensor([vocab - 1], device=DEV), logprob=logprob, entropy=entropy, top_ids=ids,
                    top_logprobs=tops, work=ops.work_buffer() if split else None)
    total = vocab - 3 + 2 * math.exp(12) + math.exp(13)
    log = math.log(total)
    mean = (24 * math.exp(12) + 13 * math.exp(13)) / total
    off = (28 + 31 + 48) * E
    assert ids.tolist() == [[vocab // 2, 7, vocab - 1, 0, 1]]
    for got, want in [(logprob[0].item(), 12 - log), *zip(tops[0].tolist(), (13 - log, 12 - log, 12 - log, -log, -log))]:
        assert abs(got - want) <= off + abs(want) * E
    assert abs(entropy.item() - (log - mean)) <= off * (2 + 2 * 13) + (log - mean) * E


@pytest.mark.parametrize("rows,vocab", [(1, 8192), (3, 20001)])
@pytest.mark.parametrize("scale", [1e-38, 3e-39, 1e-40])
@pytest.mark.parametrize("split", [False, True])
def test_logits_far_apart(rows, vocab, scale, split):
    """Logits of 1e38 to either side, scaled to a few units: what is summed is within
    range only once it is scaled. 2 E (40 + 2 mean) as for other logits."""
    g = torch.Generator(device=DEV).manual_seed(vocab)
    x = (torch.rand(rows, vocab, generator=g, device=DEV) * 2 - 1) * 1.6e38
    x[-1, ::2], x[-1, 1::2] = 1.6e38, -1.6e38
    targets = torch.arange(rows, device=DEV) + vocab // 2
    logprob, entropy = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ids, tops = torch.empty(rows, 5, dtype=torch.int64, device=DEV), torch.empty(rows, 5, device=DEV)
    ops.ii_logprobs(x, targets=targets, logprob=logprob, entropy=entropy, top_ids=ids, top_logprobs=tops, scale=scale,
                    work=ops.work_buffer() if split else None)
    logp, off, h, far = ref.logprobs(x, scale)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(ids, order)
    for got, want, bound in ((logprob, logp.gather(1, targets[:, None])[:, 0], off.gather(1, targets[:, None])[:, 0]),
                             (entropy, h, far), (tops, logp.gather(1, order), off.gather(1, order))):
        assert bool(((got.double() - want).abs() <= bound).all()), (got, want)
