"""Where NaN stands among the likeliest tokens: with -infinity, in the order of tokens."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ops  # noqa: E402  (fails loudly if libii.so is missing)

DEV = torch.device("cuda:0")
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF, NAN = math.inf, math.nan


def _rows(n, dt):
    """NaN in every tile, at the borders of tiles and parts, alone, beside infinities,
    and where fewer finite logits are left than are asked for."""
    g = torch.Generator(device=DEV).manual_seed(n)
    x = torch.empty(9, n, device=DEV).normal_(0, 3, generator=g).to(dt)
    at = torch.arange(n, device=DEV)
    x[0, at % 97 == 5] = NAN
    x[1, at % 8192 < 40] = NAN
    x[2, at % 2 == 0] = NAN
    x[3] = NAN
    x[4] = NAN
    x[4, [n // 3, n - 1]] = torch.tensor([1.0, 2.0], device=DEV).to(dt)
    x[5] = -INF
    x[5, at % 3 == 1] = NAN
    x[5, [n // 2, n // 2 + 1, n - 2]] = torch.tensor([-5.0, 7.0, 7.0], device=DEV).to(dt)
    x[6, at % 11 == 3] = NAN
    x[6, [4, n - 3]] = INF
    x[7, 0] = x[7, n - 1] = NAN
    x[8] = NAN
    x[8, ::2] = torch.finfo(dt).min
    return x


@pytest.mark.parametrize("n", [70, 8192, 20001, 131075])
@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("split", [False, True])
def test_nan_is_as_minus_infinity(n, dt, split):
    x = _rows(n, dt)
    work = ops.work_buffer() if split else None
    for top in (1, 4, 20, 64):
        ids = torch.full((9, top), -7, dtype=torch.int64, device=DEV)
        tops = torch.full((9, top), 7.0, device=DEV)
        entropy = torch.full((9,), 7.0, device=DEV)
        ops.ii_logprobs(x, entropy=entropy, top_ids=ids, top_logprobs=tops, work=work)
        want = torch.sort(torch.where(x.isnan(), -INF, x.float()), dim=1, descending=True, stable=True).indices
        assert torch.equal(ids, want[:, :top])
        assert tops.isnan().all() and entropy.isnan().all()
