"""A layer norm of rows whose mean is far above their deviation."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ops  # noqa: E402  (fails loudly if libii.so is missing)

from ops_ref import TINY, U  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
E = 2.0 ** -24


@pytest.mark.parametrize("n", [64, 128, 200, 1001, 4096, 8200, 20000])
@pytest.mark.parametrize("mean", [0.0, 1e2, -1e4, 1e6, 3e9])
@pytest.mark.parametrize("dt", [BF16, F16])
def test_layer_norm_of_a_far_mean(n, mean, dt):
    """x is 0, so that sum is the residual exactly. Of z = (y - mean) r: y - mean is
    rounded twice on its way, r and the product once each, 4 E of z in all; the mean
    is known to n 2^-53 of the largest |y| (a sum in 64 bits) and, as a float and
    what that leaves out, to E^2 of itself. The weights' product is rounded once
    and the result to its type."""
    g = torch.Generator(device=DEV).manual_seed(n)
    deviation = max(1.0, abs(mean) * 2.0 ** -22)       # of a few steps of a float at the least
    stream = torch.empty(5, n, device=DEV).normal_(0, 1, generator=g) * deviation + mean
    w = (torch.empty(n, device=DEV).normal_(0, 0.3, generator=g) + 1).to(dt)
    x, out, total = torch.zeros(5, n, dtype=dt, device=DEV), torch.empty(5, n, dtype=dt, device=DEV), torch.empty_like(stream)
    ops.ii_norm(out, x, w, residual=stream, sum=total, kind="layer", eps=1e-5)
    assert torch.equal(total, stream)
    y = stream.double()
    mu = y.mean(-1, keepdim=True)
    r = (((y - mu) ** 2).mean(-1, keepdim=True) + float(torch.tensor(1e-5))) ** -0.5
    z = (y - mu) * r
    far = 4 * E * z.abs() + (n * 2.0 ** -53 + E * E) * y.abs().amax(-1, keepdim=True) * r
    want, far = z * w.double(), far * w.double().abs() + z.abs() * w.double().abs() * E
    far = far + (want.abs() + far) * U[dt] + TINY[dt]
    bad = ~((out.double() - want).abs() <= far)
    assert not bad.any(), (int(bad.sum()), (out.double() - want).abs().max().item())
