"""ii_adapt on one tensor: base may be its output, x may not, also where base is."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ii, ops  # noqa: E402  (fails loudly if libii.so is missing)

import decoder_ref as ref  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("m,k,rank", [(1, 64, 8), (40, 1024, 16), (40, 512, 64), (700, 256, 16)])
@pytest.mark.parametrize("split", [False, True])
def test_x_is_not_the_output(m, k, rank, split):
    g = torch.Generator(device=DEV).manual_seed(m + k)
    normal = lambda *s, dt=BF16, std=1.0: torch.empty(*s, device=DEV).normal_(0, std, generator=g).to(dt)  # noqa: E731
    x, a, b = normal(m, k), normal(2, rank, k, std=k ** -0.5), normal(2, k, rank)
    ids = torch.randint(0, 2, (m,), generator=g, device=DEV).int()
    work = ops.work_buffer() if split else None
    wide = normal(m, k, dt=F32)
    narrow = wide.view(BF16)[:, :k]         # 16 bits at the same address
    for out, x_, base in ((x, x, x), (x, x, None), (wide, narrow, wide)):
        before = out.clone()
        with pytest.raises(ii.IIError) as e:
            ops.ii_adapt(out, x_, a, b, ids, base=base, work=work)
        assert e.value.name == "II_EOVERLAP", e.value
        torch.cuda.synchronize()
        assert torch.equal(out, before)
    # the same sum, x kept apart
    y = x.clone()
    want, far = ref.adapt(x, a, b, ids, None, None, y)
    ops.ii_adapt(y, x, a, b, ids, base=y, work=work)
    assert bool(((y.double() - want).abs() <= far).all())
