"""The generation example with norms, positions and log-probabilities by the
operators, against the same 64-bit model as without."""
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_generate_kept import F8, _bound, _dense  # noqa: E402

import generate  # noqa: E402
from paper_2607_18957_amd import synth  # noqa: E402


@pytest.mark.parametrize("kept", [torch.bfloat16, F8])
def test_generate_fused(kept):
    """Keys are quantised without the rounding to bf16 that the 64-bit model
    makes between: off from its codes as often as that rounding moves one, which
    the bound counts for keys that are rounded another way."""
    table = synth.tiny()
    plan, _arena, w = generate.load(table, generate.normal_blob(table))
    w64 = {k: v.cpu().double() for k, v in w.items()}
    prompts = [[3], [(5 * j) % 8192 for j in range(37)], [(11 * j + 2) % 8192 for j in range(150)]]
    model = generate.Model(w, table.meta, 64, 3, 160, page=16, cache_dtype=kept, fused=True)
    got = model.step(torch.tensor(sum(prompts, []), device="cuda"), [len(p) for p in prompts])
    for step in range(3):
        ids, logp = model.likeliest(got, 4)
        want = torch.log_softmax(got.double(), -1)
        order = torch.sort(got, dim=1, descending=True, stable=True).indices[:, :4]
        assert torch.equal(ids, order)
        assert (logp - want.gather(1, order)).abs().max() <= 2.0 ** -18
        for p, row in zip(prompts, got.double().cpu()):
            dense = _dense(w64, table.meta, 64, torch.tensor(p), kept)
            assert float((row - dense).norm() / dense.norm()) <= _bound(len(p), kept), (step, len(p))
            p.append(int(row.argmax()))
        got = model.step(torch.tensor([p[-1] for p in prompts], device="cuda"), [1, 1, 1])
    plan.free()


@pytest.mark.parametrize("top", ["3", "65", "-1"])
def test_command_line(top, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["generate.py", "--tokens", "2", "--fused", "--top", top])
    if not 0 <= int(top) <= 64:
        with pytest.raises(SystemExit) as e:
            generate.main()
        assert "0 to 64" in str(e.value)
        return
    generate.main()
    out = capsys.readouterr().out.splitlines()
    lines = [x for x in out if x.startswith("  ")]
    assert len(lines) == 6 and all(x.split()[0] == x.split()[2] for x in lines)
