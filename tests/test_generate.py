"""The generation example: loaded weights, prompts, then single tokens,
against the same model in 64 bits."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import generate  # noqa: E402
from paper_2607_18957_amd import synth  # noqa: E402


def _dense(w, meta, dim, tokens):
    """Logits of the last token, all in 64 bits, no cache."""
    w = {k: v.double() for k, v in w.items()}
    n, heads, kv = len(tokens), meta["hidden"] // dim, meta["kv"] // dim
    at = torch.arange(n, device="cuda", dtype=torch.float64)
    angle = at[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
    turn = torch.polar(torch.ones_like(angle), angle)

    def norm(x, name):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w[name]

    def split(h, name, c, rotate):
        y = (h @ w[name].T).view(n, c, dim)
        if rotate:
            z = torch.view_as_complex(y.unflatten(-1, (-1, 2)).contiguous())
            y = torch.view_as_real(z * turn[:, None]).flatten(-2)
        return y.repeat_interleave(heads // c, 1).transpose(0, 1)

    x = w["embed"][tokens]
    hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
    for i in range(meta["layers"]):
        p = f"layers.{i}."
        h = norm(x, p + "attn_norm")
        q, k, v = (split(h, p + m, c, m != "v") for m, c in (("q", heads), ("k", kv), ("v", kv)))
        s = (q @ k.transpose(1, 2).contiguous() * dim ** -0.5).masked_fill(hidden, -torch.inf)
        x = x + (torch.softmax(s, -1) @ v).transpose(0, 1).flatten(1) @ w[p + "o"].T
        h = norm(x, p + "ffn_norm")
        g = h @ w[p + "gate"].T
        x = x + (g * torch.sigmoid(g) * (h @ w[p + "up"].T)) @ w[p + "down"].T
    return norm(x[-1], "final_norm") @ w["lm_head"].T


# Ten tensors a layer are rounded to bf16 (2^-9 of an element at most), four
# layers, their errors added up at worst: 40 * 2^-9 = 0.08 of the logits' norm,
# doubled for what the norms and the gate's product amplify. An 8-bit cache adds
# 2^-4 of keys and of values in each layer.
@pytest.mark.parametrize("kept,most", [(torch.bfloat16, 0.16), (torch.float8_e4m3fn, 0.16 + 8 * 2.0 ** -4)])
def test_generate(kept, most):
    table = synth.tiny()
    plan, _arena, w = generate.load(table, generate.normal_blob(table))
    prompts = [[3], [(5 * j) % 8192 for j in range(37)], [(11 * j + 2) % 8192 for j in range(150)]]
    model = generate.Model(w, table.meta, 64, 3, 160, page=16, cache_dtype=kept)
    got = model.step(torch.tensor(sum(prompts, []), device="cuda"), [len(p) for p in prompts])
    for _ in range(3):
        for p, row in zip(prompts, got):
            want = _dense(w, table.meta, 64, torch.tensor(p, device="cuda"))
            assert (row.double() - want).norm() <= most * want.norm()
            p.append(int(row.argmax()))
        got = model.step(torch.tensor([p[-1] for p in prompts], device="cuda"), [1, 1, 1])
    plan.free()


def test_refuses_what_does_not_fit():
    """Sequences past max_len, and counts that do not fit the tokens, are refused
    before anything is launched; the model goes on as if they had not been given."""
    table = synth.tiny()
    plan, _arena, w = generate.load(table, generate.normal_blob(table))
    model = generate.Model(w, table.meta, 64, 2, 20, page=16)
    model.step(torch.arange(15, device="cuda"), [5, 10])
    for tokens, counts in ((27, [16, 11]), (18, [16, 2]), (12, [1, 11]), (2, [2, 0]), (1, [1]), (3, [1, 1]),
                           (3, [1, 1, 1])):
        with pytest.raises(ValueError):
            model.step(torch.arange(tokens, device="cuda"), counts)
    assert model.step(torch.arange(25, device="cuda"), [15, 10]).isfinite().all()
    assert model.lengths.tolist() == [20, 20]
    plan.free()


@pytest.mark.parametrize("count", ["0", "-300", "2"])
def test_command_line(count, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["generate.py", "--tokens", count])
    if int(count) < 1:
        with pytest.raises(SystemExit) as e:
            generate.main()
        assert "1 or more" in str(e.value)
    else:
        generate.main()
        assert capsys.readouterr().out.count("prompt of") == 3
