"""The generation example against a 64-bit model that keeps keys and values as
the cache does, so that quantising them is not part of the bound: a wrong
position, mask, scale, slot or order of writing is far outside it."""
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

import ops_ref  # noqa: E402

F8 = torch.float8_e4m3fn

# Mistakes planted in the oracle
FAULTS = ["no rotation", "no causal mask", "scale 1 / dim", "a window of 16", "the newest key left out",
          "the first key left out", "two keys exchanged"]


def _dense(w, meta, dim, tokens, kept, fault=""):
    """Logits of the last token in 64 bits on the CPU, no cache: keys and values
    are rounded to bf16, then to what the cache keeps."""
    n, heads, kv = len(tokens), meta["hidden"] // dim, meta["kv"] // dim
    at = torch.arange(n, dtype=torch.float64)
    angle = at[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    if fault == "no rotation":
        angle = angle * 0
    turn = torch.polar(torch.ones_like(angle), angle)
    scale = 1 / dim if fault == "scale 1 / dim" else dim ** -0.5
    hidden = torch.ones(n, n, dtype=torch.bool).triu(1)
    if fault == "no causal mask":
        hidden[:] = False
    elif fault == "a window of 16":
        hidden |= torch.ones(n, n, dtype=torch.bool).tril(-16)
    elif fault == "the newest key left out":
        hidden[-1, -1] = True
    elif fault == "the first key left out":
        hidden[1:, 0] = True

    def norm(x, name):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w[name]

    def split(h, name, c, rotate, stored):
        y = (h @ w[name].T).view(n, c, dim)
        if rotate:
            z = torch.view_as_complex(y.unflatten(-1, (-1, 2)).contiguous())
            y = torch.view_as_real(z * turn[:, None]).flatten(-2)
        if stored:
            y = y.to(torch.bfloat16)
            y = ops_ref.kept(y)[0] if kept == F8 else y.double()
        return y.repeat_interleave(heads // c, 1).transpose(0, 1)

    x = w["embed"][tokens]
    for i in range(meta["layers"]):
        p = f"layers.{i}."
        h = norm(x, p + "attn_norm")
        q, k, v = (split(h, p + m, c, m != "v", m != "q")
                   for m, c in (("q", heads), ("k", kv), ("v", kv)))
        if fault == "two keys exchanged":
            k = torch.cat([k[:, 1:2], k[:, :1], k[:, 2:]], 1)
        s = (q @ k.transpose(1, 2) * scale).masked_fill(hidden, -torch.inf)
        x = x + (torch.softmax(s, -1) @ v).transpose(0, 1).flatten(1) @ w[p + "o"].T
        h = norm(x, p + "ffn_norm")
        g = h @ w[p + "gate"].T
        x = x + (g * torch.sigmoid(g) * (h @ w[p + "up"].T)) @ w[p + "down"].T
    return norm(x[-1], "final_norm") @ w["lm_head"].T


def _bound(n, kept):
    """Of the logits' norm. Forty tensors are rounded to bf16 (2^-9 / sqrt(3) of
    an element, in the mean over magnitudes 0.7 of it), independently:
    sqrt(40) 0.7 2^-9 / sqrt(3) = 0.005, twice that for what norms and the gate's
    product amplify, twice again for chance. Into 8 bits, values off by e = 2^-9
    round to the next code where they lie that near to a step's middle, steps s
    being 2^-3 to 2^-4 of a value: sqrt(e s) = 0.014 of keys and of values in each
    of four layers, 0.04 of all, averaged over the n keys that are attended to."""
    return 0.02 + (0.04 * n ** -0.5 if kept == F8 else 0)


@pytest.mark.parametrize("kept", [torch.bfloat16, F8])
def test_generate_as_the_cache_keeps_it(kept):
    table = synth.tiny()
    plan, _arena, w = generate.load(table, generate.normal_blob(table))
    w64 = {k: v.cpu().double() for k, v in w.items()}
    prompts = [[3], [(5 * j) % 8192 for j in range(37)], [(11 * j + 2) % 8192 for j in range(150)]]
    model = generate.Model(w, table.meta, 64, 3, 160, page=16, cache_dtype=kept)

    def off(row, p, fault=""):
        want = _dense(w64, table.meta, 64, torch.tensor(p), kept, fault)
        return float((row - want).norm() / want.norm())

    got = model.step(torch.tensor(sum(prompts, []), device="cuda"), [len(p) for p in prompts])
    for step in range(4):
        rows = got.double().cpu()
        for p, row in zip(prompts, rows):
            far = off(row, p)
            assert far <= _bound(len(p), kept), (step, len(p), far)
            if step in (0, 3) and len(p) > 30:
                for fault in FAULTS:
                    assert off(row, p, fault) > _bound(len(p), kept), (fault, step, len(p))
            p.append(int(row.argmax()))
        got = model.step(torch.tensor([p[-1] for p in prompts], device="cuda"), [1, 1, 1])
    plan.free()
