"""Queries, keys and values of each head side by side in one buffer [tokens, heads,
3, dim]: queries turned in place, keys and values into the cache."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ops  # noqa: E402  (fails loudly if libii.so is missing)

import decoder_ref as ref  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def _close(got, want, bound):
    assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("tokens", [1, 50])
@pytest.mark.parametrize("heads,dim", [(1, 64), (6, 64), (5, 128)])
@pytest.mark.parametrize("kept", [BF16, F8])
def test_append_of_fused_heads(tokens, heads, dim, kept):
    g = torch.Generator(device=DEV).manual_seed(tokens + heads)
    fused = torch.empty(tokens, heads, 3, dim, device=DEV).normal_(generator=g).to(BF16)
    before = fused.clone()
    q, k, v = fused.unbind(2)
    slots = torch.randperm(64, generator=g, device=DEV)[:tokens].contiguous()
    at, freqs = torch.randint(0, 5000, (tokens,), generator=g, device=DEV), ops.ii_rotary_freqs(dim)
    cache = ops.Cache.empty(4, heads, 16, dim, kept)
    ops.ii_cache_append(cache, k, v, slots, at, freqs, q=q, q_out=q)
    want = ref.turn(before[:, :, 0], at, freqs)
    _close(q, want, ref.rounded(want, BF16))
    assert torch.equal(fused[:, :, 1:], before[:, :, 1:])
    back = [torch.empty(tokens, heads, dim, dtype=BF16, device=DEV) for _ in "kv"]
    ops.ii_cache_read(cache, slots, *back)
    turned = ref.turn(k, at, freqs)
    if kept == F8:
        assert torch.equal(back[0].double(), ref.kept(turned)[0])
        assert torch.equal(back[1].double(), ref.kept(v.double())[0])
    else:
        _close(back[0], turned, ref.rounded(turned, BF16))
        assert torch.equal(back[1], v)


@pytest.mark.parametrize("tokens", [1, 50])
def test_rotate_beside_its_input(tokens):
    g = torch.Generator(device=DEV).manual_seed(tokens)
    pair = torch.empty(tokens, 6, 2, 96, device=DEV).normal_(generator=g).to(BF16)
    before = pair.clone()
    at, freqs = torch.randint(0, 5000, (tokens,), generator=g, device=DEV), ops.ii_rotary_freqs(64)
    ops.ii_rotate(pair[:, :, 1], pair[:, :, 0], at, freqs)
    want = ref.turn(before[:, :, 0], at, freqs)
    _close(pair[:, :, 1], want, ref.rounded(want, BF16))
    assert torch.equal(pair[:, :, 0], before[:, :, 0])
