"""What the operators' checks of memory refuse and let through, without a GPU: on
addresses that count as device memory, where nothing can be launched."""
import random

import pytest

torch = pytest.importorskip("torch")

import fake_device  # noqa: E402
from paper_2607_18957_amd import ii, ops  # noqa: E402
from test_decoder_ops_abi import ADAPT, CACHE, LOGPROBS, ROTARY, TOKENS, TURN  # noqa: E402

AT = 1 << 40
LET_THROUGH = "II_EHIP"     # nothing can be launched


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    fake = fake_device.build(str(tmp_path_factory.mktemp("fake")))

    def run(*calls):
        return [ii.ERRNAMES[rc] for rc in fake_device.codes(fake, calls)]
    return run


def _adapt(**change):
    return "ii_adapt", [ops._ADAPT.pack(*{**ADAPT, **change}.values())]


@pytest.mark.parametrize("work", [dict(), dict(work=1 << 50, work_bytes=1 << 20)])
def test_adapt_x_is_not_the_output(call, work):
    """x is read by every workgroup that shares its row's columns: base may be out
    itself, x may not, also where base is."""
    square = dict(n=64, k=64, b_stride=64 * 8, out=AT, out_stride=64, base_stride=64, **work)
    apart = {**square, "x": 1 << 47}
    assert call(_adapt(**square), _adapt(**square, x=AT), _adapt(**square, x=AT, base=AT),
                _adapt(**square, x=AT, base=AT, x_stride=128), _adapt(**square, x=AT, base=AT, x_stride=0),
                _adapt(**square, x=AT, base=AT, m=1),
                _adapt(**square, x=AT, base=AT, out_dtype=7, base_dtype=7)) == ["II_EOVERLAP"] * 7
    assert call(_adapt(**apart), _adapt(**apart, base=AT), _adapt(**apart, base=1 << 48),
                _adapt(**apart, base=apart["x"]), _adapt(**apart, base=AT, out_dtype=7, base_dtype=7)) == [LET_THROUGH] * 5
    # of base in place the strides and the types agree
    assert call(_adapt(**{**apart, "base_stride": 128}, base=AT), _adapt(**apart, base=AT, out_dtype=7),
                _adapt(**apart, base=AT, base_dtype=7)) == ["II_EOVERLAP"] * 3


@pytest.mark.parametrize("what", ["adapters", "scales", "ranks", "a", "b"])
def test_adapt_other_inputs_are_not_the_output(call, what):
    at = dict(out=AT, base=AT, base_stride=32, x=1 << 47)
    assert call(_adapt(**at), _adapt(**{**at, what: AT})) == [LET_THROUGH, "II_EOVERLAP"]


def _turned(q, **change):
    return ops._TURN.pack(*{**TURN, **q, **change}.values())


def _fused(tokens, heads, dim, parts, at=AT):
    """Arrays [tokens, heads, dim] side by side for each head: [tokens, heads, parts, dim]."""
    return [dict(x=at + 2 * i * dim, x_token_stride=heads * parts * dim, x_head_stride=parts * dim,
                 out=at + 2 * i * dim, out_token_stride=heads * parts * dim, out_head_stride=parts * dim,
                 tokens=tokens, heads=heads, dim=dim) for i in range(parts)]


def _append(q, k, v, **turn):
    cache = {**CACHE, "heads": k["heads"], "dim": k["dim"]}
    tokens = {**TOKENS, "tokens": k["tokens"], "k": k["x"], "k_token_stride": k["x_token_stride"],
              "k_head_stride": k["x_head_stride"], "v": v["x"], "v_token_stride": v["x_token_stride"],
              "v_head_stride": v["x_head_stride"]}
    rotary = {**ROTARY, "positions": 1 << 50, "freqs": 1 << 51}
    return "ii_cache_append", [ops._CACHE.pack(*cache.values()), ops._TOKENS.pack(*tokens.values()),
                               ops._ROTARY.pack(*rotary.values()), _turned(q, **turn)]


@pytest.mark.parametrize("tokens", [1, 5])
@pytest.mark.parametrize("heads", [1, 6])
def test_queries_beside_the_keys_of_their_head(call, tokens, heads):
    """q, k and v of a head side by side in one buffer: q is turned in place."""
    q, k, v = _fused(tokens, heads, 64, 3)
    assert call(_append(q, k, v), _append(v, q, k), _append(k, v, q)) == [LET_THROUGH] * 3
    # a quarter of a head too far
    assert call(_append(q, k, v, x=AT + 32, out=AT + 32), _append(q, k, k, out=k["x"]),
                _append(q, k, v, out=v["x"])) == ["II_EOVERLAP"] * 3


@pytest.mark.parametrize("tokens", [1, 5])
def test_turned_heads_beside_the_others(call, tokens):
    x, out = _fused(tokens, 6, 64, 2)
    rotary = ops._ROTARY.pack(*{**ROTARY, "positions": 1 << 50, "freqs": 1 << 51}.values())
    to = {k: v for k, v in out.items() if k.startswith("out")}
    assert call(("ii_rotate", [_turned(x, **to), rotary])) == [LET_THROUGH]
    assert call(("ii_rotate", [_turned(x, **{**to, "out": to["out"] - 16}), rotary])) == ["II_EOVERLAP"]


def test_heads_that_meet_are_refused(call):
    """Random places and strides, heads of inputs that meet or are all one among them:
    whatever is let through shares no byte, and arrays of one shape at one stride
    that share none are let through."""
    rng = random.Random(5)
    held = lambda at, ts, hs, n: {at + 2 * (t * ts + h * hs + d) for t in range(n[0]) for h in range(n[1])  # noqa: E731
                                  for d in range(n[2])}
    calls, met, alike = [], [], []
    rotary = ops._ROTARY.pack(*{**ROTARY, "positions": 1 << 50, "freqs": 1 << 51, "rot_dim": 8}.values())
    for _ in range(3000):
        n = rng.choice([1, 2, 3]), rng.choice([1, 2, 3]), 8
        if rng.random() < 0.5:
            hs, ts = rng.choice([(16, 48), (24, 72), (72, 24), (48, 16)])
        else:
            hs, ts = rng.sample([8, 16, 24, 40, 48, 80], 2)
        same = rng.random() < 0.6
        xs = (ts, hs) if same else (rng.choice([0, 8, 16, 24, 48]), rng.choice([0, 8, 16, 24, 48]))
        x, out = (AT + 16 * rng.randint(0, 20) for _ in "xy")
        apart = lambda ts, hs: len(held(0, ts, hs, n)) == n[0] * n[1] * n[2]  # noqa: E731
        if x == out or not apart(ts, hs) or ts < hs * (n[1] - 1) + 8 and hs < ts * (n[0] - 1) + 8:
            continue
        calls.append(("ii_rotate", [_turned({}, tokens=n[0], heads=n[1], dim=8, x=x, x_token_stride=xs[0],
                                            x_head_stride=xs[1], out=out, out_token_stride=ts,
                                            out_head_stride=hs), rotary]))
        met.append(bool(held(x, *xs, n) & held(out, ts, hs, n)))
        alike.append(same and n[0] > 1 and n[1] > 1)
    got = call(*calls)
    assert sum(met) > 200 and sum(a and not m for a, m in zip(alike, met)) > 50
    for rc, m, a in zip(got, met, alike):
        assert rc in ("II_EOVERLAP", LET_THROUGH)
        assert rc == "II_EOVERLAP" if m else (rc == LET_THROUGH or not a)


def _logprobs(**change):
    return "ii_logprobs", [ops._LOGPROBS.pack(*{**LOGPROBS, **change}.values())]


@pytest.mark.parametrize("dtype", [5, 6, 7])
@pytest.mark.parametrize("work", [dict(), dict(work=1 << 50, work_bytes=64 << 20)])
def test_logprobs_vocabularies(call, dtype, work):
    """Up to 2^31 - 1 tokens, as the header says."""
    for vocab, rc in (((1 << 31) - 1, LET_THROUGH), ((1 << 31) - 16384, LET_THROUGH), (1, LET_THROUGH), (1 << 31, "II_EINVAL")):
        assert call(_logprobs(dtype=dtype, vocab=vocab, logits_stride=vocab, **work)) == [rc]


def test_logprobs_scales(call):
    """A logit's exponential is taken of scale / ln 2 times it, a float."""
    most = 2.3e38       # times 1.4427 the largest float
    calls = [_logprobs(scale=s) for s in (most, 1e-38, 1e-45, 3.4028234e38, 2.4e38)]
    assert call(*calls) == [LET_THROUGH] * 3 + ["II_EINVAL"] * 2
