"""The C interface of norms, rotary positions, adapters and log-probabilities
without a GPU: what their header says compiles as C, the binding lays arguments
out as it says, refusals give their codes before anything is launched."""
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2607_18957_amd import ii, ops  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
M = 1 << 31
INF, NAN = float("inf"), float("nan")

NORM = dict(dtype=5, stream_dtype=5, kind=0, post=0, m=4, n=64, x=1 << 40, x_stride=64, gate=0, gate_stride=0,
            residual=0, residual_stride=0, post_weight=0, post_bias=0, weight=1 << 41, bias=0, sum=0,
            sum_stride=0, out=1 << 42, out_stride=64, scale=1.0, eps=1e-5, offset=0.0, reserved=0)
ROTARY = dict(positions=1 << 40, freqs=1 << 41, rot_dim=64, layout=0, magnitude=1.0, reserved=0)
TURN = dict(dtype=5, heads=2, dim=64, reserved=0, tokens=3, x=1 << 42, x_token_stride=128, x_head_stride=64,
            out=1 << 43, out_token_stride=128, out_head_stride=64)
LOGPROBS = dict(dtype=7, top=2, rows=3, vocab=100, logits=1 << 40, logits_stride=100, targets=1 << 41,
                logprob=1 << 42, entropy=1 << 43, top_ids=1 << 44, top_logprobs=1 << 45, scale=1.0, reserved=0,
                work=0, work_bytes=0)
ADAPT = dict(dtype=5, out_dtype=5, base_dtype=5, rank=8, m=4, n=32, k=64, count=2, x=1 << 40, x_stride=64,
             a=1 << 41, a_stride=512, a_row_stride=64, b=1 << 42, b_stride=256, b_row_stride=8,
             adapters=1 << 43, scales=0, ranks=0, base=0, base_stride=0, out=1 << 44, out_stride=32, work=0,
             work_bytes=0)
CACHE = dict(dtype=5, heads=2, dim=64, page=16, pages=0, k=0, v=0, k_scale=0, v_scale=0, page_stride=2048,
             head_stride=1024, token_stride=64, scale_page_stride=0, scale_head_stride=0, scale_token_stride=0)
TOKENS = dict(dtype=5, reserved=0, tokens=3, k=1 << 44, k_token_stride=128, k_head_stride=64,
              v=1 << 45, v_token_stride=128, v_head_stride=64, slots=1 << 46)
STRUCTS = {"ii_norm_args": (ops._NORM, NORM), "ii_rotary": (ops._ROTARY, ROTARY), "ii_turn": (ops._TURN, TURN),
           "ii_logprobs_args": (ops._LOGPROBS, LOGPROBS), "ii_adapt_args": (ops._ADAPT, ADAPT)}


def _offsets(fmt):
    """Byte offset of each field of a struct.Struct of unpadded fields."""
    width = {"i": 4, "f": 4, "q": 8, "Q": 8}
    out, at, count = [], 0, ""
    for ch in fmt.lstrip("="):
        if ch.isdigit():
            count += ch
            continue
        for _ in range(int(count or 1)):
            out.append(at)
            at += width[ch]
        count = ""
    return out


def test_structs_are_laid_out_as_the_header_says(tmp_path):
    lines = ["#include <stddef.h>", '#include "ii_ops.h"']
    for name, (packed, fields) in STRUCTS.items():
        fmt = packed.format if isinstance(packed.format, str) else packed.format.decode()
        at = _offsets(fmt)
        assert len(at) == len(fields), name
        lines.append(f'_Static_assert(sizeof({name}) == {packed.size}, "{name}");')
        lines += [f'_Static_assert(offsetof({name}, {f}) == {o}, "{name}.{f}");' for f, o in zip(fields, at)]
    lines += [f'_Static_assert(II_MAX_TOP == {ops.MAX_TOP}, "top");',
              *(f'_Static_assert(II_NORM_{k.upper()} == {v}, "{k}");' for k, v in ops.NORMS.items()),
              *(f'_Static_assert(II_ROTARY_{k.upper()} == {v}, "{k}");' for k, v in ops.LAYOUTS.items()),
              "int main(void) { return 0; }"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines) + "\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only",
                           "-I", os.path.join(ROOT, "include"), str(src)])


def _refused(rc, name):
    assert ii.ERRNAMES[rc] == name, (ii.ERRNAMES[rc], ii.ii_last_error())
    assert ii.ii_last_error()


@pytest.mark.parametrize("name,change", [
    ("II_EINVAL", dict(dtype=7)), ("II_EINVAL", dict(stream_dtype=6)), ("II_EINVAL", dict(kind=2)),
    ("II_EINVAL", dict(kind=-1)), ("II_EINVAL", dict(post=2)), ("II_EINVAL", dict(reserved=1)),
    ("II_EINVAL", dict(m=-1)), ("II_EINVAL", dict(m=M)), ("II_EINVAL", dict(n=-1)), ("II_EINVAL", dict(n=32769)),
    ("II_EINVAL", dict(scale=INF)), ("II_EINVAL", dict(scale=NAN)), ("II_EINVAL", dict(eps=-1e-5)),
    ("II_EINVAL", dict(eps=NAN)), ("II_EINVAL", dict(offset=INF)), ("II_EINVAL", dict(post_weight=1 << 43)),
    ("II_EINVAL", dict(post_bias=1 << 43)), ("II_EINVAL", dict(out=0)), ("II_EINVAL", dict(out=0, weight=0)),
    ("II_EINVAL", dict(out=0, weight=0, bias=1 << 43, sum=1 << 44, sum_stride=64)),
    ("II_EINVAL", dict(x_stride=-64)), ("II_EINVAL", dict(gate=1 << 43, gate_stride=-1)),
    ("II_EINVAL", dict(out_stride=63)), ("II_EINVAL", dict(sum=1 << 43, sum_stride=63)), ("II_EINVAL", dict(x=0)),
    ("II_EALIGN", dict(out=(1 << 42) + 1)), ("II_EALIGN", dict(stream_dtype=7, sum=(1 << 43) + 2, sum_stride=64)),
    ("II_EOVERFLOW", dict(out_stride=1 << 62)), ("II_EOVERFLOW", dict(stream_dtype=7, sum=1 << 43, sum_stride=1 << 62)),
    ("II_EOVERFLOW", dict(out_stride=3 << 61)),
    ("II_EINVAL", dict())])   # not memory of any device
def test_norm_refusals(name, change):
    _refused(ops._call_norm(ops._NORM.pack(*{**NORM, **change}.values()), 0), name)


@pytest.mark.parametrize("name,turn,rotary", [
    ("II_EINVAL", dict(dtype=7), {}), ("II_EINVAL", dict(heads=0), {}), ("II_EINVAL", dict(heads=M - 1), {}),
    ("II_EINVAL", dict(dim=4), {}), ("II_EINVAL", dict(dim=60), {}), ("II_EINVAL", dict(dim=520), {}),
    ("II_EINVAL", dict(reserved=1), {}), ("II_EINVAL", dict(tokens=-1), {}), ("II_EINVAL", dict(tokens=1 << 41), {}),
    ("II_EINVAL", dict(x=0), {}), ("II_EINVAL", dict(out_head_stride=56), {}),
    ("II_EINVAL", dict(x_token_stride=-128), {}), ("II_EALIGN", dict(x=(1 << 42) + 8), {}),
    ("II_EALIGN", dict(x_head_stride=68), {}), ("II_EOVERFLOW", dict(x_token_stride=1 << 62), {}),
    ("II_EINVAL", dict(tokens=0), dict(rot_dim=66)), ("II_EINVAL", dict(tokens=0), dict(rot_dim=3)),
    ("II_EINVAL", dict(tokens=0), dict(rot_dim=-2)), ("II_EINVAL", dict(tokens=0), dict(layout=2)),
    ("II_EINVAL", dict(tokens=0), dict(magnitude=INF)), ("II_EINVAL", dict(tokens=0), dict(magnitude=NAN)),
    ("II_EINVAL", dict(tokens=0), dict(reserved=1)), ("II_EINVAL", {}, {})])
def test_rotate_refusals(name, turn, rotary):
    args = ops._TURN.pack(*{**TURN, **turn}.values()), ops._ROTARY.pack(*{**ROTARY, **rotary}.values())
    _refused(ops._call_rotate(*args, 0), name)


@pytest.mark.parametrize("name,cache,tokens,rotary,turn", [
    ("II_EINVAL", dict(dim=96), {}, {}, {}), ("II_EINVAL", dict(page=24), {}, {}, {}),
    ("II_EINVAL", dict(dtype=6), {}, {}, {}), ("II_EINVAL", {}, dict(tokens=-1), {}, {}),
    ("II_EINVAL", {}, dict(slots=0), {}, {}), ("II_EINVAL", {}, dict(tokens=0), dict(rot_dim=66), {}),
    ("II_EINVAL", {}, dict(tokens=0), dict(layout=-1), {}), ("II_EINVAL", {}, dict(tokens=0), {}, dict(dtype=6)),
    ("II_EINVAL", {}, dict(tokens=0), {}, dict(tokens=1)), ("II_EINVAL", {}, dict(tokens=0), {}, dict(dim=128)),
    ("II_EINVAL", {}, dict(tokens=0), {}, dict(heads=0)), ("II_EALIGN", {}, dict(slots=4), {}, {}),
    ("II_EINVAL", {}, {}, {}, {})])
def test_append_refusals(name, cache, tokens, rotary, turn):
    args = [ops._CACHE.pack(*{**CACHE, **cache}.values()), ops._TOKENS.pack(*{**TOKENS, **tokens}.values()),
            ops._ROTARY.pack(*{**ROTARY, **rotary}.values()),
            ops._TURN.pack(*{**TURN, "tokens": {**TOKENS, **tokens}["tokens"], **turn}.values())]
    _refused(ops._call_append(*args, 0), name)


@pytest.mark.parametrize("name,change", [
    ("II_EINVAL", dict(dtype=3)), ("II_EINVAL", dict(top=-1)), ("II_EINVAL", dict(top=65)),
    ("II_EINVAL", dict(top=0)), ("II_EINVAL", dict(top_ids=0)), ("II_EINVAL", dict(top_logprobs=0)),
    ("II_EINVAL", dict(targets=0)), ("II_EINVAL", dict(logprob=0)),
    ("II_EINVAL", dict(top=0, top_ids=0, top_logprobs=0, targets=0, logprob=0, entropy=0)),
    ("II_EINVAL", dict(rows=-1)), ("II_EINVAL", dict(rows=M)), ("II_EINVAL", dict(vocab=0)),
    ("II_EINVAL", dict(vocab=M)), ("II_EINVAL", dict(scale=0.0)), ("II_EINVAL", dict(scale=-1.0)),
    ("II_EINVAL", dict(scale=INF)), ("II_EINVAL", dict(scale=NAN)), ("II_EINVAL", dict(reserved=1)),
    ("II_EINVAL", dict(logits_stride=-1)), ("II_EINVAL", dict(logits=0)), ("II_EALIGN", dict(logits=(1 << 40) + 2)),
    ("II_EOVERFLOW", dict(logits_stride=1 << 62)), ("II_EINVAL", dict())])
def test_logprobs_refusals(name, change):
    _refused(ops._call_logprobs(ops._LOGPROBS.pack(*{**LOGPROBS, **change}.values()), 0), name)


@pytest.mark.parametrize("name,change", [
    ("II_EINVAL", dict(dtype=7)), ("II_EINVAL", dict(out_dtype=6)), ("II_EINVAL", dict(base_dtype=6)),
    ("II_EINVAL", dict(rank=0)), ("II_EINVAL", dict(rank=257)), ("II_EINVAL", dict(m=-1)), ("II_EINVAL", dict(n=M)),
    ("II_EINVAL", dict(k=M)), ("II_EINVAL", dict(count=-1)), ("II_EINVAL", dict(count=M)),
    ("II_EINVAL", dict(x_stride=-1)), ("II_EINVAL", dict(base=1 << 45, base_stride=-1)),
    ("II_EINVAL", dict(out_stride=31)), ("II_EINVAL", dict(out=0)), ("II_EALIGN", dict(out=(1 << 44) + 1)),
    ("II_EALIGN", dict(out_dtype=7, out=(1 << 44) + 2)), ("II_EOVERFLOW", dict(out_stride=1 << 62)),
    ("II_EINVAL", dict())])
def test_adapt_refusals(name, change):
    _refused(ops._call_adapt(ops._ADAPT.pack(*{**ADAPT, **change}.values()), 0), name)


@pytest.mark.parametrize("change", [
    dict(rot_dim=-2), dict(rot_dim=3), dict(rot_dim=(1 << 20) + 2), dict(base=0.0), dict(base=-1.0), dict(base=INF),
    dict(factor=0.0), dict(factor=NAN), dict(original=-1), dict(original=8192, low=4.0, high=4.0),
    dict(original=8192, low=NAN), dict(original=8192, high=INF)])
def test_freqs_refusals(change):
    with pytest.raises(ii.IIError) as e:
        ops.ii_rotary_freqs(**{**dict(rot_dim=8, device="cpu"), **change})
    assert e.value.name == "II_EINVAL"


def test_null_and_empty():
    import ctypes
    lib = ctypes.CDLL(ii.LIB_PATH)
    for name, n in (("ii_norm", 2), ("ii_rotate", 3), ("ii_cache_append", 5), ("ii_logprobs", 2), ("ii_adapt", 2)):
        f = getattr(lib, name)
        f.argtypes = [ctypes.c_void_p] * n
        assert f(*[None] * n) == ii.EINVAL
    # nothing to do touches no device
    for change in (dict(m=0), dict(n=0)):
        assert ops._call_norm(ops._NORM.pack(*{**NORM, **change}.values()), 0) == 0
        assert ops._call_adapt(ops._ADAPT.pack(*{**ADAPT, **change}.values()), 0) == 0
    rotary = ops._ROTARY.pack(*ROTARY.values())
    turn = ops._TURN.pack(*{**TURN, "tokens": 0}.values())
    tokens = ops._TOKENS.pack(*{**TOKENS, "tokens": 0}.values())
    assert ops._call_rotate(turn, rotary, 0) == 0
    assert ops._call_append(ops._CACHE.pack(*CACHE.values()), tokens, rotary, turn, 0) == 0
    assert ops._call_append(ops._CACHE.pack(*CACHE.values()), tokens, rotary, None, 0) == 0
    assert ops._call_logprobs(ops._LOGPROBS.pack(*{**LOGPROBS, "rows": 0}.values()), 0) == 0


def test_shapes_that_do_not_fit():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    x, w, c64 = z(4, 64), z(64), torch.complex64
    h, at, f = z(3, 2, 64), torch.arange(3), torch.ones(32, dtype=torch.float64)
    cache = ops.Cache.empty(2, 2, 16, 64, torch.bfloat16, device="cpu")
    a, b, ids = z(2, 8, 64), z(2, 32, 8), z(4, dt=torch.int32)
    logits, p = z(4, 100, dt=torch.float32), z(4, dt=torch.float32)
    for call in (lambda: ops.ii_norm(z(4, 63), x, w), lambda: ops.ii_norm(x, x, z(63)),
                 lambda: ops.ii_norm(x, x, w.float()), lambda: ops.ii_norm(x.float(), x, w),
                 lambda: ops.ii_norm(x, x, w, kind="batch"), lambda: ops.ii_norm(x, x, w, gate=z(4, 1)),
                 lambda: ops.ii_norm(x, x, w, residual=x.float(), sum=x), lambda: ops.ii_norm(x, z(64, 4).t(), w),
                 lambda: ops.ii_norm(x.to(c64), x.to(c64)), lambda: ops.ii_rotate(h, h, at.int(), f),
                 lambda: ops.ii_rotate(h, h, at, f.float()), lambda: ops.ii_rotate(h, h, at[:2], f),
                 lambda: ops.ii_rotate(z(3, 2, 32), h, at, f), lambda: ops.ii_rotate(h.float(), h, at, f),
                 lambda: ops.ii_rotate(h, h, at, f[None]), lambda: ops.ii_rotate(h, h, at, f, layout="thirds"),
                 lambda: ops.ii_rotate(h, z(3, 64, 2).transpose(1, 2), at, f),
                 lambda: ops.ii_cache_append(cache, h, h, at, at, f, q=h),
                 lambda: ops.ii_cache_append(cache, h, h, at, at, f, q_out=h),
                 lambda: ops.ii_cache_append(cache, h, h, at, at, f, q=z(2, 2, 64), q_out=z(2, 2, 64)),
                 lambda: ops.ii_cache_append(cache, h, h, at, at, f, q=h.half(), q_out=h.half()),
                 lambda: ops.ii_cache_append(cache, h, h, at, at[:2], f),
                 lambda: ops.ii_cache_append(cache, z(3, 1, 64), z(3, 1, 64), at, at, f),
                 lambda: ops.ii_adapt(z(4, 31), x, a, b, ids), lambda: ops.ii_adapt(z(4, 32), x, a, b, ids.long()),
                 lambda: ops.ii_adapt(z(4, 32), x, a, z(2, 32, 9), ids), lambda: ops.ii_adapt(z(4, 32), x, a.half(), b, ids),
                 lambda: ops.ii_adapt(z(4, 32), x, a, b, ids[:3]), lambda: ops.ii_adapt(z(4, 32), x, a, b, ids, base=x),
                 lambda: ops.ii_adapt(z(4, 32), x, a, b, ids, scales=z(2)), lambda: ops.ii_adapt(z(4, 32), x, a, b, ids, ranks=ids),
                 lambda: ops.ii_adapt(z(4, 32), x, z(2, 64, 8).transpose(1, 2), b, ids),
                 lambda: ops.ii_logprobs(logits, targets=at, logprob=p), lambda: ops.ii_logprobs(logits, entropy=p.half()),
                 lambda: ops.ii_logprobs(logits, targets=torch.arange(4)), lambda: ops.ii_logprobs(logits, logprob=p),
                 lambda: ops.ii_logprobs(logits, top_ids=torch.zeros(4, 2).long()),
                 lambda: ops.ii_logprobs(logits, top_ids=torch.zeros(4, 2).long(), top_logprobs=torch.zeros(4, 3)),
                 lambda: ops.ii_logprobs(logits, top_ids=torch.zeros(4, 2).int(), top_logprobs=torch.zeros(4, 2)),
                 lambda: ops.ii_logprobs(z(100, 4, dt=torch.float32).t(), entropy=p)):
        with pytest.raises(ValueError):
            call()
