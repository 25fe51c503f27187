"""The operators' C interface without a GPU: what their header says compiles
as C, the binding lays arguments out as it says, refusals give their codes."""
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2607_18957_amd import ii, ops  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STRUCTS = {
    "ii_linear_args": (ops._LINEAR, ["dtype", "out_dtype", "act", "reserved", "m", "n", "k", "x",
                                     "x_stride", "w", "w_stride", "w2", "w2_stride", "bias", "bias2",
                                     "residual", "residual_stride", "out", "out_stride", "work",
                                     "work_bytes"]),
    "ii_cache": (ops._CACHE, ["dtype", "heads", "dim", "page", "pages", "k", "v", "k_scale", "v_scale",
                              "page_stride", "head_stride", "token_stride", "scale_page_stride",
                              "scale_head_stride", "scale_token_stride"]),
    "ii_tokens": (ops._TOKENS, ["dtype", "reserved", "tokens", "k", "k_token_stride", "k_head_stride",
                                "v", "v_token_stride", "v_head_stride", "slots"]),
    "ii_attend_args": (ops._ATTEND, ["dtype", "heads", "rows", "seqs", "q", "q_row_stride",
                                     "q_head_stride", "out", "out_row_stride", "out_head_stride",
                                     "pages", "pages_stride", "columns", "lengths", "q_start", "max_q",
                                     "max_len", "window", "scale", "reserved", "work", "work_bytes"]),
}


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
        lines += [f'_Static_assert(offsetof({name}, {f}) == {o}, "{name}.{f}");'
                  for f, o in zip(fields, at)]
    lines += [f'_Static_assert(II_WORK_BYTES == {ops.WORK_BYTES}, "work");',
              *(f'_Static_assert(II_ACT_{k.upper()} == {v}, "{k}");' for k, v in ops.ACTS.items()),
              "int main(void) { return 0; }"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines) + "\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only",
                           "-I", os.path.join(ROOT, "include"), str(src)])


LINEAR = dict(dtype=5, out_dtype=5, act=0, reserved=0, m=4, n=32, k=64, x=1 << 40, x_stride=64,
              w=1 << 41, w_stride=64, w2=0, w2_stride=0, bias=0, bias2=0, residual=0,
              residual_stride=0, out=1 << 42, out_stride=32, work=0, work_bytes=0)
CACHE = dict(dtype=3, heads=2, dim=64, page=16, pages=4, k=1 << 40, v=1 << 41, k_scale=1 << 42,
             v_scale=1 << 43, page_stride=2048, head_stride=1024, token_stride=64,
             scale_page_stride=64, scale_head_stride=32, scale_token_stride=2)
TOKENS = dict(dtype=5, reserved=0, tokens=3, k=1 << 44, k_token_stride=128, k_head_stride=64,
              v=1 << 45, v_token_stride=128, v_head_stride=64, slots=1 << 46)
ATTEND = dict(dtype=5, heads=4, rows=2, seqs=2, q=1 << 44, q_row_stride=256, q_head_stride=64,
              out=1 << 45, out_row_stride=256, out_head_stride=64, pages=1 << 46, pages_stride=8,
              columns=8, lengths=1 << 47, q_start=0, max_q=1, max_len=0, window=0, scale=0.125,
              reserved=0, work=0, work_bytes=0)
M = 1 << 31


def _refused(rc, name):
    assert ii.ERRNAMES[rc] == name, (ii.ERRNAMES[rc], ii.ii_last_error())
    assert ii.ii_last_error()


@pytest.mark.parametrize("name,change", [
    ("II_EINVAL", dict(dtype=7)), ("II_EINVAL", dict(out_dtype=6)), ("II_EINVAL", dict(act=4)),
    ("II_EINVAL", dict(act=-1)), ("II_EINVAL", dict(reserved=1)), ("II_EINVAL", dict(m=-1)),
    ("II_EINVAL", dict(n=M)), ("II_EINVAL", dict(k=M)), ("II_EINVAL", dict(bias2=1 << 43)),
    ("II_EINVAL", dict(x_stride=-64)), ("II_EINVAL", dict(out_stride=31)), ("II_EINVAL", dict(out=0)),
    ("II_EALIGN", dict(out=(1 << 42) + 1)), ("II_EALIGN", dict(out_dtype=7, out=(1 << 42) + 2)),
    ("II_EOVERFLOW", dict(out_stride=1 << 62)),
    ("II_EINVAL", dict())])   # not memory of any device
def test_linear_refusals(name, change):
    args = ops._LINEAR.pack(*{**LINEAR, **change}.values())
    _refused(ops._call_linear(args, 0), name)


@pytest.mark.parametrize("name,change,more", [
    ("II_EINVAL", dict(dtype=7), {}), ("II_EINVAL", dict(heads=0), {}), ("II_EINVAL", dict(dim=96), {}),
    ("II_EINVAL", dict(page=24), {}), ("II_EINVAL", dict(page=0), {}), ("II_EINVAL", dict(pages=-1), {}),
    ("II_EINVAL", dict(pages=M), {}), ("II_EINVAL", dict(k=0), {}),
    ("II_EINVAL", dict(token_stride=-64), {}), ("II_EINVAL", dict(head_stride=512), {}),
    ("II_EALIGN", dict(k=(1 << 40) + 8), {}), ("II_EALIGN", dict(head_stride=1032), {}),
    ("II_EALIGN", dict(scale_token_stride=3, scale_head_stride=48), {}),
    ("II_EOVERFLOW", dict(page_stride=1 << 62), {}),
    ("II_EINVAL", dict(pages=0), dict(dtype=3)), ("II_EINVAL", dict(pages=0, dtype=6), {}),
    ("II_EINVAL", dict(pages=0), dict(tokens=-1)), ("II_EINVAL", dict(pages=0), dict(reserved=1)),
    ("II_EINVAL", dict(pages=0), dict(slots=0)), ("II_EALIGN", dict(pages=0), dict(slots=4)),
    ("II_EINVAL", dict(), {})])
def test_cache_refusals(name, change, more):
    cache = ops._CACHE.pack(*{**CACHE, **change}.values())
    tokens = ops._TOKENS.pack(*{**TOKENS, **more}.values())
    for call in (ops._call_write, ops._call_read):
        _refused(call(cache, tokens, 0), name)


@pytest.mark.parametrize("name,change", [
    ("II_EINVAL", dict(dtype=7)), ("II_EINVAL", dict(heads=5)), ("II_EINVAL", dict(heads=0)),
    ("II_EINVAL", dict(rows=-1)), ("II_EINVAL", dict(rows=3)), ("II_EINVAL", dict(seqs=-1)),
    ("II_EINVAL", dict(max_q=-1)), ("II_EINVAL", dict(max_len=-1)), ("II_EINVAL", dict(window=-1)),
    ("II_EINVAL", dict(columns=-1)), ("II_EINVAL", dict(pages_stride=-1)),
    ("II_EINVAL", dict(scale=float("nan"))), ("II_EINVAL", dict(scale=float("inf"))),
    ("II_EINVAL", dict(reserved=1)), ("II_EALIGN", dict(out_row_stride=257)),
    ("II_EALIGN", dict(out=(1 << 45) + 8)), ("II_EINVAL", dict(out_head_stride=56)),
    ("II_EINVAL", dict())])
def test_attend_refusals(name, change):
    cache = ops._CACHE.pack(*{**CACHE, "pages": 0}.values())
    args = ops._ATTEND.pack(*{**ATTEND, **change}.values())
    _refused(ops._call_attend(args, cache, 0), name)


def test_null_and_empty():
    import ctypes
    lib = ctypes.CDLL(ii.LIB_PATH)
    for name in ("ii_cache_write", "ii_cache_read", "ii_attend"):
        f = getattr(lib, name)
        f.argtypes = [ctypes.c_void_p] * 3
        assert f(None, None, None) == ii.EINVAL
    lib.ii_linear.argtypes = [ctypes.c_void_p] * 2
    assert lib.ii_linear(None, None) == ii.EINVAL
    # nothing to do touches no device
    assert ops._call_linear(ops._LINEAR.pack(*{**LINEAR, "m": 0}.values()), 0) == 0
    cache = ops._CACHE.pack(*{**CACHE, "pages": 0}.values())
    assert ops._call_write(cache, ops._TOKENS.pack(*{**TOKENS, "tokens": 0}.values()), 0) == 0
    assert ops._call_attend(ops._ATTEND.pack(*{**ATTEND, "rows": 0, "seqs": 0}.values()), cache, 0) == 0


def test_shapes_that_do_not_fit():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    x, w, out = z(4, 64), z(32, 64), z(4, 32)
    for call in (lambda: ops.ii_linear(out, x, z(32, 63)), lambda: ops.ii_linear(z(4, 31), x, w),
                 lambda: ops.ii_linear(out, x, w.float()), lambda: ops.ii_linear(out, x, w, w2=z(31, 64)),
                 lambda: ops.ii_linear(out, x, w, bias=z(31)), lambda: ops.ii_linear(out, x, w, residual=x),
                 lambda: ops.ii_linear(out, z(64, 4).t(), w),
                 lambda: ops.Cache(z(2, 1, 16, 64), z(2, 1, 16, 128)),
                 lambda: ops.Cache(z(2, 1, 16, 64), z(2, 1, 16, 64), *[z(2, 1, 16, 2, dt=torch.uint8)] * 2)):
        with pytest.raises(ValueError):
            call()
    cache = ops.Cache.empty(2, 1, 16, 64, torch.bfloat16, device="cpu")
    slots = torch.arange(3)
    q, table, n = z(1, 2, 64), z(1, 2, dt=torch.int32), z(1, dt=torch.int32)
    for call in (lambda: ops.ii_cache_write(cache, z(3, 2, 64), z(3, 2, 64), slots),
                 lambda: ops.ii_cache_write(cache, z(3, 1, 64), z(3, 1, 64), slots.int()),
                 lambda: ops.ii_cache_read(cache, slots[:2], z(3, 1, 64), z(3, 1, 64)),
                 lambda: ops.ii_attend(z(1, 2, 128), q, cache, table, n),
                 lambda: ops.ii_attend(z(1, 2, 64), q, cache, table.long(), n),
                 lambda: ops.ii_attend(z(1, 2, 64), q, cache, table, n, n)):
        with pytest.raises(ValueError):
            call()


def test_attend_refuses_more_rows_than_it_counts():
    cache = ops._CACHE.pack(*{**CACHE, "pages": 0}.values())
    args = {**ATTEND, "rows": (1 << 30) // ATTEND["heads"] + 1}
    assert ops._call_attend(ops._ATTEND.pack(*args.values()), cache, 0) == ii.EINVAL


def _places(at, width, *axes):
    """First bytes of the rows of an array: (count, stride in bytes) of its axes."""
    rows = [at]
    for count, stride in axes:
        rows = [r + i * stride for r in rows for i in range(count)]
    return [(r, r + width) for r in rows]


def _cache_arrays(c):
    """Byte ranges of the arrays of a cache (CACHE's fields)."""
    size = 1 if c["dtype"] == 3 else 2
    n = (c["pages"], c["heads"], c["page"])
    data = [(k, s * size) for k, s in zip(n, (c["page_stride"], c["head_stride"], c["token_stride"]))]
    out = [_places(c[x], c["dim"] * size, *data) for x in ("k", "v")]
    if size == 1:
        scale = list(zip(n, (c["scale_page_stride"], c["scale_head_stride"], c["scale_token_stride"])))
        out += [_places(c[x], c["dim"] // 32, *scale) for x in ("k_scale", "v_scale")]
    return out


def _meet(arrays):
    marked = set()
    for rows in arrays:
        mine = {b for first, end in rows for b in range(first, end)}
        if marked & mine:
            return True
        marked |= mine
    return False


def test_written_cache_arrays_are_apart():
    """Arrays of one buffer at random distances, in random orders of axes, against
    the bytes they hold: ii_cache_write refuses those that meet and no others;
    ii_cache_read, which writes none of them, refuses none."""
    import random
    rng = random.Random(5)
    tokens = ops._TOKENS.pack(*TOKENS.values())
    met = apart = 0
    for _ in range(1500):
        quant = rng.random() < 0.5
        n = [rng.choice([1, 1, 2, 3]), rng.choice([1, 2, 3]), rng.choice([1, 2, 4])]
        size = 1 if quant else 2
        order, strides, span = rng.sample(range(3), 3), [0, 0, 0], 64 * size
        scales, sspan = [0, 0, 0], 2
        for axis in order:      # the innermost first; room for a second array or not
            strides[axis] = span * rng.choice([1, 1, 2]) + 16 * rng.choice([0, 0, 1, 3])
            scales[axis] = sspan * rng.choice([1, 1, 2])
            span = strides[axis] * (n[axis] - 1) + span
            sspan = scales[axis] * (n[axis] - 1) + sspan
        if quant and rng.random() < 0.5:    # scales behind the codes of each page
            strides[0] = scales[0] = max(strides[0], -(-(span + 2 * sspan) // 16) * 16)
        base = 1 << 40
        c = {**CACHE, "dtype": 3 if quant else 5, "pages": n[0], "heads": n[1], "page": n[2], "k": base,
             "v": base + 16 * rng.randint(-span // 8, span // 8),
             "page_stride": strides[0] // size, "head_stride": strides[1] // size,
             "token_stride": strides[2] // size}
        if rng.random() < 0.4:
            c["v"] = base + rng.choice(strides) // 32 * 16
        if quant:
            c.update(scale_page_stride=scales[0], scale_head_stride=scales[1], scale_token_stride=scales[2],
                     k_scale=base + rng.choice([span, 1 << 20, rng.randint(0, span) & ~1]))
            c["v_scale"] = c["k_scale"] + rng.choice([sspan, 1 << 20, scales[1] // 4 * 2, 0])
        cache = ops._CACHE.pack(*c.values())
        write, read = (ii.ERRNAMES[f(cache, tokens, 0)] for f in (ops._call_write, ops._call_read))
        assert read == "II_EINVAL", (read, c)       # not memory of any device
        arrays = _cache_arrays(c)
        # what the strides do not tell apart may be refused: scales among codes
        if _meet(arrays):
            met += 1
            assert write == "II_EOVERLAP", c
        elif not (_meet([*arrays[:2]]) or quant and any(
                min(a)[0] < max(s)[1] and min(s)[0] < max(a)[1] for a in arrays[:2] for s in arrays[2:])):
            apart += 1
            assert write == "II_EINVAL", c
    assert met > 300 and apart > 300, (met, apart)


@pytest.mark.parametrize("layout", ["pages", "heads", "tokens", "positions"])
def test_keys_and_values_of_one_buffer(layout):
    """k and v side by side in every place of an axis are apart; one array twice is not."""
    p, h, t, d = 3, 2, 4, 64
    a = {"pages": (2 * h * t * d, t * d, d, h * t * d), "heads": (2 * h * t * d, 2 * t * d, d, t * d),
         "tokens": (2 * h * t * d, t * 2 * d, 2 * d, d), "positions": (2 * t * h * d, 2 * d, 2 * h * d, d)}[layout]
    c = {**CACHE, "dtype": 5, "pages": p, "heads": h, "page": t, "v": CACHE["k"] + 2 * a[3],
         "page_stride": a[0], "head_stride": a[1], "token_stride": a[2]}
    tokens = ops._TOKENS.pack(*TOKENS.values())
    for v, name in ((c["v"], "II_EINVAL"), (c["k"], "II_EOVERLAP"), (c["v"] - 16, "II_EOVERLAP"),
                    (c["k"] + 2 * a[1], "II_EOVERLAP"), (c["k"] + 2 * a[0], "II_EOVERLAP"),
                    (c["k"] + 2 * p * a[0], "II_EINVAL")):
        _refused(ops._call_write(ops._CACHE.pack(*{**c, "v": v}.values()), tokens, 0), name)


@pytest.mark.parametrize("stride", [1 << 62, (1 << 62) + 32, 3 << 61])
def test_strides_that_wrap(stride):
    """Strides whose bytes pass 64 bits, where the wrapped ones would do."""
    _refused(ops._call_linear(ops._LINEAR.pack(*{**LINEAR, "out_dtype": 7, "out_stride": stride}.values()), 0),
             "II_EOVERFLOW")
    cache = ops._CACHE.pack(*{**CACHE, "pages": 0}.values())
    _refused(ops._call_attend(ops._ATTEND.pack(*{**ATTEND, "pages_stride": stride}.values()), cache, 0),
             "II_EOVERFLOW")


def test_types_and_activations_that_are_not_known():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    x, w, out = z(4, 64), z(32, 64), z(4, 32)
    c64 = torch.complex64
    scale = z(2, 1, 16, 2, dt=torch.uint8)
    cache = ops.Cache(z(2, 1, 16, 64), z(2, 1, 16, 64))
    slots, table, n = torch.arange(3), z(1, 2, dt=torch.int32), z(1, dt=torch.int32)
    for call in (lambda: ops.ii_linear(out, x, w, act="tanh"),
                 lambda: ops.ii_linear(out, x.to(c64), w.to(c64)), lambda: ops.ii_linear(out.to(c64), x, w),
                 lambda: ops.Cache(z(2, 1, 16, 64, dt=c64), z(2, 1, 16, 64, dt=c64)),
                 lambda: ops.Cache(*[z(2, 1, 16, 64, dt=torch.float8_e4m3fn)] * 2, scale),
                 lambda: ops.ii_cache_write(cache, *[z(3, 1, 64, dt=c64)] * 2, slots),
                 lambda: ops.ii_attend(*[z(1, 2, 64, dt=c64)] * 2, cache, table, n)):
        with pytest.raises(ValueError):
            call()
