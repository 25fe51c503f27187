"""Cases of the operators between a decoder's products and its answer: norms at
the borders of blocks, rotary positions, the cache they are written to, low-rank
adapters beside a shared projection, log-probabilities of tokens.

A case's `op` says which:

  norm      ops.ii_norm: y = x, normalised if `post`; sum = scale * gate * y + residual;
            out = sum normalised
  rotate    ops.ii_rotate: heads turned by their token's position
  append    ops.ii_cache_append, then ops.ii_cache_read of the same tokens: queries
            and keys turned, keys and values put into pages, and taken out again
  logprobs  ops.ii_logprobs: log-probabilities of given tokens, entropy, the likeliest tokens
  adapt     ops.ii_adapt: out = base + scale_a B_a (A_a x), a the adapter of each row

`dtype` is the type of activations. `pad` widens the rows of the inputs by so
many elements (views of a fused buffer). `far` is the farthest position, `factor`
stretches the positions of a long context. The plain form computes in float32, or
in float64 where angles, sums and values next to a border of 8 bits ask for it,
and rounds once at the end.
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 32          # elements of the cache that share a scale
WORK_BYTES = 64 << 20
EPS = 1e-5

NORM = dict(op="norm", dtype="bf16", kind="rms", stream="same", post=False, gate="none",
            residual=True, bias=False, offset=0.0, scale=1.0, pad=0)
ROTATE = dict(op="rotate", dtype="bf16", dim=128, rot=128, layout="half", far=8192, factor=1.0, pad=0)
APPEND = dict(op="append", dtype="bf16", dim=128, rot=128, layout="half", far=8192, factor=1.0, pad=0,
              cache="fp8", page=64)
LOGPROBS = dict(op="logprobs", dtype="f32", top=0, targets=True, entropy=True, scale=1.0, masked=False,
                pad=0)
ADAPT = dict(op="adapt", dtype="bf16", out="same", base="same", rank=16, run=1, mixed=False, pad=0)

# the largest listed case of each kind bounds the drawn ones
MOST_NORM = 16384 * 8192            # elements of x
MOST_TURNED = 16384 * 40 * 128      # elements turned
MOST_LOGITS = 2047 * 128256
MOST_ADAPTED = 4099 * 8 * 64 * (4096 + 14336)   # products of the plain form: rows, adapters, rank, k + n


def listed():
    return [
        # one token of the tiny model before its feed-forward block: the smallest norm
        dict(NORM, name="norm-token-tiny", m=1, n=256),
        # long prompts of a 70B-shaped model whose blocks are normalised before and after, with a
        # gate for each element and a residual stream in 32 bits: the largest
        dict(NORM, name="norm-blocks", m=16384, n=8192, post=True, gate="each", stream="f32",
             offset=1.0, scale=0.5),
        # queries of a decoding batch of a 70B model, out of a fused q/k/v buffer
        dict(ROTATE, name="rotate-batch", tokens=256, heads=64, pad=2048, far=131072, factor=8.0),
        # a whole prompt, neighbouring pairs in half of each head, in f16
        dict(ROTATE, name="rotate-prompt", tokens=8191, heads=32, rot=64, layout="interleaved",
             dtype="f16"),
        # one token of the tiny model, cache in bf16
        dict(APPEND, name="append-token-tiny", tokens=1, heads=4, kv_heads=4, dim=64, rot=64, page=16,
             layout="interleaved", cache="same", far=512),
        # long prompts of an 8B model, stretched positions
        dict(APPEND, name="append-prompt", tokens=16384, heads=32, kv_heads=8, far=131072, factor=8.0),
        # the next token of one request to the tiny model with its likeliest alternatives
        dict(LOGPROBS, name="logprobs-token-tiny", rows=1, vocab=8192, top=5),
        # next tokens of a decoding batch of an 8B model, some of the vocabulary forbidden
        dict(LOGPROBS, name="logprobs-batch", rows=48, vocab=128256, top=20, scale=1.25, masked=True),
        # every token of a prompt of an 8B model, logits in bf16
        dict(LOGPROBS, name="logprobs-prompt", rows=2047, vocab=128256, dtype="bf16"),
        # a few decoding requests with adapters of their own beside an 8B model's output projection
        dict(ADAPT, name="adapt-token", m=4, k=4096, n=4096, adapters=4),
        # a decoding batch, some of its requests sharing adapters, beside the down projection
        dict(ADAPT, name="adapt-batch", m=250, k=14336, n=4096, adapters=32, mixed=True),
        # prompts of several requests beside the gate projection, kept in 32 bits until here
        dict(ADAPT, name="adapt-prompt", m=4099, k=4096, n=14336, adapters=8, rank=64, run=700,
             base="f32"),
    ]


def _log_uniform(rng, lo, hi):
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return x - 1 + x % 2 if x > 2048 else x  # the long ones are odd


def _stepped(rng, lo, hi, steps):
    step = rng.choice(steps)
    x = _log_uniform(rng, lo, hi)
    return step * (x // step - 1 + x // step % 2) if x >= step else step


def draw(rng):
    op = rng.choice(["norm", "rotate", "append", "logprobs", "adapt", "adapt"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    pad = rng.choice([0, 0, 8 * (2 * rng.randint(0, 255) + 1)])
    if op == "norm":
        c = dict(NORM, dtype=dtype, kind=rng.choice(["rms", "rms", "layer"]), pad=pad,
                 stream=rng.choice(["same", "same", "f32"]), post=rng.random() < 0.4,
                 gate=rng.choice(["none", "none", "row", "each"]), residual=rng.random() < 0.8,
                 bias=rng.random() < 0.3, offset=rng.choice([0.0, 0.0, 1.0]),
                 scale=rng.choice([1.0, 1.0, 0.25]))
        c["n"] = _stepped(rng, 64, 32768, [256, 64, 8, 1])
        c["m"] = _log_uniform(rng, 1, min(16384, MOST_NORM // c["n"]))
        return c
    if op in ("rotate", "append"):
        dim = rng.choice([64, 128, 128]) if op == "append" else rng.choice([64, 80, 96, 128, 128, 256])
        c = dict(ROTATE if op == "rotate" else APPEND, dtype=dtype, dim=dim, pad=pad,
                 rot=rng.choice([dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)]),
                 layout=rng.choice(["half", "half", "interleaved"]),
                 far=_log_uniform(rng, 512, 1048576), factor=rng.choice([1.0, 1.0, 8.0]))
        c["heads"] = rng.choice([1, 3, 4, 8, 16, 32, 32, 64])
        heads = c["heads"]
        if op == "append":
            c["kv_heads"] = rng.choice([h for h in (1, 2, 3, 4, 8, 16) if heads % h == 0])
            c["cache"] = rng.choice(["fp8", "fp8", "same"])
            c["page"] = rng.choice([16, 32, 64, 128, 256])
            heads += 2 * c["kv_heads"]
        c["tokens"] = _log_uniform(rng, 1, min(32768, MOST_TURNED // (heads * dim)))
        return c
    if op == "logprobs":
        c = dict(LOGPROBS, dtype=rng.choice(["f32", "f32", "bf16", "f16"]), pad=rng.choice([0, 0, 8, 3]),
                 top=rng.choice([0, 1, 5, 20, rng.randint(1, 64)]), entropy=rng.random() < 0.7,
                 scale=rng.choice([1.0, 1.0, 0.7, 1.25]), masked=rng.random() < 0.3)
        c["targets"] = rng.random() < 0.7 or not (c["top"] or c["entropy"])
        c["vocab"] = _stepped(rng, 256, 262144, [64, 8, 1])
        # the plain form sorts the rows whose likeliest tokens it wants
        most = MOST_LOGITS // (4 if c["top"] else 1)
        c["rows"] = _log_uniform(rng, 1, max(1, min(4096, most // c["vocab"])))
        return c
    c = dict(ADAPT, dtype=dtype, out=rng.choice(["same", "same", "f32"]), pad=pad,
             base=rng.choice(["none", "same", "same", "f32"]),
             rank=rng.choice([8, 16, 16, 32, 64, 128, rng.randint(1, 128)]), mixed=rng.random() < 0.4)
    c["k"] = _stepped(rng, 64, 16384, [256, 64, 8, 8, 1])
    c["n"] = _stepped(rng, 64, 32768, [256, 64, 8, 8, 1])
    c["adapters"] = _log_uniform(rng, 1, 64)
    most = MOST_ADAPTED // (c["adapters"] * c["rank"] * (c["k"] + c["n"]))
    c["m"] = _log_uniform(rng, 1, max(1, min(8192, most)))
    c["run"] = rng.choice([1, _log_uniform(rng, 1, 1024)])
    return c


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        m, n = case["m"], case["n"]
        stream = 4 if case["stream"] == "f32" else size
        moved = 2 * size + stream * (2 if case["residual"] else 1)
        moved += size if case["gate"] == "each" else 0
        vectors = (1 + case["post"]) * (1 + case["bias"]) + (case["gate"] == "row")
        return {"bytes": moved * m * n + vectors * n * size, "flops": (8 if case["post"] else 5) * m * n}
    if case["op"] in ("rotate", "append"):
        tokens, heads, dim = case["tokens"], case["heads"], case["dim"]
        moved = 2 * tokens * heads * dim * size + 8 * tokens
        turned = heads
        if case["op"] == "append":
            kept = 1 + 1 / BLOCK if case["cache"] == "fp8" else size
            moved += 2 * tokens * case["kv_heads"] * dim * (2 * size + 2 * kept) + 8 * tokens
            turned += case["kv_heads"]
        return {"bytes": int(moved), "flops": 3 * tokens * turned * case["rot"]}
    if case["op"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        moved = rows * vocab * size + rows * (12 * case["targets"] + 4 * case["entropy"] + 12 * case["top"])
        return {"bytes": moved, "flops": 5 * rows * vocab}
    m, n, k = case["m"], case["n"], case["k"]
    pairs = sum(r for _, r in _ranks_of_rows(case))
    used = {a: r for a, r in _ranks_of_rows(case) if a >= 0}
    base = {"none": 0, "same": size, "f32": 4}[case["base"]]
    moved = m * k * size + m * n * (base + (4 if case["out"] == "f32" else size)) + 4 * m
    moved += sum(used.values()) * (k + n) * size
    return {"bytes": moved, "flops": 2 * pairs * (k + n)}


# ---------------------------------------------------------------------------
# sizes of a batch with adapters: the case's alone, whatever the seed


def ranks(case):
    """The rank of each adapter: what `rank` leaves room for."""
    r, n = case["rank"], case["adapters"]
    return [max(1, r >> (i % 3)) for i in range(n)] if case["mixed"] else [r] * n


def owners(case):
    """The adapter of each row, in runs; the last of many runs has none."""
    m, n, run = case["m"], case["adapters"], case["run"]
    runs = -(-m // run)
    ids = list(range(min(runs, n)))
    ids += [int(n * math.modf(i * 0.6180339887)[0]) for i in range(len(ids), runs)]
    if runs > 4:
        ids[-1] = -1
    # requests of one adapter are not neighbours
    ids = [ids[i] for i in sorted(range(runs), key=lambda i: math.modf(i * 0.7548776662)[0])]
    return [a for a in ids for _ in range(run)][:m]


def _ranks_of_rows(case):
    r = ranks(case)
    return [(a, r[a] if a >= 0 else 0) for a in owners(case)]


# ---------------------------------------------------------------------------
# inputs


def _normal(g, *shape, dtype, std=1.0, pad=0):
    """Normal values whose rows lie `pad` elements further apart than they are long."""
    row = shape[-1] if len(shape) == 2 else shape[-2] * shape[-1]
    wide = torch.empty(shape[0], row + pad, dtype=dtype, device="cuda")
    wide.normal_(0.0, std, generator=g)
    return wide[:, :row].unflatten(1, shape[1:]) if len(shape) > 2 else wide[:, :row]


def _freqs(case):
    """Radians a position of each pair; with a factor, pairs that turn less than
    once over the 8192 positions known before turn that many times slower, pairs
    that turn four times keep their pace."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64)
    f = 500000.0 ** (-2 * i / case["rot"])
    if case["factor"] != 1:
        keep = ((8192 * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
        f = f * keep + f / case["factor"] * (1 - keep)
    return f.cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]
    s = dict(case=case)
    if case["op"] == "norm":
        m, n, pad = case["m"], case["n"], case["pad"]
        stream = TYPES[case["stream"]] if case["stream"] != "same" else dt
        vector = lambda mean: (_normal(g, 1, n, dtype=torch.float32, std=0.1)[0] + mean).to(dt)  # noqa: E731
        s["x"] = _normal(g, m, n, dtype=dt, pad=pad)
        s["weight"] = vector(1 - case["offset"])
        s["bias"] = vector(0.0) if case["bias"] else None
        s["post_weight"] = vector(1 - case["offset"]) if case["post"] else None
        s["post_bias"] = vector(0.0) if case["post"] and case["bias"] else None
        s["gate"] = {"none": lambda: None, "row": lambda: vector(0.5).expand(m, n),
                     "each": lambda: _normal(g, m, n, dtype=dt, pad=pad)}[case["gate"]]()
        s["residual"] = _normal(g, m, n, dtype=stream, std=3.0, pad=pad) if case["residual"] else None
        s["sum"] = torch.empty(m, n, dtype=stream, device="cuda")
        s["out"] = torch.empty(m, n, dtype=dt, device="cuda")
        return s
    if case["op"] in ("rotate", "append"):
        t, h, d, pad = case["tokens"], case["heads"], case["dim"], case["pad"]
        far = case["far"]
        # prompts one after another, or any position for the tokens of a batch
        start = torch.randint(0, max(1, far - t), (1,), generator=g, device="cuda")
        at = start + torch.arange(t, device="cuda")
        any_at = torch.randint(0, far, (t,), generator=g, device="cuda")
        s["positions"] = (at % far if t > 1024 else any_at).contiguous()
        s["freqs"] = _freqs(case)
        s["q"] = _normal(g, t, h, d, dtype=dt, pad=pad)
        s["q_out"] = torch.empty(t, h, d, dtype=dt, device="cuda")
        if case["op"] == "rotate":
            return s
        hk, page, fp8 = case["kv_heads"], case["page"], case["cache"] == "fp8"
        pages = -(-t // page) + 1
        order = torch.randperm(pages, generator=g, device="cuda")
        rows = torch.randperm(pages * page, generator=g, device="cuda")
        runs = (order[:, None] * page + torch.arange(page, device="cuda")).flatten()
        s["slots"] = (runs if t > 1024 else rows)[:t].contiguous()
        s["k"] = _normal(g, t, hk, d, dtype=dt, pad=pad)
        s["v"] = _normal(g, t, hk, d, dtype=dt, pad=pad)
        s["k_back"] = torch.empty(t, hk, d, dtype=dt, device="cuda")
        s["v_back"] = torch.empty(t, hk, d, dtype=dt, device="cuda")
        s["cache"] = [torch.zeros(pages, hk, page, d, dtype=F8 if fp8 else dt, device="cuda") for _ in "kv"]
        if fp8:
            s["cache"] += [torch.zeros(pages, hk, page, d // BLOCK, dtype=torch.uint8, device="cuda")
                           for _ in "kv"]
        return s
    s["work"] = torch.zeros(WORK_BYTES, dtype=torch.uint8, device="cuda")
    if case["op"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        s["logits"] = _normal(g, rows, vocab, dtype=dt, std=3.0, pad=case["pad"])
        if case["masked"]:
            hidden = torch.rand(vocab, generator=g, device="cuda") < 0.4
            s["logits"].masked_fill_(hidden, -math.inf)
        f32 = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
        s["targets"] = s["logprob"] = s["entropy"] = s["top_ids"] = s["top_logprobs"] = None
        if case["targets"]:
            s["targets"] = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
            s["logprob"] = f32(rows)
        if case["entropy"]:
            s["entropy"] = f32(rows)
        if case["top"]:
            s["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int64, device="cuda")
            s["top_logprobs"] = f32(rows, case["top"])
        return s
    m, n, k, r, count = (case[x] for x in ("m", "n", "k", "rank", "adapters"))
    types = {"none": None, "same": dt, "f32": torch.float32}
    s["x"] = _normal(g, m, k, dtype=dt, pad=case["pad"])
    s["a"] = torch.empty(count, r, k, dtype=dt, device="cuda").normal_(0, k ** -0.5, generator=g)
    s["b"] = torch.empty(count, n, r, dtype=dt, device="cuda").normal_(0, r ** -0.5, generator=g)
    s["scales"] = torch.rand(count, generator=g, device="cuda") + 0.5
    s["adapters"] = torch.tensor(owners(case), dtype=torch.int32, device="cuda")
    s["ranks"] = torch.tensor(ranks(case), dtype=torch.int32, device="cuda") if case["mixed"] else None
    s["base"] = None if case["base"] == "none" else _normal(g, m, n, dtype=types[case["base"]],
                                                            pad=case["pad"])
    s["out"] = torch.empty(m, n, dtype=types[case["out"]], device="cuda")
    return s


# ---------------------------------------------------------------------------
# plain forms


def _normalised(y, weight, bias, case):
    if case["kind"] == "layer":
        y = y - y.mean(-1, keepdim=True)
    y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * (weight.float() + case["offset"])
    return y if bias is None else y + bias.float()


def _plain_norm(s):
    case = s["case"]
    y = s["x"].float()
    if case["post"]:
        y = _normalised(y, s["post_weight"], s["post_bias"], case)
    if s["gate"] is not None:
        y = y * s["gate"].float()
    y = y * case["scale"]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["sum"].dtype), _normalised(y, s["weight"], s["bias"], case).to(s["x"].dtype)


def _turn(x, s):
    """x turned, in 64 bits."""
    case = s["case"]
    rot = case["rot"]
    angle = s["positions"].double()[:, None, None] * s["freqs"]
    cos, sin = torch.cos(angle), torch.sin(angle)
    y = x.double()
    head, rest = y[..., :rot], y[..., rot:]
    if case["layout"] == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, rest), -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), rest), -1)


def _two_to(e):
    """2^e exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x, f16):
    """Codes and scale exponents of the last axis of float64 values: in each block
    of 32 the scale is the least power of two that brings the largest value to 448."""
    y = x.unflatten(-1, (-1, BLOCK))
    part, e = torch.frexp(y.abs().amax(-1))                   # in [0.5, 1) times 2^e; 448 = 0.875 * 2^9
    e = (e - 9 + (part > 0.875)).clamp(-126, 120)
    y = y * _two_to(-e[..., None])
    # eight steps in each power of two, of 2^-9 below 2^-6
    _, at = torch.frexp(y)
    step = _two_to((at - 1).clamp(min=-6) - 3)
    y = torch.round(y / step) * step
    if f16:     # what is read back has to fit the type
        most = torch.where(e == 8, 240.0, 448.0)[..., None]
        y = torch.minimum(torch.maximum(y, -most), most)
    return y.flatten(-2).float().to(F8), (e + 127).to(torch.uint8)


def _plain_append(s):
    case, dt = s["case"], s["k"].dtype
    page, row = s["slots"] // case["page"], s["slots"] % case["page"]
    q, k, v = _turn(s["q"], s).to(dt), _turn(s["k"], s), s["v"]
    back = []
    for i, x in enumerate((k, v)):
        codes = s["cache"][i]
        if case["cache"] == "same":
            codes[page, :, row] = x.to(dt)
            back.append(codes[page, :, row].clone())
            continue
        raw, scales = codes.view(torch.uint8), s["cache"][2 + i]
        y, e = _quantise(x.double(), dt == torch.float16)
        raw[page, :, row], scales[page, :, row] = y.view(torch.uint8), e
        y = raw[page, :, row].view(F8).float().unflatten(-1, (-1, BLOCK))
        scale = (scales[page, :, row].to(torch.int32) << 23).view(torch.float32)
        back.append((y * scale[..., None]).flatten(-2).to(dt))
    return q, *back


def _plain_logprobs(s):
    case = s["case"]
    x = s["logits"].float()
    z = x * case["scale"]
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    log = torch.log(total)
    out = {}
    if s["targets"] is not None:
        out["logprob"] = ((z - top).gather(1, s["targets"][:, None]).double() - log)[:, 0].float()
    if s["entropy"] is not None:
        below = torch.where(e > 0, e * (z - top), 0.0).sum(-1, keepdim=True, dtype=torch.float64)
        out["entropy"] = (log - below / total)[:, 0].float()
    if case["top"]:
        # equal logits in the order of their tokens
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :case["top"]]
        out["top_ids"] = order
        out["top_logprobs"] = ((z - top).gather(1, order).double() - log).float()
    return out


def _plain_adapt(s):
    case = s["case"]
    count, r = case["adapters"], case["rank"]
    mine = s["adapters"][:, None] == torch.arange(count, device="cuda")              # m adapters
    held = torch.full((count,), r, device="cuda") if s["ranks"] is None else s["ranks"]
    mine = mine[..., None] & (torch.arange(r, device="cuda") < held[:, None])        # m adapters r
    h = (s["x"].float() @ s["a"].float().flatten(0, 1).t()).unflatten(1, (count, r))
    h = torch.where(mine, h * s["scales"][:, None], 0.0)
    y = h.flatten(1) @ s["b"].float().transpose(1, 2).reshape(count * r, -1)
    if s["base"] is not None:
        y = y + s["base"].float()
    return y.to(s["out"].dtype)


def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "rotate":
            return _turn(s["q"], s).to(s["q"].dtype)
        return {"norm": _plain_norm, "append": _plain_append, "logprobs": _plain_logprobs,
                "adapt": _plain_adapt}[case["op"]](s)
    from paper_2607_18957_amd import ops
    stream = torch.cuda.current_stream()
    if case["op"] == "norm":
        ops.ii_norm(s["out"], s["x"], s["weight"], bias=s["bias"], post=case["post"],
                    post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"],
                    residual=s["residual"], sum=s["sum"], scale=case["scale"], kind=case["kind"],
                    eps=EPS, offset=case["offset"], stream=stream)
        return s["sum"], s["out"]
    if case["op"] == "rotate":
        ops.ii_rotate(s["q_out"], s["q"], s["positions"], s["freqs"], layout=case["layout"], stream=stream)
        return s["q_out"]
    if case["op"] == "append":
        cache = ops.Cache(*s["cache"])
        ops.ii_cache_append(cache, s["k"], s["v"], s["slots"], s["positions"], s["freqs"], q=s["q"],
                            q_out=s["q_out"], layout=case["layout"], stream=stream)
        ops.ii_cache_read(cache, s["slots"], s["k_back"], s["v_back"], stream=stream)
        return s["q_out"], s["k_back"], s["v_back"]
    if case["op"] == "logprobs":
        names = ("logprob", "entropy", "top_ids", "top_logprobs")
        ops.ii_logprobs(s["logits"], targets=s["targets"], **{x: s[x] for x in names}, scale=case["scale"],
                        work=s["work"], stream=stream)
        return {x: s[x] for x in names if s[x] is not None}
    ops.ii_adapt(s["out"], s["x"], s["a"], s["b"], s["adapters"], scales=s["scales"], ranks=s["ranks"],
                 base=s["base"], work=s["work"], stream=stream)
    return s["out"]


# ---------------------------------------------------------------------------
# the definitions in 64 bits


def _exact_norm(s):
    case = s["case"]
    d = lambda t: None if t is None else t.double()  # noqa: E731

    def norm(y, w, b):
        var, mean = torch.var_mean(y, -1, correction=0, keepdim=True)
        if case["kind"] == "rms":
            var, mean = var + mean ** 2, 0.0
        y = torch.addcmul(torch.zeros_like(w) if b is None else b, (y - mean) * torch.rsqrt(var + EPS),
                          w + case["offset"])
        return y

    sums, outs = [], []
    step = max(1, (1 << 27) // case["n"])
    for i in range(0, case["m"], step):
        rows = {k: d(s[k][i:i + step]) if s[k] is not None else None for k in ("x", "gate", "residual")}
        y = rows["x"]
        if case["post"]:
            y = norm(y, d(s["post_weight"]), d(s["post_bias"]))
        y = y * case["scale"] * (1.0 if rows["gate"] is None else rows["gate"])
        y = y if rows["residual"] is None else y + rows["residual"]
        sums.append(y)
        outs.append(norm(y, d(s["weight"]), d(s["bias"])))
    return torch.cat(sums), torch.cat(outs)


def _exact_turn(x, s):
    case = s["case"]
    half = case["rot"] // 2
    angle = torch.outer(s["positions"].double(), s["freqs"])
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.double().clone()
    if case["layout"] == "half":
        z = torch.complex(y[..., :half], y[..., half:2 * half]) * turn
        y[..., :half], y[..., half:2 * half] = z.real, z.imag
    else:
        pairs = y[..., :2 * half].unflatten(-1, (half, 2)).contiguous()
        y[..., :2 * half] = torch.view_as_real(torch.view_as_complex(pairs) * turn).flatten(-2)
    return y


def _kept(y, case):
    """Float64 values as the cache holds them."""
    if case["cache"] == "same":
        return y
    z = y.unflatten(-1, (-1, BLOCK))
    # the least power of two: up from one that is too small
    top = z.abs().amax(-1, keepdim=True)
    scale = _two_to(torch.floor(torch.log2(top.clamp(min=2.0 ** -110) / 448)).long() - 1)
    for _ in range(3):
        scale = torch.where(top > 448 * scale, 2 * scale, scale)
    z = z / scale
    exponent = (z.view(torch.int64) >> 52 & 2047) - 1023
    unit = _two_to(exponent.clamp(min=-6) - 3)
    z = torch.round(z / unit) * unit * scale
    if case["dtype"] == "f16":  # 61440 is the largest such value that fits
        z = z.clamp(-61440, 61440)
    return z.flatten(-2)


def _exact_logprobs(s):
    case = s["case"]
    parts = []
    step = max(1, (1 << 26) // case["vocab"])
    for i in range(0, case["rows"], step):
        x = s["logits"][i:i + step].double()
        logp = torch.log_softmax(x * case["scale"], -1)
        part = {}
        if s["targets"] is not None:
            at = s["targets"][i:i + step]
            part["logprob"] = logp[torch.arange(len(at), device="cuda"), at]
        if s["entropy"] is not None:
            part["entropy"] = torch.special.entr(torch.exp(logp)).sum(-1)
        if case["top"]:
            part["top_ids"] = torch.argsort(-x, dim=-1, stable=True)[:, :case["top"]].contiguous()
            part["top_logprobs"] = torch.take_along_dim(logp, part["top_ids"], 1)
        parts.append(part)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_adapt(s):
    case = s["case"]
    shape = (case["m"], case["n"])
    out = torch.zeros(shape, dtype=torch.float64, device="cuda") if s["base"] is None else s["base"].double()
    owner = owners(case)
    for a, r in enumerate(ranks(case)):
        rows = [i for i, x in enumerate(owner) if x == a]
        if rows:
            rows = torch.tensor(rows, device="cuda")
            h = torch.nn.functional.linear(s["x"][rows].double(), s["a"][a, :r].double())
            y = torch.nn.functional.linear(h, s["b"][a, :, :r].double())
            out[rows] += s["scales"][a].double() * y
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "rotate":
        return _exact_turn(s["q"], s)
    if case["op"] == "append":
        return _exact_turn(s["q"], s), _kept(_exact_turn(s["k"], s), case), _kept(s["v"].double(), case)
    if case["op"] == "logprobs":
        return _exact_logprobs(s)
    return _exact_adapt(s)
