"""A decoder's step from its residual stream to log-probabilities, all of it the
operators, one after another: each against its definition on what it was given,
on a stream of its own, then captured and replayed with new inputs between eager
work."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_18957_amd import ops  # noqa: E402  (fails loudly if libii.so is missing)

import decoder_ref as ref  # noqa: E402
import ops_ref  # noqa: E402

DEV = torch.device("cuda:0")
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def _close(got, want, bound, what):
    bad = ~(((got.double() - want).abs() <= bound) | (got.double() == want))
    assert not bad.any(), (what, int(bad.sum()), bad.numel())


class Step:
    """New tokens of `counts` each after `held` ones, through one block and the head."""

    def __init__(self, held, counts, work, hidden=256, heads=8, kv_heads=2, dim=64, vocab=5000, page=16, rank=16,
                 adapters=3, kept=F8):
        g = self.g = torch.Generator(device=DEV).manual_seed(1)
        t, self.work = sum(counts), work
        normal = lambda *s, std=1.0: torch.empty(*s, device=DEV).normal_(0, std, generator=g).to(BF16)  # noqa: E731
        empty = lambda *s, dt=BF16: torch.zeros(*s, dtype=dt, device=DEV)  # noqa: E731
        width = (heads + 2 * kv_heads) * dim
        self.heads, self.kv_heads, self.dim, self.counts, self.held = heads, kv_heads, dim, counts, held
        self.w = {k: normal(n, m, std=m ** -0.5) for k, (n, m) in dict(
            qkv=(width, hidden), o=(hidden, heads * dim), head=(vocab, hidden)).items()}
        self.norms = {k: (normal(hidden, std=0.1) + 1).to(BF16) for k in ("attn", "post", "ffn")}
        self.a, self.b = normal(adapters, rank, hidden, std=hidden ** -0.5), normal(adapters, width, rank, std=0.25)
        self.ids = torch.randint(-1, adapters, (t,), generator=g, device=DEV).int()
        lengths = [h + c for h, c in zip(held, counts)]
        columns = -(-max(lengths) // page)
        self.cache = ops.Cache.empty(len(counts) * columns, kv_heads, page, dim, kept)
        self.table = torch.randperm(len(counts) * columns, generator=g, device=DEV).int().view(len(counts), columns)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        starts = [sum(counts[:i]) for i in range(len(counts) + 1)]
        self.starts = torch.tensor(starts, dtype=torch.int32, device=DEV)
        seq = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)).to(DEV)
        self.at = torch.cat([torch.arange(h, h + c) for h, c in zip(held, counts)]).to(DEV)
        self.slots = self.table[seq, self.at // page].long() * page + self.at % page
        self.freqs = ops.ii_rotary_freqs(dim)
        if sum(held):      # what came before
            slots = torch.cat([self.table[i, torch.arange(h, device=DEV) // page].long() * page
                               + torch.arange(h, device=DEV) % page for i, h in enumerate(held)])
            ops.ii_cache_write(self.cache, *(normal(sum(held), kv_heads, dim) for _ in "kv"), slots)
        self.block, self.stream = normal(t, hidden), empty(t, hidden, dt=F32)
        self.targets = torch.randint(0, vocab, (t,), generator=g, device=DEV)
        self.h, self.plain, self.fused = empty(t, hidden), empty(t, width, dt=F32), empty(t, width)
        self.mixed, self.y, self.total, self.z = empty(t, heads, dim), empty(t, hidden), empty(t, hidden, dt=F32), empty(t, hidden)
        self.logits, self.logprob, self.entropy = empty(t, vocab, dt=F32), empty(t, dt=F32), empty(t, dt=F32)
        self.ids_top, self.top = empty(t, 7, dt=torch.int64), empty(t, 7, dt=F32)

    def parts(self):
        q, k = self.heads * self.dim, self.kv_heads * self.dim
        cut = self.fused[:, :q], self.fused[:, q:q + k], self.fused[:, q + k:]
        return [x.unflatten(1, (-1, self.dim)) for x in cut]

    def run(self, stream):
        q, k, v = self.parts()
        kw = dict(stream=stream)
        ops.ii_norm(self.h, self.block, self.norms["attn"], residual=self.stream, sum=self.stream, **kw)
        ops.ii_linear(self.plain, self.h, self.w["qkv"], work=self.work, **kw)
        ops.ii_adapt(self.fused, self.h, self.a, self.b, self.ids, base=self.plain, work=self.work, **kw)
        ops.ii_cache_append(self.cache, k, v, self.slots, self.at, self.freqs, q=q, q_out=q, **kw)
        ops.ii_attend(self.mixed, q, self.cache, self.table, self.lengths, self.starts, max_q=max(self.counts),
                      work=self.work, **kw)
        ops.ii_linear(self.y, self.mixed.flatten(1), self.w["o"], work=self.work, **kw)
        ops.ii_norm(self.z, self.y, self.norms["ffn"], post=True, post_weight=self.norms["post"],
                    residual=self.stream, sum=self.total, scale=0.5, **kw)
        ops.ii_linear(self.logits, self.z, self.w["head"], work=self.work, **kw)
        ops.ii_logprobs(self.logits, targets=self.targets, logprob=self.logprob, entropy=self.entropy,
                        top_ids=self.ids_top, top_logprobs=self.top, work=self.work, **kw)

    def check(self, before):
        """What came out of a run that began with the stream `before`."""
        (total, far), (h, h_far) = ref.norm(self.block, self.norms["attn"], residual=before, stream=F32)
        _close(self.stream, total, far, "stream")
        _close(self.h, h, h_far, "h")
        _close(self.plain, *ops_ref.linear(self.h, self.w["qkv"], F32), "qkv")
        # q was turned in place: the adapted rows again, apart
        fused = torch.empty_like(self.fused)
        ops.ii_adapt(fused, self.h, self.a, self.b, self.ids, base=self.plain)
        _close(fused, *ref.adapt(self.h, self.a, self.b, self.ids, None, None, self.plain, BF16), "adapted")
        q, k, v = self.parts()
        width = self.heads * self.dim
        turned = ref.turn(fused[:, :width].unflatten(1, (-1, self.dim)), self.at, self.freqs)
        _close(q, turned, ref.rounded(turned, BF16) + turned.abs() * ref.U[BF16], "q")  # h in another split
        back = [torch.empty(k.shape, dtype=BF16, device=DEV) for _ in "kv"]
        ops.ii_cache_read(self.cache, self.slots, *back)
        assert torch.equal(back[0].double(), ref.kept(ref.turn(k, self.at, self.freqs))[0])
        assert torch.equal(back[1].double(), ref.kept(v.double())[0])
        want, far, _ = ops_ref.attend(q, self.cache, self.table.tolist(), self.lengths.tolist(), self.starts.tolist())
        _close(self.mixed, want, far, "attention")
        (total, far), (z, z_far) = ref.norm(self.y, self.norms["ffn"], post=True, post_weight=self.norms["post"],
                                            residual=self.stream, scale=0.5, stream=F32)
        _close(self.total, total, far, "total")
        _close(self.z, z, z_far, "z")
        _close(self.logits, *ops_ref.linear(self.z, self.w["head"], F32), "logits")
        logp, off, entropy, far = ref.logprobs(self.logits)
        at = self.targets[:, None]
        _close(self.logprob, logp.gather(1, at)[:, 0], off.gather(1, at)[:, 0], "logprob")
        _close(self.entropy, entropy, far, "entropy")
        order = torch.sort(self.logits, dim=1, descending=True, stable=True).indices[:, :7]
        assert torch.equal(self.ids_top, order)
        _close(self.top, logp.gather(1, order), off.gather(1, order), "top")


@pytest.mark.parametrize("held,counts", [([0, 0, 0], [5, 37, 130]), ([300, 5, 90], [1, 1, 1]), ([40, 0, 700], [1, 60, 3])])
def test_step(held, counts):
    s = Step(held, counts, ops.work_buffer())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        before = s.stream.clone()
        s.run(side)
    side.synchronize()
    s.check(before)


def test_captured_steps():
    """Two graphs share their scratch; each replay is that of the inputs it finds."""
    work = ops.work_buffer()
    steps = [Step([300, 5, 90], [1, 1, 1], work), Step([0, 33], [70, 1], work)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for s in steps:
        with torch.cuda.stream(side):
            s.run(side)
        side.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            s.run(torch.cuda.current_stream())
    for i in range(3):
        for s, graph in zip(steps, graphs):
            s.block.normal_(generator=s.g)
            s.stream.normal_(generator=s.g)
            s.ids.copy_(s.ids.roll(1))
            s.targets.copy_(s.targets.roll(1))
            s.fused.zero_()
            before = s.stream.clone()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            s.check(before)
    assert not work[:65536].any()


def test_calls_on_two_streams():
    """Two steps at once, each with scratch of its own."""
    steps = [Step([300, 5, 90], [1, 1, 1], ops.work_buffer()), Step([0, 33], [70, 1], ops.work_buffer())]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(3):
        before = [s.stream.clone() for s in steps]
        torch.cuda.synchronize()
        for s, side in zip(steps, streams):
            with torch.cuda.stream(side):
                s.run(side)
        torch.cuda.synchronize()
        for s, b in zip(steps, before):
            s.check(b)
