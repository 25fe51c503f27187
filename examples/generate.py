"""Load a model's weights with one plan and answer prompts from where they lie.

    python examples/generate.py [--model tiny|llama8b] [--tokens 8] [--cache fp8|bf16]

The weights of a decoder-only transformer (synth's tables, filled with seeded
normal values) are loaded by ii_load into one arena; every matrix is then used
there, in place, by the operators of paper_2607_18957_amd.ops: ii_linear for
all products (with the gate, the activation and the residual stream in their
epilogues), ii_cache_write for new keys and values, ii_attend for prompts of
different lengths at once, then for single tokens.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2607_18957_amd import ii, ops, synth


def normal_blob(table, seed: int = 0) -> np.ndarray:
    """A blob of the table's layout: norms of ones, other weights normal."""
    blob = np.zeros(table.blob_bytes, dtype=np.uint8)
    g = torch.Generator().manual_seed(seed)
    for name, shape, at in zip(table.names, table.shapes, table.src_offset):
        w = torch.ones(shape) if len(shape) == 1 else torch.empty(shape).normal_(
            0, 1.0 if name == "embed" else shape[1] ** -0.5, generator=g)
        raw = w.to(torch.bfloat16).view(torch.uint8).flatten().numpy()
        blob[int(at):int(at) + raw.size] = raw
    return blob


def load(table, blob):
    """(plan, arena, name -> weight): one load, views of its arena."""
    plan = ii.ii_plan(table)
    arena = torch.empty(plan.arena_bytes, dtype=torch.uint8, device="cuda")
    _, off = plan.tensors()
    ii.ii_load(plan, blob, arena.data_ptr() + off, torch.cuda.current_stream())
    return plan, arena, ii.arena_views(plan, table, arena)


class Model:
    """A decoder over loaded weights, with a paged cache for `seqs` sequences
    of up to `max_len` tokens."""

    def __init__(self, weights, meta, dim: int, seqs: int, max_len: int, page: int = 64,
                 cache_dtype=torch.float8_e4m3fn):
        self.w, self.layers, self.dim = weights, meta["layers"], dim
        self.heads, self.kv_heads = meta["hidden"] // dim, meta["kv"] // dim
        self.page, self.max_len, columns = page, max_len, -(-max_len // page)
        self.caches = [ops.Cache.empty(seqs * columns, self.kv_heads, page, dim, cache_dtype)
                       for _ in range(self.layers)]
        # any order of pages will do
        self.pages = torch.randperm(seqs * columns, device="cuda").to(torch.int32).view(seqs, columns)
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.held = [0] * seqs      # the same on the host, to refuse what does not fit
        self.work = ops.work_buffer()
        angle = torch.arange(max_len, device="cuda")[:, None] * 10000.0 ** (
            -torch.arange(0, dim, 2, device="cuda") / dim)
        self.turn = torch.polar(torch.ones_like(angle), angle)

    def linear(self, x, name, n, **kw):
        out = torch.empty(x.shape[0], n, dtype=kw.pop("out", x.dtype), device="cuda")
        ops.ii_linear(out, x, self.w[name], work=self.work, stream=torch.cuda.current_stream(), **kw)
        return out

    def norm(self, x, name):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5) * self.w[name]).to(x.dtype)

    def rotate(self, x, at):
        y = torch.view_as_complex(x.float().unflatten(-1, (-1, 2)).contiguous())
        return torch.view_as_real(y * self.turn[at, None]).flatten(-2).to(x.dtype)

    def step(self, tokens, counts):
        """Logits of each sequence's last token after `counts` more tokens of
        each (a list of 1 or more), given one after another."""
        held = [a + b for a, b in zip(self.held, counts)]
        if len(counts) != len(self.held) or min(counts) < 1 or max(held) > self.max_len \
                or sum(counts) != len(tokens):
            raise ValueError(f"{counts} more tokens ({len(tokens)} given) after {self.held}, of up to "
                             f"{self.max_len} each")
        self.held = held
        stream = torch.cuda.current_stream()
        n = torch.tensor(counts, device="cuda")
        start = torch.zeros(len(counts) + 1, dtype=torch.int32, device="cuda")
        start[1:] = n.cumsum(0)
        seq = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), n)
        at = torch.arange(len(tokens), device="cuda") - start[seq] + self.lengths[seq]
        slots = self.pages[seq, at // self.page].long() * self.page + at % self.page
        self.lengths += n.to(torch.int32)
        hidden = self.heads * self.dim
        x = self.w["embed"][tokens]
        for i, cache in enumerate(self.caches):
            p = f"layers.{i}."
            h = self.norm(x, p + "attn_norm")
            q, k, v = (self.linear(h, p + m, c * self.dim).unflatten(1, (c, self.dim)) for m, c in
                       (("q", self.heads), ("k", self.kv_heads), ("v", self.kv_heads)))
            q, k = self.rotate(q, at), self.rotate(k, at)
            ops.ii_cache_write(cache, k, v, slots, stream=stream)
            out = torch.empty_like(q)
            ops.ii_attend(out, q, cache, self.pages, self.lengths, start, max_q=max(counts),
                          max_len=self.max_len, work=self.work, stream=stream)
            x = self.linear(out.flatten(1), p + "o", hidden, residual=x)
            h = self.norm(x, p + "ffn_norm")
            h = self.linear(h, p + "gate", self.w[p + "up"].shape[0], w2=self.w[p + "up"], act="silu")
            x = self.linear(h, p + "down", hidden, residual=x)
        last = self.norm(x[start[1:].long() - 1], "final_norm")
        return self.linear(last, "lm_head", self.w["lm_head"].shape[0], out=torch.float32)


def main() -> None:
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--model", choices=["tiny", "llama8b"], default="tiny")
    a.add_argument("--tokens", type=int, default=8)
    a.add_argument("--cache", choices=["fp8", "bf16"], default="fp8")
    a = a.parse_args()
    if a.tokens < 1:
        raise SystemExit("--tokens has to be 1 or more")
    table = getattr(synth, a.model)()
    plan, _arena, weights = load(table, normal_blob(table))
    prompts = [[(7 * i + j) % table.meta["vocab"] for j in range(n)] for i, n in enumerate((5, 37, 300))]
    model = Model(weights, table.meta, 64 if a.model == "tiny" else 128, len(prompts), 300 + a.tokens,
                  cache_dtype=torch.float8_e4m3fn if a.cache == "fp8" else torch.bfloat16)
    logits = model.step(torch.tensor(sum(prompts, []), device="cuda"), [len(p) for p in prompts])
    answers = []
    for _ in range(a.tokens):
        torch.cuda.synchronize()
        t = time.perf_counter()
        answers.append(logits.argmax(-1))
        logits = model.step(answers[-1], [1] * len(prompts))
        torch.cuda.synchronize()
    print(f"{a.model}: last step {1e3 * (time.perf_counter() - t):.2f} ms")
    for p, row in zip(prompts, torch.stack(answers, 1).tolist()):
        print(f"prompt of {len(p)}: {row}")
    plan.free()


if __name__ == "__main__":
    main()
