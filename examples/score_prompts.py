#!/usr/bin/env python3
"""Scores prompts: the log probability of each of their tokens, with the model's uncertainty and its own choices, in chunks that are packed.

Prompts of different lengths are worked on at once, so many tokens a pass: each pass takes the next tokens of the prompts that are not done, one prompt behind the other, and
runs them through the decoder's layers.  Per layer: the stacked q/k/v projection (`mpgemm_f32`, ternary weights), norms and rotation of the heads with
the new keys and values put into their pages (`append_kv`), attention of the chunks over each prompt's pages (`chunk_attention`), the
output projection, its residual with the norm before the feed-forward block (`residual_norm`), the stacked gate|up projection, their product
and its norm (`gated_norm`), the down projection, and its residual with the next layer's norm (`residual_norm`).  Behind the last layer the
logits (a library product) and what is wanted of them (`token_logprobs`).

    python examples/score_prompts.py --prompts 6 --longest 3000 --budget 2048

Synthetic weights of 2.4B-style layers (2560 features, 20 query heads and 5 key heads of 128, 6912 features inside) and synthetic tokens.
Prints one line: passes, time and tokens per second.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch  # noqa: E402
from shared_prefix_decode import Pages, rotation  # noqa: E402

from paper_2512_06443_amd import binding as vlut  # noqa: E402


class Linear:
    """Ternary weights int8 [rows][features] and their scale."""

    def __init__(self, rows: int, features: int, seed: int):
        from paper_2512_06443_amd import workloads as wl
        self.rows, self.scale = rows, features ** -0.5
        self.packed = vlut.pack_weights(torch.from_numpy(wl.ternary(seed, rows, features, 0.4)).cuda())

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        return vlut.mpgemm_f32(self.packed, self.scale, x, self.rows)[0]


class Layer:
    """A decoder layer whose pages are its own."""

    def __init__(self, features: int, inner: int, q_heads: int, k_heads: int, D: int, pages: int, page_size: int, seed: int):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        norm = lambda n: 1 + 0.1 * torch.randn(n, generator=gen, device="cuda")  # noqa: E731
        self.q_heads, self.k_heads, self.inner = q_heads, k_heads, inner
        self.qkv, self.o = Linear((q_heads + 2 * k_heads) * D, features, 8 * seed), Linear(features, q_heads * D, 8 * seed + 1)
        self.gate_up, self.down = Linear(2 * inner, features, 8 * seed + 2), Linear(features, inner, 8 * seed + 3)
        self.norm, self.ffn_norm, self.inner_norm, self.q_norm, self.k_norm = norm(features), norm(features), norm(inner), norm(D), norm(D)
        self.pages = Pages(pages, k_heads, page_size, D)

    def attend(self, x, step, cos, sin):
        """x: fp32 [tokens][features], normed; the tokens' keys and values go to their slots."""
        y = self.qkv(x).view(x.shape[0], self.q_heads + 2 * self.k_heads, -1)
        q, k, v = y.split([self.q_heads, self.k_heads, self.k_heads], 1)
        q = vlut.append_kv(k, v, step.slots, self.pages.k, self.pages.v, positions=step.positions, cos=cos, sin=sin, k_weight=self.k_norm, q=q, q_weight=self.q_norm)
        out, _ = vlut.chunk_attention(q, self.pages.k, self.pages.v, step.table, step.starts, step.lens, step.max_queries, step.max_len, dtype=torch.float32)
        return self.o(out.flatten(1))

    def forward(self, h, x, next_norm, step, cos, sin):
        """The residual stream h and its norm x -> those of the next layer."""
        h, x = vlut.residual_norm(self.attend(x, step, cos, sin), h, next_weight=self.ffn_norm, out=h)
        y = self.gate_up(x)
        x = vlut.gated_norm(y[:, self.inner:], y[:, :self.inner], "relu2", self.inner_norm)
        return vlut.residual_norm(self.down(x), h, next_weight=next_norm, out=h)


class Step:
    """The next tokens of some prompts: (prompt, first token, tokens) each, one behind the other."""

    def __init__(self, chunks, tables, page_size):
        new = lambda x, dtype=torch.int32: torch.tensor(x, dtype=dtype, device="cuda")  # noqa: E731
        self.chunks = chunks
        starts = [0]
        for _, _, n in chunks:
            starts.append(starts[-1] + n)
        self.starts, self.lens = new(starts), new([first + n for _, first, n in chunks])
        self.max_queries, self.max_len = max(n for _, _, n in chunks), max(first + n for _, first, n in chunks)
        of = [tables[prompt] for prompt, _, _ in chunks]
        width = -(-self.max_len // page_size)
        self.table = torch.stack([torch.nn.functional.pad(t, (0, max(0, width - t.numel())), value=-1)[:width] for t in of])
        self.positions = torch.cat([torch.arange(first, first + n, device="cuda") for _, first, n in chunks])
        page = torch.cat([t[torch.arange(first, first + n, device="cuda") // page_size] for t, (_, first, n) in zip(of, chunks)])
        self.slots = page.long() * page_size + self.positions % page_size


def steps(lengths, budget):
    """Passes of at most `budget` tokens over prompts of these lengths, in order."""
    first, chunks, room = 0, [], budget
    for prompt, length in enumerate(lengths):
        first = 0
        while first < length:
            n = min(room, length - first)
            chunks.append((prompt, first, n))
            first, room = first + n, room - n
            if room == 0:
                yield chunks
                chunks, room = [], budget
    if chunks:
        yield chunks


class Model:
    def __init__(self, layers=2, vocabulary=32000, features=2560, inner=6912, q_heads=20, k_heads=5, D=128, pages=64, page_size=64, positions=65536, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(1000 + seed)
        self.layers = [Layer(features, inner, q_heads, k_heads, D, pages, page_size, seed + i) for i in range(layers)]
        self.embedding = torch.randn((vocabulary, features), generator=gen, device="cuda")
        self.head = (torch.randn((features, vocabulary), generator=gen, device="cuda") * features ** -0.5).bfloat16()
        self.norm, self.page_size = 1 + 0.1 * torch.randn(features, generator=gen, device="cuda"), page_size
        self.cos, self.sin = rotation(positions, D)

    def forward(self, tokens, step):
        """int64 [tokens] -> logits bf16 [tokens][vocabulary]."""
        h = self.embedding[tokens]
        h, x = vlut.residual_norm(torch.zeros_like(h), h, next_weight=self.layers[0].norm, out=h)
        for layer, after in zip(self.layers, [*[of.norm for of in self.layers[1:]], self.norm]):
            h, x = layer.forward(h, x, after, step, self.cos, self.sin)
        return x.bfloat16() @ self.head

    def score(self, prompts, budget, top=5, temperature=1.0):
        """int64 prompts on the GPU -> for each the log probabilities of its tokens behind the first, the entropies ahead of them, and the `top` tokens (and
        their log probabilities) that were the likeliest there; the last of these are of the token that would follow."""
        lengths = [p.numel() for p in prompts]
        tables = [self.layers[0].pages.take(n) for n in lengths]               # (the layers' pages are numbered alike)
        got = [[] for _ in prompts]
        for chunks in steps(lengths, budget):
            step = Step(chunks, tables, self.page_size)
            tokens = torch.cat([prompts[i][first:first + n] for i, first, n in chunks])
            # the token behind each; -1, which none is, behind a prompt's last
            targets = torch.cat([torch.nn.functional.pad(prompts[i], (0, 1), value=-1)[first + 1:first + n + 1] for i, first, n in chunks])
            result = vlut.token_logprobs(self.forward(tokens, step), targets, top=top, temperature=temperature)
            for (i, _, _), *parts in zip(chunks, *[r.split([n for _, _, n in chunks]) for r in result]):
                got[i].append(parts)
        joined = [[torch.cat(x) for x in zip(*parts)] for parts in got]
        return [(logprob[:-1], *rest) for logprob, *rest in joined]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompts", type=int, default=6)
    ap.add_argument("--longest", type=int, default=3000, help="tokens of the longest prompt; the others are shorter")
    ap.add_argument("--budget", type=int, default=2048, help="tokens of a pass")
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args()
    if min(a.prompts, a.budget, a.layers) < 1 or a.longest < 2:
        ap.error("a prompt of two tokens, a token a pass and a layer at least")
    lengths = [max(2, a.longest * (i + 1) // a.prompts) for i in range(a.prompts)]
    model = Model(layers=a.layers, pages=2 * sum(-(-n // 64) for n in lengths), positions=a.longest)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    prompts = [torch.randint(0, 32000, (n,), generator=gen, device="cuda") for n in lengths]
    model.score(prompts, a.budget)                         # (kernels are loaded at their first launch)
    torch.cuda.synchronize()
    began = time.perf_counter()
    scored = model.score(prompts, a.budget)
    torch.cuda.synchronize()
    took = time.perf_counter() - began
    assert all(s[0].isfinite().all() and s[0].numel() == n - 1 for s, n in zip(scored, lengths))
    print(f"{sum(lengths)} tokens of {a.prompts} prompts in {sum(1 for _ in steps(lengths, a.budget))} passes through {a.layers} layers: {took * 1e3:.2f} ms "
          f"({sum(lengths) / took / 1e3:.1f} thousand tokens/s)")


if __name__ == "__main__":
    main()
