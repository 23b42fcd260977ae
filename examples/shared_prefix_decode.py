#!/usr/bin/env python3
"""The attention block of a decoder layer, decoding for a batch of sequences that continue one prompt.

Per step and layer: the stacked q/k/v projection (`mpgemm_f32`, ternary weights), norms and rotation of the heads with the new keys and values
put into their pages (`append_kv`), attention over the shared prompt and each sequence's own tokens (`shared_prefix_attention`, fp32
out), the output projection (`mpgemm_f32`), and the residual.  The prompt is worked on once, by the same calls, with its tokens as
one sequence's own; afterwards its pages are everybody's prefix.  A sequence's first token comes from the prompt's last one, whose keys are there
already: its queries alone are made (`norm_rope`).

    python examples/shared_prefix_decode.py --sequences 64 --prompt 4096 --steps 32

Synthetic weights of the 2.4B-style layer's q, k, v and o (2560 features, 20 query heads and 5 key heads of 128) and synthetic tokens.
Prints one line: the time of the prompt and of a decoding step (captured as a graph and replayed).
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2512_06443_amd import binding as vlut  # noqa: E402


class Pages:
    """A paged cache of keys and values and which of its pages are free; [pages][heads][page_size][D]."""

    def __init__(self, pages: int, heads: int, page_size: int, D: int, dtype: torch.dtype = torch.bfloat16):
        self.k, self.v = (torch.zeros((pages, heads, page_size, D), dtype=dtype, device="cuda") for _ in range(2))
        self.page_size, self.free = page_size, list(range(pages))

    def take(self, tokens: int) -> torch.Tensor:
        """Pages with room for so many tokens, int32."""
        count = -(-tokens // self.page_size)
        if count > len(self.free):
            raise RuntimeError(f"{count} pages are wanted, {len(self.free)} are free")
        got, self.free = self.free[:count], self.free[count:]
        return torch.tensor(got, dtype=torch.int32, device="cuda")

    def slots(self, pages: torch.Tensor, at: torch.Tensor) -> torch.Tensor:
        """Where the tokens `at` of the rows of `pages` are: pages [..., count], at [...] (or pages [count], at [tokens])."""
        if pages.dim() == 1:
            page = pages[at // self.page_size]
        else:
            page = pages.gather(-1, (at // self.page_size).unsqueeze(-1)).squeeze(-1)
        return page.long() * self.page_size + at % self.page_size


class AttentionBlock:
    """q/k/v and o of ternary weights int8 [rows][features] with their scales, weights of the heads' norms, tables of the rotation."""

    def __init__(self, w_qkv, qkv_scales, w_o, o_scale, q_heads, k_heads, D, q_norm, k_norm, cos, sin, eps=1e-6):
        self.q_heads, self.k_heads, self.D = q_heads, k_heads, D
        self.rows, self.features = w_qkv.shape
        if self.rows != (q_heads + 2 * k_heads) * D or tuple(w_o.shape) != (self.features, q_heads * D):
            raise ValueError("w_qkv: [(q_heads + 2 * k_heads) * D][features], w_o: [features][q_heads * D]")
        self.qkv, self.qkv_scales = vlut.pack_weights(w_qkv), qkv_scales
        self.o, self.o_scale = vlut.pack_weights(w_o), o_scale
        self.q_norm, self.k_norm, self.cos, self.sin, self.eps = q_norm, k_norm, cos, sin, eps

    def project(self, x):
        """fp32 [tokens][features] -> views q, k, v [tokens][heads][D] of the stacked projection's rows."""
        y = vlut.mpgemm_f32(self.qkv, self.qkv_scales, x, self.rows)[0].view(x.shape[0], -1, self.D)
        return y[:, :self.q_heads], y[:, self.q_heads:self.q_heads + self.k_heads], y[:, self.q_heads + self.k_heads:]

    def append(self, x, positions, slots, pages):
        """The tokens' keys and values to their slots; their queries, of the cache's type."""
        q, k, v = self.project(x)
        return vlut.append_kv(k, v, slots, pages.k, pages.v, positions=positions, cos=self.cos, sin=self.sin, k_weight=self.k_norm, eps=self.eps,
                              q=q, q_weight=self.q_norm)

    def queries(self, x, positions, dtype):
        """The queries alone, of tokens whose keys are there already."""
        return vlut.norm_rope(self.project(x)[0], positions=positions, cos=self.cos, sin=self.sin, q_weight=self.q_norm, eps=self.eps, dtype=dtype)[0]

    def attend(self, q, sequences, pages, prefix_pages, prefix_len, table, own_lens, max_own_len):
        """[tokens][heads][D] queries, the same number for each sequence -> fp32 [tokens][q_heads * D]."""
        out, _ = vlut.shared_prefix_attention(q.view(sequences, -1, self.q_heads, self.D), pages.k, pages.v, prefix_pages, prefix_len, table, own_lens,
                                              max_own_len=max_own_len, dtype=torch.float32)
        return out.view(q.shape[0], -1)

    def output(self, x, attended):
        return x + vlut.mpgemm_f32(self.o, self.o_scale, attended, self.features)[0]

    def prompt(self, x, pages):
        """Works on a prompt: returns (its tokens' outputs, its pages)."""
        at = torch.arange(x.shape[0], device="cuda")
        own = pages.take(x.shape[0])
        q = self.append(x, at, pages.slots(own, at), pages)
        length = torch.tensor([x.shape[0]], dtype=torch.int32, device="cuda")
        return self.output(x, self.attend(q, 1, pages, None, 0, own[None], length, x.shape[0])), own

    def first(self, x, pages, prefix_pages, prefix_len):
        """The output of the prompt's last token (x: [1][features]) again, from the cache: what each sequence starts from."""
        q = self.queries(x, torch.tensor([prefix_len - 1], device="cuda"), pages.k.dtype)
        none = torch.zeros(1, dtype=torch.int32, device="cuda")
        return self.output(x, self.attend(q, 1, pages, prefix_pages, prefix_len, None, none, 0))

    def decode(self, x, pages, prefix_pages, prefix_len, table, own_lens, max_own_len):
        """One token per sequence, x [sequences][features], behind own_lens (int32) own tokens; own_lens counts it in afterwards."""
        at = own_lens.long()
        q = self.append(x, at + prefix_len, pages.slots(table, at), pages)
        own_lens.add_(1)
        return self.output(x, self.attend(q, x.shape[0], pages, prefix_pages, prefix_len, table, own_lens, max_own_len))


def rotation(positions: int, D: int, base: float = 10000.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def synthetic_block(features=2560, q_heads=20, k_heads=5, D=128, positions=65536, seed=0) -> AttentionBlock:
    from paper_2512_06443_amd import workloads as wl
    rows = [q_heads * D, k_heads * D, k_heads * D]
    w = [torch.from_numpy(wl.ternary(seed * 7 + i, m, features, 0.4)).cuda() for i, m in enumerate(rows)]
    w_o = torch.from_numpy(wl.ternary(seed * 7 + 3, features, q_heads * D, 0.4)).cuda()
    scale = features ** -0.5
    scales = torch.cat([torch.full((m,), scale * (1 + 0.1 * i), device="cuda") for i, m in enumerate(rows)])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    norm = lambda: 1 + 0.1 * torch.randn(D, generator=gen, device="cuda")  # noqa: E731
    return AttentionBlock(torch.cat(w), scales, w_o, scale, q_heads, k_heads, D, norm(), norm(), *rotation(positions, D))


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sequences", type=int, default=64)
    ap.add_argument("--prompt", type=int, default=4096, help="tokens that all sequences share")
    ap.add_argument("--steps", type=int, default=32, help="tokens that each sequence goes on by")
    ap.add_argument("--page-size", type=int, default=64)
    a = ap.parse_args()
    if a.sequences < 1 or a.prompt < 1 or a.steps < 2:
        ap.error("a sequence, a token of the prompt and two steps at least")
    block = synthetic_block(positions=a.prompt + a.steps)
    per = -(-a.steps // a.page_size)
    pages = Pages(-(-a.prompt // a.page_size) + a.sequences * per, block.k_heads, a.page_size, block.D)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn((a.prompt, block.features), generator=gen, device="cuda")
    block.prompt(x, Pages(-(-a.prompt // a.page_size), block.k_heads, a.page_size, block.D))      # (kernels are loaded at their first launch)
    torch.cuda.synchronize()
    began = time.perf_counter()
    y, prefix = block.prompt(x, pages)
    torch.cuda.synchronize()
    prompt_ms = (time.perf_counter() - began) * 1e3
    start = block.first(x[-1:], pages, prefix, a.prompt)
    assert torch.allclose(start, y[-1:], rtol=1e-2, atol=1e-2 * y[-1].abs().max().item())
    table = torch.stack([pages.take(a.steps) for _ in range(a.sequences)])
    own = torch.zeros(a.sequences, dtype=torch.int32, device="cuda")
    state = start + torch.randn((a.sequences, block.features), generator=gen, device="cuda")      # (each sequence draws a token of its own)
    step = lambda: block.decode(state, pages, prefix, a.prompt, table, own, a.steps)  # noqa: E731
    state.copy_(step())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
        state.copy_(out)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.steps - 1):
        graph.replay()
    torch.cuda.synchronize()
    step_us = (time.perf_counter() - began) / (a.steps - 1) * 1e6
    assert own.eq(a.steps).all() and state.isfinite().all()
    print(f"prompt of {a.prompt}: {prompt_ms:.2f} ms; {a.sequences} sequences, {a.steps} tokens each: {step_us:.1f} us a step "
          f"({a.sequences / step_us:.2f} M tokens/s of this block)")


if __name__ == "__main__":
    main()
