"""examples/shared_prefix_decode.py: the operators together, against their formulas in 64 bits."""
from __future__ import annotations

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E(vlut_lib_path):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("shared_prefix_decode", os.path.join(ROOT, "examples", "shared_prefix_decode.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rotated(block, heads, weight, positions):
    """Norm and rotation in 64 bits: heads [tokens][heads][D], halves in pairs."""
    x = heads.double()
    x = x / (x.square().mean(-1, keepdim=True) + block.eps).sqrt() * weight.double()
    c, s = block.cos[positions].double()[:, None], block.sin[positions].double()[:, None]
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def close(got, want):
    """Rounded once to bf16, from fp32 values that are off by 2^-18 at most (norms and tables: a dozen roundings of 2^-24 of a pair's magnitudes)."""
    assert ((got.double() - want).abs() <= want.abs() * 2.0 ** -8 + 2.0 ** -18 * want.abs().amax(-1, keepdim=True)).all()


def tokens_of(pages, of, count):
    """The first tokens of a list of pages, k and v [tokens][heads][D]."""
    return [c[of.long()].transpose(1, 2).flatten(0, 1)[:count] for c in (pages.k, pages.v)]


def attended(block, q, k, v):
    """One sequence's queries q [n][q_heads][D], its last, over k and v [tokens][k_heads][D], in 64 bits: the results and their bounds (weights in two
    terms of bf16; scores off by (D + 4) 2^-24 of their magnitudes, of which those of normed heads are at most 1.5^2 D^0.5)."""
    n, T, G = q.shape[0], k.shape[0], block.q_heads // block.k_heads
    q, k, v = q.double(), k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    s = torch.stack([q[:, h] @ k[:, h].T for h in range(block.q_heads)]) * block.D ** -0.5
    s = s.masked_fill(torch.arange(T, device="cuda") > torch.arange(T - n, T, device="cuda")[:, None], -float("inf"))
    w = torch.softmax(s, -1)
    out, size = (torch.stack([w[h] @ x[:, h] for h in range(block.q_heads)], 1) for x in (v, v.abs()))
    return out, size * (2.0 ** -16 + 2 * (block.D + 4) * 2.0 ** -24 * 2.25 * block.D ** 0.5 + T * 2.0 ** -24 + 2.0 ** -20)


@pytest.mark.parametrize("sequences,prompt,page", [(3, 70, 16), (40, 333, 64)])
def test_prompt_first_and_steps(E, sequences, prompt, page):
    block = E.synthetic_block(features=512, q_heads=8, k_heads=2, D=64, positions=prompt + 8)
    pages = E.Pages(-(-prompt // page) + sequences, block.k_heads, page, block.D)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.randn((prompt, 512), generator=gen, device="cuda")
    y, prefix = block.prompt(x, pages)
    # what the prompt left in its pages
    q, k, v = block.project(x)
    at = torch.arange(prompt, device="cuda")
    pk, pv = tokens_of(pages, prefix, prompt)
    close(pk, rotated(block, k, block.k_norm, at))
    assert torch.equal(pv, v.bfloat16())
    q = block.queries(x, at, torch.bfloat16)
    close(q, rotated(block, block.project(x)[0], block.q_norm, at))
    want, bound = attended(block, q, pk, pv)
    length = torch.tensor([prompt], dtype=torch.int32, device="cuda")
    got = block.attend(q, 1, pages, None, 0, prefix[None], length, prompt)
    assert ((got.view(want.shape).double() - want).abs() <= bound).all()
    assert torch.equal(y, block.output(x, got))
    # the last token again, from the cache
    last = block.attend(block.queries(x[-1:], at[-1:], torch.bfloat16), 1, pages, prefix, prompt, None, torch.zeros_like(length), 0)
    assert ((last.view(want[-1:].shape).double() - want[-1:]).abs() <= bound[-1:]).all()
    assert torch.equal(block.first(x[-1:], pages, prefix, prompt), block.output(x[-1:], last))
    # steps
    table = torch.stack([pages.take(8) for _ in range(sequences)])
    own = torch.zeros(sequences, dtype=torch.int32, device="cuda")
    for step in range(3):
        x = torch.randn((sequences, 512), generator=gen, device="cuda")
        y = block.decode(x, pages, prefix, prompt, table, own, 8)
        assert own.eq(step + 1).all()
        q, k, v = block.project(x)
        now = torch.full((sequences,), prompt + step, device="cuda")
        rows = [torch.stack([c[table[b, 0], :, step] for b in range(sequences)]) for c in (pages.k, pages.v)]
        close(rows[0], rotated(block, k, block.k_norm, now))
        assert torch.equal(rows[1], v.bfloat16())
        q = block.queries(x, now, torch.bfloat16)
        got = block.attend(q, sequences, pages, prefix, prompt, table, own, 8)
        assert torch.equal(y, block.output(x, got))
        for b in range(sequences):
            ok, ov = tokens_of(pages, table[b], step + 1)
            want, bound = attended(block, q[b:b + 1], torch.cat([pk, ok]), torch.cat([pv, ov]))
            assert ((got[b].view(want.shape).double() - want).abs() <= bound).all(), (step, b)


def test_command(E, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["shared_prefix_decode.py", "--sequences", "5", "--prompt", "300", "--steps", "4"])
    E.main()
    assert "5 sequences, 4 tokens each" in capsys.readouterr().out
