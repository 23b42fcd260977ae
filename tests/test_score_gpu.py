"""examples/score_prompts.py: chunks, norms and log probabilities together, each call of a run against its formula in 64 bits."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

import test_chunk_gpu as chunks
import test_layer_gpu as layers

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E(vlut_lib_path):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("score_prompts", os.path.join(ROOT, "examples", "score_prompts.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


class Checked:
    """The framework's calls, of which those that are the subject here are checked one by one."""

    def __init__(self, of):
        self.of, self.calls = of, dict(chunk_attention=0, residual_norm=0, gated_norm=0, token_logprobs=0)

    def __getattr__(self, name):
        return getattr(self.of, name)

    def chunk_attention(self, q, k, v, table, starts, lens, max_queries, max_len, dtype):
        self.calls["chunk_attention"] += 1
        got = self.of.chunk_attention(q, k, v, table, starts, lens, max_queries, max_len, dtype=dtype, want_lse=True)
        chunks.check(dict(q=q, k_cache=k, v_cache=v, page_table=table, query_starts=starts, lens=lens), *got)
        return got

    def residual_norm(self, y, residual, next_weight, out):
        self.calls["residual_norm"] += 1
        before = residual.clone()
        h, x = self.of.residual_norm(y, residual, next_weight=next_weight, out=out)
        layers.check_residual(y, before, None, None, None, 1.0, next_weight, h, x)
        return h, x

    def gated_norm(self, x, gate, activation, weight):
        self.calls["gated_norm"] += 1
        got = self.of.gated_norm(x, gate, activation, weight)
        t = layers.act(gate.double(), activation) * x.double()
        # of t 8 roundings and the product's own; an error of t moves the norm by as much at most
        layers.check(got, layers.rms(t, weight), layers.rms(t, weight).abs() * (layers.NORM + 2 * 9 * layers.U), "gated norm")
        return got

    def token_logprobs(self, logits, tokens, top, temperature):
        self.calls["token_logprobs"] += 1
        got = self.of.token_logprobs(logits, tokens, top=top, temperature=temperature)
        there = tokens >= 0
        assert bool(got[0][~there].isnan().all())
        layers.check_logprobs(logits[there], tokens[there], top, temperature, [x[there] for x in got])
        layers.check_logprobs(logits[~there], None, top, temperature, [None, *[x[~there] for x in got[1:]]]) if not there.all() else None
        return got


@pytest.mark.parametrize("lengths,budget", [([150, 2, 333, 40], 128), ([70, 5, 61], 1000), ([260], 65), ([9, 30, 2], 1)])
def test_each_call_of_a_run(E, monkeypatch, lengths, budget):
    checked = Checked(E.vlut)
    monkeypatch.setattr(E, "vlut", checked)
    model = E.Model(layers=2, vocabulary=1000, features=512, inner=1408, q_heads=8, k_heads=2, D=64, pages=200, page_size=16, positions=max(lengths))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    prompts = [torch.randint(0, 1000, (n,), generator=gen, device="cuda") for n in lengths]
    passes = -(-sum(lengths) // budget)
    got = model.score(prompts, budget, top=7, temperature=0.8)
    assert checked.calls == dict(chunk_attention=2 * passes, residual_norm=5 * passes, gated_norm=2 * passes, token_logprobs=passes)
    for (logprob, entropy, ids, probs), prompt in zip(got, prompts):
        n = prompt.numel()
        assert logprob.shape == (n - 1,) and entropy.shape == (n,) and ids.shape == probs.shape == (n, 7)
        # a token that is among the likeliest has the log probability that it has there
        at = (ids[:-1] == prompt[1:, None]).nonzero()
        assert torch.equal(logprob[at[:, 0]], probs[at[:, 0], at[:, 1]])


def test_the_passes_of_a_run(E):
    """Every token of every prompt once, in order, no pass of more than the budget."""
    for lengths, budget in (([150, 2, 333, 40], 128), ([5], 1), ([3, 3], 100), ([64, 64], 64)):
        seen = []
        for step in E.steps(lengths, budget):
            assert 0 < sum(n for _, _, n in step) <= budget
            seen += [(i, t) for i, first, n in step for t in range(first, first + n)]
        assert seen == [(i, t) for i, length in enumerate(lengths) for t in range(length)]


def test_command(E, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["score_prompts.py", "--prompts", "3", "--longest", "500", "--budget", "300"])
    E.main()
    assert "3 prompts in 4 passes through 2 layers" in capsys.readouterr().out
