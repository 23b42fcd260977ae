"""Attention of chunks with infinite values that queries see, keys in several parts: the formula's infinities and NaN, wherever a key is and whatever its part weighs."""
from __future__ import annotations

import pytest
import torch

from test_chunk_gpu import BF16, F16, F32, INF, NAN, U, case, check, reference, run
from paper_2512_06443_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def device():
    torch.cuda.set_device(0)


def scored(news, lens, Hq, Hk, D, dtype, page, scores, **more):
    """Every query and key of sequence 0 has one feature, so that token t scores scores[t] (a scale of 1)."""
    c = case(news, lens, Hq, Hk, D, dtype, page, **more)
    c["q"].zero_()
    c["q"][..., 0] = 1
    for i, number in enumerate(c["page_table"][0, :-(-lens[0] // page)].tolist()):
        part = scores[i * page:(i + 1) * page]
        c["k_cache"][number, :, :part.numel(), 0] = part.to(dtype)
    return c


def value(c, t, h, feature, x):
    page = c["k_cache"].shape[2]
    c["v_cache"][int(c["page_table"][0, t // page]), h, t % page, feature] = x


SHAPES = {"few": ([2], [3000], 4, 2, 64, 16), "few_100": ([1], [2500], 4, 4, 100, 32), "few_256": ([3], [2000], 2, 1, 256, 16), "few_registers": ([2], [3000], 4, 2, 64, 4),
          "many": ([150], [2100], 8, 2, 64, 16), "many_100": ([150], [2600], 4, 4, 100, 16), "many_256": ([150], [2100], 4, 1, 256, 32), "many_registers": ([150], [2100], 8, 2, 128, 2),
          "few_one_part": ([2], [100], 4, 2, 64, 16), "many_one_part": ([60], [400], 4, 2, 128, 16)}


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("low", [-300.0, -INF])
def test_infinite_values_of_keys_that_weigh_nothing_beside_others(name, low, dtype, out):
    """The keys of a part, of one wave of it, and of one of two groups of waves are far below all others (their weights are 0 in 32 bits) or score -inf: an infinite value
    is infinite still, or NaN where the score is -inf."""
    news, lens, Hq, Hk, D, page = SHAPES[name]
    n, m = news[0], lens[0]
    few, few_parts, few_keys, many, many_parts, many_keys = B.query_chunk_attention(n + 3, 1, Hq, Hk, D, n, m)
    parts, keys = (few_parts, few_keys) if few else (many_parts, many_keys)
    assert (parts > 1) != name.endswith("one_part")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    t = torch.arange(m, device="cuda")
    for which in ("first", "second_32", "every_other_64"):
        hidden = {"first": t < min(keys, m // 2), "second_32": (t // 32 == 1), "every_other_64": (t // 64) % 2 == 0}[which]
        scores = torch.where(hidden, low, torch.randn(m, generator=gen, device="cuda").mul(0.5).to(dtype).float())
        c = scored(news, lens, Hq, Hk, D, dtype, page, scores, seed=D)
        for h in range(Hk):                                # (each head of its own kind, or the odd ones would be in every head)
            c["v_cache"][:, h, :, 3] = 1 + h
        clean, clean_lse = run(c, 0, out, scale=1.0, max_len=m, max_queries=n)
        seen = (t < m - n).nonzero()[:, 0]                 # by all queries
        below = seen[hidden[seen]]
        one, other = int(below[below.numel() // 3]), int(below[-1])
        above = int(seen[~hidden[seen]][-1])
        given = [(one, 5, INF), (one, 7, -INF), (one, 11, INF), (above, 11, -INF), (other, 13, NAN), (above, 17, INF), (other, 19, INF)]
        odd = {}
        for token, f, x in given:
            value(c, token, Hk - 1, f, x)
            odd.setdefault(f, []).append(0.0 * x if low == -INF and token != above else x)
        got, lse = run(c, 0, out, scale=1.0, max_len=m, max_queries=n)
        G = Hq // Hk
        last = slice(Hq - G, Hq)
        want = torch.full((n, G, D), 0.0, dtype=out, device="cuda")
        for f, xs in odd.items():
            want[..., f] = sum(xs)
            its = got[:n, last, f]
            same = (its == want[..., f]) | (its.isnan() & want[..., f].isnan())
            assert bool(same.all()), (which, f, xs, its[~same][:4])
        rest = [f for f in range(D) if f not in odd]
        assert bool(got[:n, :, rest].isfinite().all() and got[:n, :Hq - G].isfinite().all())
        ref = reference(c, 0, 1.0)
        spread = torch.full_like(ref[3], (D + 4) * U * 4.0)                # (of the scores that count)
        mended = got.clone()
        for f in odd:
            mended[:n, last, f] = ref[0][:n, last, f].to(out)
        check(c, mended, lse, ref=(ref[0], ref[1], ref[2], torch.where(ref[3].isfinite() & (ref[3] < 1e-3), ref[3], spread)))
        assert torch.equal(lse, clean_lse) or bool((lse[:n] - clean_lse[:n]).abs().max() < 1e-5)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F32)])
@pytest.mark.parametrize("name", list(SHAPES))
def test_queries_whose_keys_all_score_minus_infinity(name, dtype, out):
    """0, and lse -inf, whatever values they see."""
    news, lens, Hq, Hk, D, page = SHAPES[name]
    c = scored(news, lens, Hq, Hk, D, dtype, page, torch.full((lens[0],), -INF, device="cuda"), seed=D)
    for t in (0, lens[0] // 2, lens[0] - 1):
        value(c, t, 0, 5, INF)
        value(c, t, 0, 6, NAN)
    got, lse = run(c, 0, out, scale=1.0, max_len=lens[0], max_queries=news[0])
    assert bool((got[:news[0]] == 0).all() and (lse[:news[0]] == -INF).all())
