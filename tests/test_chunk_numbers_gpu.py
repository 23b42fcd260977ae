"""Attention of chunks, what its numbers may lose: the bits of the weights, on every way that keys come in and for few and many rows."""
from __future__ import annotations

import pytest
import torch

from test_chunk_gpu import BF16, F16, F32, HALF, U, case, check, reference, run
from paper_2512_06443_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def device():
    torch.cuda.set_device(0)


# How keys come in -> query heads, key heads, features, page, the pages' order.
LOADS = {
    "whole_64": (8, 2, 64, 16, False),
    "whole_128": (8, 2, 128, 64, True),
    "whole_256": (4, 1, 256, 16, False),
    "vectors_40": (6, 2, 40, 16, False),
    "vectors_96": (4, 4, 96, 8, False),
    "vectors_160": (4, 2, 160, 32, True),
    "runs_60": (5, 1, 60, 16, False),
    "runs_100": (4, 4, 100, 32, False),
    "dwords_36": (4, 2, 36, 16, True),
    "dwords_100": (4, 4, 100, 16, True),
    "dwords_132": (2, 2, 132, 16, False),
    "registers_72": (8, 2, 72, 4, False),
    "registers_128": (8, 2, 128, 2, True),
}
# Single tokens, drafts, the same in parts, tiles whose keys two groups of waves share, the same in parts.
ROWS = {"few": ([1, 3, 2], [9, 70, 300]), "few_in_parts": ([1, 2], [3000, 77]), "many": ([60, 140], [60, 200]), "many_in_parts": ([150], [2100])}


def sharp(c):
    """Queries of one feature: scores are single products, of a spread of one or two, whose fp32 values are nearly exact."""
    D = c["q"].shape[2]
    c["q"][..., 1:] = 0
    c["q"][..., 0] = (c["q"][..., 0].float().abs() + 0.5).mul(D ** 0.5).to(c["q"].dtype)
    return c


def bound_of(c, out, window=0):
    """Weights in two terms: each is off by half a step of the rest that the first term leaves, HALF^2 of it, and in fp16, whose smallest number is 2^-24, by
    2^-25 of a reference that is so large beside l that (16 + n / 32) U of the largest value are the most for n keys; fp32 sums and scores as in test_chunk_gpu.check; the
    output's own half step."""
    ref = want, _, size, spread = reference(c, window)
    n = int(c["lens"].max())
    kind = c["k_cache"].dtype
    flushed = (16 + n / 32) * U * float(c["v_cache"].abs().max()) if kind == F16 else 0.0
    bound = size * (2 * spread[..., None] + U * (24 + n / 32) + HALF[kind] ** 2) * 1.02 + HALF[out] * want.abs() * 1.01 + flushed + (2.0 ** -25 if out == F16 else 1e-40)
    return ref, bound


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("load", list(LOADS))
def test_weights_keep_their_bits_for_outputs_of_16_bits(load, rows, dtype):
    """Where terms cancel, the output's own rounding says nothing, and one term of the cache's type would be off by up to HALF of their magnitudes."""
    Hq, Hk, D, page, token_major = LOADS[load]
    news, lens = ROWS[rows]
    c = sharp(case(news, lens, Hq, Hk, D, dtype, page, seed=D, token_major=token_major))
    for window in (0, 50):
        got, _ = run(c, window)
        (want, want_lse, _, _), bound = bound_of(c, dtype, window)
        real = ~want_lse.isnan().any(-1)
        off = ((got.double() - want).abs() / bound)[real]
        assert bool((off <= 1.0).all()), float(off.max())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_weights_keep_their_bits_in_tiles_enough_for_all_units(dtype):
    """Two workgroups of four waves a unit."""
    for D in (128, 64, 100):
        c = sharp(case([1200], [1230], 64, 64, D, dtype, 64, seed=D))
        assert B.query_chunk_attention(1203, 1, 64, 64, D, 1200, 1230)[3:5] == (128, 1)
        got, _ = run(c, max_len=1230, max_queries=1200)
        (want, _, _, _), bound = bound_of(c, dtype)
        off = ((got.double() - want).abs() / bound)[:1200]
        assert bool((off <= 1.0).all()), float(off.max())


@pytest.mark.parametrize("dtype,out", [(F16, F32), (F16, F16), (BF16, F32)])
def test_tails_far_below_a_key_that_few_others_stand_beside_at_first(dtype, out):
    """One key 17.4 nats, 2^25.07, above all 8191 others of the windows, in whose first steps it is among 1 to 15.  The others are 2.3e-4 of the result and of the sum of
    weights, and may be off by 4.4e-5 of it in all: in fp16 their weights are lost unless the key's own is far above 1, and each alone is less than half a step
    of a sum in 32 bits."""
    n, m, window = 200, 9000, 8192
    c = case([n], [m], 256, 256, 8, dtype, 32, seed=24)
    assert B.query_chunk_attention(n + 3, 1, 256, 256, 8, n, m, window)[3:5] == (128, 1)
    c["q"].zero_()
    c["q"][..., 0] = 1
    c["k_cache"][..., 0] = -17.375
    c["v_cache"].abs_().add_(0.5)
    loud = m - n - window + 1 + 62                         # the first key of query 62
    c["k_cache"][int(c["page_table"][0, loud // 32]), :, loud % 32, 0] = 0
    got, lse = run(c, window, out, scale=1.0, max_len=m, max_queries=n)
    check(c, got, lse, window, 1.0, reference(c, window, 1.0))


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("load", ["whole_64", "whole_128", "whole_256", "runs_100", "registers_72"])
def test_values_near_the_types_largest(load, rows, out):
    """Their mean is a number of the type, though their sum is none: sums of up to 3000 weights times values of 2^127."""
    Hq, Hk, D, page, token_major = LOADS[load]
    news, lens = ROWS[rows]
    c = sharp(case(news, lens, Hq, Hk, D, BF16, page, seed=D, token_major=token_major))
    c["v_cache"].sign_().add_(0.5).mul_(2.0 ** 126)        # 1.5 and -0.5 times 2^126
    got, lse = run(c, 0, out)
    assert bool(got[:sum(news)].isfinite().all())
    check(c, got, lse)


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("load", ["whole_64", "whole_128", "whole_256", "runs_100", "registers_72"])
def test_values_near_the_types_largest_in_two_places(load, rows, out):
    """Two keys that count, of two waves or parts, whose values are numbers each, but not together."""
    Hq, Hk, D, page, token_major = LOADS[load]
    news, lens = ROWS[rows]
    for second in (40, 69, max(lens) - 10):
        c = case(news, lens, Hq, Hk, D, BF16, page, seed=D, token_major=token_major)
        c["q"].zero_()
        c["q"][..., 0] = 1
        c["k_cache"][..., 0] = -60
        c["v_cache"].fill_(1.875 * 2.0 ** 127)
        for b, n in enumerate(lens):
            for t in (5, second):
                if t < n:
                    c["k_cache"][int(c["page_table"][b, t // page]), :, t % page, 0] = 0
        got, lse = run(c, 0, out, scale=1.0)
        assert bool(got[:sum(news)].isfinite().all())
        check(c, got, lse, scale=1.0)


@pytest.mark.parametrize("out,exponent", [(BF16, -112), (F32, -104)])
@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("load", ["whole_64", "whole_128", "whole_256", "runs_100", "registers_72"])
def test_small_values_behind_scores_that_rise(load, rows, out, exponent):
    """Parts that are begun again: their weights are not so small that products with values of 2^-112 lose their bits."""
    Hq, Hk, D, page, token_major = LOADS[load]
    news, lens = ROWS[rows]
    c = case(news, lens, Hq, Hk, D, BF16, page, seed=D, token_major=token_major)
    c["q"].zero_()
    c["q"][..., 0] = 1
    c["v_cache"].mul_(2.0 ** exponent)
    c["k_cache"][..., 0] = c["k_cache"][..., 0].clamp(-1, 1)
    for b, n in enumerate(lens):
        t = torch.arange(3, n, 7, device="cuda")
        c["k_cache"][c["page_table"][b].long()[t // page], :, t % page, 0] += (t.clamp(max=400) / 5.0).to(BF16)[:, None]
    got, lse = run(c, 0, out, scale=1.0)
    check(c, got, lse, scale=1.0)
