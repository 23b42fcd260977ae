"""Attention of chunks where pages cannot be: who sees no key of such a page gets what it gets without them, on every way that keys come in."""
from __future__ import annotations

import pytest
import torch

from test_chunk_gpu import BF16, F16, F32, case, check, reference, run
from test_chunk_numbers_gpu import LOADS

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def device():
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F32)])
@pytest.mark.parametrize("load", list(LOADS))
@pytest.mark.parametrize("news,lens,window", [([1], [700], 300), ([3, 1, 2], [500, 90, 331], 40), ([70], [900], 333), ([130, 1], [400, 300], 100), ([300], [300], 64), ([40], [2500], 2000)])
def test_pages_behind_the_window_that_are_given_back(load, news, lens, window, dtype, out):
    """Pages that no query of a sequence sees any more are none (-1): not a bit of any output changes."""
    Hq, Hk, D, page, token_major = LOADS[load]
    page = min(page, 16)
    c = case(news, lens, Hq, Hk, D, dtype, page, seed=D + len(news), token_major=token_major)
    want, want_lse = run(c, window, out)
    check(c, want, want_lse, window)
    table = c["page_table"].clone()
    given = 0
    for b, (n, length) in enumerate(zip(news, lens)):
        behind = max(0, length - n - window + 1) // page
        table[b, :behind] = -1
        given += behind
    assert given or max(lens) <= max(news)
    got, lse = run(dict(c, page_table=table), window, out)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F32)])
@pytest.mark.parametrize("load", list(LOADS))
@pytest.mark.parametrize("news,lens,window", [([5], [260], 0), ([6, 1], [1500, 3], 0), ([100], [300], 0), ([128], [700], 400), ([200, 30], [200, 430], 0)])
def test_a_page_that_only_a_tiles_last_rows_see(load, news, lens, window, dtype, out):
    """Those get NaN; the others, of the same tile or not, are as right as without it."""
    Hq, Hk, D, page, token_major = LOADS[load]
    page = min(page, 16)
    c = case(news, lens, Hq, Hk, D, dtype, page, seed=D + len(news), token_major=token_major)
    b = len(news) - 1 if len(news) == 2 and news[1] > 1 else 0
    start, n, length = int(c["query_starts"][b]), news[b], lens[b]
    for seen_from in {length - 2, length - n // 2}:
        first = seen_from // page
        table = c["page_table"].clone()
        table[b, first] = 2 ** 30
        got, lse = run(dict(c, page_table=table), window, out)
        positions = torch.arange(length - n, length, device="cuda")
        hit = positions >= first * page                    # (the page is within the window of all of these)
        assert bool(hit.any())
        assert bool(got[start:start + n][hit].isnan().all() and lse[start:start + n][hit].isnan().all())
        ref = want, want_lse, size, spread = [x.clone() for x in reference(c, window)]
        want[start:start + n][hit] = want_lse[start:start + n][hit] = float("nan")     # (rows of NaN are not compared)
        check(c, got, lse, window, ref=ref)
