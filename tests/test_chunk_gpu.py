"""Attention of packed chunks of new tokens over a paged cache, against its formula in 64 bits."""
from __future__ import annotations

import itertools
import math

import pytest
import torch

from paper_2512_06443_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = math.inf, math.nan
# Half a step of a type, relative.
HALF = {t: torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def device():
    torch.cuda.set_device(0)


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def case(news, lens, Hq, Hk, D, dtype, page, seed=0, token_major=False, spare=2, rows_behind=3, scale_q=1.0):
    """q, the caches, the page table (pages behind a sequence's end are no numbers of pages), query_starts, lens; rows behind the last sequence."""
    gen = generator(seed)
    Bn, width = len(news), max(1, -(-max(lens) // page)) + 1
    pages = Bn * width + spare
    shape = (pages, page, Hk, D) if token_major else (pages, Hk, page, D)
    k, v = (torch.randn(shape, generator=gen, device="cuda", dtype=F32).to(dtype) for _ in "kv")
    if token_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    table = torch.randperm(pages, generator=gen, device="cuda")[:Bn * width].to(torch.int32).reshape(Bn, width)
    for b, n in enumerate(lens):
        table[b, -(-max(n, 0) // page):] = -7
    starts = torch.tensor(list(itertools.accumulate(news, initial=0)), dtype=torch.int32, device="cuda")
    q = (scale_q * torch.randn(sum(news) + rows_behind, Hq, D, generator=gen, device="cuda")).to(dtype)
    return dict(q=q, k_cache=k, v_cache=v, page_table=table, query_starts=starts, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))


def reference(c, window=0, scale=None):
    """(out, lse, weighted |v|) in 64 bits; rows of no sequence NaN."""
    q, table = c["q"].double(), c["page_table"].tolist()
    N, Hq, D = q.shape
    Hk, page = c["k_cache"].shape[1:3]
    G = Hq // Hk
    starts, lens = c["query_starts"].tolist(), c["lens"].tolist()
    out, size = torch.full((N, Hq, D), NAN, dtype=torch.float64, device="cuda"), torch.zeros((N, Hq, D), dtype=torch.float64, device="cuda")
    lse, spread = torch.full((N, Hq), NAN, dtype=torch.float64, device="cuda"), torch.zeros((N, Hq), dtype=torch.float64, device="cuda")
    scale = D ** -0.5 if scale is None else scale
    for b in range(len(lens)):
        n, m = starts[b + 1] - starts[b], lens[b]
        if n <= 0:
            continue
        ids = table[b][:-(-m // page)]
        k, v = (torch.cat([x[i].double() for i in ids] or [torch.zeros(Hk, 0, D, dtype=torch.float64, device="cuda")], dim=1)[:, :m] for x in (c["k_cache"], c["v_cache"]))
        pos = torch.arange(m - n, m, device="cuda")[:, None]
        t = torch.arange(m, device="cuda")[None]
        seen = (t <= pos) & ((t > pos - window) if window else True)
        for h in range(Hq):
            qh = q[starts[b]:starts[b + 1], h]
            s = (qh @ k[h // G].T) * scale
            s = torch.where(seen, s, -INF)
            top = s.amax(-1, keepdim=True) if m else torch.full((n, 1), -INF, dtype=torch.float64, device="cuda")
            e = torch.exp(s - torch.where(top == -INF, 0.0, top))
            e = torch.where(seen, e, 0.0)
            l = e.sum(-1, keepdim=True)
            vh = v[h // G]
            w = e / torch.where(l == 0, 1.0, l)
            out[starts[b]:starts[b + 1], h] = w @ torch.where(torch.isfinite(vh), vh, 0.0)
            size[starts[b]:starts[b + 1], h] = w @ torch.where(torch.isfinite(vh), vh, 0.0).abs()
            lse[starts[b]:starts[b + 1], h] = (torch.log(l) + torch.where(top == -INF, 0.0, top))[:, 0]
            # how far an fp32 score may be off: D products and the accumulation's roundings, D terms one after the other at most
            spread[starts[b]:starts[b + 1], h] = (((qh.abs() @ k[h // G].abs().T) * scale * seen).amax(-1) if m else 0.0) * (D + 4) * U
    return out, lse, size, spread


def check(c, got, lse, window=0, scale=None, ref=None):
    """What may be off, relative to sum w |v|: the weights by their scores (twice: weight and sum), exponentials and sums of fp32 (up to 2^-12 of them for the
    longest lengths here, as terms are of one sign: 16 U + 2 U per 64 keys), the weights' rounding to the cache's type for 16-bit outputs (half a step; for fp32
    outputs less than U remains), and the output's own half step."""
    want, want_lse, size, spread = reference(c, window, scale) if ref is None else ref
    rows = ~want_lse.isnan().any(-1)
    cache_half = 0.0 if got.dtype == F32 else HALF[c["k_cache"].dtype]
    longest = int(c["lens"].max())
    sums = U * (24 + longest / 32)
    bound = size * (2 * spread[..., None] + sums + cache_half) * 1.02 + HALF[got.dtype] * (want.abs() + size * cache_half) + (2.0 ** -25 if got.dtype == F16 else 1e-40)
    off = (got.double() - want).abs()[rows]
    assert bool((off <= bound[rows]).all()), (off / bound[rows]).max()
    if lse is not None:
        finite = rows[:, None] & (want_lse > -INF)
        assert bool((lse[rows[:, None] & (want_lse == -INF)] == -INF).all())
        assert bool(((lse.double() - want_lse).abs() <= spread + sums + 4 * U * want_lse.abs() + 2 * U)[finite].all())


def run(c, window=0, dtype=None, **more):
    """Both outputs into tensors of a known content: rows of no sequence stay as they are."""
    out = torch.full(c["q"].shape, 123.0, dtype=c["q"].dtype if dtype is None else dtype, device="cuda")
    got, lse = B.chunk_attention(**c, window=window, out=out, want_lse=True, **more)
    assert got is out
    last = int(c["query_starts"][-1])
    assert bool((out[last:] == 123.0).all())
    lse[last:] = 0                                          # (left as torch made them)
    return out, lse


HEADS = [(20, 5, 128), (4, 4, 100), (16, 2, 64), (8, 1, 256), (6, 2, 96), (3, 3, 8), (5, 1, 60), (2, 1, 132), (64, 1, 64), (90, 2, 36)]
LENGTHS = [([1], [1]), ([1], [40]), ([1, 1, 1], [700, 1, 129]), ([5, 1, 8], [5, 33, 400]), ([40], [40]), ([130], [515]), ([3, 0, 200, 1, 17], [3, 9, 200, 1000, 64]),
           ([257, 64], [300, 900]), ([9], [6])]


@pytest.mark.parametrize("Hq,Hk,D", HEADS)
@pytest.mark.parametrize("news,lens", LENGTHS)
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
def test_chunks_of_every_head_and_length(Hq, Hk, D, news, lens, dtype, out):
    for page, token_major, window in ((16, False, 0), (64, True, 0), (8, False, 50), (2, True, 7)):
        c = case(news, lens, Hq, Hk, D, dtype, page, seed=len(news) + D, token_major=token_major)
        got, lse = run(c, window, out)
        check(c, got, lse, window)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F32)])
@pytest.mark.parametrize("Hq,Hk,D", [(32, 8, 128), (16, 16, 64), (8, 2, 256), (32, 32, 100)])
@pytest.mark.parametrize("news,lens,window", [([1024], [1024], 0), ([600], [3000], 0), ([700, 1, 300], [700, 5000, 2000], 333), ([1] * 33, [61 * i + 1 for i in range(33)], 0),
                                              ([1] * 7, [9000, 1, 64, 127, 128, 129, 4000], 1000)])
def test_longer_ones(Hq, Hk, D, news, lens, window, dtype, out):
    c = case(news, lens, Hq, Hk, D, dtype, 32, seed=D)
    got, lse = run(c, window, out)
    check(c, got, lse, window)
    again, again_lse = run(c, window, out)
    assert torch.equal(got, again) and torch.equal(lse, again_lse)


def test_many_tiles():
    """More tiles than two for each unit, every type and way of loading."""
    for Hq, Hk, D, dtype, out in ((64, 64, 128, BF16, BF16), (64, 16, 64, F16, F16), (64, 64, 100, F16, F32), (64, 32, 128, BF16, F32), (64, 8, 96, BF16, BF16)):
        n = 4096 + 77
        assert B.query_chunk_attention(n, 1, Hq, Hk, D, n, n)[3:5] == (128, 1)
        c = case([n], [n + 20], Hq, Hk, D, dtype, 64, seed=1)
        for window in (0, 100):
            got, lse = run(c, window, out)
            check(c, got, lse, window)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lens", [([1], [3000]), ([300], [1200]), ([4], [2500])])
def test_scores_that_leave_the_first_ones_far_behind(news, lens, dtype):
    """Rising scores: weights of the first step's maximum would leave the type's range; and falling ones."""
    for sign in (1.0, -1.0):
        c = case(news, lens, 4, 2, 64, dtype, 16, seed=5)
        c["q"].fill_(4.0)
        ramp = sign * torch.linspace(-6, 6, lens[0], device="cuda")          # scores of +-192 / sqrt(64) ... times 64 * 4 / 8
        for i, page in enumerate(c["page_table"][0, :-(-lens[0] // 16)].tolist()):
            part = ramp[16 * i:16 * i + 16]
            c["k_cache"][page, :, :part.numel()] = part.to(dtype)[None, :, None]
        for out in (dtype, F32):
            got, lse = run(c, 0, out)
            check(c, got, lse)
        got, lse = run(c, 200, dtype)
        check(c, got, lse, 200)


def page_of(c, b, t):
    page = c["k_cache"].shape[2]
    return int(c["page_table"][b, t // page]), t % page


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F32), (F16, F16)])
@pytest.mark.parametrize("news,lens", [([6], [500]), ([150], [400]), ([1, 100], [77, 300]), ([5], [2500])])
@pytest.mark.parametrize("D", [128, 100, 36])
def test_values_and_keys_that_are_no_numbers(D, news, lens, dtype, out):
    """Behind a query's position, outside its window or behind the sequence's end they have no influence; seen, an infinity makes its feature infinite."""
    window = 60
    Hq, Hk = 6, 3
    c = case(news, lens, Hq, Hk, D, dtype, 16, seed=9)
    clean = {w: run(c, w, out) for w in (0, window)}
    b = len(news) - 1
    n, m, start = news[b], lens[b], int(c["query_starts"][b])
    # behind the sequence's end, in its last page
    if m % 16:
        page, _ = page_of(c, b, m - 1)
        c["v_cache"][page, :, m % 16:] = NAN
        c["k_cache"][page, :, m % 16:] = INF
    for w in (0, window):
        again = run(c, w, out)
        assert all(torch.equal(x, y) for x, y in zip(clean[w], again))
    # a value and a key that only queries from the third last on see
    t = m - 3
    page, at = page_of(c, b, t)
    c["v_cache"][page, 1, at, 5] = INF
    c["v_cache"][page, 1, at, 6] = -INF
    c["v_cache"][page, 2, at, 7] = NAN
    # and one that only those within the window see
    t2 = m - n // 2 - window
    if 0 <= t2 < t:
        page, at = page_of(c, b, t2)
        c["v_cache"][page, 0, at, 9] = INF
    for w in (0, window):
        got, lse = run(c, w, out)
        want = clean[w][0].clone()
        G = Hq // Hk
        sees = torch.zeros(want.shape[0], dtype=torch.bool, device="cuda")
        for row in range(n):
            pos = m - n + row
            if pos >= t and (not w or pos - w < t):
                want[start + row, G:2 * G, 5], want[start + row, G:2 * G, 6], want[start + row, 2 * G:3 * G, 7] = INF, -INF, NAN
                sees[start + row] = True
            if 0 <= t2 < t and pos >= t2 and (not w or pos - w < t2):
                want[start + row, :G, 9] = INF
                sees[start + row] = True
        odd = ~torch.isfinite(want)
        assert torch.equal(odd, ~torch.isfinite(got))
        assert torch.equal(want[odd & ~want.isnan()], got[odd & ~want.isnan()]) and torch.equal(want.isnan(), got.isnan())
        # no influence on those that do not see them: the same bits (parts with an infinity are worked on twice, with another m)
        assert torch.equal(got[~sees], want[~sees]) and torch.equal(lse[~sees], clean[w][1][~sees])
        ref = reference(c, w)
        check(c, torch.where(odd, ref[0], got.double()).to(got.dtype), lse, w, ref=ref)
    page, at = page_of(c, b, t)
    c["v_cache"][page, 0, at, 9] = -INF                     # with an infinity of the other sign: NaN for those that see both
    c["k_cache"][page, 1, at] = NAN
    got, lse = run(c, 0, out)
    G = Hq // Hk
    assert bool(got[start + n - 3 if n > 2 else start:start + n, G:2 * G].isnan().all() and lse[start + max(0, n - 3):start + n, G:2 * G].isnan().all())
    if n > 3:
        assert torch.allclose(lse[start:start + n - 3], clean[0][1][start:start + n - 3], rtol=0, atol=1e-4) and not bool(got[start:start + n - 3, G:2 * G].isnan().any())


def test_keys_that_score_minus_infinity():
    c = case([3, 70], [200, 200], 2, 2, 64, BF16, 16, seed=3)
    c["q"].copy_(c["q"].abs())
    for b in range(2):
        for t in list(range(0, 150)) + [199]:
            page, at = page_of(c, b, t)
            c["k_cache"][page, 0, at] = -INF
        for t in range(200):
            page, at = page_of(c, b, t)
            c["k_cache"][page, 1, at] = -INF               # every key of the second head: nothing
    got, lse = run(c)
    want, want_lse, size, spread = reference(c)
    spread = torch.nan_to_num(spread, posinf=0.0) + 68 * U * 30
    spread[spread > 1e-3] = 68 * U * 30
    check(c, got, lse, ref=(want, want_lse, size, spread))
    assert bool((got[:73, 1] == 0).all() and (lse[:73, 1] == -INF).all())
    # rows that see only such keys of the first head
    assert bool((lse[3:3 + 20, 0] == -INF).all() and (got[3:23, 0] == 0).all())


@pytest.mark.parametrize("D", [64, 60])
def test_lengths_pages_and_starts_that_cannot_be(D):
    """Found on the device: nothing is read, and who depends on it gets NaN."""
    c = case([2, 80, 1, 3], [100, 200, 150, 60], 4, 2, D, BF16, 16, seed=4)
    clean, clean_lse = run(c, max_len=200)
    rows = [slice(0, 2), slice(2, 82), slice(82, 83), slice(83, 86)]
    for b, length in ((0, 201), (1, -1), (1, 2 ** 30), (2, -2 ** 31)):
        d = dict(c, lens=c["lens"].clone())
        d["lens"][b] = length
        got, lse = run(d, max_len=200)
        for i, r in enumerate(rows):
            if i == b:
                assert bool(got[r].isnan().all() and lse[r].isnan().all())
            else:
                assert torch.equal(got[r], clean[r]) and torch.equal(lse[r], clean_lse[r])
    for b, number in ((0, -1), (1, 2 ** 31 - 1), (1, c["k_cache"].shape[0]), (2, -2 ** 31)):
        for place in (0, 3):
            d = dict(c, page_table=c["page_table"].clone())
            d["page_table"][b, place] = number
            got, _ = run(d, max_len=200)
            for i, r in enumerate(rows):
                if i == b:
                    positions = torch.arange(int(c["lens"][b]) - (r.stop - r.start), int(c["lens"][b]), device="cuda")
                    hit = positions >= 16 * place
                    assert bool(got[r][hit].isnan().all()) and torch.equal(got[r][~hit], clean[r][~hit])
                else:
                    assert torch.equal(got[r], clean[r])
    # sequences whose starts are out of place have no rows
    d = dict(c, query_starts=torch.tensor([0, 2, 82, 83, 500], dtype=torch.int32, device="cuda"))
    out = torch.full_like(c["q"], 5.0)
    B.chunk_attention(**d, out=out, max_len=200)
    assert torch.equal(out[:83], clean[:83]) and bool((out[83:] == 5).all())
    d["query_starts"] = torch.tensor([-4, 2, 82, 83, 86], dtype=torch.int32, device="cuda")
    out.fill_(5.0)
    B.chunk_attention(**d, out=out, max_len=200)
    assert bool((out[:2] == 5).all()) and torch.equal(out[2:86], clean[2:86])
    # more queries than said: NaN where few rows are all there is
    got, lse = run(c, max_len=200, max_queries=3)
    assert torch.equal(got[:2], clean[:2]) and torch.equal(got[82:86], clean[82:86]) and bool(got[2:82].isnan().all() and lse[2:82].isnan().all())


@pytest.mark.parametrize("D", [128, 60])
def test_pages_that_cannot_be_in_parts(D):
    """Of few rows and of many: whoever sees the keys of such a page gets NaN, whatever part they are in."""
    c = case([2, 1, 3], [4000, 2500, 100], 4, 2, D, BF16, 16, seed=14)
    assert B.query_chunk_attention(6, 3, 4, 2, D, 3, 4000)[1] > 2
    clean, clean_lse = run(c, max_len=4000, max_queries=3)
    check(c, clean, clean_lse)
    d = case([1, 80], [300, 3000], 4, 2, D, BF16, 16, seed=15)
    assert B.query_chunk_attention(81, 2, 4, 2, D, 80, 3000)[4] > 2
    clean_many, _ = run(d, max_len=3000, max_queries=80)
    for place in (0, 40, 130):
        bad = dict(c, page_table=c["page_table"].clone())
        bad["page_table"][0, place] = -1
        got, lse = run(bad, max_len=4000, max_queries=3)
        assert bool(got[:2].isnan().all() and lse[:2].isnan().all()) and torch.equal(got[2:6], clean[2:6])
        bad = dict(d, page_table=d["page_table"].clone())
        bad["page_table"][1, place] = 2 ** 30
        got, _ = run(bad, max_len=3000, max_queries=80)
        assert bool(got[1:81].isnan().all()) and torch.equal(got[:1], clean_many[:1])


def test_views_and_a_workspace_of_the_callers():
    N, Hq, Hk, D = 90, 8, 2, 64
    c = case([90], [1400], Hq, Hk, D, BF16, 16, seed=6, rows_behind=0)
    wide = torch.randn(N, Hq + 3, D + 2, device="cuda", generator=generator(7)).to(BF16)
    q = wide[:, 2:2 + Hq, 2:]
    q.copy_(c["q"])
    first = B.chunk_attention(**c, max_len=1416)[0]
    d = dict(c, q=q, max_len=1416)
    into = torch.zeros(N, 2 * Hq, D, dtype=BF16, device="cuda")
    assert torch.equal(B.chunk_attention(**d, out=into[:, ::2])[0], first) and bool((into[:, 1::2] == 0).all())
    need = B.chunk_attention_bytes(N, 1, Hq, Hk, D, N, 1416)
    assert need > 0
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(B.chunk_attention(**c, max_len=1416, workspace=ws[:need])[0], first) and bool((ws[need:] == 255).all())


@pytest.mark.parametrize("Hq,Hk,D", [(2, 1, 128), (6, 3, 36)])
def test_more_sequences_than_a_wave_has_lanes(Hq, Hk, D):
    """Of all kinds in any order, long ones among them in parts, and prompts whose tiles are found among all sequences'."""
    news = [(0, 1, 2, 45, 1, 7, 0, 130, 1, 3)[(7 * i + i // 10) % 10] for i in range(150)]
    lens = [n + (0, 5, 3100, 64, 700)[(3 * i + i // 7) % 5] for i, n in enumerate(news)]
    c = case(news, lens, Hq, Hk, D, BF16, 16, seed=21)
    assert B.query_chunk_attention(sum(news) + 3, 150, Hq, Hk, D, 130, max(lens))[1] >= (2 if Hk == 1 else 1)
    for window in (0, 200):
        got, lse = run(c, window, max_queries=130, max_len=max(lens))
        check(c, got, lse, window)


def test_parts_of_more_keys_than_page_numbers_are_kept_for():
    """A part whose pages' numbers come in several loads: of few rows where workgroups are many, of many rows where tiles are."""
    gen = generator(23)
    k, v = (torch.randn(400, 8, 16, 64, generator=gen, device="cuda").to(BF16) for _ in "kv")
    lens = torch.tensor([{5: 5000, 700: 4097, 1199: 4096}.get(i, 1 + i % 7) for i in range(1200)], dtype=torch.int32, device="cuda")
    table = torch.stack([torch.randperm(400, generator=gen, device="cuda")[:313] for _ in range(1200)]).int()
    c = dict(q=torch.randn(1200, 8, 64, generator=gen, device="cuda").to(BF16), k_cache=k, v_cache=v, page_table=table,
             query_starts=torch.arange(1201, dtype=torch.int32, device="cuda"), lens=lens)
    assert B.query_chunk_attention(1200, 1200, 8, 8, 64, 1, 5000)[1:3] == (1, 5120)
    got, lse = run(c, max_queries=1, max_len=5000)
    check(c, got, lse)
    c = case([200], [9000], 256, 256, 8, F16, 32, seed=24)
    parts, keys = B.query_chunk_attention(203, 1, 256, 256, 8, 200, 9000)[4:]
    assert parts == 1 and keys >= 9000
    got, lse = run(c, max_len=9000, max_queries=200)
    check(c, got, lse)


def test_scale_nothing_to_do_and_pages_for_all():
    c = case([70, 3, 1], [90, 300, 1500], 8, 2, 64, F16, 16, seed=22)
    for scale in (1e-3, 0.02, 0.7):
        got, lse = run(c, scale=scale)
        check(c, got, lse, scale=scale, ref=reference(c, 0, scale))
    # no sequence has a token: nothing is written, whatever the lengths say
    d = dict(c, query_starts=torch.zeros(4, dtype=torch.int32, device="cuda"))
    run(d)
    run(d, max_queries=0)
    # nothing is to be seen: 0
    d = dict(c, lens=torch.zeros(3, dtype=torch.int32, device="cuda"))
    got, lse = run(d, max_len=0)
    assert bool((got[:74] == 0).all() and (lse[:74] == -INF).all())
    # one row of pages for all sequences
    d = dict(c, page_table=c["page_table"][2:3].expand(3, -1))
    got, lse = run(d)
    check(d, got, lse)
    e = dict(d, page_table=d["page_table"].contiguous())
    assert torch.equal(run(e)[0], got)


def test_a_cache_past_32_bits():
    """Pages whose elements lie past 2^31, and with strides past what 31 bits hold (the path of addresses per key)."""
    Hk, page, D = 2, 64, 128
    big = torch.zeros((2 ** 31 // (Hk * page * D) + 40, Hk, page, D), dtype=BF16, device="cuda")
    small = case([1, 90], [300, 200], 4, 2, D, BF16, page, seed=8)
    far = small["page_table"].clone()
    far[far >= 0] += big.shape[0] - small["k_cache"].shape[0]
    big[-small["k_cache"].shape[0]:] = small["k_cache"]
    want = B.chunk_attention(**small)[0]
    got = B.chunk_attention(**dict(small, k_cache=big, v_cache=big, page_table=far))[0]
    alone = B.chunk_attention(**dict(small, v_cache=small["k_cache"]))[0]
    assert torch.equal(got[:91], alone[:91]) and not torch.equal(want[:91], alone[:91])
    spread = big.view(-1).as_strided((2, Hk, page, D), (2 ** 30 + 64, page * D, D, 1))
    d = case([1, 90], [60, 64], 4, 2, D, BF16, page, seed=8)
    d["page_table"] = torch.tensor([[0, -1], [1, -1]], dtype=torch.int32, device="cuda")
    k = torch.randn(2, Hk, page, D, device="cuda", generator=generator(3)).to(BF16)
    spread.copy_(k)
    got = B.chunk_attention(**dict(d, k_cache=spread, v_cache=spread))[0]
    d = dict(d, k_cache=k, v_cache=k)
    check(d, got, None)


def test_chunks_in_graphs_that_share_a_workspace_and_on_another_stream():
    c = case([1, 130, 4], [900, 300, 1200], 8, 2, 128, BF16, 16, seed=10)
    need = B.chunk_attention_bytes(c["q"].shape[0], 3, 8, 2, 128, 130, 1216)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    call = lambda w: B.chunk_attention(**c, max_queries=130, window=w, want_lse=True, max_len=1216 if w == 0 else None, workspace=ws if w == 0 else None)  # noqa: E731
    first = call(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call(0)
    torch.cuda.current_stream().wait_stream(side)
    last = int(c["query_starts"][-1])
    assert torch.equal(first[0][:last], second[0][:last])
    graphs, outs = [], []
    for w in (0, 100, 0):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(w))
        graphs.append((g, w))
    for turn in range(4):
        c["q"].mul_(1.1)
        c["lens"].sub_(7)
        for (g, w), out in zip(graphs, outs):
            want = call(w)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(want[0][:last], out[0][:last]) and torch.equal(want[1][:last], out[1][:last]), (turn, w)


def test_chunks_agree_with_the_attention_behind_a_prefix_and_in_both_forms(monkeypatch):
    """The same tokens by the other attention of the library (no prefix, padded queries), and by the call's Python form."""
    c = case([4, 4, 4], [300, 64, 5], 8, 2, 128, BF16, 16, seed=11, rows_behind=0)
    got, lse = B.chunk_attention(**c, dtype=F32, want_lse=True)
    other, other_lse = B.shared_prefix_attention(c["q"].view(3, 4, 8, 128), c["k_cache"], c["v_cache"], None, 0, c["page_table"], c["lens"], dtype=F32, want_lse=True)
    assert torch.allclose(got.view_as(other), other, rtol=0, atol=2e-5) and torch.allclose(lse.view_as(other_lse), other_lse, rtol=0, atol=2e-5)
    assert B._native is not None
    monkeypatch.setattr(B, "_native", None)
    again, again_lse = B.chunk_attention(**c, dtype=F32, want_lse=True)
    assert torch.equal(got, again) and torch.equal(lse, again_lse)
