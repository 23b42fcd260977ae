"""shared_prefix_attention against its formula in 64 bits."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
U = {torch.float32: U32, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # unit roundoffs


@pytest.fixture(scope="module")
def B(vlut_lib_path):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2512_06443_amd import binding
    binding.lib()
    return binding


class Case:
    """Inputs of a call; pages in a shuffled order, NaN wherever nobody may look."""

    def __init__(self, B, n, Hq, Hk, D, P, lens, page, dtype=torch.bfloat16, queries=None, token_major=False, seed=0, spread=1.0, stale=float("nan")):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.shape, self.P, self.lens, self.queries, self.page = (B, n, Hq, Hk, D), P, lens, queries if queries is not None else [n] * B, page
        own_pages = max(1, -(-max(lens) // page))
        prefix_pages = -(-P // page)
        pages = prefix_pages + B * own_pages + 1
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        self.prefix_pages, self.table = order[:prefix_pages].contiguous(), order[prefix_pages:prefix_pages + B * own_pages].reshape(B, own_pages).contiguous()
        shape = (pages, page, Hk, D) if token_major else (pages, Hk, page, D)
        self.k, self.v = (torch.full(shape, stale, dtype=dtype, device="cuda") for _ in range(2))
        if token_major:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.q = (torch.randn((B, n, Hq, D), generator=gen, device="cuda") * spread).to(dtype)
        rand = lambda m: torch.randn((m, Hk, D), generator=gen, device="cuda").to(dtype)  # noqa: E731
        self.prefix = rand(P), rand(P)
        self.own = [(rand(m), rand(m)) for m in lens]
        self.write()
        self.own_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.query_lens = torch.tensor(self.queries, dtype=torch.int32, device="cuda") if queries is not None else None

    def write(self):
        """The tokens to their pages."""
        for pages, tokens in [(self.prefix_pages, self.prefix)] + list(zip(self.table, self.own)):
            at = torch.arange(tokens[0].shape[0], device="cuda")
            ids = pages.long()[at // self.page]
            self.k[ids, :, at % self.page] = tokens[0]
            self.v[ids, :, at % self.page] = tokens[1]

    def run(self, B, **more):
        return B.shared_prefix_attention(self.q, self.k, self.v, self.prefix_pages, self.P, self.table, self.own_lens, query_lens=self.query_lens, **more)

    def check(self, out, lse=None, scale=None, only=None):
        """Every query's output is within its bound.  A score is off by (D + 4) 2^-24 of the sum of its products' magnitudes at most (A; log2(e) and the
        subtraction of the maximum included, the latter 2 roundings of the scores' range) and so are weights, relatively, above and below the
        fraction; weights are rounded to the cache's type (once, or with what that left: twice) for the product alone; sums of N terms are off by
        N 2^-24; exponentials and the joining of parts add 2^-20 at most; then the output's rounding."""
        Bn, n, Hq, Hk, D = self.shape
        G = Hq // Hk
        u = U[self.k.dtype]
        out = out.cpu().double() if out.dtype == torch.float32 else out.cpu()
        kind = torch.float32 if out.dtype == torch.float64 else out.dtype
        for b in range(Bn) if only is None else only:
            k = torch.cat([self.prefix[0], self.own[b][0]]).cpu().double()
            v = torch.cat([self.prefix[1], self.own[b][1]]).cpu().double()
            for j in range(n):
                see = self.P + max(0, self.lens[b] - self.queries[b] + j + 1) if j < self.queries[b] else 0
                for h in range(Hq):
                    got = out[b, j, h].double()
                    if see <= 0:
                        assert (got == 0).all(), (b, j, h)
                        assert lse is None or lse[b, j, h].item() == -math.inf
                        continue
                    q, kk, vv = self.q[b, j, h].cpu().double(), k[:see, h // G], v[:see, h // G]
                    c = D ** -0.5 if scale is None else scale
                    s = kk @ q * c
                    w = torch.softmax(s, 0)
                    want, size = w @ vv, w @ vv.abs()
                    A = (kk.abs() @ q.abs()).max().item() * c
                    spread = (s.max() - s.min()).item()
                    score = (D + 4) * U32 * A + 4 * U32 * (spread + abs(s.max().item()))
                    weights = u if kind != torch.float32 else u * u
                    tiny = 2.0 ** -24 if self.k.dtype == torch.float16 else 0.0            # weights below fp16's normal range: an absolute error
                    bound = size * (weights + 2 * score + see * U32 + 2.0 ** -20) + vv.abs().sum(0) * tiny + want.abs() * U[kind] + 1e-30
                    worst = ((got - want).abs() / bound).max().item()
                    assert worst <= 1.0, f"sequence {b}, query {j}, head {h}: {worst:.3f} of the bound"
                    if lse is not None:
                        assert abs(lse[b, j, h].item() - torch.logsumexp(s, 0).item()) <= 2 * score + see * U32 + 2.0 ** -20 + 4 * U32 * abs(s.max().item())


CASES = {
    # few query rows: tiles of 16 and 32 rows
    "one": dict(B=1, n=1, Hq=4, Hk=1, D=128, P=100, lens=[5], page=16),
    "no_prefix": dict(B=3, n=1, Hq=4, Hk=2, D=128, P=0, lens=[1, 37, 300], page=16),
    "no_own": dict(B=2, n=1, Hq=4, Hk=2, D=64, P=77, lens=[0, 0], page=8),
    "nothing_at_all": dict(B=2, n=1, Hq=4, Hk=2, D=64, P=0, lens=[0, 0], page=8),
    "one_key": dict(B=1, n=1, Hq=1, Hk=1, D=8, P=1, lens=[0], page=1),
    "empty_among_others": dict(B=4, n=1, Hq=2, Hk=1, D=96, P=0, lens=[0, 130, 0, 64], page=32),
    "rows_32": dict(B=6, n=1, Hq=10, Hk=2, D=100, P=333, lens=[3, 40, 0, 129, 128, 127], page=16, dtype=torch.float16),
    "rows_64": dict(B=5, n=3, Hq=8, Hk=2, D=128, P=515, lens=[3, 40, 260, 129, 7], page=64),
    "rows_64_d64": dict(B=15, n=1, Hq=8, Hk=2, D=64, P=700, lens=list(range(15)), page=16, dtype=torch.float16, token_major=True),
    "d256": dict(B=2, n=1, Hq=8, Hk=1, D=256, P=600, lens=[17, 64], page=16),
    "d200_rows_32": dict(B=3, n=1, Hq=16, Hk=2, D=200, P=150, lens=[17, 64, 1], page=4, dtype=torch.float16),
    # own tokens of many pages, several parts
    "long_own": dict(B=1, n=1, Hq=8, Hk=2, D=128, P=0, lens=[5000], page=16),
    "long_own_and_prefix": dict(B=2, n=2, Hq=4, Hk=2, D=64, P=3001, lens=[4097, 2], page=128, dtype=torch.float16),
    # more query rows than a tile
    "rows_128": dict(B=33, n=1, Hq=8, Hk=2, D=128, P=200, lens=[(7 * i) % 150 for i in range(33)], page=16),
    "rows_128_tail": dict(B=17, n=2, Hq=8, Hk=1, D=100, P=1001, lens=[1 + (13 * i) % 90 for i in range(17)], page=32, dtype=torch.float16, token_major=True),
    "rows_128_d64": dict(B=40, n=1, Hq=16, Hk=2, D=64, P=65, lens=[i % 5 for i in range(40)], page=8),
    "rows_128_d256": dict(B=9, n=1, Hq=16, Hk=1, D=256, P=450, lens=[i * 30 for i in range(9)], page=16),
    "rows_128_d132": dict(B=70, n=1, Hq=2, Hk=1, D=132, P=90, lens=[1] * 70, page=16, dtype=torch.float16),
    # drafts: several queries, of which a sequence has some
    "drafts": dict(B=4, n=5, Hq=8, Hk=4, D=128, P=130, lens=[5, 33, 200, 64], page=16, queries=[5, 1, 3, 0]),
    "drafts_past_their_tokens": dict(B=3, n=4, Hq=2, Hk=2, D=64, P=0, lens=[0, 2, 9], page=16, queries=[4, 3, 4]),
    "drafts_past_with_prefix": dict(B=3, n=4, Hq=2, Hk=2, D=64, P=40, lens=[0, 2, 9], page=16, queries=[4, 3, 4]),
    "prompt": dict(B=1, n=150, Hq=4, Hk=2, D=128, P=0, lens=[150], page=16),
    "prompt_behind_prefix": dict(B=2, n=45, Hq=4, Hk=2, D=64, P=70, lens=[45, 60], page=16, dtype=torch.float16),
    "one_head_each": dict(B=3, n=1, Hq=5, Hk=5, D=128, P=50, lens=[9, 10, 11], page=2),
}

# Many query rows over a long prefix: a launch of its own, 32 rows for each of four waves or eight.
MANY = {
    "four_waves": dict(B=20, n=1, Hq=32, Hk=8, D=64, P=31401, lens=[(11 * i) % 70 for i in range(20)], page=16),
    "four_waves_d100": dict(B=3, n=8, Hq=32, Hk=8, D=100, P=13100, lens=[8, 100, 31], page=64, dtype=torch.float16, queries=[8, 3, 5]),
    "eight_waves": dict(B=40, n=1, Hq=32, Hk=8, D=128, P=7950, lens=[(7 * i) % 150 for i in range(40)], page=16),
    "eight_waves_d100": dict(B=21, n=2, Hq=32, Hk=8, D=100, P=7501, lens=[2 + (13 * i) % 90 for i in range(21)], page=32, dtype=torch.float16, token_major=True),
    "eight_waves_d64": dict(B=41, n=1, Hq=16, Hk=2, D=64, P=31999, lens=[1] * 41, page=128, dtype=torch.float16),
    "d256": dict(B=20, n=1, Hq=32, Hk=4, D=256, P=15777, lens=[i * 9 for i in range(20)], page=16),
    "d132": dict(B=33, n=1, Hq=16, Hk=4, D=132, P=19001, lens=[3] * 33, page=16, dtype=torch.float16),
    "pages_of_8": dict(B=40, n=1, Hq=32, Hk=8, D=128, P=7950, lens=[5] * 40, page=8),          # (too short for that launch: tiles)
    "no_own": dict(B=40, n=1, Hq=32, Hk=8, D=64, P=15901, lens=[0] * 40, page=16),
}


@pytest.mark.parametrize("dtype", ["cache", "fp32"])
@pytest.mark.parametrize("name", list(MANY))
def test_many_rows_against_64_bits(B, name, dtype):
    case = Case(**MANY[name])
    print(name, dtype, B.query_shared_prefix_attention(*case.shape, case.P, max(case.lens)), flush=True)
    out, lse = case.run(B, dtype=torch.float32 if dtype == "fp32" else None, want_lse=True, max_own_len=max(case.lens))
    case.check(out, lse.cpu(), only=[0, case.shape[0] - 1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_many_rows_whose_scores_rise(B, dtype):
    """Scores far above those of the first keys: the range is worked on again.  In one range, in the last ones, and everywhere."""
    for where in (slice(1000, 1001), slice(7000, 7940), slice(70, None)):
        case = Case(B=40, n=1, Hq=32, Hk=8, D=128, P=7950, lens=[4] * 40, page=16, dtype=dtype)
        case.prefix[0][where] *= 40
        case.write()
        out, lse = case.run(B, dtype=torch.float32, want_lse=True)
        case.check(out, lse.cpu(), only=[0, 39])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Bn,P,page", [(1, 40000, 16), (1, 40000, 4), (40, 15950, 16)])
@pytest.mark.parametrize("where", [0, 0.6])
def test_one_key_far_above_many(B, dtype, Bn, P, page, where):
    """Weights of 2^-26 of the largest, of which there are so many that they count: where the largest one's value is 0 they are the whole output.
    Bound: the scores' and the sums' of Case.check(); weights in two terms of the type, for fp16 32 rows a wave: to 2^-24 of 2^7 times the largest."""
    D = 64
    case = Case(B=Bn, n=1, Hq=32, Hk=8, D=D, P=P, lens=[0] * Bn, page=page, dtype=dtype)
    case.q.zero_()
    case.q[..., 5] = 16.0
    k, v = case.prefix
    top = int(where * P)
    k.zero_()
    k[:, :, 5] = -13 * math.log(2) / 2
    k[top, :, 5] = 13 * math.log(2) / 2
    v.copy_(v.abs() + 1)
    v[top] = 0
    case.write()
    out, lse = case.run(B, dtype=torch.float32, want_lse=True)
    s = 2.0 * k[:, 0, 5].cpu().double()
    w = torch.softmax(s, 0)
    want = torch.einsum("p,phd->hd", w, v.cpu().double()).repeat_interleave(4, 0)
    score = (D + 4) * U32 * 10 + 4 * U32 * 30
    tiny = 2.0 ** -31 * P * 3 if dtype == torch.float16 and Bn > 1 else 0.0
    bound = want * (U[dtype] ** 2 + 2 * score + P * U32 + 2.0 ** -20) + tiny
    assert ((out.cpu().double()[:, 0] - want).abs() <= bound).all()
    assert (lse.cpu().double() - torch.logsumexp(s, 0)).abs().max() <= 2 * score + P * U32 + 2.0 ** -20


def test_many_rows_with_infinities_and_pages_that_cannot_be(B):
    case = Case(**MANY["eight_waves"])
    want, _ = case.run(B)
    assert want.isfinite().all()
    case.prefix[1][5000, 3, 7] = float("inf")                             # one value of one key head: that feature of its query heads
    case.write()
    out, _ = case.run(B)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[:, :, 12:16, 7] = True
    assert torch.equal(out[~hit], want[~hit]) and not out[hit].isfinite().any()
    case = Case(**MANY["eight_waves"])
    case.prefix_pages[300] = case.k.shape[0]
    out, _ = case.run(B)
    assert out.isnan().all()


@pytest.mark.parametrize("dtype", ["cache", "fp32"])
@pytest.mark.parametrize("name", list(CASES))
def test_against_64_bits(B, name, dtype):
    case = Case(**CASES[name])
    print(name, dtype, B.query_shared_prefix_attention(*case.shape, case.P, max(case.lens)), flush=True)
    out, lse = case.run(B, dtype=torch.float32 if dtype == "fp32" else None, want_lse=True)
    assert out.dtype == (torch.float32 if dtype == "fp32" else case.k.dtype)
    case.check(out, lse.cpu())
    # an upper bound of the lengths that is just met: the same numbers up to how keys are parted
    tight, none = case.run(B, dtype=torch.float32 if dtype == "fp32" else None, max_own_len=max(case.lens))
    assert none is None
    case.check(tight)


def test_every_tile_is_among_the_cases(B):
    rows = {B.query_shared_prefix_attention(c["B"], c["n"], c["Hq"], c["Hk"], c["D"], c["P"], max(c["lens"]))[0] for c in [*CASES.values(), *MANY.values()]}
    assert rows == {16, 32, 128, 256}


def test_scale_and_large_scores(B):
    case = Case(B=3, n=1, Hq=4, Hk=2, D=64, P=300, lens=[10, 20, 30], page=16, spread=30.0)
    out, lse = case.run(B, dtype=torch.float32, scale=0.5, want_lse=True)
    case.check(out, lse.cpu(), scale=0.5)
    case = Case(B=40, n=1, Hq=8, Hk=2, D=64, P=300, lens=[1] * 40, page=16, spread=30.0)
    out, lse = case.run(B, dtype=torch.float32, scale=0.5, want_lse=True)
    case.check(out, lse.cpu(), scale=0.5, only=[0, 17, 39])


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("n,P", [(3, 0), (3, 40), (40, 0)])
def test_what_is_not_seen_has_no_influence(B, n, P, what):
    """Infinities and NaN in keys and values of later tokens reach the queries that see them, and no other."""
    lens = [n + 9, n + 50]
    case = Case(B=2, n=n, Hq=4, Hk=2, D=64, P=P, lens=lens, page=16)
    clean, _ = case.run(B)
    for own in case.own:
        own[0][-1], own[1][-1] = what, what                               # the last token: seen by the last query alone
    case.write()
    out, _ = case.run(B)
    assert torch.equal(out[:, :-1], clean[:, :-1])
    assert not out[:, -1].isfinite().all(-1).any()


def test_strided_and_given_tensors(B):
    Bn, n, Hq, Hk, D = 4, 2, 4, 2, 64
    case = Case(B=Bn, n=n, Hq=Hq, Hk=Hk, D=D, P=90, lens=[5, 6, 70, 8], page=16)
    want, want_lse = case.run(B, want_lse=True)
    # queries as views of wider rows, sequences behind each other in memory the other way round, tables and outputs with room between rows
    wide = torch.zeros((n, Bn, Hq * D + 6), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 2:2 + Hq * D] = case.q.transpose(0, 1).reshape(n, Bn, Hq * D)
    q = wide[:, :, 2:2 + Hq * D].unflatten(2, (Hq, D)).transpose(0, 1)
    table = torch.full((Bn, 3 * case.table.shape[1] + 1), 1 << 20, dtype=torch.int32, device="cuda")
    table[:, :case.table.shape[1]] = case.table
    room = torch.full((Bn, n, Hq, D + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    out = room[..., 4:4 + D]
    ws = torch.empty(B.shared_prefix_attention_bytes(Bn, n, Hq, Hk, D, 90, 70), dtype=torch.uint8, device="cuda")
    got, lse = B.shared_prefix_attention(q, case.k, case.v, case.prefix_pages, 90, table, case.own_lens, max_own_len=70, out=out, workspace=ws, want_lse=True)
    assert got is out
    case.check(out, lse.cpu())
    assert (room[..., :4] == 3.0).all() and (room[..., 4 + D:] == 3.0).all()
    assert torch.allclose(got.float(), want.float(), atol=0.03) and torch.allclose(lse, want_lse, atol=1e-5)


def test_lengths_and_pages_that_cannot_be_are_nan(B):
    """Found on the device; nothing outside the cache is read, and other sequences keep their results."""
    case = Case(B=4, n=2, Hq=4, Hk=2, D=64, P=50, lens=[20, 20, 20, 20], page=16)
    want, _ = case.run(B)
    other = torch.tensor([True, False, True, True], device="cuda")
    for field, value in (("own_lens", -1), ("own_lens", 33), ("own_lens", 1 << 30), ("query_lens", 3), ("query_lens", -1)):
        bad = Case(B=4, n=2, Hq=4, Hk=2, D=64, P=50, lens=[20, 20, 20, 20], page=16, queries=[2, 2, 2, 2])
        getattr(bad, field)[1] = value
        out, lse = bad.run(B, want_lse=True)
        assert out[1].isnan().all() and lse[1].isnan().all(), field
        assert torch.equal(out[other], want[other]), field
    for page in (-1, case.k.shape[0], 1 << 30):
        table = case.table.clone()
        table[1, 0] = page
        out, _ = B.shared_prefix_attention(case.q, case.k, case.v, case.prefix_pages, 50, table, case.own_lens)
        assert out[1].isnan().all() and torch.equal(out[other], want[other])
        prefix = case.prefix_pages.clone()
        prefix[1] = page
        out, _ = B.shared_prefix_attention(case.q, case.k, case.v, prefix, 50, case.table, case.own_lens)
        assert out.isnan().all()
    many = Case(B=40, n=1, Hq=8, Hk=2, D=64, P=200, lens=[3] * 40, page=16)
    many.prefix_pages[3] = -5
    out, _ = many.run(B)
    assert out.isnan().all()
    # an entry of the table that no length reaches is not looked at
    table = torch.cat([case.table, torch.full((4, 2), -7, dtype=torch.int32, device="cuda")], dim=1)
    out, _ = B.shared_prefix_attention(case.q, case.k, case.v, case.prefix_pages, 50, table, case.own_lens, max_own_len=32)
    assert torch.equal(out, want)


def test_pages_past_32_bits(B):
    """A cache of 2^33 bytes each way, whose last pages are the ones in use."""
    page, Hk, Hq, D = 64, 8, 16, 128
    pages = (1 << 32) // (page * Hk * D) + 8
    caches = [torch.empty((pages, Hk, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for Bn in (2, 70):
        case = Case(B=Bn, n=1, Hq=Hq, Hk=Hk, D=D, P=130, lens=[3] * Bn, page=page)
        used = case.k.shape[0]
        near = case.run(B)[0]
        if used <= 8:
            for c, x in zip(caches, (case.k, case.v)):
                c[-used:] = x
            out, _ = B.shared_prefix_attention(case.q, *caches, case.prefix_pages + pages - used, 130, case.table + pages - used, case.own_lens)
        else:                                                   # the prefix alone at the end
            for c, x in zip(caches, (case.k, case.v)):
                c[:used] = x
                c[-3:] = x[case.prefix_pages.long()]
            out, _ = B.shared_prefix_attention(case.q, *caches, torch.arange(pages - 3, pages, dtype=torch.int32, device="cuda"), 130, case.table, case.own_lens)
        assert torch.equal(out, near)


def test_other_stream_repeats_and_graph(B):
    for Bn in (3, 40):
        case = Case(B=Bn, n=1, Hq=8, Hk=2, D=128, P=700, lens=[1 + 9 * i for i in range(Bn)], page=16)
        want, _ = case.run(B)
        assert all(torch.equal(case.run(B)[0], want) for _ in range(3))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out, _ = case.run(B)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want)
        out = torch.empty_like(want)
        ws = torch.empty(B.shared_prefix_attention_bytes(*case.shape, 700, max(case.lens)), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            case.run(B, out=out, workspace=ws, max_own_len=max(case.lens))
        for step in range(4):
            case.q.mul_(0.8)
            case.own_lens.sub_(1 if step == 1 else 0).clamp_(min=0)       # lengths are read on the device at each replay
            ws.fill_(255)                                                 # (NaN in every float of the workspace)
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            eager, _ = case.run(B, max_own_len=max(case.lens))
            assert torch.equal(got, eager)


def test_refusals(B):
    case = Case(B=2, n=1, Hq=4, Hk=2, D=64, P=20, lens=[5, 6], page=16)
    q, k, v, pages, table, lens = case.q, case.k, case.v, case.prefix_pages, case.table, case.own_lens
    f = B.shared_prefix_attention
    for call in (lambda: f(q.cpu(), k, v, pages, 20, table, lens), lambda: f(q[0], k, v, pages, 20, table, lens), lambda: f(q, k, v[:1], pages, 20, table, lens),
                 lambda: f(q, k, v, pages.long(), 20, table, lens), lambda: f(q, k, v, pages, 33, table, lens), lambda: f(q, k, v, None, 20, table, lens),
                 lambda: f(q, k, v, pages, 20, table.long(), lens), lambda: f(q, k, v, pages, 20, table[:1], lens), lambda: f(q, k, v, pages, 20, table, lens.long()),
                 lambda: f(q, k, v, pages, 20, table, lens[:1]), lambda: f(q, k, v, pages, 20, table, lens, max_own_len=17),
                 lambda: f(q, k, v, pages, 20, None, lens, max_own_len=1), lambda: f(q, k, v, pages, 20, table, lens, query_lens=lens[:1]),
                 lambda: f(q, k, v, pages, 20, table, lens, out=torch.empty_like(q)[:1]), lambda: f(q[..., :32], k, v, pages, 20, table, lens)):
        with pytest.raises(ValueError):
            call()
    odd = torch.zeros((2, 1, 4, 65), dtype=torch.bfloat16, device="cuda")
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    for call, status in ((lambda: f(q.half(), k, v, pages, 20, table, lens), B.VLUT_ERR_SHAPE), (lambda: f(q[:, :, :3], k, v, pages, 20, table, lens), B.VLUT_ERR_SHAPE),
                         (lambda: f(q, k, v, pages, 20, table, lens, dtype=torch.float16), B.VLUT_ERR_SHAPE),
                         (lambda: f(q[:0], k, v, pages, 20, table[:0], lens[:0]), B.VLUT_ERR_SHAPE), (lambda: f(q, k, v, pages, -1, table, lens), B.VLUT_ERR_SHAPE),
                         (lambda: f(odd[..., 1:], k, v, pages, 20, table, lens), B.VLUT_ERR_UNSUPPORTED),
                         (lambda: f(q, k, v, pages, 20, table, lens, scale=0.0), B.VLUT_ERR_UNSUPPORTED),
                         (lambda: f(q, k, v, pages, 20, table, lens, scale=float("nan")), B.VLUT_ERR_UNSUPPORTED),
                         (lambda: f(q[..., :62], k[..., :62], v[..., :62], pages, 20, table, lens), B.VLUT_ERR_UNSUPPORTED),
                         (lambda: f(q, k[:, :, :12], v[:, :, :12], pages, 20, table, lens), B.VLUT_ERR_UNSUPPORTED),
                         (lambda: f(q.float(), k.float(), v.float(), pages, 20, table, lens), B.VLUT_ERR_UNSUPPORTED),
                         (lambda: f(q, k, v, pages, 20, table, lens, workspace=small), B.VLUT_ERR_SMALL_BUFFER)):
        with pytest.raises(B.VlutError) as e:
            call()
        assert e.value.status == status


def test_native_and_python_form_agree(B, monkeypatch):
    """The calls without their native form: the same numbers, to the bit."""
    if B._native is None:
        pytest.skip("built with a torch for ROCm only")
    case = Case(B=3, n=2, Hq=8, Hk=2, D=64, P=100, lens=[5, 40, 2], page=16, queries=[2, 1, 2])
    x = torch.randn((6, 12, 64), device="cuda")
    angle = torch.rand((50, 32), device="cuda")
    rotation = dict(positions=torch.arange(6, device="cuda") * 9, cos=angle.cos(), sin=angle.sin())
    weight = torch.rand(64, device="cuda")

    def run():
        k, v = (torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        slots = torch.tensor([3, -1, 17, 0, 31, 5], device="cuda")
        q = B.append_kv(x[:, 8:10], x[:, 10:], slots, k, v, q=x[:, :8], q_weight=weight, k_weight=weight, **rotation)
        return [q, k, v, *B.norm_rope(x[:, :8], x[:, 8:10], q_weight=weight, dtype=torch.float16, interleaved=True, **rotation),
                *case.run(B, dtype=torch.float32, want_lse=True, scale=0.3)]

    native = run()
    monkeypatch.setattr(B, "_native", None)
    monkeypatch.setattr(B, "_load_native", lambda L: None)
    assert all(torch.equal(a, b) for a, b in zip(native, run()))
