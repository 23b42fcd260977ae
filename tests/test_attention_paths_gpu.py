"""shared_prefix_attention on each of its paths: what one of them could lose and another keep.

A path is the kernel and the tile that a call's sizes lead to; every case says which one it is for and finds that it runs."""
from __future__ import annotations

import copy

import pytest

torch = pytest.importorskip("torch")

from test_attention_gpu import U, U32, Case  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B(vlut_lib_path):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2512_06443_amd import binding
    binding.lib()
    return binding


BF16, F16 = torch.bfloat16, torch.float16

# Rows of a workgroup (16, 32: waves that share a tile; 128, 256: a launch of its own for the prefix, four or eight waves of 32) -> sizes.
PATHS = {
    "16_d64": (16, dict(B=4, n=1, Hq=8, Hk=2, D=64, P=700, lens=[3, 0, 40, 9], page=16)),
    "16_d128": (16, dict(B=1, n=1, Hq=4, Hk=1, D=128, P=900, lens=[70], page=64)),
    "16_d200": (16, dict(B=9, n=1, Hq=8, Hk=2, D=200, P=1000, lens=[1] * 9, page=16)),
    "16_pages_of_4": (16, dict(B=4, n=1, Hq=8, Hk=2, D=96, P=700, lens=[3, 0, 40, 9], page=4)),
    "32_d64": (32, dict(B=16, n=1, Hq=32, Hk=8, D=64, P=4200, lens=[5 * i for i in range(16)], page=16)),
    "32_d100": (32, dict(B=16, n=1, Hq=32, Hk=8, D=100, P=4200, lens=[5 * i for i in range(16)], page=32)),
    "32_d128": (32, dict(B=8, n=2, Hq=32, Hk=8, D=128, P=4321, lens=[40, 2, 3, 70, 100, 31, 32, 33], page=16)),
    "32_drafts_d128": (32, dict(B=2, n=9, Hq=8, Hk=2, D=128, P=333, lens=[9, 77], page=16)),
    "128_d64": (128, dict(B=32, n=1, Hq=32, Hk=8, D=64, P=19600, lens=[3] * 32, page=16)),
    "128_d100": (128, dict(B=24, n=1, Hq=32, Hk=8, D=100, P=13100, lens=[3] * 24, page=32)),
    "128_d132": (128, dict(B=33, n=1, Hq=16, Hk=4, D=132, P=7001, lens=[3] * 33, page=16)),
    "128_d256": (128, dict(B=40, n=1, Hq=16, Hk=4, D=256, P=5600, lens=[3] * 40, page=16)),
    "256_d64": (256, dict(B=41, n=1, Hq=16, Hk=2, D=64, P=31999, lens=[1] * 41, page=128)),
    "256_d100": (256, dict(B=21, n=2, Hq=32, Hk=8, D=100, P=7501, lens=[2] * 21, page=32)),
    "256_d128": (256, dict(B=40, n=1, Hq=32, Hk=8, D=128, P=7950, lens=[4] * 40, page=16)),
}


def path(B, name, dtype, **more) -> Case:
    rows, sizes = PATHS[name]
    case = Case(**sizes, dtype=dtype, **more)
    got = B.query_shared_prefix_attention(*case.shape, case.P, case.table.shape[1] * case.page)
    assert got[0] == rows
    print(name, dtype, got, flush=True)
    return case


def per_key_head(case, x):
    """[B][n][Hq][...] -> [Hk][rows of it][...] in 64 bits."""
    Bn, n, Hq, Hk, _ = case.shape
    return x.double().unflatten(2, (Hk, Hq // Hk)).movedim(2, 0).flatten(1, 3)


def sharp_weights(case, rest=-25.0, ahead=-9.0):
    """Queries and keys of one feature: scores are single products and exact.  Every feature of V has two keys of its own, whose weights are
    e^-2 to 1 (and cancel in the odd features); all other keys are `rest`, too low to count, but for one of `ahead` in 32, ahead of the others, from which the
    largest score of any range's first keys is no further than what 32 bits' scores tell exactly.  Own tokens: `rest`."""
    Bn, n, Hq, Hk, D = case.shape
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    case.q.zero_()
    case.q[..., 0] = 1 + torch.randint(0, 8, (Bn, n, Hq), generator=gen, device="cuda") / 128
    k, v = case.prefix
    k.zero_()
    v.zero_()
    k[:, :, 0] = rest
    k[::32, :, 0] = ahead
    for own in case.own:
        own[0].zero_()
        own[0][:, :, 0] = rest
        own[1].zero_()
    for h in range(Hk):
        at = torch.randperm(case.P, generator=gen, device="cuda")[:2 * D]
        at = torch.where(at % 32 == 0, at + 1, at).clamp_(max=case.P - 1).unique()
        at = at[:at.numel() // 2 * 2]
        a, b = at[0::2], at[1::2]
        k[at, h, 0] = (-2 * torch.rand(at.numel(), generator=gen, device="cuda")).to(k.dtype)
        f = torch.arange(a.numel(), device="cuda")
        x = (1 + torch.rand(a.numel(), generator=gen, device="cuda")).to(v.dtype)
        v[a, h, f] = x
        odd = f % 2 == 1
        v[b[odd], h, f[odd]] = -x[odd]
    case.write()


def formula(case):
    """Of the prefix alone, per key head in 64 bits: (output, sum of the terms' magnitudes, log of the sum of exponentials); scale 1, scores of feature 0."""
    q = per_key_head(case, case.q)[..., 0]
    k, v = (x.double().transpose(0, 1) for x in case.prefix)
    outs = []
    for h in range(case.shape[3]):
        s = q[h][:, None] * k[h][None, :, 0]
        w = torch.softmax(s, -1)
        outs.append((w @ v[h], w @ v[h].abs(), torch.logsumexp(s, -1)))
    return [torch.stack(x) for x in zip(*outs)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", list(PATHS))
def test_weights_keep_their_bits_for_outputs_of_16_bits(B, name, dtype):
    """out * exp(lse), of which the sum of weights cancels, is off by its output's rounding and by 2^-16 (two terms of bf16; fp16 less) of its terms'
    magnitudes for the weights; by 2^-18 of those at most for all else: scores times log2(e) above a maximum within 16 (2^-20.5), an exponential (2^-23), sums of
    two keys' terms (six additions, 2^-21), parts joined (2^-21), lse (2^-20.5).  One term of bf16 alone would be 2^-9."""
    case = path(B, name, dtype)
    sharp_weights(case)
    out, lse = case.run(B, scale=1.0, want_lse=True)
    want, size, want_lse = formula(case)
    got, got_lse = per_key_head(case, out), per_key_head(case, lse)
    factor = (got_lse - want_lse).exp()[..., None]
    off = (got * factor - want).abs()
    tiny = 2.0 ** -24 if dtype == F16 else 1e-38                          # outputs below fp16's normal range
    bound = want.abs() * U[dtype] * 1.01 + size * (2.0 ** -16 + 2.0 ** -18) + tiny
    assert (off / bound).max().item() <= 1.0


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", list(PATHS))
def test_weights_keep_their_bits_for_outputs_of_fp32(B, name, dtype):
    """The same for fp32 outputs: weights in three terms of bf16 (2^-24) or two of fp16 (2^-22), 1.2 * 2^-19 of the terms' magnitudes with all else.
    Two terms of bf16 would be 2^-18 off at most, which so many weights come near."""
    case = path(B, name, dtype)
    sharp_weights(case)
    out, lse = case.run(B, scale=1.0, dtype=torch.float32, want_lse=True)
    want, size, want_lse = formula(case)
    got, got_lse = per_key_head(case, out), per_key_head(case, lse)
    off = (got * (got_lse - want_lse).exp()[..., None] - want).abs()
    worst = (off / (want.abs() * U32 + size * (1.2 * 2.0 ** -19) + 1e-38)).max().item()
    assert worst <= 1.0


def check_without(case, hidden, out, lse):
    """The formula without the keys `hidden` [P] of the prefix."""
    seen = copy.copy(case)
    seen.prefix = tuple(x[~hidden] for x in case.prefix)
    seen.P = seen.prefix[0].shape[0]
    seen.check(out, lse.cpu(), only=[0, case.shape[0] - 1])


def range_of(B, case):
    """Keys of one part of the prefix, where the prefix has a launch of its own (a multiple of 64, or of 32 over 128 features)."""
    keys, parts = 64 if case.shape[4] <= 128 else 32, B.query_shared_prefix_attention(*case.shape, case.P, case.table.shape[1] * case.page)[1]
    return -(-(-(-case.P // parts)) // keys) * keys


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", list(PATHS))
@pytest.mark.parametrize("where", ["one_range", "every_range", "all_but_one", "all"])
def test_keys_of_minus_infinity_count_for_nothing(B, name, dtype, where):
    """Keys that score -inf in front of others: of the first part alone, of every part, everywhere but at one key, everywhere.  The others as they come,
    and so low (-375 and below) that they would be nothing above any other reference than their own."""
    for low in (False, True):
        case = path(B, name, dtype)
        at, part = torch.arange(case.P, device="cuda"), range_of(B, case)
        hidden = {"one_range": at < 70, "every_range": at % part < 70, "all_but_one": at != case.P - 9, "all": at >= 0}[where]
        case.q[..., 0] = 1
        if low:
            case.prefix[0][..., 0] = -375 * case.shape[4] ** 0.5
            for own in case.own:
                own[0][..., 0] = -375 * case.shape[4] ** 0.5
        # (by an infinite key, and, in bf16, by its lowest value, whose product passes 32 bits)
        case.prefix[0][hidden, :, 0] = float("-inf")
        if dtype == BF16 and not low:
            case.q[..., 0] = 4
            case.prefix[0][hidden, :, 0] = torch.finfo(BF16).min
        case.write()
        for kind in (torch.float32, None):
            out, lse = case.run(B, dtype=kind, want_lse=True)
            assert out.isfinite().all()
            check_without(case, hidden, out, lse)


# Besides the paths above: one part, whose workgroups store the result.
ONE_PART = {
    "prefix_alone": dict(B=2, n=1, Hq=4, Hk=2, D=64, P=77, lens=[0, 0], page=16),
    "prefix_alone_d256": dict(B=3, n=2, Hq=4, Hk=1, D=256, P=128, lens=[0, 0, 0], page=4),
    "own_alone": dict(B=3, n=3, Hq=4, Hk=2, D=128, P=0, lens=[20, 37, 5], page=16),
    "own_alone_of_one_wave": dict(B=300, n=1, Hq=16, Hk=8, D=100, P=0, lens=[30 - i % 20 for i in range(300)], page=16),
    "own_alone_many_queries": dict(B=2, n=40, Hq=4, Hk=2, D=64, P=0, lens=[40, 90], page=64),
}


@pytest.mark.parametrize("kind", ["cache", "fp32"])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", [*PATHS, *ONE_PART])
def test_infinite_values_that_are_seen(B, name, dtype, kind):
    """The formula's infinities and NaN, wherever the key is, in the features of the queries that see them, and no other number changed."""
    inf, nan = float("inf"), float("nan")
    case = path(B, name, dtype) if name in PATHS else Case(**ONE_PART[name], dtype=dtype)
    Bn, n, Hq, Hk, D = case.shape
    h, G, P = Hk - 1, Hq // Hk, case.P
    case.q[..., 0] = 1
    of, length = (case.prefix, P) if P else (case.own[Bn - 1], case.lens[Bn - 1])
    of[0][2, h, 0] = -inf                                                 # a key that weighs nothing
    case.write()
    run = lambda: case.run(B, dtype=torch.float32 if kind == "fp32" else None, want_lse=True, max_own_len=max(case.lens))  # noqa: E731
    clean, clean_lse = run()
    assert clean.isfinite().all()
    # token (of those that several sequences see, where there is a prefix) and feature -> value
    last, middle = length - 1, length // 2
    given = [(1, 3, inf), (middle, 7, -inf), (middle, 11, inf), (last, 11, -inf), (1, 15, nan), (last, 19, inf), (1, 23, -inf), (last, 23, -inf), (2, 27, inf), (0, D - 1, inf)]
    want = clean.clone()
    for t, f, x in given:
        of[1][t, h, f] = x
    for b in range(Bn) if P else [Bn - 1]:
        for j in range(n):
            sees = P if P else length - n + j + 1
            for f in {f for _, f, _ in given}:
                seen = [0.0 * x if t == 2 else x for t, g, x in given if g == f and t < sees]
                if seen:
                    want[b, j, h * G:(h + 1) * G, f] = sum(seen)
    # a sequence's last own token: its last query's alone
    for b in {0, Bn // 2}:
        if P and case.lens[b] >= n:
            case.own[b][1][-1, 0, 30] = -inf
            want[b, n - 1, :G, 30] = -inf if want[b, n - 1, 0, 30].isfinite() else nan
    case.write()
    got, lse = run()
    assert torch.equal(lse, clean_lse)
    same = (got == want) | (got.isnan() & want.isnan())
    assert same.all(), (same.logical_not().nonzero()[:4].tolist(), got[~same][:4].tolist(), want[~same][:4].tolist())


def test_infinite_values_of_sequences_that_cannot_be(B):
    """Lengths out of range are NaN, whatever the prefix holds."""
    case = Case(B=3, n=1, Hq=4, Hk=2, D=64, P=77, lens=[0, 0, 0], page=16)
    case.prefix[1][3, :, 5] = float("inf")
    case.write()
    case.own_lens[1] = 17
    out, lse = case.run(B, want_lse=True)
    assert out[1].isnan().all() and lse[1].isnan().all()
    assert (out[[0, 2]][..., 5] == float("inf")).all() and out[[0, 2]][..., :5].isfinite().all() and out[[0, 2]][..., 6:].isfinite().all()


# Every kernel that is compiled for one type of the cache: features of the accumulators (64, 128, 256) filled or not, pages of 16 tokens and more or less, tiles of
# 16 rows for both parts, of 32 and 16, of 32 and 32, and 128 or 256 rows for the prefix with tiles of 16 or 32 for the own tokens.
TILES = {
    "16_16": (16, dict(B=4, n=1, Hq=8, Hk=2, P=300, lens=[3, 0, 140, 9])),
    "32_16": (32, dict(B=64, n=1, Hq=16, Hk=8, P=300, lens=[260 - 31 * i % 200 for i in range(64)])),
    "32_32": (32, dict(B=3, n=9, Hq=8, Hk=2, P=333, lens=[9, 77, 200])),
    "128_16": (128, dict(B=32, n=1, Hq=32, Hk=8, lens=[3 + 4 * i for i in range(32)])),
    "128_32": (128, dict(B=6, n=5, Hq=32, Hk=8, lens=[3, 5, 8, 13, 21, 34])),
    "256_16": (256, dict(B=40, n=1, Hq=32, Hk=8, lens=[3 + 4 * i for i in range(40)])),
    "256_32": (256, dict(B=8, n=5, Hq=32, Hk=8, lens=[3, 5, 8, 13, 21, 34, 55, 89])),
}


def instances():
    for D in (64, 48, 128, 100, 256, 200):
        for page in (16, 4):
            for tiles in ("16_16",) if D > 128 else ("16_16", "32_16", "32_32"):
                yield D, page, tiles
        for tiles in ("128_16", "128_32") if D > 128 else ("128_16", "128_32", "256_16", "256_32"):
            yield D, 16, tiles


@pytest.mark.parametrize("kind", ["cache", "fp32"])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,page,tiles", list(instances()))
def test_every_kernel_against_64_bits(B, D, page, tiles, dtype, kind):
    rows, sizes = TILES[tiles]
    sizes = dict(sizes)
    if "P" not in sizes:                                                  # long enough for a launch of its own
        own = sizes["B"] * sizes["n"] * sizes["Hq"] // sizes["Hk"] * sizes["Hk"]
        sizes["P"] = (3500000 if D > 128 else 1280000000 // (64 if D <= 64 else 128)) // own + 77
    case = Case(**sizes, D=D, page=page, dtype=dtype)
    got = B.query_shared_prefix_attention(*case.shape, case.P, max(case.lens))
    print(D, page, tiles, dtype, kind, got, flush=True)
    assert got[0] == (128 if D > 128 and rows > 128 else rows)
    out, lse = case.run(B, dtype=torch.float32 if kind == "fp32" else None, want_lse=True, max_own_len=max(case.lens))
    case.check(out, lse.cpu(), only=[0, case.shape[0] - 1])


@pytest.mark.parametrize("kind", ["cache", "fp32"])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", [name for name in PATHS if PATHS[name][0] > 32])
def test_scores_that_rise_above_a_ranges_first(B, name, dtype, kind):
    """Ranges that are worked on again with their largest score: one, the last ones, all of them."""
    for where in (slice(1000, 1001), slice(-900, -10), slice(70, None)):
        case = path(B, name, dtype)
        case.prefix[0][where] *= 40
        case.write()
        out, lse = case.run(B, dtype=torch.float32 if kind == "fp32" else None, want_lse=True)
        case.check(out, lse.cpu(), only=[0, case.shape[0] - 1])


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", ["32_d128", "32_drafts_d128", "256_d100"])
def test_own_tokens_that_are_not_seen_have_no_influence(B, name, dtype, what):
    """The last own token, seen by the last query alone, in keys and values."""
    case = path(B, name, dtype)
    some = torch.tensor([m >= case.shape[1] for m in case.lens])
    clean, clean_lse = case.run(B, want_lse=True)
    for own in case.own:
        own[0][-1], own[1][-1] = what, what
    case.write()
    out, lse = case.run(B, want_lse=True)
    assert torch.equal(out[:, :-1], clean[:, :-1]) and torch.equal(lse[:, :-1], clean_lse[:, :-1])
    assert not out[some][:, -1].isfinite().all(-1).any()


@pytest.mark.parametrize("name", list(PATHS))
def test_replays_of_a_graph(B, name):
    """The call captured once; new queries and lengths, eager work and a workspace of NaN between the replays."""
    case = path(B, name, BF16)
    bound = max(case.lens)
    want, _ = case.run(B, max_own_len=bound)
    out = torch.empty_like(want)
    ws = torch.empty(B.shared_prefix_attention_bytes(*case.shape, case.P, bound), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        case.run(B, out=out, workspace=ws, max_own_len=bound)
    for step in range(4):
        case.q.mul_(0.8)
        case.own_lens.sub_(1 if step == 1 else 0).clamp_(min=0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        eager, _ = case.run(B, max_own_len=bound)
        assert torch.equal(got, eager) and got.isfinite().all()


@pytest.mark.parametrize("name", list(PATHS))
def test_large_values_behind_low_scores(B, name):
    """Values of 2^100 whose scores are 2^33 and more above those of their range's first keys: the product of both is past 32 bits, the result is not.
    Bound: as for fp32 outputs above, with scores up to 36 from the maximum that a tile's waves begin with (2^-19 * log(2) more)."""
    case = path(B, name, BF16)
    sharp_weights(case, ahead=-25.0)
    case.prefix[1].mul_(2.0 ** 100)
    case.write()
    out, lse = case.run(B, scale=1.0, dtype=torch.float32, want_lse=True)
    want, size, want_lse = formula(case)
    got, got_lse = per_key_head(case, out), per_key_head(case, lse)
    off = (got * (got_lse - want_lse).exp()[..., None] - want).abs()
    assert (off <= want.abs() * U32 + size * (1.2 + 0.7) * 2.0 ** -19 + 1e-38).all()
