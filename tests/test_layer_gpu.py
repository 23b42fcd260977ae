"""Norms before and after a block with its gate and residual, and log probabilities of logits, against their formulas in 64 bits."""
from __future__ import annotations

import itertools
import math

import pytest
import torch

from paper_2512_06443_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24                              # half a step of fp32, relative
EPS = 1e-6
# Half a step of an output, relative, and of its smallest numbers.
HALF = {t: torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}
TINY = {t: torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}
INF, NAN = math.inf, math.nan


@pytest.fixture(autouse=True)
def device():
    torch.cuda.set_device(0)


def act(x, name):
    return {None: lambda: x, "sigmoid": lambda: torch.sigmoid(x), "silu": lambda: x * torch.sigmoid(x), "relu2": lambda: torch.relu(x) ** 2,
            "gelu": lambda: 0.5 * x * torch.special.erfc(x * -math.sqrt(0.5))}[name]()


def act_error(x, name):
    """Of act(x), relative: a few roundings; of gelu erfc's 16 steps and the rounding of its argument, which the tail's slope x^2 lifts."""
    return U * (40 + 2 * x * x) if name == "gelu" else 8 * U


# The sum of squares: up to 32 terms in a thread, 6 exchanges, 16 waves, one after the other: 54 roundings, halved by the root; 5 more of products.
NORM = 32 * U


def rms(x, weight):
    return x if weight is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.double()


def inverse(x):
    return 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)


def check(got, want, error, what=""):
    """error: of the fp32 value ahead of its one rounding."""
    bound = error * 1.01 + HALF[got.dtype] * (want.abs() + error) + TINY[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what}: {(off / bound).max().item()} of the bound"


def check_residual(y, r, weight, gate, activation, scale, next_weight, h, x):
    y64, r64 = y.double(), r.double()
    t = rms(y64, weight)
    g = act(gate.double(), activation) if gate is not None else torch.ones_like(t)
    s = scale * t * g
    h64 = r64 + s
    error = s.abs() * (NORM + 3 * U + (act_error(gate.double(), activation) if gate is not None else 0)) + U * h64.abs()
    check(h, h64, error, "h")
    if next_weight is None:
        assert x is None
        return
    x64 = rms(h64, next_weight)
    # an error of h moves its own feature, and by the norm all of them: sum(h error) / sum(h^2) of each
    moved = (h64.abs() * error).sum(-1, keepdim=True) / (h64 * h64).sum(-1, keepdim=True).clamp(min=1e-300)
    check(x, x64, (inverse(h64) * next_weight.double()).abs() * error + x64.abs() * (NORM + moved), "x")


def weights(K, gen, on=True):
    return (1.0 + 0.1 * torch.randn(K, generator=gen, device="cuda")) if on else None


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


SIZES = [(1, 1), (3, 7), (1, 2560), (5, 33), (2, 1037), (640, 128), (530, 2052), (9, 4096), (2, 8640), (3, 14336), (2, 16388), (2, 32768), (2, 32766)]


@pytest.mark.parametrize("N,K", SIZES)
@pytest.mark.parametrize("src,res,dst", [(F32, F32, F32), (BF16, BF16, BF16), (F16, F32, F16), (F32, BF16, F16), (BF16, F32, F32), (F16, F16, BF16), (F32, F16, F32),
                                         (BF16, F16, F16), (F16, BF16, F32)])
def test_residual_norm_of_every_size_and_type(N, K, src, res, dst):
    gen = generator(N * 7 + K)
    new = lambda dtype: torch.randn(N, K, generator=gen, device="cuda").to(dtype)  # noqa: E731
    y, r = new(src), 3 * new(res)
    for norm, gate, activation, following in ((True, new(src), "sigmoid", True), (False, None, None, True), (True, weights(K, gen), None, False)):
        w, nw = weights(K, gen, norm), weights(K, gen, following)
        h, x = B.residual_norm(y, r, weight=w, gate=gate, activation=activation, scale=0.5, next_weight=nw, eps=EPS, dtype=dst)
        assert h.dtype == res and (x is None or x.dtype == dst)
        check_residual(y, r, w, gate, activation, 0.5, nw, h, x)


@pytest.mark.parametrize("N,K", SIZES)
@pytest.mark.parametrize("src,dst", list(itertools.product((F32, BF16, F16), repeat=2)))
@pytest.mark.parametrize("activation", [None, "sigmoid", "silu", "relu2", "gelu"])
def test_gated_norm_of_every_size_and_type(N, K, src, dst, activation):
    gen = generator(N * 5 + K)
    both = torch.randn(N, 2 * K, generator=gen, device="cuda").mul_(2).to(src)
    gate, up = both.split(K, dim=1)
    for g, weight in ((gate, weights(K, gen)), (gate, None), (None, weights(K, gen)), (gate[0], None)):
        out = B.gated_norm(up, g, activation=activation, weight=weight, eps=EPS, dtype=dst)
        a = act((up if g is None else g).double(), activation)
        t = a if g is None else a * up.double()
        error = t.abs() * (act_error((up if g is None else g).double(), activation) + U)
        want = rms(t, weight)
        if weight is not None:
            moved = (t.abs() * error).sum(-1, keepdim=True) / (t * t).sum(-1, keepdim=True).clamp(min=1e-300)
            error = (inverse(t) * weight.double()).abs() * error + want.abs() * (NORM + moved)
        check(out, want, error)


def test_rows_strides_alignment_and_in_place():
    gen = generator(3)
    N, K = 37, 1000
    for shift, pad in ((0, 0), (1, 0), (0, 1), (2, 2), (4, 4), (3, 5)):
        wide = lambda dtype: torch.randn(N * (K + pad) + shift, generator=gen, device="cuda").to(dtype)[shift:].unflatten(0, (N, K + pad))[:, :K]  # noqa: E731
        y, r, gate = wide(BF16), wide(F32), wide(BF16)
        w, nw = weights(K + shift, gen)[shift:], weights(K + shift, gen)[shift:]
        h, x = B.residual_norm(y, r, w, gate, "silu", 1.0, nw, EPS, F32)
        check_residual(y, r, w, gate, "silu", 1.0, nw, h, x)
        outer = torch.full((N, K + pad + 3), 7.0, device="cuda", dtype=F32)
        r2, y2 = r.clone(), y.clone()
        h2, x2 = B.residual_norm(y2, r2, w, gate, "silu", 1.0, nw, EPS, out=r2, next_out=outer[:, 3:3 + K])
        # (an output at an odd place is worked on in single features, whose squares are added in another order: no bits to compare)
        check_residual(y, r, w, gate, "silu", 1.0, nw, h2, outer[:, 3:3 + K])
        assert h2 is r2 and bool((outer[:, :3] == 7).all() and (outer[:, 3 + K:] == 7).all())
        _, x3 = B.residual_norm(y2, r, w, gate, "silu", 1.0, nw, EPS, next_out=y2)
        check_residual(y, r, w, gate, "silu", 1.0, nw, h, x3)
        assert x3 is y2
        up = y.clone()
        assert torch.equal(B.gated_norm(y, gate, weight=w), B.gated_norm(up, gate, weight=w, out=up))


def test_rows_of_other_numbers():
    """Zeros are normed to zeros; what is no number stays in its row."""
    gen = generator(4)
    y = torch.randn(8, 600, generator=gen, device="cuda")
    y[1] = 0
    y[2, 5] = NAN
    y[3, 599] = INF
    r, w = torch.zeros_like(y), torch.ones(600, device="cuda")
    h, x = B.residual_norm(y, r, weight=w, next_weight=w)
    clean = [0, 4, 5, 6, 7]
    check_residual(y[clean], r[clean], w, None, None, 1.0, w, h[clean], x[clean])
    assert bool((h[1] == 0).all() and (x[1] == 0).all()) and bool(h[2].isnan().all() and x[2].isnan().all() and x[3].isnan().all())
    big = torch.full((2, 64), 1e4, device="cuda", dtype=F16)
    assert bool((B.gated_norm(big, big, activation=None) == INF).all())       # rounded as the type does
    out = B.gated_norm(torch.tensor([[-200.0, -20.0, 0.0, 20.0, 200.0, INF, -INF, NAN]], device="cuda"), activation="silu")       # (20 / (1 + exp(-20)) is 20 in 24 bits)
    assert out[0, 2:6].tolist() == [0.0, 20.0, 200.0, INF] and abs(out[0, 0]) == 0 and bool(out[0, 7].isnan())
    out = B.gated_norm(torch.tensor([[-200.0, -INF, INF, NAN, 3.0]], device="cuda"), activation="relu2")
    assert out[0, :3].tolist() == [0.0, 0.0, INF] and bool(out[0, 3].isnan()) and out[0, 4] == 9


def test_rows_past_32_bits():
    """Rows whose offsets pass 2^31 elements (strides; nothing between them is touched)."""
    base = torch.zeros(2 ** 31 + 5000, dtype=BF16, device="cuda")
    y = base.as_strided((3, 256), (2 ** 30 + 8, 1))
    y.copy_(torch.randn(3, 256, generator=generator(5), device="cuda"))
    w = torch.ones(256, device="cuda")
    before = base.sum(dtype=torch.float64)
    check(B.gated_norm(y, weight=w, activation=None, dtype=F32), rms(y.double(), w), rms(y.double(), w).abs() * NORM)
    logits = y[:, :250]
    got = B.token_logprobs(logits, torch.tensor([3, 4, 5], device="cuda"))
    check_logprobs(logits, torch.tensor([3, 4, 5], device="cuda"), 0, 1.0, got)
    assert base.sum(dtype=torch.float64) == before


# ---- log probabilities
def check_logprobs(logits, tokens, top, temperature, got):
    """Errors in units of U: an exponent u (in nats below the maximum) is off by 2 u + 2, so that the weighted mean of that and of the sum's own roundings is what
    log l has; a thread adds at most V / 256 terms one after the other in each part (and 32 parts' worth of exchanges)."""
    N, V = logits.shape
    z = logits.double() / temperature
    m = z.amax(-1, keepdim=True)
    none = m == -INF                        # nothing is allowed: log probabilities of -inf, an entropy of 0
    m = torch.where(none, 0.0, m)
    e = torch.exp(z - m)
    l = torch.where(none[:, 0], 1.0, e.sum(-1))
    u = torch.where(e > 0, m - z, 0.0)
    mean, square = (e * u).sum(-1) / l, (e * u * u).sum(-1) / l
    lse = l.log()
    serial = V / 256 + 90
    of_log = U * (2 * mean + 4 + serial)
    lp, entropy, ids, lps = got
    if tokens is not None:
        want = z.gather(1, tokens[:, None])[:, 0] - m[:, 0] - lse
        finite = want >= -torch.finfo(F32).max          # (past that it is -inf in 32 bits)
        assert bool((lp[~finite] == -INF).all())
        off = (lp.double() - want).abs()[finite]
        assert bool((off <= (of_log + 6 * U * (want.abs() + lse))[finite]).all()), off.max()
    if entropy is not None:
        want = lse + mean
        assert bool(((entropy.double() - want).abs() <= of_log + U * (2 * square + (serial + 10) * mean + 6 * want)).all())
    if top:
        order = torch.sort(logits.double(), dim=-1, descending=True, stable=True).indices[:, :top]
        assert ids.dtype == torch.int64 and torch.equal(ids, order)
        want = z.gather(1, order) - m - lse[:, None]
        finite = want >= -torch.finfo(F32).max          # (past that it is -inf in 32 bits)
        assert bool((lps[~finite] == -INF).all())
        assert bool(((lps.double() - want).abs() <= of_log[:, None] + 6 * U * (want.abs() + lse[:, None]))[finite].all())
    else:
        assert ids is None and lps is None


def logits_of(kind, N, V, dtype, gen):
    x = torch.randn(N, V, generator=gen, device="cuda") * 3
    if kind == "peaked":
        x.scatter_(1, torch.randint(0, V, (N, 1), generator=gen, device="cuda"), 40.0)
    elif kind == "equal":
        x = torch.full_like(x, 2.5)
    elif kind == "few":                     # a handful allowed, far apart
        keep = torch.randint(0, V, (N, 4), generator=gen, device="cuda")
        x = torch.full_like(x, -INF).scatter_(1, keep, x.gather(1, keep))
    elif kind == "steps":                   # many ties
        x = (x * 1.5).round()
    elif kind == "rising":
        x = torch.arange(V, device="cuda").float().expand(N, V) * (50.0 / V)
    elif kind == "falling":
        x = torch.arange(V, 0, -1, device="cuda").float().expand(N, V) * (50.0 / V)
    elif kind == "half":
        x[:, V // 2:] = -INF
    elif kind == "lowest":                  # masked by the type's lowest value; of some rows everything is
        low = torch.finfo(dtype).min
        x[:, V // 3:] = low
        x[::2] = low
    elif kind == "far":
        x = x * 1e3 + 1e5
    return x.to(dtype)


@pytest.mark.parametrize("kind", ["normal", "peaked", "equal", "few", "steps", "rising", "falling", "half", "lowest", "far"])
@pytest.mark.parametrize("N,V", [(1, 1), (2, 5), (3, 64), (1, 300), (5, 2048), (2, 2049), (3, 9001), (1, 32000), (2, 50001), (70, 32000), (300, 12288), (1100, 1500), (1025, 8196),
                                 (1, 128000), (1, 270000)])
def test_token_logprobs(kind, N, V):
    gen = generator(N + V)
    for dtype, temperature in ((F32, 1.0), (BF16, 0.7), (F16, 1.6)):
        if dtype == F16 and kind == "far":
            continue
        logits = logits_of(kind, N, V, dtype, gen)
        tokens = torch.randint(0, V, (N,), generator=gen, device="cuda")
        for top in sorted({0, 1, min(V, 20), min(V, 64)}):
            check_logprobs(logits, tokens, top, temperature, B.token_logprobs(logits, tokens, top=top, temperature=temperature))


def test_token_logprobs_strides_wants_and_odd_tokens():
    gen = generator(8)
    wide = torch.randn(6, 5003, generator=gen, device="cuda")
    tokens = torch.randint(0, 4000, (6,), generator=gen, device="cuda")
    for first in (0, 1, 2, 4):
        logits = wide[:, first:first + 4000]
        check_logprobs(logits, tokens, 7, 1.0, B.token_logprobs(logits, tokens, top=7))
    logits = wide[:, :4000]
    full = B.token_logprobs(logits, tokens, top=7)
    alone = B.token_logprobs(logits, top=7, want_entropy=False)
    assert alone[0] is None and alone[1] is None and torch.equal(alone[2], full[2]) and torch.equal(alone[3], full[3])
    assert torch.equal(B.token_logprobs(logits, tokens, want_entropy=False)[0], full[0])
    odd = tokens.clone()
    odd[0], odd[1], odd[2], odd[3] = -1, 4000, 2 ** 40, -2 ** 40
    lp = B.token_logprobs(logits, odd)[0]
    assert bool(lp[:4].isnan().all()) and torch.equal(lp[4:], full[0][4:])


@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_token_logprobs_of_rows_that_allow_nothing_or_hold_no_numbers(V):
    x = torch.randn(8, V, generator=generator(V), device="cuda")
    x[1] = -INF
    x[2, 7] = NAN
    x[3, 8] = INF
    x[4] = -INF
    x[4, V - 1] = -3e38                      # the only one, far down
    x[5, 3:] = -INF
    x[6] = NAN
    tokens = torch.full((8,), V - 1, device="cuda")
    lp, entropy, ids, lps = B.token_logprobs(x, tokens, top=20)
    clean = [0, 7]
    check_logprobs(x[clean], tokens[clean], 20, 1.0, (lp[clean], entropy[clean], ids[clean], lps[clean]))
    assert lp[1] == -INF and entropy[1] == 0 and ids[1].tolist() == list(range(20)) and bool((lps[1] == -INF).all())
    for row in (2, 3, 6):
        assert bool(lp[row].isnan() and entropy[row].isnan() and lps[row].isnan().all())
    assert ids[3, 0] == 8 and 7 not in ids[2].tolist()[:19] and ids[6].tolist() == list(range(20))
    assert lp[4] == 0 and entropy[4] == 0 and ids[4].tolist() == [V - 1] + list(range(19)) and lps[4, 0] == 0 and bool((lps[4, 1:] == -INF).all())
    assert sorted(ids[5, :3].tolist()) == [0, 1, 2] and ids[5, 3:].tolist() == list(range(3, 20)) and abs(lps[5, :3].double().exp().sum().item() - 1) < 1e-6


def test_layer_calls_in_a_graph_and_on_another_stream():
    gen = generator(11)
    y, r = torch.randn(65, 2560, generator=gen, device="cuda"), torch.randn(65, 2560, generator=gen, device="cuda")
    w = weights(2560, gen)
    logits, tokens = torch.randn(5, 70001, generator=gen, device="cuda"), torch.arange(5, device="cuda")

    def everything():
        h, x = B.residual_norm(y, r, w, None, None, 0.5, w)
        return [h, x, B.gated_norm(x, h, weight=w, dtype=BF16), *B.token_logprobs(logits, tokens, top=9)]

    first = everything()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = everything()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = everything()
    for turn in range(4):
        y.add_(0.25)
        logits.mul_(0.9)
        want = everything()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, captured)), turn


def test_the_native_form_and_the_python_form_agree(monkeypatch):
    gen = generator(12)
    y, r, w = torch.randn(9, 640, generator=gen, device="cuda").to(BF16), torch.randn(9, 640, generator=gen, device="cuda"), weights(640, gen)
    calls = [lambda: B.residual_norm(y, r, w, y, "sigmoid", 0.5, w, 1e-5, F32), lambda: B.residual_norm(y, r), lambda: B.residual_norm(y, r, gate=w),
             lambda: [B.gated_norm(y, w.to(BF16), "gelu", w, 1e-5, F32)], lambda: B.token_logprobs(r, top=3), lambda: B.token_logprobs(y, torch.arange(9, device="cuda"), 5, 0.5)]
    native = [c() for c in calls]
    assert B._native is not None
    monkeypatch.setattr(B, "_native", None)
    for a, b in zip(native, [c() for c in calls]):
        assert all((s is None and t is None) or torch.equal(s, t) for s, t in zip(a, b))
