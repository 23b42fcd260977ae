"""norm_rope and append_kv against their formulas in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

# Unit roundoffs.  A value is x * inverse * weight (the sum of squares of D <= 256 products in fp32: (D + 8) * 2^-24 of the root's argument at most,
# half of it after the root, and a handful of single roundings) and two products and a sum of the rotation: below (D / 2 + 16) * 2^-24
# of |a cos| + |b sin|, then one rounding to the output's type.
U32 = 2.0 ** -24
U = {torch.float32: U32, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}      # (the smallest subnormal of fp16)


@pytest.fixture(scope="module")
def B(vlut_lib_path):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2512_06443_amd import binding
    binding.lib()
    return binding


def definition(x, weight, eps, positions, cos, sin, interleaved):
    """(the result, the sum of the magnitudes that make it up) in 64 bits on the CPU."""
    x = x.detach().cpu().double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.cpu().double()
    size = x.abs()
    if cos is not None:
        R = 2 * cos.shape[1]
        c, s = (t.cpu().double()[positions.cpu()][:, None, :] for t in (cos, sin))
        first = slice(0, R, 2) if interleaved else slice(0, R // 2)
        second = slice(1, R, 2) if interleaved else slice(R // 2, R)
        a, b = x[..., first].clone(), x[..., second].clone()
        x, size = x.clone(), size.clone()
        x[..., first], x[..., second] = a * c - b * s, b * c + a * s
        size[..., first], size[..., second] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return x, size


def near(got, want, size, D, what=""):
    got = got.cpu()
    bound = want.abs() * U[got.dtype] + size * (1 + U[got.dtype]) * ((D / 2 + 16) * U32) + TINY[got.dtype]
    off = (got.double() - want).abs()
    worst = (off / bound).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


def tables(gen, rows, R):
    angle = torch.rand((rows, R // 2), generator=gen, device="cuda") * 6.28
    return angle.cos(), angle.sin()


CASES = [  # N, Hq, Hk, D, R, in, out, norm, interleaved
    (1, 20, 5, 128, 128, torch.float32, torch.bfloat16, True, False),
    (3, 1, 1, 2, 2, torch.float32, torch.float32, True, False),
    (5, 4, 2, 64, 64, torch.bfloat16, torch.bfloat16, True, True),
    (7, 3, 3, 100, 100, torch.float32, torch.float16, True, False),
    (7, 3, 3, 100, 52, torch.float16, torch.float32, True, True),
    (33, 2, 1, 250, 250, torch.float32, torch.float32, True, False),      # pairs of single features, two units per lane
    (33, 2, 1, 250, 126, torch.bfloat16, torch.float16, True, True),
    (9, 8, 1, 256, 256, torch.float32, torch.bfloat16, True, False),
    (9, 8, 1, 256, 64, torch.float32, torch.bfloat16, False, False),
    (65, 5, 3, 96, 0, torch.float32, torch.bfloat16, True, False),        # no rotation
    (65, 5, 3, 96, 0, torch.float16, torch.float32, False, False),        # neither: a conversion
    (130, 7, 1, 6, 2, torch.float32, torch.float32, True, True),
]


@pytest.mark.parametrize("N,Hq,Hk,D,R,src,dst,norm,interleaved", CASES)
def test_norm_rope(B, N, Hq, Hk, D, R, src, dst, norm, interleaved):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N * 1000 + D)
    q = torch.randn((N, Hq, D), generator=gen, device="cuda").to(src) * 3
    k = torch.randn((N, Hk, D), generator=gen, device="cuda").to(src)
    k[0, 0] = 0                                                           # mean 0: eps alone
    qw, kw = (torch.randn((Hq, D), generator=gen, device="cuda"), torch.randn(D, generator=gen, device="cuda")) if norm else (None, None)
    cos, sin = tables(gen, 50, R) if R else (None, None)
    positions = torch.randint(0, 50, (N,), generator=gen, device="cuda") if R else None
    got = B.norm_rope(q, k, positions, cos, sin, qw, kw, eps=1e-5, interleaved=interleaved, dtype=dst)
    for g, x, w in zip(got, (q, k), (qw, kw)):
        assert g.dtype == dst and g.shape == x.shape
        near(g, *definition(x, w, 1e-5, positions, cos, sin, interleaved), D)
    alone, none = B.norm_rope(q, None, positions, cos, sin, qw, eps=1e-5, interleaved=interleaved, dtype=dst)
    assert none is None and torch.equal(alone, got[0])


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
def test_norm_rope_of_views_at_any_alignment(B, src, shift):
    """Heads of a stacked projection whose rows are padded, starting at any element; outputs into such rows."""
    N, Hq, Hk, D = 11, 6, 2, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(shift)
    rows = torch.randn((N, (Hq + 2 * Hk) * D + 7), generator=gen, device="cuda").to(src)
    q = rows[:, shift:shift + Hq * D].unflatten(1, (Hq, D))
    k = rows[:, shift + Hq * D:shift + (Hq + Hk) * D].unflatten(1, (Hk, D))
    cos, sin = tables(gen, 9, D)
    positions = torch.arange(N, device="cuda") % 9
    w = torch.randn(D + 3, generator=gen, device="cuda")[shift:shift + D]
    room = torch.full((N, Hq * D + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    q_out = room[:, shift:shift + Hq * D].unflatten(1, (Hq, D))
    got, k_got = B.norm_rope(q, k, positions, cos, sin, w, w, q_out=q_out)
    assert got is q_out
    near(q_out, *definition(q, w, 1e-6, positions, cos, sin, False), D)
    near(k_got, *definition(k, w, 1e-6, positions, cos, sin, False), D)
    edge = torch.cat([room[:, :shift], room[:, shift + Hq * D:]], dim=1)
    assert (edge == 7.0).all()
    # heads ahead of tokens in memory, and an output that is the input
    t = q.transpose(0, 1).contiguous().transpose(0, 1)
    same, _ = B.norm_rope(t, None, positions, cos, sin, w, q_out=t)
    near(same, *definition(q, w, 1e-6, positions, cos, sin, False), D)


def test_positions_outside_the_tables_are_nan(B):
    N, H, D, R = 6, 3, 64, 32
    x = torch.randn((N, H, D), device="cuda")
    angle = torch.rand((4, R // 2), device="cuda")
    positions = torch.tensor([0, 3, 4, -1, 1 << 40, 2], device="cuda")
    y, _ = B.norm_rope(x, None, positions, angle.cos(), angle.sin())
    bad = torch.tensor([False, False, True, True, True, False])
    assert torch.equal(y[..., :R].isnan().all(-1).all(-1).cpu(), bad) and torch.equal(y[..., :R].isnan().any(-1).any(-1).cpu(), bad)
    assert torch.equal(y[..., R:], x[..., R:])


@pytest.mark.parametrize("page,token_major", [(1, False), (16, False), (64, True), (8, True)])
@pytest.mark.parametrize("D,R,src,dst,norm,with_q", [
    (128, 128, torch.float32, torch.bfloat16, True, True), (100, 52, torch.float16, torch.float16, False, False),
    (64, 0, torch.bfloat16, torch.float16, True, True), (250, 250, torch.float32, torch.bfloat16, True, True)])
def test_append_kv(B, page, token_major, D, R, src, dst, norm, with_q):
    N, Hq, Hk = 45, 6, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(page + D)
    pages = -(-2 * N // page)
    shape = (pages, page, Hk, D) if token_major else (pages, Hk, page, D)
    caches = [torch.randn(shape, generator=gen, device="cuda").to(dst) for _ in range(2)]
    caches = [c.transpose(1, 2) for c in caches] if token_major else caches
    before = [c.clone() for c in caches]
    qkv = torch.randn((N, (Hq + 2 * Hk) * D), generator=gen, device="cuda").to(src)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], dim=1))
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:N].contiguous()
    slots[::7] = -1
    slots[3] = pages * page                                               # past the cache
    slots[4] = 1 << 45
    cos, sin = tables(gen, 30, R) if R else (None, None)
    positions = torch.randint(0, 30, (N,), generator=gen, device="cuda") if R else None
    kw, qw = (torch.randn((Hk, D), generator=gen, device="cuda"), torch.randn(D, generator=gen, device="cuda")) if norm else (None, None)
    got = B.append_kv(k, v, slots, *caches, positions, cos, sin, k_weight=kw, q=q if with_q else None, q_weight=qw if with_q else None)
    if with_q:
        assert got.dtype == dst
        near(got, *definition(q, qw, 1e-6, positions, cos, sin, False), D, "q")
    else:
        assert got is None
    kept = ((slots >= 0) & (slots < pages * page)).cpu()
    at = slots.cpu()[kept]
    want_k, size = definition(k, kw, 1e-6, positions, cos, sin, False)
    flat = [c.permute(0, 2, 1, 3).reshape(pages * page, Hk, D).cpu() for c in caches]
    near(flat[0][at], want_k[kept], size[kept], D, "keys")
    assert torch.equal(flat[1][at], v.cpu()[kept].to(dst))
    untouched = torch.ones(pages * page, dtype=torch.bool)
    untouched[at] = False
    for c, b in zip(flat, before):
        assert torch.equal(c[untouched], b.permute(0, 2, 1, 3).reshape(pages * page, Hk, D).cpu()[untouched])


def test_append_kv_to_slots_past_32_bits(B):
    """A cache of 2^33 bytes each way: offsets of the last pages pass 32 bits in elements."""
    page, Hk, D = 64, 8, 128
    pages = (1 << 32) // (page * Hk * D) + 2
    k_cache = torch.empty((pages, Hk, page, D), dtype=torch.bfloat16, device="cuda")
    v_cache = torch.empty((pages, Hk, page, D), dtype=torch.bfloat16, device="cuda")
    k_cache[0], v_cache[0] = 0, 0
    k, v = torch.randn((2, Hk, D), device="cuda"), torch.randn((2, Hk, D), device="cuda")
    slots = torch.tensor([pages * page - 1, (pages - 1) * page], device="cuda")
    B.append_kv(k, v, slots, k_cache, v_cache)
    for c, x in ((k_cache, k), (v_cache, v)):
        assert torch.equal(c[-1, :, -1], x[0].to(torch.bfloat16)) and torch.equal(c[-1, :, 0], x[1].to(torch.bfloat16)) and (c[0] == 0).all()


def test_heads_on_another_stream_and_in_a_graph(B):
    N, Hq, Hk, D = 20, 4, 2, 128
    x = torch.randn((N, Hq, D), device="cuda")
    kv = torch.randn((2, N, Hk, D), device="cuda")
    angle = torch.rand((N, D // 2), device="cuda")
    positions, slots = torch.arange(N, device="cuda"), torch.arange(N, device="cuda")
    caches = torch.zeros((2, 2, Hk, 16, D), dtype=torch.bfloat16, device="cuda")
    args = (kv[0], kv[1], slots, caches[0], caches[1], positions, angle.cos(), angle.sin())
    q_out = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda")
    B.append_kv(*args, q=x, q_out=q_out)
    want, want_q = caches.clone(), q_out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        caches.zero_()
        B.append_kv(*args, q=x, q_out=q_out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(caches, want) and torch.equal(q_out, want_q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.append_kv(*args, q=x, q_out=q_out)
    for scale in (1.0, 2.0, 0.5):
        x.mul_(scale)
        kv.mul_(scale)
        caches.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, got_q = caches.clone(), q_out.clone()
        B.append_kv(*args, q=x, q_out=q_out)
        assert torch.equal(caches, got) and torch.equal(q_out, got_q)


def test_refusals(B):
    x = torch.zeros((4, 2, 64), device="cuda")
    t = torch.zeros((8, 32), device="cuda")
    pos = torch.zeros(4, dtype=torch.int64, device="cuda")
    cache = torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: B.norm_rope(x.cpu()), lambda: B.norm_rope(x.double()), lambda: B.norm_rope(x[0]), lambda: B.norm_rope(x.transpose(1, 2)),
                 lambda: B.norm_rope(x, x[:3]), lambda: B.norm_rope(x, None, pos, t, None), lambda: B.norm_rope(x, None, pos.int(), t, t),
                 lambda: B.norm_rope(x, None, pos[:3], t, t), lambda: B.norm_rope(x, None, pos, t.half(), t), lambda: B.norm_rope(x, q_weight=t[0]),
                 lambda: B.norm_rope(x, q_out=x[:3]), lambda: B.append_kv(x, x, pos.int(), cache, cache), lambda: B.append_kv(x, x[:3], pos, cache, cache),
                 lambda: B.append_kv(x, x, pos, cache, cache[:1]), lambda: B.append_kv(x, x, pos, cache[..., :32], cache[..., :32]),
                 lambda: B.append_kv(x, x, pos, cache, cache, q=x[:2])):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: B.norm_rope(x[:0]), B.VLUT_ERR_SHAPE), (lambda: B.norm_rope(x[..., :63]), B.VLUT_ERR_SHAPE),
                         (lambda: B.norm_rope(x, eps=-1.0), B.VLUT_ERR_SHAPE), (lambda: B.norm_rope(x, eps=float("nan")), B.VLUT_ERR_SHAPE),
                         (lambda: B.norm_rope(x[..., :32], None, pos, t, t), B.VLUT_ERR_SHAPE),      # more features rotated than there are
                         (lambda: B.norm_rope(x, x.half()), B.VLUT_ERR_SHAPE),
                         (lambda: B.norm_rope(torch.zeros((1, 1, 258), device="cuda")), B.VLUT_ERR_SHAPE),
                         (lambda: B.append_kv(x[:, :1], x[:, :1], pos, cache, cache), B.VLUT_ERR_SHAPE),
                         (lambda: B.append_kv(x, x, pos, cache.float(), cache.float()), B.VLUT_ERR_UNSUPPORTED),
                         (lambda: B.append_kv(x, x, pos, cache[:, :, :12], cache[:, :, :12]), B.VLUT_ERR_UNSUPPORTED)):
        with pytest.raises(B.VlutError) as e:
            call()
        assert e.value.status == status


def test_no_norm_reads_no_more_than_its_row(B):
    """Infinities and NaN of one head stay in it."""
    x = torch.randn((3, 4, 64), device="cuda")
    y = x.clone()
    y[1, 2] = float("nan")
    y[2, 0, 5] = float("inf")
    w = torch.ones(64, device="cuda")
    a, _ = B.norm_rope(x, q_weight=w)
    b, _ = B.norm_rope(y, q_weight=w)
    same = torch.ones((3, 4), dtype=torch.bool, device="cuda")
    same[1, 2] = same[2, 0] = False
    assert torch.equal(a[same], b[same]) and b[1, 2].isnan().all() and b[2, 0, 5].isnan() and (np.delete(b[2, 0].cpu().numpy(), 5) == 0).all()


def test_more_heads_than_a_launch_has_threads_for(B):
    """2^24 - 1 tokens (all the same ones: a stride of 0) of five heads, four of them to a workgroup."""
    N, H, D = (1 << 24) - 1, 5, 66
    if torch.cuda.mem_get_info()[0] < 3 * N * H * D * 2:
        pytest.skip("no room")
    x = torch.randn((1, H, D), device="cuda").to(torch.bfloat16)
    w = torch.rand(D, device="cuda")
    want, _ = B.norm_rope(x, q_weight=w)
    got, _ = B.norm_rope(x.expand(N, H, D), q_weight=w)
    for part in got.split(1 << 22):
        assert (part == want).all()


def sample(N):
    """Tokens to be compared: the first, the last, and some between."""
    return torch.tensor(sorted({0, 1, N - 1, *range(5, N, max(1, N // 61))}), device="cuda")


# Rows enough (tokens * heads of 2048 workgroups with a head per group of lanes) for several heads of a token to go together: two of vectors of four, four of
# vectors of two; head counts that these do not divide.
TOGETHER = [  # N, Hq, Hk, D, R, in, out, norm, interleaved
    (6000, 7, 5, 128, 128, torch.float32, torch.bfloat16, True, False),
    (6000, 5, 1, 128, 64, torch.bfloat16, torch.bfloat16, True, True),
    (40000, 1, 1, 128, 128, torch.float32, torch.float32, False, False),
    (5000, 7, 5, 100, 100, torch.float32, torch.float16, True, False),
    (5000, 6, 3, 100, 52, torch.float16, torch.float32, True, True),
    (30000, 1, 2, 100, 0, torch.bfloat16, torch.float16, True, False),
    (3000, 9, 2, 256, 256, torch.float32, torch.bfloat16, True, False),
    (7000, 5, 7, 64, 40, torch.float16, torch.float16, False, True),
    (12000, 5, 7, 12, 12, torch.float32, torch.float32, True, False),
]


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("N,Hq,Hk,D,R,src,dst,norm,interleaved", TOGETHER)
def test_several_heads_together(B, N, Hq, Hk, D, R, src, dst, norm, interleaved, per_head):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + D)
    q, k = (torch.randn((N, H, D), generator=gen, device="cuda").to(src) for H in (Hq, Hk))
    weight = lambda H: torch.randn((H, D) if per_head else (D,), generator=gen, device="cuda") if norm else None  # noqa: E731
    qw, kw = weight(Hq), weight(Hk)
    cos, sin = tables(gen, 50, R) if R else (None, None)
    positions = torch.randint(0, 50, (N,), generator=gen, device="cuda") if R else None
    more = dict(eps=1e-5, interleaved=interleaved)
    got = B.norm_rope(q, k, positions, cos, sin, qw, kw, dtype=dst, **more)
    at = sample(N)
    for g, x, w in zip(got, (q, k), (qw, kw)):
        near(g[at], *definition(x[at], w, 1e-5, None if positions is None else positions[at], cos, sin, interleaved), D)
    few = B.norm_rope(q[:20], k[:20], None if positions is None else positions[:20], cos, sin, qw, kw, dtype=dst, **more)      # one head at a time
    assert torch.equal(few[0], got[0][:20]) and torch.equal(few[1], got[1][:20])
    same = B.norm_rope(q, k, positions, cos, sin, qw, kw, dtype=src, **more)
    B.norm_rope(q, k, positions, cos, sin, qw, kw, q_out=q, k_out=k, **more)                       # in place
    assert torch.equal(q, same[0]) and torch.equal(k, same[1])


@pytest.mark.parametrize("page,token_major", [(16, False), (64, True)])
@pytest.mark.parametrize("N,Hq,Hk,D,R,src,dst,norm,interleaved", [c for c in TOGETHER if c[6] != torch.float32])
@pytest.mark.parametrize("with_q", [False, True])
def test_append_of_several_heads_together(B, N, Hq, Hk, D, R, src, dst, norm, interleaved, page, token_major, with_q):
    N = N if with_q else max(N, -(-33000 // Hk))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + D + page)
    pages = -(-N * 9 // 8 // page)
    shape = (pages, page, Hk, D) if token_major else (pages, Hk, page, D)
    caches = [torch.randn(shape, generator=gen, device="cuda").to(dst) for _ in range(2)]
    caches = [c.transpose(1, 2) for c in caches] if token_major else caches
    before = [c.clone() for c in caches]
    qkv = torch.randn((N, (Hq + 2 * Hk) * D), generator=gen, device="cuda").to(src)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], dim=1))
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:N].contiguous()
    slots[::7] = -1
    slots[3], slots[4], slots[N - 2] = pages * page, 1 << 45, -(1 << 40)
    cos, sin = tables(gen, 30, R) if R else (None, None)
    positions = torch.randint(0, 30, (N,), generator=gen, device="cuda") if R else None
    kw, qw = (torch.randn((Hk, D), generator=gen, device="cuda"), torch.randn(D, generator=gen, device="cuda")) if norm else (None, None)
    got = B.append_kv(k, v, slots, *caches, positions, cos, sin, k_weight=kw, interleaved=interleaved, q=q if with_q else None, q_weight=qw if with_q else None)
    at = sample(N)
    if with_q:
        near(got[at], *definition(q[at], qw, 1e-6, None if positions is None else positions[at], cos, sin, interleaved), D, "q")
    kept = (slots >= 0) & (slots < pages * page)
    flat = [c.permute(0, 2, 1, 3).reshape(pages * page, Hk, D) for c in caches]
    at = at[kept[at]]
    near(flat[0][slots[at]], *definition(k[at], kw, 1e-6, None if positions is None else positions[at], cos, sin, interleaved), D, "keys")
    keys = B.norm_rope(k, None, positions, cos, sin, kw, interleaved=interleaved, dtype=dst)[0]      # all of them, by the other call
    assert torch.equal(flat[0][slots[kept]], keys[kept]) and torch.equal(flat[1][slots[kept]], v[kept].to(dst))
    untouched = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    untouched[slots[kept]] = False
    for c, b in zip(flat, before):
        assert torch.equal(c[untouched], b.permute(0, 2, 1, 3).reshape(pages * page, Hk, D)[untouched])
