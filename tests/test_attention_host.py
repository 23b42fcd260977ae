"""Heads, paged append and shared-prefix attention on the host: argument errors ahead of any device call, sizes and plans, the native form's refusals.
(There is no GPU here: a call that got as far as a launch would report VLUT_ERR_DEVICE.)"""
from __future__ import annotations

import ctypes
import itertools
import math

import pytest
import torch

from paper_2512_06443_amd import binding as B

P = 1 << 20                                                               # an address that nobody reads
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L(vlut_lib_path):
    return B.lib()


def heads(data=P, weight=None, token=64 * 8, head=64, weight_stride=0, n=8, type=1):
    return B._Heads(data, weight, token, head, weight_stride, n, type)


def cache(k=P, v=P, pages=10, page_size=16, strides=(8 * 16 * 64, 16 * 64, 64), n=8, type=1, v_strides=None):
    return B._Cache(k, v, pages, page_size, *strides, *(v_strides or strides), n, type)


def rotation(cos=P, sin=P, positions=P, rows=100, features=64, interleaved=0):
    return B._Rotation(cos, sin, positions, rows, features, interleaved)


def ref(s):
    return None if s is None else ctypes.byref(s)


def norm_rope(L, q=heads(), k=None, eps=1e-6, rot=None, N=4, D=64, q_out=heads(), k_out=None):
    return L.vlut_norm_rope(ref(q), ref(k), eps, ref(rot), N, D, ref(q_out), ref(k_out), None)


def append(L, k=heads(), v=heads(), q=None, eps=1e-6, rot=None, slots=P, N=4, D=64, c=cache(), q_out=None):
    return L.vlut_append_kv(ref(k), ref(v), ref(q), eps, ref(rot), slots, N, D, ref(c), ref(q_out), None)


def attend(L, q=heads(n=16), stride=64 * 16, c=cache(), prefix=P, prefix_len=40, table=P, lens=P, max_own=20, queries=None, Bn=2, n=1, D=64, scale=0.125,
           out=heads(n=16), lse=None, ws=P, ws_bytes=1 << 40):
    return L.vlut_shared_prefix_attention(ref(q), stride, ref(c), prefix, prefix_len, table, 3, lens, max_own, queries, Bn, n, D, scale, ref(out), stride, lse, ws,
                                          ws_bytes, None)


def test_the_calls_that_are_changed_one_by_one_below_are_accepted(L):
    if torch.cuda.is_available():
        pytest.skip("addresses of nothing")
    assert norm_rope(L) == append(L) == attend(L) == B.VLUT_ERR_DEVICE


def test_norm_rope_refusals(L):
    null, shape = B.VLUT_ERR_NULL, B.VLUT_ERR_SHAPE
    for more in (dict(q=None), dict(q_out=None), dict(k=heads()), dict(k_out=heads()), dict(q=heads(data=None)), dict(q_out=heads(data=None)),
                 dict(rot=rotation(cos=None)), dict(rot=rotation(sin=None)), dict(rot=rotation(positions=None))):
        assert norm_rope(L, **more) == null, more
    for more in (dict(N=0), dict(N=-1), dict(N=1 << 24), dict(D=0), dict(D=1), dict(D=63), dict(D=258), dict(eps=-1e-6), dict(eps=NAN), dict(q=heads(n=0)),
                 dict(q=heads(n=1 << 16)), dict(q=heads(type=3)), dict(q=heads(type=-1)), dict(q_out=heads(type=7)), dict(q_out=heads(n=7)),
                 dict(k=heads(type=0), k_out=heads()), dict(k=heads(), k_out=heads(type=0)), dict(k=heads(n=3), k_out=heads(n=2)),
                 dict(rot=rotation(features=66)), dict(rot=rotation(features=63)), dict(rot=rotation(features=0)), dict(rot=rotation(rows=0)),
                 dict(N=(1 << 24) - 1, q=heads(n=200), q_out=heads(n=200))):
        assert norm_rope(L, **more) == shape, more


def test_append_kv_refusals(L):
    for more in (dict(k=None), dict(v=None), dict(slots=None), dict(c=None), dict(c=cache(k=None)), dict(c=cache(v=None)), dict(q=heads()), dict(q_out=heads()),
                 dict(k=heads(data=None)), dict(v=heads(data=None)), dict(rot=rotation(positions=None))):
        assert append(L, **more) == B.VLUT_ERR_NULL, more
    for more in (dict(N=0), dict(D=65), dict(k=heads(n=7)), dict(v=heads(n=9)), dict(v=heads(type=0)), dict(q=heads(type=0), q_out=heads()),
                 dict(q=heads(n=32), q_out=heads(n=31)), dict(q=heads(), q_out=heads(type=2)), dict(c=cache(pages=0)), dict(c=cache(n=0)), dict(c=cache(page_size=0)),
                 dict(eps=-INF), dict(rot=rotation(rows=-1))):
        assert append(L, **more) == B.VLUT_ERR_SHAPE, more
    for more in (dict(c=cache(page_size=12)), dict(c=cache(page_size=1 << 17)), dict(c=cache(type=0)), dict(c=cache(type=5))):
        assert append(L, **more) == B.VLUT_ERR_UNSUPPORTED, more


def test_attention_refusals(L):
    for more in (dict(q=None), dict(out=None), dict(c=None), dict(c=cache(k=None)), dict(q=heads(data=None, n=16)), dict(out=heads(data=None, n=16)), dict(lens=None),
                 dict(prefix=None), dict(table=None), dict(ws=None)):
        assert attend(L, **more) == B.VLUT_ERR_NULL, more
    for more in (dict(Bn=0), dict(n=0), dict(Bn=1 << 24), dict(n=1 << 24), dict(prefix_len=-1), dict(max_own=-1), dict(prefix_len=1 << 30), dict(max_own=1 << 30),
                 dict(D=0), dict(q=heads(n=12), out=heads(n=12)), dict(q=heads(n=15), out=heads(n=15)), dict(out=heads(n=8)), dict(q=heads(n=16, type=2)),
                 dict(out=heads(n=16, type=2)), dict(c=cache(n=0)), dict(c=cache(pages=1 << 31)), dict(Bn=1 << 20, n=1 << 10)):
        assert attend(L, **more) == B.VLUT_ERR_SHAPE, more
    for more in (dict(D=4), dict(D=66), dict(D=260), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(c=cache(page_size=24)),
                 dict(c=cache(type=0), q=heads(n=16, type=0)), dict(q=heads(data=P + 2, n=16)), dict(q=heads(n=16, head=65)), dict(q=heads(n=16, token=1025)),
                 dict(stride=1025), dict(out=heads(n=16, head=65)), dict(out=heads(data=P + 2, n=16)), dict(c=cache(k=P + 2)), dict(c=cache(v=P + 2)),
                 dict(c=cache(strides=(8193, 1024, 64))), dict(c=cache(strides=(8192, 1023, 64))), dict(c=cache(v_strides=(8192, 1024, 65))), dict(ws=P + 8)):
        assert attend(L, **more) == B.VLUT_ERR_UNSUPPORTED, more
    need = B.shared_prefix_attention_bytes(2, 1, 16, 8, 64, 40, 20)
    assert need > 0 and attend(L, ws_bytes=63) == B.VLUT_ERR_SMALL_BUFFER
    assert attend(L, out=heads(data=P + 4, n=16, head=65, type=0), ws=P + 8) == B.VLUT_ERR_UNSUPPORTED      # (of the workspace alone: fp32 rows start at any float)


SHAPES = [*itertools.product((1, 2, 31, 64, 256), (1, 5), ((8, 1), (20, 5), (32, 32), (7, 7)), (8, 64, 100, 128, 256), (0, 1, 500, 8192, 1 << 20), (0, 1, 300, 70000))]


def test_plans_and_workspaces(L):
    """Every shape has a plan whose parts are in the workspace that is asked for, and whose workgroups are neither none nor many rounds."""
    for Bn, n, (Hq, Hk), D, prefix, own in SHAPES:
        rows, prefix_parts, own_parts, groups = B.query_shared_prefix_attention(Bn, n, Hq, Hk, D, prefix, own)
        all_rows, parts = Bn * n * Hq, prefix_parts + own_parts
        case = (Bn, n, Hq, Hk, D, prefix, own)
        assert rows in (16, 32, 128, 256) and parts >= 1 and groups >= 1, case
        assert (prefix_parts == 0) == (prefix == 0) and (own_parts == 0) <= (own == 0), case
        assert prefix_parts <= math.ceil(prefix / 128) and own_parts <= max(1, math.ceil(own / 32)), case
        need = B.shared_prefix_attention_bytes(Bn, n, Hq, Hk, D, prefix, own)
        if parts > 1:
            assert need >= all_rows * parts * (D * 4 + 8), case
        assert need <= all_rows * 2048 * (D * 4 + 8) + 4096, case
    for bad in ((0, 1, 8, 1, 64, 1, 1), (1, 1, 8, 3, 64, 1, 1), (1, 1, 8, 1, 66, 1, 1), (1, 1, 8, 1, 64, -1, 1)):
        assert B.shared_prefix_attention_bytes(*bad) == 0
        with pytest.raises(B.VlutError):
            B.query_shared_prefix_attention(*bad)
    assert L.vlut_query_shared_prefix_attention(1, 1, 8, 1, 64, 1, 1, None) == B.VLUT_ERR_NULL


def test_python_form_refuses_what_is_not_on_the_gpu(L):
    x, c = torch.zeros(2, 4, 8, dtype=torch.bfloat16), torch.zeros(3, 4, 16, 8, dtype=torch.bfloat16)
    one, slots = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: B.norm_rope(x), lambda: B.append_kv(x, x, slots, c, c), lambda: B.shared_prefix_attention(x[:, None], c, c, None, 0, None, one)):
        with pytest.raises(ValueError):
            call()


def test_native_form_declines_what_it_does_not_know(L):
    if B._native is None:
        pytest.skip("built with a torch for ROCm only")
    n, x, c = B._native, torch.zeros(2, 4, 8, dtype=torch.bfloat16), torch.zeros(3, 4, 16, 8, dtype=torch.bfloat16)
    one, slots = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    assert n.norm_rope(x, None, None, None, None, None, None, 1e-6, False, None, None, None) is None
    assert n.norm_rope(x) is None and n.norm_rope("x", *[None] * 11) is None
    assert n.append_kv(x, x, slots, c, c, None, None, None, None, 1e-6, False, None, None, None) is None
    assert n.append_kv(x, x) is None
    assert n.shared_prefix_attention(x[:, None], c, c, None, 0, None, one, None, None, None, None, None, False, None) is None
    assert n.shared_prefix_attention() is None
    with pytest.raises(TypeError):
        n.bind_attention(1)


def parts_of(L, Bn, n, Hq, Hk, D, prefix, own, page_size):
    """Parts of a call over such a cache, prefix and own tokens together, by the workspace that it asks for (0: a single one)."""
    rows = Bn * n * Hq
    c = cache(page_size=page_size, strides=(Hk * page_size * D, page_size * D, D), n=Hk)
    q = heads(token=Hq * D, head=D, n=Hq)
    call = lambda size: attend(L, q=q, out=q, stride=n * Hq * D, c=c, prefix_len=prefix, max_own=own, Bn=Bn, n=n, D=D, ws=P if size else None, ws_bytes=size)  # noqa: E731
    if call(0) != B.VLUT_ERR_NULL:
        return 0
    low, high = 0, 4096                                                   # parts; the workspace of `high` is enough, that of `low` is not
    need = lambda parts: (rows * parts * D * 4 + 255) // 256 * 256 + rows * parts * 8  # noqa: E731
    assert call(need(high)) == B.VLUT_ERR_DEVICE
    while high - low > 1:
        middle = (low + high) // 2
        low, high = (middle, high) if call(need(middle)) == B.VLUT_ERR_SMALL_BUFFER else (low, middle)
    return high


# Sizes at which a part of the prefix would have more keys than 32 bits hold if it went by the work of all rows alone.
LARGE = [(1, 2097152, 1, 1, 128, 1, 33554304), (1, 1048576, 32, 8, 128, 1, 1048576), (1, 1 << 20, 32, 8, 128, 100, 1 << 20), (16, 1 << 16, 32, 8, 128, 1, 1 << 16),
         (1, 1, 65535, 65535, 128, 1 << 20, 1), (1, 1, 60000, 60000, 8, (1 << 30) - 1, 0), (2, 1 << 19, 8, 8, 64, 1000, (1 << 30) - 1)]


@pytest.mark.parametrize("page_size", [1, 8, 16, 64])
@pytest.mark.parametrize("sizes", LARGE)
def test_plans_of_many_rows_and_long_ranges(L, sizes, page_size):
    """Each has its prefix among its parts, for pages of any size."""
    if torch.cuda.is_available():
        pytest.skip("addresses of nothing")
    Bn, n, Hq, Hk, D, prefix, own = sizes
    need = B.shared_prefix_attention_bytes(*sizes)
    parts = parts_of(L, *sizes, page_size)
    assert (parts >= 2) if own else (parts == 0 or parts >= 2)
    assert parts <= math.ceil(prefix / 128) + max(1, math.ceil(own / 32))
    assert need >= Bn * n * Hq * parts * (D * 4 + 8)
    rows, prefix_parts, own_parts, groups = B.query_shared_prefix_attention(*sizes)
    assert prefix_parts >= 1 and own_parts >= (own > 0) and groups >= 1


def test_attention_refuses_more_than_a_launch_or_64_bits_hold(L):
    """Workgroups of 256 threads past 2^32 threads, by own ranges, by the prefix' tiles and by rows whose parts are joined, and rows past 2^63."""
    most = (1 << 24) - 1
    for sizes in ((most, most, 65535, 1, 64, 10, 10), (most, most, 65535, 1, 64, 0, 0), (1 << 23, 1 << 23, 1 << 15, 1, 8, 5, 5),
                  (most, 1, 8, 8, 64, 0, 16), (most, 1, 8, 8, 64, 20, 16), (most, 1, 16, 8, 128, 100000, 0)):
        assert B.shared_prefix_attention_bytes(*sizes) == 0, sizes
        with pytest.raises(B.VlutError) as e:
            B.query_shared_prefix_attention(*sizes)
        assert e.value.status == B.VLUT_ERR_SHAPE
        Bn, n, Hq, Hk, D, prefix, own = sizes
        q = heads(token=Hq * D, head=D, n=Hq)
        c = cache(n=Hk, strides=(Hk * 16 * D, 16 * D, D))
        assert attend(L, q=q, out=q, stride=n * Hq * D, c=c, prefix_len=prefix, max_own=own, Bn=Bn, n=n, D=D) == B.VLUT_ERR_SHAPE
    for sizes in ((1 << 22, 1, 8, 8, 64, 0, 16), (1 << 20, 4, 8, 8, 64, 20, 16), (1, 1 << 22, 32, 8, 128, 0, 1 << 22), (1, most, 4, 4, 128, 0, most)):
        assert B.query_shared_prefix_attention(*sizes)[3] < 1 << 24
