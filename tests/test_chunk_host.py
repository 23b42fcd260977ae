"""Attention of chunks on the host: argument errors ahead of any device call, sizes and plans, refusals of the Python and native forms.
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


def heads(data=P, token=64 * 16, head=64, n=16, type=1):
    return B._Heads(data, None, token, head, 0, n, type)


def cache(k=P, v=P, pages=10, page_size=16, strides=(8 * 16 * 64, 16 * 64, 64), n=8, type=1, v_strides=None):
    return B._Cache(k, v, pages, page_size, *strides, *(v_strides or strides), n, type)


def ref(s):
    return None if s is None else ctypes.byref(s)


def attend(L, q=heads(), c=cache(), table=P, starts=P, lens=P, N=40, Bn=3, D=64, queries=30, max_len=2000, window=0, scale=0.125, out=heads(), lse=None, ws=P, ws_bytes=1 << 40):
    return L.vlut_chunk_attention(ref(q), ref(c), table, 125, starts, lens, N, Bn, D, queries, max_len, window, scale, ref(out), lse, ws, ws_bytes, None)


def test_the_call_that_is_changed_below_is_accepted(L):
    if torch.cuda.is_available():
        pytest.skip("addresses of nothing")
    for more in (dict(), dict(lse=P), dict(out=heads(type=0)), dict(c=cache(type=2), q=heads(type=2), out=heads(type=2)), dict(max_len=0, table=None), dict(queries=0),
                 dict(queries=1000), dict(window=1), dict(c=cache(strides=(8194, 1026, 66))), dict(q=heads(head=66)), dict(out=heads(data=P + 4)), dict(N=1, Bn=1, queries=1),
                 dict(q=heads(n=8), out=heads(n=8)), dict(q=heads(n=320), out=heads(n=320)), dict(c=cache(page_size=1)), dict(c=cache(page_size=1 << 16)), dict(Bn=100)):
        assert attend(L, **more) == B.VLUT_ERR_DEVICE, more


def test_refusals(L):
    for more in (dict(q=None), dict(out=None), dict(c=None), dict(c=cache(k=None)), dict(c=cache(v=None)), dict(q=heads(data=None)), dict(out=heads(data=None)), dict(table=None),
                 dict(starts=None), dict(lens=None), dict(Bn=30, max_len=20000, c=cache(pages=40000), ws=None)):
        assert attend(L, **more) == B.VLUT_ERR_NULL, more
    for more in (dict(N=0), dict(N=-1), dict(N=1 << 24), dict(Bn=0), dict(Bn=1 << 24), dict(D=0), dict(queries=-1), dict(max_len=-1), dict(max_len=1 << 30), dict(window=-1),
                 dict(window=1 << 30), dict(q=heads(n=12), out=heads(n=12)), dict(q=heads(n=0), out=heads(n=0)), dict(q=heads(n=1 << 16), out=heads(n=1 << 16)), dict(out=heads(n=8)),
                 dict(q=heads(type=2)), dict(q=heads(type=0)), dict(out=heads(type=2)), dict(c=cache(n=0)), dict(c=cache(pages=0)), dict(c=cache(pages=1 << 31)),
                 dict(N=(1 << 24) - 1, q=heads(n=64), out=heads(n=64))):
        assert attend(L, **more) == B.VLUT_ERR_SHAPE, more
    for more in (dict(D=4), dict(D=66), dict(D=260), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(c=cache(page_size=24)), dict(c=cache(page_size=1 << 17)),
                 dict(c=cache(type=0)), dict(q=heads(data=P + 2)), dict(q=heads(head=65)), dict(q=heads(token=1025)), dict(out=heads(head=65)), dict(out=heads(data=P + 2)),
                 dict(out=heads(data=P + 2, type=0)), dict(c=cache(k=P + 2)), dict(c=cache(v=P + 2)), dict(c=cache(strides=(8193, 1024, 64))), dict(c=cache(strides=(8192, 1023, 64))),
                 dict(c=cache(v_strides=(8192, 1024, 65))), dict(ws=P + 8)):
        assert attend(L, **more) == B.VLUT_ERR_UNSUPPORTED, more
    need = B.chunk_attention_bytes(40, 3, 16, 8, 64, 30, 2000)
    assert need > 0 and attend(L, ws_bytes=need - 1) == B.VLUT_ERR_SMALL_BUFFER
    assert B.chunk_attention_bytes(40, 3, 16, 8, 64, 30, 20) == 0
    if not torch.cuda.is_available():
        assert attend(L, ws_bytes=need) == B.VLUT_ERR_DEVICE
        assert attend(L, max_len=20, ws=None, ws_bytes=0) == B.VLUT_ERR_DEVICE


SHAPES = [s for s in itertools.product((1, 2, 40, 4096, 100000), (1, 2, 64, 3000), ((8, 1), (20, 5), (32, 32), (7, 7), (64, 1)), (8, 64, 100, 128, 256), (1, 8, 5000),
                                       (0, 1, 300, 8192, 1 << 20), (0, 1, 1000))]


def test_plans_and_workspaces(L):
    """Every shape has a plan of whose parts a tile's keys are never more than there are, all of which the workspace holds, in workgroups that a launch has."""
    for N, Bn, (Hq, Hk), D, queries, max_len, window in SHAPES:
        case = (N, Bn, Hq, Hk, D, queries, max_len, window)
        few, few_parts, few_keys, many, many_parts, many_keys = B.query_chunk_attention(*case)
        need, G = B.chunk_attention_bytes(*case), Hq // Hk
        most = min(queries, N) * G
        # a sequence of any number of rows that the bounds allow has its workgroups
        assert few in range(33) and many in (0, 128) and (few or many), case
        assert many or few == min(32, max(1, min(queries, N)) * G) >= most, case
        assert many == 0 or most > 32, case
        assert not (many and few) or (Bn > 1 and few % G == 0), case
        if many and Bn > 1 and G <= 32:
            assert few >= G, case
        # the keys of tokens that are neighbours: from up to 31 in front of the first one's first to the last one's own
        for rows, parts, keys in ((few, few_parts, few_keys), (many, many_parts, many_keys)):
            if rows:
                tokens = min(N, (rows + G - 2) // G + 1)                  # of a tile's rows at most, whatever head it begins with
                seen = min(max_len, window + tokens - 1) if window else max_len
                assert keys >= 32 and keys % 32 == 0 and parts >= 1 and parts * keys >= seen + (31 if window else 0), case
        sums = 0
        if few and few_parts > 1:
            sums += few_parts * Bn * Hk * few * (D * 4 + 8)
        if many and many_parts > 1:
            sums += many_parts * N * Hq * (D * 4 + 8)
        assert sums <= need <= sums + 4 * 256, case
    for bad in ((0, 1, 8, 1, 64, 1, 1), (1, 0, 8, 1, 64, 1, 1), (1, 1, 8, 3, 64, 1, 1), (1, 1, 8, 1, 66, 1, 1), (1, 1, 8, 1, 64, -1, 1), (1, 1, 8, 1, 64, 1, -1), (1, 1, 8, 1, 64, 1, 1, -1)):
        assert B.chunk_attention_bytes(*bad) == 0
        with pytest.raises(B.VlutError):
            B.query_chunk_attention(*bad)
    assert L.vlut_query_chunk_attention(1, 1, 8, 1, 64, 1, 1, 0, None) == B.VLUT_ERR_NULL


def test_more_than_a_launch_holds(L):
    """Workgroups of few rows, of tiles, and of those that join parts; refused ahead of a launch."""
    for sizes in (((1 << 24) - 1, (1 << 24) - 1, 8, 8, 64, 1, 10), (1 << 20, 1 << 20, 64, 64, 8, 1, 10), (1 << 23, 1, 64, 64, 64, 1 << 23, 1), ((1 << 24) - 1, 2, 32, 1, 256, 1 << 20, 1 << 20)):
        assert B.chunk_attention_bytes(*sizes) == 0
        with pytest.raises(B.VlutError) as e:
            B.query_chunk_attention(*sizes)
        assert e.value.status == B.VLUT_ERR_SHAPE
        N, Bn, Hq, Hk, D, queries, max_len = sizes
        q = heads(token=Hq * D, head=D, n=Hq)
        assert attend(L, q=q, out=q, c=cache(n=Hk, strides=(Hk * 16 * D, 16 * D, D)), N=N, Bn=Bn, D=D, queries=queries, max_len=max_len) == B.VLUT_ERR_SHAPE
    for sizes in ((1 << 20, 1, 32, 8, 128, 1 << 20, 1 << 20), (1 << 16, 1 << 16, 32, 8, 128, 1, 1 << 20), (1 << 20, 1 << 18, 8, 8, 64, 1, 10)):
        assert B.query_chunk_attention(*sizes)


def test_longer_waits_for_nobody(L):
    """One long sequence's keys are in parts enough to fill the card, of many as few as there may be."""
    assert B.query_chunk_attention(1, 1, 32, 8, 128, 1, 1 << 17)[1] >= 20
    assert B.query_chunk_attention(128, 1, 32, 8, 128, 128, 1 << 17)[4] >= 8
    assert B.query_chunk_attention(16384, 1, 32, 8, 128, 16384, 16384)[4] == 1
    assert math.prod(B.query_chunk_attention(4096, 4096, 32, 8, 128, 1, 200)[:2]) == 4
    assert B.query_chunk_attention(64, 64, 32, 8, 128, 1, 4096)[1] == 1


def test_python_form_refuses_what_is_not_on_the_gpu(L):
    x, c = torch.zeros(4, 4, 8, dtype=torch.bfloat16), torch.zeros(3, 4, 16, 8, dtype=torch.bfloat16)
    table, starts, lens = torch.zeros(2, 3, dtype=torch.int32), torch.tensor([0, 2, 4], dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.chunk_attention(x, c, c, table, starts, lens)


def test_native_form_declines_what_it_does_not_know(L):
    if B._native is None:
        pytest.skip("built with a torch for ROCm only")
    n, x, c = B._native, torch.zeros(4, 4, 8, dtype=torch.bfloat16), torch.zeros(3, 4, 16, 8, dtype=torch.bfloat16)
    table, starts, lens = torch.zeros(2, 3, dtype=torch.int32), torch.tensor([0, 2, 4], dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    assert n.chunk_attention(x, c, c, table, starts, lens, None, None, 0, None, None, None, False, None) is None
    assert n.chunk_attention() is None and n.chunk_attention("x", *[None] * 13) is None
    with pytest.raises(TypeError):
        n.bind_layer(1)
