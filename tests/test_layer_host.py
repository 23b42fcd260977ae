"""Norms around a block and log probabilities on the host: argument errors ahead of any device call, workspaces, refusals of the Python and native forms.
(There is no GPU here: a call that got as far as a launch would report VLUT_ERR_DEVICE.)"""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2512_06443_amd import binding as B

P = 1 << 20                                                               # an address that nobody reads
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L(vlut_lib_path):
    return B.lib()


def rows(data=P, stride=512, type=1):
    return B._Rows(data, stride, type)


def ref(s):
    return None if s is None else ctypes.byref(s)


def residual(L, y=rows(), weight=P, gate=None, activation=0, scale=1.0, r=rows(type=0), next_weight=P, eps=1e-6, N=4, K=512, h=rows(type=0), x=rows()):
    return L.vlut_residual_norm(ref(y), weight, ref(gate), activation, scale, ref(r), next_weight, eps, N, K, ref(h), ref(x), None)


def gated(L, x=rows(), gate=rows(), activation=2, weight=None, eps=1e-6, N=4, K=512, out=rows()):
    return L.vlut_gated_norm(ref(x), ref(gate), activation, weight, eps, N, K, ref(out), None)


def logprobs(L, x=rows(stride=32000, type=0), tokens=P, temperature=1.0, top=8, N=4, V=32000, logprob=P, entropy=P, ids=P, probs=P, ws=P, ws_bytes=1 << 40):
    return L.vlut_token_logprobs(ref(x), tokens, temperature, top, N, V, logprob, entropy, ids, probs, ws, ws_bytes, None)


def test_the_calls_that_are_changed_one_by_one_below_are_accepted(L):
    if torch.cuda.is_available():
        pytest.skip("addresses of nothing")
    for more in (dict(), dict(weight=None), dict(next_weight=None, x=None), dict(gate=rows()), dict(gate=rows(type=0), activation=4), dict(gate=rows(stride=0), activation=1), dict(scale=0.0),
                 dict(scale=-2.0), dict(eps=0.0), dict(K=1), dict(K=32768), dict(K=511), dict(y=rows(data=P + 2)), dict(N=(1 << 24) - 1), dict(r=rows(type=2), h=rows(type=2))):
        assert residual(L, **more) == B.VLUT_ERR_DEVICE, more
    for more in (dict(), dict(gate=None), dict(gate=None, activation=0), dict(weight=P), dict(out=rows(type=2)), dict(gate=rows(type=0))):
        assert gated(L, **more) == B.VLUT_ERR_DEVICE, more
    for more in (dict(), dict(tokens=None, logprob=None), dict(entropy=None), dict(top=0, ids=None, probs=None), dict(V=1, top=1), dict(top=64), dict(temperature=1e-3),
                 dict(x=rows(stride=0)), dict(N=(1 << 24) - 1, V=5, top=5), dict(V=(1 << 30) - 1)):
        assert logprobs(L, **more) == B.VLUT_ERR_DEVICE, more


def test_refusals_of_residual_norm(L):
    for more in (dict(y=None), dict(r=None), dict(h=None), dict(x=None), dict(next_weight=None), dict(y=rows(data=None)), dict(gate=rows(data=None)), dict(r=rows(data=None, type=0)),
                 dict(h=rows(data=None, type=0)), dict(x=rows(data=None))):
        assert residual(L, **more) == B.VLUT_ERR_NULL, more
    for more in (dict(N=0), dict(N=-1), dict(N=1 << 24), dict(K=0), dict(eps=-1e-6), dict(eps=NAN), dict(scale=NAN), dict(scale=INF), dict(activation=-1), dict(activation=5, gate=rows()),
                 dict(activation=2), dict(gate=rows(type=2)), dict(y=rows(type=3)), dict(y=rows(type=-1)), dict(gate=rows(type=9)), dict(r=rows(type=1)), dict(r=rows(type=3), h=rows(type=3)),
                 dict(x=rows(type=3))):
        assert residual(L, **more) == B.VLUT_ERR_SHAPE, more
    assert residual(L, K=32769) == B.VLUT_ERR_UNSUPPORTED


def test_refusals_of_gated_norm(L):
    for more in (dict(x=None), dict(out=None), dict(x=rows(data=None)), dict(gate=rows(data=None)), dict(out=rows(data=None))):
        assert gated(L, **more) == B.VLUT_ERR_NULL, more
    for more in (dict(N=0), dict(N=1 << 24), dict(K=0), dict(eps=-1.0), dict(activation=5), dict(gate=rows(type=2)), dict(x=rows(type=3)), dict(out=rows(type=3))):
        assert gated(L, **more) == B.VLUT_ERR_SHAPE, more
    assert gated(L, K=32769) == B.VLUT_ERR_UNSUPPORTED


def test_refusals_of_token_logprobs(L):
    for more in (dict(x=None), dict(x=rows(data=None, type=0)), dict(tokens=None), dict(logprob=None), dict(ids=None), dict(probs=None), dict(top=0), dict(ws=None),
                 dict(tokens=None, logprob=None, entropy=None, top=0, ids=None, probs=None)):
        assert logprobs(L, **more) == B.VLUT_ERR_NULL, more
    for more in (dict(N=0), dict(N=1 << 24), dict(V=0), dict(V=1 << 30), dict(top=-1), dict(V=7), dict(x=rows(type=3)), dict(temperature=0.0), dict(temperature=-1.0),
                 dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-39)):
        assert logprobs(L, **more) == B.VLUT_ERR_SHAPE, more
    assert logprobs(L, top=65) == logprobs(L, ws=P + 8) == B.VLUT_ERR_UNSUPPORTED
    need = B.token_logprobs_bytes(4, 32000, 8)
    assert need > 0 and logprobs(L, ws_bytes=need - 1) == B.VLUT_ERR_SMALL_BUFFER
    if not torch.cuda.is_available():
        assert logprobs(L, ws_bytes=need) == B.VLUT_ERR_DEVICE


def test_workspaces(L):
    """Rows of their own need none where they are many or short; long ones a part for every 2048 logits at most, 64 of them at most."""
    assert B.token_logprobs_bytes(4096, 128000, 20) == B.token_logprobs_bytes(1, 2048, 64) == 0
    for bad in ((0, 10, 0), (1, 0, 0), (1, 10, 11), (1, 100, 65), (1, 100, -1)):
        assert B.token_logprobs_bytes(*bad) == 0
    for N in (1, 3, 100, 500):
        for V in (2049, 9001, 32000, 262144, 1 << 24):
            for top in (0, 1, 64):
                parts, rest = divmod(B.token_logprobs_bytes(N, V, top), N * (16 + 8 * top))
                assert rest == 0 and parts != 1 and parts <= min(64, -(-V // 2048), -(-1024 // N)), (N, V, top)


def test_python_forms_refuse(L):
    """What is not on the GPU, and names that are no activation."""
    x, r = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(4, 16)
    for call in (lambda: B.residual_norm(x, r), lambda: B.gated_norm(x, x), lambda: B.token_logprobs(r), lambda: B.residual_norm(x, r, gate=x, activation="swish")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        B._activation("swish")


def test_native_forms_decline_what_they_do_not_know(L):
    if B._native is None:
        pytest.skip("built with a torch for ROCm only")
    n, x, r = B._native, torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(4, 16)
    assert n.residual_norm(x, r, None, None, None, 1.0, None, 1e-6, None, None, None) is None
    assert n.residual_norm(x) is None and n.residual_norm("x", *[None] * 10) is None
    assert n.gated_norm(x, x, "silu", None, 1e-6, None, None) is None and n.gated_norm() is None
    assert n.token_logprobs(r, None, 0, 1.0, True, None) is None and n.token_logprobs("x", *[None] * 5) is None
