"""A workspace of the caller's own that kernels cannot write as they would: refused ahead of any launch, by every call that takes one."""
from __future__ import annotations

import pytest
import torch

from paper_2512_06443_amd import binding as B

BF16 = torch.bfloat16


def calls(make):
    """Every call with a workspace, of small tensors that `make` makes: (name, call with that workspace)."""
    new = lambda shape, dtype=torch.float32: make(torch.zeros(shape, dtype=dtype))  # noqa: E731
    q, out, cache = new((4, 4, 64), BF16), new((4, 4, 64), BF16), new((3, 2, 16, 64), BF16)
    table, lens = new((2, 3), torch.int32), new(2, torch.int32)
    starts = new(3, torch.int32)
    packed, codes, scales, x = new(64 * 80, torch.uint8), new((1, 320, 8), torch.int8), new(8), new((8, 320))
    rows = new(64)
    return [("chunk_attention", lambda w: B.chunk_attention(q, cache, cache, table, starts, lens, out=out, workspace=w)),
            ("shared_prefix_attention", lambda w: B.shared_prefix_attention(q.view(2, 2, 4, 64), cache, cache, None, 0, table, lens, out=out.view(2, 2, 4, 64), workspace=w)),
            ("token_logprobs", lambda w: B.token_logprobs(x, workspace=w)),
            ("mpgemm", lambda w: B.mpgemm(packed, 1.0, codes, scales, 64, workspace=w)),
            ("mpgemm_rows", lambda w: B.mpgemm_rows(packed, rows, codes, scales, 64, workspace=w)),
            ("mpgemm_f32", lambda w: B.mpgemm_f32(packed, 1.0, x, 64, workspace=w)),
            ("mpgemm_g5", lambda w: B.mpgemm_g5(packed, 1.0, codes, scales, 64, workspace=w))]


class OnGpu(torch.Tensor):
    """Host memory that says it is the GPU's, as far as arguments are looked at."""
    is_cuda = True


def strange(make):
    """Of one byte said to be many, and of every other byte."""
    return [make(torch.zeros(1, dtype=torch.uint8)).expand(1 << 20), make(torch.zeros(1 << 21, dtype=torch.uint8))[::2]]


NAMES = ["chunk_attention", "shared_prefix_attention", "token_logprobs", "mpgemm", "mpgemm_rows", "mpgemm_f32", "mpgemm_g5"]


@pytest.mark.parametrize("name", NAMES)
def test_python_forms_refuse_them(vlut_lib_path, name, monkeypatch):
    if torch.cuda.is_available():
        pytest.skip("host memory in the place of the GPU's")
    B.lib()
    monkeypatch.setattr(B, "_native", None)
    monkeypatch.setattr(B, "_here", lambda *tensors: None)
    monkeypatch.setattr(B, "_stream", lambda: None)
    make = lambda t: t.as_subclass(OnGpu)  # noqa: E731
    call = dict(calls(make))[name]
    # (what the call comes to without a GPU, where the workspace is in order)
    with pytest.raises(B.VlutError) as e:
        call(make(torch.zeros(1 << 20, dtype=torch.uint8)))
    assert e.value.status == B.VLUT_ERR_DEVICE
    for workspace in [torch.zeros(1 << 20, dtype=torch.uint8), *strange(make)]:
        with pytest.raises(ValueError, match="workspace"):
            call(workspace)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_native_forms_refuse_them(name):
    B.lib()
    assert B._native is not None
    make = lambda t: t.cuda()  # noqa: E731
    call = dict(calls(make))[name]
    for workspace in [torch.zeros(1 << 20, dtype=torch.uint8), *strange(make)]:
        with pytest.raises(ValueError, match="workspace"):
            call(workspace)
