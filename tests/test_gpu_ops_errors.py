"""A C call that fails after it has queued some of its launches is not made again."""
import ctypes

import pytest
import torch

from paper_2110_02861_amd import bq, optim
from tests.gpu_helpers import needs_gpu, say

pytestmark = [pytest.mark.gpu, needs_gpu]


def params(n):
    out = []
    for i in range(n):
        p = torch.nn.Parameter(torch.zeros(64, device="cuda"))
        p.grad = torch.full((64,), float(i + 1), device="cuda")
        out.append(p)
    return out


def check(ps, calls):
    kept = [p.grad.clone() for p in ps]
    versions = [p.grad._version for p in ps]
    with pytest.raises(bq.BQError) as e:
        optim.clip_grad_norm_(ps, 0.5)
    assert e.value.status == bq.BQ_ERR_HIP
    assert len(calls) == 1
    # the stand-in has changed nothing, and a second call would have; what saved the
    # gradients before the call is told that they may have changed
    for p, k, v in zip(ps, kept, versions):
        assert torch.equal(p.grad, k) and p.grad._version > v


def test_clip_native():
    say("clip fails, native")
    from paper_2110_02861_amd import _bqhost
    calls = []

    @ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int, ctypes.c_double,
                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p)
    def failing(*args):
        calls.append(args[1])
        return bq.BQ_ERR_HIP

    bq.host()
    entries = [ctypes.cast(getattr(bq.lib(), n), ctypes.c_void_p).value for n in bq._HOST_OPS]
    at = bq._HOST_OPS.index("bq_clip_grad_norm")
    stub = ctypes.cast(failing, ctypes.c_void_p).value
    try:
        _bqhost.bind_ops(tuple(entries[:at] + [stub] + entries[at + 1:]))
        check(params(5), calls)
    finally:
        _bqhost.bind_ops(tuple(entries))
    assert calls == [5]
    ps = params(3)
    optim.clip_grad_norm_(ps, 0.5)
    assert abs(float(optim.grad_norm(ps)) - 0.5) <= 1e-5


def test_clip_python(monkeypatch):
    say("clip fails, python")
    calls = []
    monkeypatch.setattr(bq, "_host_module", bq._PythonOnly())
    monkeypatch.setattr(bq.lib(), "bq_clip_grad_norm",
                        lambda *args: calls.append(args[1]) or bq.BQ_ERR_HIP)
    check(params(5), calls)
