"""The calls on weights of 4 bits refuse what they cannot do before any GPU call: checked without a GPU, with addresses that are never followed."""
import ctypes as C

import pytest
import torch

import paper_1706_07191_amd as B
from tests.test_model_ops_cpu import ARG, AT, BF16, BUDGET, F16, F32, F64, OK
from tests.test_model_ops_edges_cpu import NoLibrary, on, two_devices  # noqa: F401


def quantize(**kw):
    a = dict(X=AT, ldx=300, rows=200, cols=300, dtype=F32, Q=AT, ldq=150, S=AT)
    a.update(kw)
    return B.lib().brsvd_quantize_e2m1(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(X=None), dict(Q=None), dict(S=None), dict(ldx=299), dict(ldq=149), dict(cols=301, ldx=301, ldq=150), dict(rows=-1), dict(cols=-1), dict(dtype=F64),
                                 dict(dtype=9), dict(rows=1 << 40), dict(cols=(1 << 33) + 1, ldx=1 << 34, ldq=1 << 33), dict(ldx=1 << 62), dict(ldq=1 << 40)])
def test_quantize_refuses(bad):
    assert quantize(**bad) == ARG
    assert quantize(rows=0) == OK and quantize(cols=0, X=None) == OK


def dequantize(**kw):
    a = dict(Q=AT, ldq=150, S=AT, rows=200, cols=300, dtype=BF16, X=AT, ldx=300)
    a.update(kw)
    return B.lib().brsvd_dequantize_e2m1(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(Q=None), dict(S=None), dict(X=None), dict(ldq=149), dict(ldx=299), dict(dtype=F64), dict(rows=-3), dict(ldx=2 ** 63 - 1), dict(rows=1 << 62)])
def test_dequantize_refuses(bad):
    assert dequantize(**bad) == ARG and dequantize(rows=0) == OK


def linear(backward=False, **kw):
    a = dict(X=AT, ldx=512, dtype=F16, W=AT, ldw=256, SW=AT, m=100, n=512, k=512, Y=AT, ldy=512, scratch=AT, bytes=1 << 50)
    a.update(kw)
    return (B.lib().brsvd_linear_e2m1_backward if backward else B.lib().brsvd_linear_e2m1)(*a.values(), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [dict(X=None), dict(W=None), dict(SW=None), dict(Y=None), dict(ldx=511), dict(ldw=255), dict(ldy=511), dict(dtype=F32), dict(dtype=F64), dict(m=-1),
                                 dict(n=-1), dict(k=-2), dict(m=1 << 31), dict(n=1 << 31), dict(k=1 << 21, ldx=1 << 21, ldw=1 << 20, ldy=1 << 22), dict(ldx=1 << 21), dict(ldw=1 << 21),
                                 dict(ldy=1 << 40), dict(ldx=2 ** 62), dict(m=(1 << 31) - 1, n=1 << 16, ldy=1 << 16), dict(k=513, ldx=513, ldw=256, ldy=513)])
def test_linear_refuses(bad, backward):
    assert linear(backward, **bad) == ARG
    assert linear(backward, m=0, X=None, Y=None) == OK
    assert linear(backward, **({"k": 0} if backward else {"n": 0}), Y=None, W=None) == OK


@pytest.mark.parametrize("backward", [False, True])
def test_scratch(backward):
    size = B.lib().brsvd_linear_e2m1_scratch_bytes
    need = size(100, 4096, 4096, 0, backward)
    assert size(100, 4096, 4096, 1, backward) < need
    wide = dict(n=4096, k=4096, ldx=4096, ldw=2048, ldy=4096)
    assert need > 0                                            # few tiles: the contraction is cut; rows may have to be laid out
    assert linear(backward, **wide, bytes=100) == BUDGET and linear(backward, **wide, scratch=None) == ARG and linear(backward, **wide, scratch=C.c_void_p(4100)) == ARG
    assert linear(backward, **dict(wide, ldx=4097), bytes=need - 1) == BUDGET        # rows that begin at any address
    assert size(-1, 3, 3, 0, backward) == 0 and size(0, 3, 3, 0, backward) == 0 and size(5, 1 << 31, 3, 0, backward) == 0
    if not backward:
        assert size(16, 512, 4096, 0, 0) == 0 and size(64, 4096, 4096, 0, 0) == 0 and linear(m=16, scratch=None, bytes=1, X=None) == ARG


def test_operands_on_several_devices_are_refused(two_devices):  # noqa: F811
    X, W, S = on(0, 4, 64), on(1, 6, 32, dtype=torch.uint8), on(1, 6, 2, dtype=torch.uint8)
    for call in (lambda: B.brsvd_linear_e2m1(X, W, S), lambda: B.brsvd_linear_e2m1_backward(on(0, 4, 6), W, S), lambda: B.brsvd_dequantize_e2m1(W, on(0, 6, 2)),
                 lambda: B.brsvd_linear_e2m1(on(1, 4, 64), W, S, out=on(0, 4, 6))):
        with pytest.raises(TypeError, match="one device"):
            call()


def test_results_whatever_torchs_default_type(monkeypatch):
    monkeypatch.setattr(B, "torch", torch)
    monkeypatch.setattr(B, "lib", NoLibrary)
    monkeypatch.setattr(B, "_current", lambda device: None)
    for name in ("empty", "empty_strided"):
        monkeypatch.setattr(torch, name, lambda *a, real=getattr(torch, name), device=None, **kw: real(*a, **kw))
    torch.set_default_dtype(torch.float64)
    try:
        Q, S = B.brsvd_quantize_e2m1(on(0, 4, 70))
        X = B.brsvd_dequantize_e2m1(on(0, 4, 35, dtype=torch.float4_e2m1fn_x2), on(0, 4, 3, dtype=torch.float8_e8m0fnu))
    finally:
        torch.set_default_dtype(torch.float32)
    assert Q.dtype == torch.float4_e2m1fn_x2 and Q.shape == (4, 35) and Q.stride() == (48, 1) and S.dtype == torch.float8_e8m0fnu and S.shape == (4, 3)
    assert X.dtype == torch.float32 and X.shape == (4, 70)
