"""The calls on a model's matrices refuse what they cannot do before any GPU call: checked without a GPU, with addresses that are never followed."""
import ctypes as C

import pytest

import paper_1706_07191_amd as B

AT = C.c_void_p(4096)          # 256-byte aligned
BF16, F16, F32, F64 = B.BRSVD_DTYPE_BF16, B.BRSVD_DTYPE_F16, B.BRSVD_DTYPE_F32, B.BRSVD_DTYPE_F64
ARG, BUDGET, OK = B.BRSVD_ERR_ARG, B.BRSVD_ERR_BUDGET, B.BRSVD_OK


def quantize(**kw):
    a = dict(X=AT, ldx=300, rows=200, cols=300, dtype=F32, block=1, Q=AT, ldq=304, S=AT, Qt=None, ldqt=0, St=None)
    a.update(kw)
    return B.lib().brsvd_quantize_e4m3(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(X=None), dict(ldx=299), dict(rows=-1), dict(cols=-1), dict(dtype=F64), dict(dtype=7), dict(block=0), dict(block=64), dict(Q=None),
                                 dict(S=None), dict(ldq=299), dict(Qt=AT, ldqt=199, St=AT), dict(Qt=AT, ldqt=200), dict(rows=1 << 40)])
def test_quantize_refuses(bad):
    assert quantize(**bad) == ARG
    assert quantize(rows=0) == OK and quantize(cols=0, X=None) == OK


def dequantize(**kw):
    a = dict(Q=AT, ldq=300, S=AT, rows=200, cols=300, block=128, dtype=BF16, X=AT, ldx=300)
    a.update(kw)
    return B.lib().brsvd_dequantize_e4m3(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(Q=None), dict(S=None), dict(X=None), dict(ldq=299), dict(ldx=299), dict(block=2), dict(dtype=F64), dict(rows=-3)])
def test_dequantize_refuses(bad):
    assert dequantize(**bad) == ARG and dequantize(rows=0) == OK


def gemm(**kw):
    a = dict(A=AT, lda=512, SA=AT, Bm=AT, ldb=512, SB=AT, block=128, m=100, n=300, k=512, dtype=BF16, C=AT, ldc=300, scratch=AT, bytes=1 << 40)
    a.update(kw)
    return B.lib().brsvd_gemm_e4m3(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(A=None), dict(Bm=None), dict(SA=None), dict(SB=None), dict(C=None), dict(lda=511), dict(ldb=511), dict(ldc=299), dict(m=-1), dict(n=-1),
                                 dict(k=-1), dict(dtype=F64), dict(block=3), dict(lda=1 << 22), dict(k=1 << 22, lda=1 << 23, ldb=1 << 23), dict(m=1 << 31),
                                 dict(m=1 << 30, n=1 << 30)])
def test_gemm_refuses(bad):
    assert gemm(**bad) == ARG
    assert gemm(m=0, C=None) == OK and gemm(n=0) == OK


def test_gemm_scratch():
    need = B.lib().brsvd_gemm_e4m3_scratch_bytes(100, 300, 4096, 128, BF16)
    assert need > 0                                            # few tiles: the contraction is cut
    big = dict(k=4096, lda=4096, ldb=4096)
    assert gemm(**big, bytes=need - 1) == BUDGET
    assert gemm(**big, scratch=None) == ARG and gemm(**big, scratch=C.c_void_p(4097)) == ARG
    assert B.lib().brsvd_gemm_e4m3_scratch_bytes(8192, 8192, 4096, 128, BF16) == 0
    assert B.lib().brsvd_gemm_e4m3_scratch_bytes(-1, 3, 3, 128, BF16) == 0


def linear(**kw):
    a = dict(X=AT, ldx=512, dtype=F16, W=AT, ldw=512, SW=AT, m=100, n=300, k=512, Y=AT, ldy=300, scratch=AT, bytes=1 << 40)
    a.update(kw)
    return B.lib().brsvd_linear_e4m3(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(X=None), dict(W=None), dict(SW=None), dict(Y=None), dict(ldx=511), dict(ldw=511), dict(ldy=299), dict(dtype=F64), dict(m=-1), dict(k=-2)])
def test_linear_refuses(bad):
    assert linear(**bad) == ARG and linear(m=0) == OK
    need = B.lib().brsvd_linear_e4m3_scratch_bytes(100, 300, 512, F16)
    assert need >= 100 * 512 + 100 * 4 * 4 and linear(bytes=need - 1) == BUDGET and linear(scratch=None) == ARG
    assert B.lib().brsvd_linear_e4m3_scratch_bytes(8, 300, 512, F16) == 0


def xent(backward=False, **kw):
    a = dict(H=AT, ldh=64, W=AT, ldw=64, labels=AT)
    if backward:
        a.update(lse=AT, grad=AT, stride=1)
    a.update(tokens=10, vocab=1000, dim=64)
    if backward:
        a.update(piece=0)
    a.update(dtype=BF16)
    a.update(dict(dH=AT, lddh=64, dW=AT, lddw=64) if backward else dict(loss=AT, lse=AT))
    a.update(ws=AT, bytes=1 << 50)
    a.update(kw)
    return (B.lib().brsvd_xent_backward if backward else B.lib().brsvd_xent_forward)(*a.values(), None)


COMMON = [dict(H=None), dict(W=None), dict(labels=None), dict(ldh=63), dict(ldw=63), dict(tokens=-1), dict(vocab=0), dict(dim=0), dict(dtype=F32), dict(dtype=F64),
          dict(lse=None), dict(ws=None), dict(ws=C.c_void_p(4100)), dict(tokens=1 << 30), dict(ldw=1 << 21)]


@pytest.mark.parametrize("bad", COMMON + [dict(loss=None)])
def test_xent_forward_refuses(bad):
    assert xent(**bad) == ARG
    need = B.lib().brsvd_head_workspace_bytes(10, 1000, 64, 0, 0, 0)
    assert need > 0 and xent(bytes=need - 1) == BUDGET and xent(tokens=0) == OK


@pytest.mark.parametrize("bad", COMMON + [dict(grad=None), dict(stride=-1), dict(piece=-1), dict(dH=None, dW=None), dict(lddh=63), dict(lddw=63)])
def test_xent_backward_refuses(bad):
    assert xent(True, **bad) == ARG
    need = B.lib().brsvd_head_workspace_bytes(10, 1000, 64, 0, 0, 1)
    assert xent(True, bytes=need - 1) == BUDGET
    assert xent(True, tokens=0, dW=None, H=None, ws=None) == OK


def distill(**kw):
    a = dict(H=AT, ldh=64, W=AT, ldw=64, ids=AT, logits=AT, top=5, tau=2.0, tokens=10, vocab=1000, dim=64, dtype=BF16, loss=AT, lse=AT, z=AT, ws=AT, bytes=1 << 50)
    a.update(kw)
    return B.lib().brsvd_distill_forward(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(ids=None), dict(logits=None), dict(top=0), dict(top=-1), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")),
                                 dict(z=None), dict(loss=None), dict(lse=None), dict(dtype=F32), dict(W=None), dict(ldh=1)])
def test_distill_refuses(bad):
    assert distill(**bad) == ARG and distill(tokens=0) == OK


def test_workspace_grows_with_what_is_kept():
    size = B.lib().brsvd_head_workspace_bytes
    # of the logits nothing is kept: a few numbers per token and 256 words forward, a piece of 16-bit numbers backward
    assert size(8192, 100000, 4096, 0, 0, 0) < 8192 * 100000 * 2 / 50
    assert size(8192, 100000, 4096, 256, 0, 1) < size(8192, 100000, 4096, 0, 0, 1) < 2 ** 28 + 8192 * 4096 * (2 + 4) + 2 ** 20
    assert size(100, 1000, 64, 0, 20, 1) >= size(100, 1000, 64, 0, 0, 1) + 100 * 20 * 4
    assert size(0, 1000, 64, 0, 0, 1) == 0 and size(10, 0, 64, 0, 0, 1) == 0 and size(10, 10, 64, -1, 0, 1) == 0
