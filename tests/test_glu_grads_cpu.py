"""The calls on a gated feed-forward block and on lists of gradients refuse what they cannot do before any GPU call: checked without a GPU, with addresses that are
never followed."""
import ctypes as C

import pytest
import torch

import paper_1706_07191_amd as B
from tests.test_model_ops_cpu import ARG, AT, BF16, BUDGET, F16, F32, F64, OK
from tests.test_model_ops_edges_cpu import on, two_devices  # noqa: F401

HIP = B.BRSVD_ERR_HIP


def glu(backward=False, **kw):
    a = dict(X=AT, ldx=64, Wg=AT, ldwg=64, Wu=AT, ldwu=64)
    if backward:
        a.update(G=AT, ldg=200, U=AT, ldu=200, dH=AT, lddh=200)
    a.update(tokens=100, dim=64, width=200, dtype=F16, act=0)
    a.update(dict(dX=AT, lddx=64, dWg=AT, lddwg=64, dWu=AT, lddwu=64) if backward else dict(H=AT, ldh=200, G=AT, ldg=200, U=AT, ldu=200))
    a.update(ws=AT, bytes=1 << 60)
    a.update(kw)
    return (B.lib().brsvd_glu_backward if backward else B.lib().brsvd_glu_forward)(*a.values(), None)


COMMON = [dict(X=None), dict(Wg=None), dict(Wu=None), dict(ldx=63), dict(ldwg=63), dict(ldwu=63), dict(tokens=-1), dict(dim=-1), dict(width=-1), dict(dtype=F32), dict(dtype=F64), dict(act=-1),
          dict(act=3), dict(tokens=1 << 30), dict(ldwg=1 << 21), dict(ldx=2 ** 62), dict(ldwu=2 ** 63 - 1), dict(G=None), dict(ldg=199), dict(ldu=199), dict(U=None), dict(ldg=1 << 40),
          dict(tokens=(1 << 30) - 1, width=1 << 20, ldg=1 << 20, ldu=1 << 20)]


@pytest.mark.parametrize("bad", COMMON + [dict(H=None), dict(ldh=199), dict(ldh=1 << 40), dict(width=1 << 21, ldh=1 << 21, ldg=1 << 21, ldu=1 << 21), dict(dim=1 << 21, ldx=1 << 21)])
def test_glu_forward_refuses(bad):
    assert glu(**bad) == ARG
    assert glu(tokens=0, X=None, H=None, ws=None) == OK and glu(width=0, H=None) == OK
    assert glu(ldx=65, bytes=1000) == BUDGET and glu(ldx=65, ws=None) == ARG and glu(ldx=65, ws=C.c_void_p(4100)) == ARG


@pytest.mark.parametrize("bad", COMMON + [dict(dH=None), dict(lddh=199), dict(dX=None, dWg=None, dWu=None), dict(dWg=None), dict(dWu=None), dict(lddx=63), dict(lddwg=63), dict(lddwu=63),
                                          dict(lddx=1 << 40)])
def test_glu_backward_refuses(bad):
    assert glu(True, **bad) == ARG
    need = B.lib().brsvd_glu_workspace_bytes(100, 64, 200, 1, 1)
    assert need >= 100 * 200 * 4 and glu(True, bytes=need - 1) == BUDGET and glu(True, ws=None) == ARG
    assert glu(True, tokens=0, dWg=None, dWu=None, X=None, G=None, ws=None) == OK and glu(True, dim=0, dX=None, dWg=None, dWu=None, ws=None) == OK
    assert glu(True, width=0, dX=None, ws=None) == OK


def test_glu_workspace():
    size = B.lib().brsvd_glu_workspace_bytes
    assert size(32, 4096, 12000, 0, 0) == 0 and size(64, 1000, 500, 0, 0) == 0 and size(4096, 4096, 12000, 1, 0) == 0          # few tokens go from memory, many tiles need no parts
    assert size(4096, 4096, 12000, 0, 0) >= 2 * (4096 + 2 * 12000) * 4096
    assert size(70, 4096, 500, 1, 0) > 0                                                      # few tiles: the contraction is cut
    assert size(4096, 4095, 12000, 1, 1) > size(4096, 4096, 12000, 1, 1) >= 4 * 4096 * 12000
    for bad in ((-1, 8, 8), (8, -1, 8), (8, 8, -1), (1 << 30, 8, 8), (8, 1 << 21, 8), (0, 8, 8)):
        assert size(*bad, 0, 1) == 0
    for t, d, f in ((5, 70, 33), (100, 1000, 64), (999, 5000, 1000), (70, 64, 20000)):
        for backward in (0, 1):
            assert size(t, d, f, 0, backward) >= size(t, d, f, 1, backward) and size(t, d, f, 0, backward) % 256 == 0


def tensor(**kw):
    a = dict(data=4096, rows=10, cols=20, ld=20, dtype=F32)
    a.update(kw)
    return B.brsvd_tensor(**a)


BAD = [dict(data=None), dict(rows=-1), dict(cols=-1), dict(ld=19), dict(dtype=F64), dict(dtype=-1), dict(dtype=1 << 32), dict(cols=1 << 45, rows=1), dict(rows=1 << 31), dict(rows=2, ld=1 << 44),
       dict(rows=1 << 22, cols=1 << 23, ld=1 << 23)]


def norm(tensors, **kw):
    a = dict(list=(B.brsvd_tensor * len(tensors))(*tensors), count=len(tensors), scale=1.0, norm=AT, ws=AT, bytes=1 << 50)
    a.update(kw)
    return B.lib().brsvd_grad_norm(*a.values(), None)


@pytest.mark.parametrize("bad", BAD)
def test_norm_refuses(bad):
    good = [tensor(), tensor(dtype=BF16)]
    assert norm(good + [tensor(**bad)]) == ARG
    assert B.lib().brsvd_grad_norm_workspace_bytes((B.brsvd_tensor * 1)(tensor(**bad)), 1) == 0
    for kw in (dict(list=None), dict(count=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(norm=None), dict(ws=None), dict(ws=C.c_void_p(4100))):
        assert norm(good, **kw) == ARG
    need = B.lib().brsvd_grad_norm_workspace_bytes((B.brsvd_tensor * 2)(*good), 2)
    assert need == 256 and norm(good, bytes=need - 1) == BUDGET
    assert B.lib().brsvd_grad_norm_workspace_bytes((B.brsvd_tensor * 1)(tensor(rows=1, cols=1 << 30)), 1) >= 8 << 15


def clip(tensors, outs, **kw):
    a = dict(list=(B.brsvd_tensor * len(tensors))(*tensors), out=(B.brsvd_tensor * len(outs))(*outs), count=len(tensors), scale=1.0, most=1.0, norm=AT)
    a.update(kw)
    return B.lib().brsvd_grad_clip(*a.values(), None)


@pytest.mark.parametrize("bad", BAD + [dict(rows=11), dict(cols=21, ld=21), dict(rows=20, cols=10)])
def test_clip_refuses(bad):
    good, other = [tensor(), tensor(data=8192, dtype=BF16)], [tensor(data=16384), tensor(data=32768, dtype=F16)]
    assert clip(good + [tensor(data=1 << 16)], other + [tensor(**dict(dict(data=1 << 17), **bad))]) == ARG
    for kw in (dict(list=None), dict(out=None), dict(count=-1), dict(scale=float("nan")), dict(norm=None), dict(most=-1.0), dict(most=float("nan"))):
        assert clip(good, other, **kw) == ARG
    assert clip([], [], out=None) == OK


def test_clip_refuses_memory_of_others():
    a, b, c = tensor(), tensor(data=8192), tensor(data=16384)
    assert clip([a, a], [a, a]) == ARG and clip([a, b], [c, c]) == ARG and clip([a, b], [b, a]) == ARG and clip([a, b], [b, c]) == ARG
    assert clip([a], [tensor(dtype=BF16)]) == ARG and clip([a], [tensor(ld=30)]) == ARG
    none = tensor(rows=0)
    assert clip([none, none], [none, none]) == OK


def test_operands_on_several_devices_are_refused(two_devices):  # noqa: F811
    X, W = on(0, 4, 64), on(1, 6, 64)
    for call in (lambda: B.brsvd_glu_forward(X, W, W), lambda: B.brsvd_glu_backward(X, on(0, 6, 64), on(0, 6, 64), on(0, 4, 6), on(1, 4, 6), on(0, 4, 6)),
                 lambda: B.brsvd_grad_norm([on(0, 4), on(1, 4)]), lambda: B.brsvd_grad_clip([on(1, 4)], on(0, 1, dtype=torch.float32), 1.0),
                 lambda: B.brsvd_grad_clip([on(0, 4)], on(0, 1, dtype=torch.float32), 1.0, out=(on(0, 4), on(1, 4)))):
        with pytest.raises(TypeError, match="one device"):
            call()
    seen = []
    B._scoped(lambda tensors: seen.append(two_devices[0]))([on(1, 4), on(1, 5)])
    assert seen == [1] and two_devices == [0]


@pytest.mark.parametrize("lists,error,text", [
    (([torch.ones(3)],), TypeError, r"tensors\[0\] must be a CUDA tensor"), (([None],), TypeError, r"tensors\[0\]"), ((torch.ones(3),), TypeError, "tensors must be a list"),
    (([], torch.ones(3)), TypeError, "out must be a list"), (([], [torch.ones(3)]), ValueError, "out has 1 tensors, expected 0"), (((torch.ones(3).to_sparse(),),), TypeError, r"tensors\[0\]"),
    ((), TypeError, "one list or two"), (([], [], []), TypeError, "one list or two")])
def test_lists_refuse(lists, error, text):
    with pytest.raises(error, match=text):
        B._tensors(*lists)


def test_empty_lists():
    assert B._tensors([]) == (b"",) and B._tensors((), []) == (b"", b"")


def wrote(*pairs):
    """What clip says to tensors that are read and written; a sound list would go on to the GPU, so a refused one behind it says so."""
    return clip([a for a, _ in pairs], [b for _, b in pairs])


def test_clip_refuses_parts_of_others():
    whole, part = tensor(), tensor(data=4096 + 400, rows=1, cols=100, ld=100)
    other, far = tensor(data=65536), tensor(data=131072, rows=1, cols=100, ld=100)
    assert wrote((whole, whole), (part, part)) == ARG and wrote((part, part), (whole, whole)) == ARG            # a matrix and its lower half, in place
    assert wrote((other, whole), (far, part)) == ARG and wrote((whole, other), (far, part)) == ARG and wrote((part, far), (other, whole)) == ARG
    assert wrote((whole, tensor(data=4096 + 4))) == ARG                                                          # one tensor, shifted
    small = tensor(data=4096, dtype=BF16)
    assert wrote((other, small), (far, tensor(data=4096 + 398, rows=1, cols=100, ld=100))) == ARG
    left, right = tensor(rows=10, cols=20, ld=64), tensor(data=4096 + 4 * 19, rows=10, cols=20, ld=64)
    assert wrote((left, left), (right, right)) == ARG and wrote((left, left), (tensor(data=4096 + 4 * 50, ld=64), tensor(data=4096 + 4 * 50, ld=64))) == ARG
    assert wrote((left, left), (tensor(data=4096 + 80, ld=63), tensor(data=4096 + 80, ld=63))) == ARG
    long = tensor(rows=1, cols=1000, ld=1000)
    assert wrote((long, long), (other, other), (tensor(data=8092, rows=1, cols=1, ld=1), far)) == ARG            # its last number, read
