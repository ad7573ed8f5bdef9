"""Every way that the products on a layer go to the GPU, in both types: few rows by their tiles, tiles of 64, 128 and 256 rows, two of these sizes in a launch each, contractions in
parts.  Against 64 bits within the bounds of the operators' own tests."""
import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.layer_sizes import BACKWARD, GLU, GLU_DW, GLU_DX, LINEAR
from tests.test_gpu_e2m1 import HALF, check_product, four_bits
from tests.test_gpu_e4m3 import randn
from tests.test_gpu_glu import ACTS, check_forward, check_gradients, problem

pytestmark = pytest.mark.gpu


def ways(table):
    return [pytest.param(*size, id="-".join(map(str, way + size))) for way, size in table.items()]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m,n,k", ways(LINEAR))
def test_linear(m, n, k, dtype):
    dev = need_gpu()
    W, S, w = four_bits(m + 7 * n + k, n, k, dev)
    X = (randn(m + k, m, k) * 3).to(dtype).to(dev)
    out = torch.full((m + 1, n), 5.0, dtype=dtype, device=dev)
    y = B.brsvd_linear_e2m1(X, W, S, out=out[:m])
    check_product(y, X.double().cpu(), w.t())
    assert bool((out[m] == 5).all()) and torch.equal(B.brsvd_linear_e2m1(X, W, S), y)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m,n,k", ways(BACKWARD))
def test_linear_backward(m, n, k, dtype):
    dev = need_gpu()
    W, S, w = four_bits(m + 7 * n + k, n, k, dev)
    dY = (randn(m + n, m, n) * 0.1).to(dtype).to(dev)
    out = torch.full((m + 1, k), 5.0, dtype=dtype, device=dev)
    dX = B.brsvd_linear_e2m1_backward(dY, W, S, cols=k, out=out[:m])
    check_product(dX, dY.double().cpu(), w)
    assert bool((out[m] == 5).all()) and torch.equal(B.brsvd_linear_e2m1_backward(dY, W, S, cols=k), dX)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("t,d,f", ways(GLU))
def test_glu(t, d, f, dtype):
    dev = need_gpu()
    act = ACTS[(t + d + f) % 3]
    X, Wg, Wu = problem(t, d, f, dtype, dev)
    H, G, U = B.brsvd_glu_forward(X, Wg, Wu, act=act, keep=True)
    check_forward(X, Wg, Wu, act, H, G, U)
    assert torch.equal(B.brsvd_glu_forward(X, Wg, Wu, act=act), H)


def gradients(t, d, f, dtype, **needs):
    dev = need_gpu()
    act = ACTS[(t + d + f) % 3]
    X, Wg, Wu = problem(t, d, f, dtype, dev)
    G, U, dH = (randn(i + t + f, t, f).to(dtype).to(dev) for i in range(3))
    grads = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH, act=act, **needs)
    check_gradients(X, Wg, Wu, G, U, dH, act, *grads)
    again = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH, act=act)
    assert all(a is None or torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("t,d,f", ways(GLU_DX))
def test_glu_dX(t, d, f, dtype):
    gradients(t, d, f, dtype, need_dW=False)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("t,d,f", ways(GLU_DW))
def test_glu_dW(t, d, f, dtype):
    gradients(t, d, f, dtype, need_dX=False)
