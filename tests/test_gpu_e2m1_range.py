"""Numbers of 4 bits at the ends of what the activations' types hold: each number with each scale through a product of its own, and casts whose results no type holds."""
import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e2m1 import HALF, TYPES, bytes_of, unpacked, values

pytestmark = pytest.mark.gpu
INF = float("inf")


def every_number():
    """All 16 numbers (rows of 32, each twice) with all 255 scales that are powers: (255, 32) in fp64, codes and scale bytes."""
    code = torch.arange(32)[None].repeat(255, 1) % 16
    s = torch.arange(255)[:, None]
    return values(code, s), code, s


def held(v, dtype):
    """Whether the documents say that the type holds v."""
    a = v.abs()
    return (a == 0) | ((a >= 2.0 ** -128) & (a <= 1.5 * 2.0 ** 127) if dtype == torch.bfloat16 else (a >= 2.0 ** -23) & (a <= 49152))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m", [1, 20, 60, 65, 300])
def test_products_of_one_number(m, dtype):
    """Sums of one product with 1: the number itself where the type holds it, rounded or infinite where it does not."""
    dev = need_gpu()
    v, code, s = every_number()
    want = v.to(dtype)
    assert torch.equal(want.double()[held(v, dtype)], v[held(v, dtype)])
    least = 2.0 ** (128 if dtype == torch.bfloat16 else 16)
    assert torch.equal(torch.isinf(want), v.abs() >= least) and bool((held(v, dtype) | torch.isinf(want) | (v.abs() < 2.0 ** -23)).all())
    # forward: a row of W for each number;  backward: one row of W, a group for each scale
    W = code.view(-1, 1).to(torch.uint8).to(dev).view(torch.float4_e2m1fn_x2)
    S = s.repeat(1, 32).view(-1, 1).to(torch.uint8).to(dev).view(torch.float8_e8m0fnu)
    y = B.brsvd_linear_e2m1(torch.ones(m, 1, dtype=dtype, device=dev), W, S).cpu()
    assert torch.equal(y, want.view(1, -1).expand(m, -1))
    W = (code[:, ::2] | code[:, 1::2] << 4).view(1, -1).to(torch.uint8).to(dev).view(torch.float4_e2m1fn_x2)
    S = s.view(1, -1).to(torch.uint8).to(dev).view(torch.float8_e8m0fnu)
    dx = B.brsvd_linear_e2m1_backward(torch.ones(m, 1, dtype=dtype, device=dev), W, S).cpu()
    assert torch.equal(dx, want.view(1, -1).expand(m, -1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_finite_numbers_that_stand_for_infinity(dtype):
    """From 3.5 2^126 on the nearest of 3 and 4 times the scale 2^126 is 2^128; a step below it is 3 2^126; other numbers of the group, and other groups, are as they were."""
    dev = need_gpu()
    top = 2.0 ** 126
    step = torch.finfo(dtype).eps * 2
    X = torch.zeros(4, 70, dtype=torch.float64)
    X[0, 3], X[0, 4], X[0, 5], X[0, 40] = 3.5 * top, (3.5 - step) * top, -top, 1.0
    X[1, 69], X[1, 0] = -torch.finfo(dtype).max, 5.0
    X[2, 32] = 3.0 * top
    X[3, 0] = (3.0 + step) * top
    Q, S = B.brsvd_quantize_e2m1(X.to(dtype).to(dev))
    want = torch.zeros(4, 70, dtype=torch.float64)
    want[0, 3], want[0, 4], want[0, 5], want[0, 40] = INF, 3 * top, -top, 1.0
    want[1, 69], want[1, 0] = -INF, 4.0                # 5 at a scale of 1 lies between 4 and 6: the even code
    want[2, 32] = want[3, 0] = 3 * top
    assert bytes_of(S)[:, 0].tolist() == [253, 127, 127, 253] and bytes_of(S)[2, 1] == 252 and bytes_of(S)[1, 2] == 253
    assert unpacked(Q, 70)[0, 3] == 6 and unpacked(Q, 70)[0, 4] == 5
    for out in TYPES:
        assert torch.equal(B.brsvd_dequantize_e2m1(Q, S, cols=70, dtype=out).cpu().double(), want.to(out).double())
    for m in (1, 40, 100):
        x = torch.zeros(m, 70, dtype=torch.bfloat16, device=dev)
        x[:, 5] = 0.5
        y = B.brsvd_linear_e2m1(x, Q, S)
        assert bool(torch.isnan(y[:, :2]).all()) and not bool(y[:, 2:].any())        # 0 times infinity, as in any product with it
        x[:, 3], x[:, 69] = 2.0 ** -20, 2.0 ** -20
        y = B.brsvd_linear_e2m1(x[:, :4].contiguous(), Q[:, :2], S[:, :1].contiguous())
        assert bool((y[:, 0] == INF).all()) and not bool(y[:, 1:].any())
