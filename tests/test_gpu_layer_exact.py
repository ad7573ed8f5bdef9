"""Products on a layer with sums that are whole numbers and exact in the result's type, over long contractions: each group of 32 numbers, and each step of 64 tokens, is met
alone or beside few others, so that one that is lost, taken twice or multiplied with another one's scale shows, however long the contraction."""
import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e2m1 import HALF

pytestmark = pytest.mark.gpu
TERMS = 24              # of a sum: each is 8 at most, so that sums stay within the 256 up to which bf16 has all whole numbers


def ones_with_scales(seed, n, k, dev):
    """W of 1 and -1 with scales from 1 to 8 (some other numbers behind an odd row's end), as bytes, and its values (n, k) as 8-bit integers."""
    g = torch.Generator(device=dev).manual_seed(seed)
    sign = torch.randint(0, 2, (n, k + k % 2), generator=g, device=dev, dtype=torch.uint8)
    code = 2 + 8 * sign
    power = torch.randint(0, 4, (n, -(-k // 32)), generator=g, device=dev, dtype=torch.uint8)
    W, S = code[:, ::2] | code[:, 1::2] << 4, power + 127
    value = (1 - 2 * sign[:, :k].to(torch.int8)) * (1 << power.to(torch.int8)).repeat_interleave(32, 1)[:, :k]
    return W.view(torch.float4_e2m1fn_x2), S.view(torch.float8_e8m0fnu), value


def sparse(seed, rows, length, unit, dtype, dev):
    """Matrices of 1, -1 and mostly 0, rows x length: in each row one place of TERMS units (of `unit` places), in all of them together one of every unit, and the last place."""
    g = torch.Generator().manual_seed(seed)
    units = -(-length // unit)
    order = torch.randperm(units, generator=g)
    per = rows * TERMS
    for first in range(0, units, per):
        X = torch.zeros(rows, length, dtype=dtype, device=dev)
        some = order[first:first + per]
        at = some * unit + torch.randint(0, unit, some.shape, generator=g)
        at = torch.where(some == units - 1, length - 1, at)
        r = torch.arange(some.numel()) % rows
        X[r.to(dev), at.to(dev)] = (1 - 2 * torch.randint(0, 2, some.shape, generator=g)).to(dtype).to(dev)
        yield X


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m,n,k,few", [(3, 40, 49253, True), (16, 33, 98437, True), (5, 17, 49024, True), (1, 16, 49025, True), (9, 4112, 24481, True), (16, 4112, 49900, True), (20, 12000, 19264, True),
                                       (12, 8300, 33000, True), (16, 17775, 19301, True), (50, 200, 4999, False), (50, 20001, 2100, True), (100, 300, 40001, False), (300, 600, 9001, False),
                                       (700, 8200, 2049, False), (2100, 4000, 1500, False)])
def test_every_group_of_a_long_contraction(m, n, k, few, dtype):
    dev = need_gpu()
    assert bool(B.brsvd_linear_e2m1_plan(m, n, k)[0]) == few
    W, S, value = ones_with_scales(m + n + k, n, k, dev)
    for i, X in enumerate(sparse(k, m, k, 32, dtype, dev)):
        want = torch.zeros(m, n, dtype=torch.float64, device=dev)
        for rows in torch.arange(n, device=dev).split(2048):
            want[:, rows] = X.double() @ value[rows].double().t().contiguous()
        assert float(want.abs().max()) <= 8 * TERMS and torch.equal(B.brsvd_linear_e2m1(X, W, S).double(), want), i


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m,n,k", [(1, 40001, 40), (70, 30000, 301), (300, 20001, 1000), (1000, 9000, 2500)])
def test_every_row_of_a_long_contraction_back(m, n, k, dtype):
    """The contraction runs down W's rows, each with scales of its own."""
    dev = need_gpu()
    W, S, value = ones_with_scales(m + n + k, n, k, dev)
    for i, dY in enumerate(sparse(n, m, n, 8, dtype, dev)):
        want = dY.double() @ value.double()
        assert float(want.abs().max()) <= 8 * TERMS and torch.equal(B.brsvd_linear_e2m1_backward(dY, W, S, cols=k).double(), want), i


def test_weights_gradients_over_more_than_4_gib():
    """140 000 tokens, G, U and dH of more than 2^32 bytes: dH is zero but for 200 tokens a call, of which each step of 64 has one in some call, and so has the last, which is half
    a step.  G is 128, where the activation is G and its slope 1: dWg sums ones, dWu 128s."""
    dev = need_gpu()
    t, d, f, some = 140000, 64, 16008, 200
    g = torch.Generator(device=dev).manual_seed(3)
    signs = lambda *s: (1 - 2 * torch.randint(0, 2, s, generator=g, device=dev, dtype=torch.int8)).bfloat16()  # noqa: E731
    X, Wg, Wu = signs(t, d), signs(f, d), signs(f, d)
    G = torch.full((t, f), 128.0, dtype=torch.bfloat16, device=dev)
    U, dH = signs(997, f).repeat(-(-t // 997), 1)[:t], torch.zeros(t, f, dtype=torch.bfloat16, device=dev)
    steps = torch.randperm(-(-t // 64), generator=g, device=dev)
    for part in steps.split(some):
        tokens = (64 * part + torch.randint(0, 64, part.shape, generator=g, device=dev)).clamp(max=t - 1)
        dH[tokens] = signs(part.numel(), f)
        none, dWg, dWu = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH, need_dX=False)
        x, h, u = X[tokens].double(), dH[tokens].double(), U[tokens].double()
        assert none is None and torch.equal(dWg.double(), (h * u).t().contiguous() @ x) and torch.equal(dWu.double(), 128 * (h.t().contiguous() @ x))
        dH[tokens] = 0
