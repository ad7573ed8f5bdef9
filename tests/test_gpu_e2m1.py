"""Weights of 4 bits: casting and back against the definition in 64 bits to the bit, products and the gradient of the activations against the
values that the numbers stand for, at the ends of groups, chunks and tiles, for rows at any alignment."""
import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e4m3 import placed, randn

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = [torch.bfloat16, torch.float16]
# Half a step relative to the lower end of a binade: numbers from 1 to 2 have 7 (fp16: 10) bits of fraction, steps of 2^-7 (2^-10), of which half is
# finfo.eps / 2; and half of the finest step.
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FINEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def cast_by_definition(x):
    """x (fp64): codes of 4 bits of the nearest of the values of x / s (the even one where two are as near), and exponents plus 127: loops over the groups."""
    rows, cols = x.shape
    q, s = torch.zeros(rows, cols, dtype=torch.int64), torch.zeros(rows, -(-cols // 32), dtype=torch.int64)
    for j in range(s.shape[1]):
        part = x[:, 32 * j:32 * j + 32]
        good = torch.isfinite(part).all(dim=1)
        top = torch.where(good, part.abs().amax(dim=1), 0.0)
        e = torch.full((rows,), -126)
        for _ in range(260):
            e = torch.where(top > 6 * torch.exp2(e.double()), e + 1, e)
        e = torch.where(top > 0, e, 0)
        u = (part / torch.exp2(e.double())[:, None]).abs().nan_to_num(0.0, 0.0)
        d = (u[..., None] - VALUES).abs()
        tie = (d == d.min(dim=-1, keepdim=True).values) * (2 - torch.arange(8) % 2)
        code = tie.argmax(dim=-1) + 8 * torch.signbit(part)
        q[:, 32 * j:32 * j + 32] = torch.where(good[:, None], code, 0)
        s[:, j] = torch.where(good, e + 127, 255)
    return q, s


def unpacked(Q, cols):
    """Codes of the numbers, and that nothing stands behind a row's last one."""
    b = Q.contiguous().view(torch.uint8).long().cpu()
    code = torch.stack([b & 15, b >> 4], dim=2).view(b.shape[0], -1)
    assert not bool(code[:, cols:].any())
    return code[:, :cols]


def values(code, s):
    """What codes with scale bytes stand for, in fp64 (NaN for a scale of 255)."""
    v = VALUES[code & 7] * torch.where(code >= 8, -1.0, 1.0).double()
    scale = torch.where(s == 255, float("nan"), torch.exp2(s.double() - 127))
    return v * scale.repeat_interleave(32, 1)[:, :code.shape[1]]


def bytes_of(S):
    return S.view(torch.uint8).long().cpu()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 32, 0, 0), (3, 31, 1, 0), (5, 33, 0, 1), (64, 64, 0, 0), (127, 300, 4, 3), (260, 8, 8, 0), (2, 2001, 0, 0),
                                                 (700, 7, 0, 0), (33, 1024, 0, 5)])
def test_cast_and_back(rows, cols, pad, shift, dtype):
    dev = need_gpu()
    x = randn(rows * 1000 + cols, rows, cols) * torch.exp2(torch.randint(-9, 9, (rows, cols), generator=torch.Generator().manual_seed(1)).double())
    X = placed(x, dtype, dev, pad, shift)
    Q, S = B.brsvd_quantize_e2m1(X)
    q, s = cast_by_definition(X.double().cpu())
    assert torch.equal(unpacked(Q, cols), q) and torch.equal(bytes_of(S), s)
    for out in TYPES:
        assert torch.equal(B.brsvd_dequantize_e2m1(Q, S, cols=cols, dtype=out).cpu(), values(q, s).to(out))


def test_cast_of_ties():
    """Every tie between two values, at several scales and with either sign."""
    dev = need_gpu()
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for e in (-126, -100, 0, 3, 125):
        X = torch.cat([ties, -ties, ties * (1 + 2.0 ** -20), ties * (1 - 2.0 ** -20)])[None] * 2.0 ** e
        X[X.abs() > 6 * 2.0 ** e] = 0
        Q, S = B.brsvd_quantize_e2m1(X.to(dev))
        q, s = cast_by_definition(X.double())
        assert torch.equal(unpacked(Q, 32), q) and torch.equal(bytes_of(S), s) and s[0, 0] == e + 127
        assert q[0, :7].tolist() == [0, 2, 2, 4, 4, 6, 6]


@pytest.mark.parametrize("shuffled", [False, True])
def test_cast_of_every_pattern_of_16_bits(shuffled):
    """All bf16 numbers; a group with an infinity or a NaN becomes NaN, the others know nothing of it."""
    dev = need_gpu()
    X = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    if shuffled:
        X = X[torch.randperm(65536, generator=torch.Generator().manual_seed(2))]
    X = X.view(256, 256)
    Q, S = B.brsvd_quantize_e2m1(X.to(dev))
    q, s = cast_by_definition(X.double())
    assert torch.equal(unpacked(Q, 256), q) and torch.equal(bytes_of(S), s)
    back = B.brsvd_dequantize_e2m1(Q, S).cpu()
    assert torch.equal(torch.isnan(back), (s == 255).repeat_interleave(32, 1))
    fine = ~torch.isnan(back)
    assert torch.equal(back[fine], values(q, s).float()[fine])


def test_cast_of_zeros_tiny_and_large_numbers():
    dev = need_gpu()
    X = torch.zeros(6, 96)
    X[1, :32] = 1e-42
    X[2, 33] = 3.4e38
    X[3, 0], X[3, 40], X[3, 95] = float("inf"), 2.0, float("nan")
    X[4, 3], X[5, 5] = -0.0, -1e-45
    Q, S = B.brsvd_quantize_e2m1(X.to(dev))
    q, s = cast_by_definition(X.double())
    assert torch.equal(unpacked(Q, 96), q) and torch.equal(bytes_of(S), s)
    assert s[0].tolist() == [127] * 3 and s[3].tolist() == [255, s[3, 1], 255] and s[1, 0] == 1


@pytest.mark.parametrize("dtype", TYPES)
def test_back_from_every_number_and_scale(dtype):
    """256 scales, both places in a byte: rounded to the type to nearest, beyond its largest to infinity."""
    dev = need_gpu()
    byte = torch.arange(256).to(torch.uint8).repeat(256, 1)
    s = torch.arange(256).to(torch.uint8)[:, None].repeat(1, 16)
    got = B.brsvd_dequantize_e2m1(byte.view(torch.float4_e2m1fn_x2).to(dev), s.view(torch.float8_e8m0fnu).to(dev), dtype=dtype).cpu()
    want = values(torch.stack([byte & 15, byte >> 4], dim=2).view(256, -1).long(), s.long()).to(dtype)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(1.0, 2.0, 3.0), want.nan_to_num(1.0, 2.0, 3.0))


def four_bits(seed, rows, cols, dev, pad=0, spread=4):
    """Random 4-bit numbers in rows of ceil(cols/2) + pad bytes (what is behind a row's end is no zero), random scales, and the values they stand for."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    width = (cols + 1) // 2
    store = torch.randint(0, 256, (rows, width + pad), generator=g).to(torch.uint8)
    s = torch.randint(127 - spread, 128 + spread, (rows, -(-cols // 32)), generator=g).to(torch.uint8)
    b = store[:, :width].long()
    value = values(torch.stack([b & 15, b >> 4], dim=2).view(rows, -1)[:, :cols], s.long())
    return store.to(dev).view(torch.float4_e2m1fn_x2)[:, :width], s.to(dev).view(torch.float8_e8m0fnu), value


def check_product(got, a, b):
    """Each result (a @ b) within a bound for sums in any order: products of a number of 4 bits and one of 16 are exact in fp32, each addition loses at most a
    step (not rounded but cut off), parts of a cut contraction are added by 16 more, those of eight waves by eight; and the rounding to the result's type."""
    dtype = got.dtype
    want, size = a @ b, a.abs() @ b.abs()
    bound = size * 2.0 ** -23 * (a.shape[1] + 32)
    bound = bound + ROUND[dtype] * (want.abs() + bound) + FINEST[dtype]
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), float((err / bound.clamp(min=1e-300)).max())


SIZES = [(1, 1, 1, 0, 0, 0), (1, 16, 32, 0, 0, 0), (2, 3, 129, 0, 1, 0), (15, 130, 128, 0, 0, 0), (16, 300, 127, 1, 0, 1), (17, 257, 300, 0, 4, 0), (33, 64, 1000, 8, 8, 0),
         (64, 129, 2000, 0, 0, 3), (65, 128, 256, 0, 0, 0), (66, 257, 15, 1, 1, 1), (100, 300, 4001, 0, 0, 0), (128, 512, 144, 0, 0, 0), (129, 256, 640, 0, 3, 0),
         (257, 513, 129, 0, 0, 0), (300, 70, 1001, 7, 15, 0), (513, 300, 1008, 8, 16, 0), (200, 1, 63, 0, 0, 0), (70, 65, 64, 0, 0, 0), (3, 8200, 260, 0, 0, 0), (20, 20, 5000, 0, 0, 0)]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m,n,k,pad_x,pad_w,shift", SIZES)
def test_linear_and_its_gradient(m, n, k, pad_x, pad_w, shift, dtype):
    dev = need_gpu()
    W, S, w = four_bits(m + 7 * n + k, n, k, dev, pad_w)
    X = placed(randn(m + k, m, k) * 3, dtype, dev, pad_x, shift)
    dY = placed(randn(m + n, m, n) * 0.1, dtype, dev, pad_x, shift)
    wide = torch.full((m, n + 3), 5.0, dtype=dtype, device=dev)
    check_product(B.brsvd_linear_e2m1(X, W, S, out=wide[:, 1:n + 1]), X.double().cpu(), w.t())
    assert bool((wide[:, 0] == 5).all() and (wide[:, n + 1:] == 5).all())
    assert torch.equal(B.brsvd_linear_e2m1(X, W, S), wide[:, 1:n + 1])
    wide = torch.full((m, k + 3), 5.0, dtype=dtype, device=dev)
    check_product(B.brsvd_linear_e2m1_backward(dY, W, S, cols=k, out=wide[:, 1:k + 1]), dY.double().cpu(), w)
    assert bool((wide[:, 0] == 5).all() and (wide[:, k + 1:] == 5).all())


@pytest.mark.parametrize("m,n,k", [(5, 8200, 300), (20, 16400, 700), (40, 8193, 300), (130, 8200, 260), (1000, 2100, 400), (500, 34433, 203)])
def test_linear_with_many_columns(m, n, k):
    """The ways that few rows are multiplied by their number and that of the columns, and tiles of both sizes, cut by their last round."""
    dev = need_gpu()
    W, S, w = four_bits(m + 7 * n + k, n, k, dev)
    X = randn(m + k, m, k).bfloat16().to(dev)
    check_product(B.brsvd_linear_e2m1(X, W, S), X.double().cpu(), w.t())
    dY = randn(m + n, m, n).bfloat16().to(dev)
    check_product(B.brsvd_linear_e2m1_backward(dY, W, S, cols=k), dY.double().cpu(), w)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m,n,k", [(1, 40, 200), (30, 40, 200), (60, 40, 200), (70, 260, 200), (300, 300, 520)])
def test_products_of_whole_numbers_are_exact(m, n, k, dtype):
    """Whole numbers whose sums are below 2^8 (bf16 holds them): any index that is off shows."""
    dev = need_gpu()
    g = torch.Generator().manual_seed(m)
    code = torch.tensor([0, 0, 0, 0, 0, 0, 2, 10])[torch.randint(0, 8, (n, k), generator=g)]       # 0, 1, -1
    W = (code[:, ::2] | code[:, 1::2] << 4).to(torch.uint8).to(dev).view(torch.float4_e2m1fn_x2)
    S = torch.full((n, -(-k // 32)), 127, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu)
    w = values(code, torch.full((n, -(-k // 32)), 127))
    X, dY = (torch.randint(-1, 2, s, generator=g).to(dtype).to(dev) for s in ((m, k), (m, n)))
    y, dx = X.double().cpu() @ w.t(), dY.double().cpu() @ w
    assert float(y.abs().max()) < 256 and float(dx.abs().max()) < 256
    assert torch.equal(B.brsvd_linear_e2m1(X, W, S).double().cpu(), y) and torch.equal(B.brsvd_linear_e2m1_backward(dY, W, S).double().cpu(), dx)


@pytest.mark.parametrize("m", [1, 20, 64, 65, 300])
def test_scales_at_the_ends_of_their_range(m):
    """Scales from 2^-127 to 2^125 in one row each, activations of the reciprocal size: bf16 holds every number, and so does the result."""
    dev = need_gpu()
    W, _, _ = four_bits(3, 300, 256, dev)
    b = W.view(torch.uint8).long().cpu()
    code = torch.stack([b & 15, b >> 4], dim=2).view(300, -1)
    s = (torch.arange(300) % 253).to(torch.uint8)[:, None].repeat(1, 8)
    w = values(code, s.long())
    X = (randn(4, m, 256) * 2.0 ** -6).bfloat16().to(dev)
    got = B.brsvd_linear_e2m1(X, W, s.to(dev).view(torch.float8_e8m0fnu))
    want, size = X.double().cpu() @ w.t(), X.double().cpu().abs() @ w.abs().t()
    bound = size * 2.0 ** -23 * 288 + 2.0 ** -149 * 288
    bound = bound + ROUND[torch.bfloat16] * (want.abs() + bound) + FINEST[torch.bfloat16]
    assert bool(((got.double().cpu() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("m", [1, 20, 50, 100, 300])
def test_nan_stays_in_its_row_and_column(m, dtype):
    """A scale NaN makes its row's results NaN, a number that is not finite those of its row of X; nothing else changes a bit."""
    dev = need_gpu()
    W, S, _ = four_bits(5, 290, 300, dev)
    X, dY = randn(4, m, 300).to(dtype).to(dev), randn(6, m, 290).to(dtype).to(dev)
    y, dx = B.brsvd_linear_e2m1(X, W, S), B.brsvd_linear_e2m1_backward(dY, W, S)
    s = S.view(torch.uint8).clone()
    s[289, 9] = 255                          # numbers 288 to 299 of the last row
    s = s.view(torch.float8_e8m0fnu)
    got, gdx = B.brsvd_linear_e2m1(X, W, s), B.brsvd_linear_e2m1_backward(dY, W, s)
    assert torch.equal(got[:, :289], y[:, :289]) and bool(torch.isnan(got[:, 289]).all())
    assert torch.equal(gdx[:, :288], dx[:, :288]) and bool(torch.isnan(gdx[:, 288:]).all())
    X[m - 1, 299], dY[m - 1, 3] = float("nan"), float("inf")
    got, gdx = B.brsvd_linear_e2m1(X, W, S), B.brsvd_linear_e2m1_backward(dY, W, S)
    assert torch.equal(got[:m - 1], y[:m - 1]) and bool(torch.isnan(got[m - 1]).all())
    assert torch.equal(gdx[:m - 1], dx[:m - 1]) and not bool(torch.isfinite(gdx[m - 1]).any())


@pytest.mark.parametrize("m", [3, 100])
def test_half_byte_behind_a_row_is_no_number(m):
    """Odd rows whose last byte has a 6 behind the number, at a scale whose 6 no bf16 holds: it must not become 0 times infinity."""
    dev = need_gpu()
    code = torch.full((40, 34), 7)
    code[:, 32] = 1
    W = (code[:, ::2] | code[:, 1::2] << 4).to(torch.uint8).to(dev).view(torch.float4_e2m1fn_x2)
    s = torch.tensor([[100, 254]], dtype=torch.uint8).repeat(40, 1)
    X = torch.ones(m, 33, dtype=torch.bfloat16)
    X[:, 32] = 2.0 ** -100
    got = B.brsvd_linear_e2m1(X.to(dev), W, s.to(dev).view(torch.float8_e8m0fnu))
    assert bool((got == 2.0 ** 26).all())
    back = B.brsvd_dequantize_e2m1(W, s.to(dev).view(torch.float8_e8m0fnu), cols=33)
    assert bool((back[:, 32] == 2.0 ** 126).all())
    dx = B.brsvd_linear_e2m1_backward(torch.full((m, 40), 2.0 ** -100, dtype=torch.bfloat16, device=dev), W, s.to(dev).view(torch.float8_e8m0fnu), cols=33)
    assert bool((dx[:, 32] == 40 * 2.0 ** 26).all())


def test_sizes_of_zero():
    dev = need_gpu()
    for rows, cols in ((0, 5), (5, 0)):
        Q, S = B.brsvd_quantize_e2m1(torch.empty(rows, cols, device=dev))
        assert tuple(Q.shape) == (rows, (cols + 1) // 2) and B.brsvd_dequantize_e2m1(Q, S, cols=cols).shape == (rows, cols)
    W, S, _ = four_bits(1, 6, 20, dev)
    none = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    assert B.brsvd_linear_e2m1(none(0, 20), W, S).shape == (0, 6) and B.brsvd_linear_e2m1_backward(none(0, 6), W, S).shape == (0, 20)
    assert B.brsvd_linear_e2m1(none(3, 20), W[:0], S[:0]).shape == (3, 0)
    dx = B.brsvd_linear_e2m1_backward(none(3, 0), W[:0], S[:0])
    assert dx.shape == (3, 20) and not bool(dx.any())
    y = B.brsvd_linear_e2m1(none(3, 0), W[:, :0], S[:, :0])
    assert y.shape == (3, 6) and not bool(y.any()) and B.brsvd_linear_e2m1_backward(none(3, 6), W[:, :0], S[:, :0]).shape == (3, 0)


def test_offsets_beyond_32_bits():
    """A matrix of more than 2^32 bytes: the last rows are multiplied as they are alone, and cast."""
    dev = need_gpu()
    rows, cols = 140000, 65536
    W = torch.zeros(rows, cols // 2, dtype=torch.uint8, device=dev)
    S = torch.full((rows, cols // 32), 127, dtype=torch.uint8, device=dev)
    tail, ts, w = four_bits(7, 300, cols, dev)
    W[-300:], S[-300:] = tail.view(torch.uint8), ts.view(torch.uint8)
    W, S = W.view(torch.float4_e2m1fn_x2), S.view(torch.float8_e8m0fnu)
    X = randn(4, 100, cols).bfloat16().to(dev)
    for m in (4, 100):
        got = B.brsvd_linear_e2m1(X[:m], W, S)
        check_product(got[:, -300:], X[:m].double().cpu(), w.t())
        assert not bool(got[:, :-300].any())
    dY = torch.zeros(70, rows, dtype=torch.bfloat16, device=dev)
    dY[:, -300:] = randn(5, 70, 300).bfloat16().to(dev)
    dx = B.brsvd_linear_e2m1_backward(dY, W, S)
    want, size = dY[:, -300:].double().cpu() @ w, dY[:, -300:].double().cpu().abs() @ w.abs()
    bound = size * 2.0 ** -23 * 332
    assert bool(((dx.double().cpu() - want).abs() <= bound + ROUND[torch.bfloat16] * (want.abs() + bound)).all())
    back = B.brsvd_dequantize_e2m1(W[-70000:], S[-70000:], dtype=torch.bfloat16)
    assert torch.equal(back[-300:].double().cpu(), w) and not bool(back[:-300].any())
    Q, s = B.brsvd_quantize_e2m1(back)
    assert torch.equal(B.brsvd_dequantize_e2m1(Q[-300:], s[-300:], dtype=torch.bfloat16), back[-300:]) and not bool(Q[:-300].view(torch.uint8).any())


def test_casts_of_more_groups_than_a_launch_takes():
    """2^31 + 300 columns in one row, and rows whose groups are more than 2^30 in all: the ends are cast as they are alone."""
    dev = need_gpu()
    cols = 2 ** 31 + 300
    X = torch.zeros(1, cols, dtype=torch.bfloat16, device=dev)
    tail = randn(5, 1, 556).bfloat16().to(dev)
    X[:, -556:] = tail                     # from a multiple of 32 on
    Q, S = B.brsvd_quantize_e2m1(X)
    q, s = B.brsvd_quantize_e2m1(tail)
    assert torch.equal(Q[:, -278:].view(torch.uint8), q.view(torch.uint8)) and torch.equal(S[:, -18:].view(torch.uint8), s.view(torch.uint8))
    X.zero_()
    assert torch.equal(B.brsvd_dequantize_e2m1(Q, S, dtype=torch.bfloat16)[:, -556:], B.brsvd_dequantize_e2m1(q, s, dtype=torch.bfloat16))
    del X, Q, S
    rows, period = 2 ** 30 + 77, 2 ** 20
    x = randn(11, period).bfloat16().to(dev)
    Q, S = B.brsvd_quantize_e2m1(x.repeat(-(-rows // period))[:rows, None])
    q, s = B.brsvd_quantize_e2m1(x[:, None])
    for i in (0, period, 2 ** 29, rows // period * period - period, rows // period * period):
        n = min(period, rows - i)
        assert torch.equal(Q[i:i + n].view(torch.uint8), q[:n].view(torch.uint8)) and torch.equal(S[i:i + n].view(torch.uint8), s[:n].view(torch.uint8)), i


@pytest.mark.parametrize("m", [5, 100, 300])
def test_repeats_itself_in_graphs_and_on_other_streams(m):
    dev = need_gpu()
    X, dY = randn(8, m, 701).bfloat16().to(dev), randn(9, m, 400).bfloat16().to(dev)
    W, S, _ = four_bits(2, 400, 701, dev)
    y, dx = B.brsvd_linear_e2m1(X, W, S), B.brsvd_linear_e2m1_backward(dY, W, S, cols=701)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.brsvd_linear_e2m1(X, W, S, stream=side), B.brsvd_linear_e2m1_backward(dY, W, S, cols=701, stream=side)
    side.synchronize()
    assert torch.equal(got[0], y) and torch.equal(got[1], dx)
    # the matrix cores do not round a sum and its negative alike: each replay is held to the call on the same numbers
    other = B.brsvd_linear_e2m1(-X, W, S), B.brsvd_linear_e2m1_backward(-dY, W, S, cols=701)
    graph = torch.cuda.CUDAGraph()
    x, g = X.clone(), dY.clone()
    with torch.cuda.graph(graph):
        a, b = B.brsvd_linear_e2m1(x, W, S), B.brsvd_linear_e2m1_backward(g, W, S, cols=701)
        q, s = B.brsvd_quantize_e2m1(x)
        c = B.brsvd_dequantize_e2m1(q, s, cols=701)
    back = B.brsvd_dequantize_e2m1(*B.brsvd_quantize_e2m1(X), cols=701)
    for i in range(4):
        sign = 1 if i % 2 == 0 else -1
        x.copy_(X * sign)
        g.copy_(dY * sign)
        graph.replay()
        torch.cuda.synchronize()
        want = (y, dx) if sign == 1 else other
        assert torch.equal(a, want[0]) and torch.equal(b, want[1]) and torch.equal(c, sign * back)
        torch.randn(1000, 1000, device=dev).sum().item()


def test_refusals():
    dev = need_gpu()
    X = torch.ones(4, 256, dtype=torch.bfloat16, device=dev)
    Q, S = B.brsvd_quantize_e2m1(X)
    for call in (lambda: B.brsvd_quantize_e2m1(X.double()), lambda: B.brsvd_quantize_e2m1(X.cpu()), lambda: B.brsvd_quantize_e2m1(X.t()), lambda: B.brsvd_quantize_e2m1(X[0]),
                 lambda: B.brsvd_linear_e2m1(X.float(), Q, S), lambda: B.brsvd_linear_e2m1(X[:, :128], Q, S), lambda: B.brsvd_linear_e2m1(X, Q[:, :64], S),
                 lambda: B.brsvd_linear_e2m1(X, Q, S[:, :4]), lambda: B.brsvd_linear_e2m1(X, Q, S.view(torch.uint8)), lambda: B.brsvd_linear_e2m1(X, Q.view(torch.uint8), S),
                 lambda: B.brsvd_linear_e2m1(X, Q, S, out=torch.empty(4, 5, device=dev)), lambda: B.brsvd_linear_e2m1(X[0], Q, S),
                 lambda: B.brsvd_linear_e2m1_backward(X, Q, S), lambda: B.brsvd_dequantize_e2m1(X, S), lambda: B.brsvd_dequantize_e2m1(Q, S, dtype=torch.float64),
                 lambda: B.brsvd_dequantize_e2m1(Q, S[:2])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.brsvd_dequantize_e2m1(Q, S, cols=254), lambda: B.brsvd_dequantize_e2m1(Q, S, cols=257), lambda: B.brsvd_linear_e2m1_backward(X[:, :4], Q, S, cols=12)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("m,n,k", [(530001, 64, 4099), (70001, 33000, 64)])
def test_products_of_more_than_4_gib(m, n, k):
    """Operands and results whose bytes, and results whose numbers, pass 32 bits: rows at both ends and where they pass."""
    dev = need_gpu()
    W, S, w = four_bits(m, n, k, dev)
    X = randn(m, 997, k).bfloat16().to(dev).repeat(-(-m // 997), 1)[:m]
    Y = B.brsvd_linear_e2m1(X, W, S)
    dX = B.brsvd_linear_e2m1_backward(Y, W, S, cols=k)
    widest = max(n, k)
    for first in (0, 2 ** 31 // widest - 20, 2 ** 32 // (2 * widest) + 1, m - 60):
        at = slice(min(first, m - 60), min(first, m - 60) + 60)
        check_product(Y[at], X[at].double().cpu(), w.t())
        check_product(dX[at], Y[at].double().cpu(), w)


@pytest.mark.parametrize("m,n,k", [(3, 40, 49153 + 100), (16, 33, 98437), (5, 17, 49024), (9, 4112, 24448 + 33), (20, 12000, 9600 * 2 + 64)])
def test_more_scales_than_a_workgroup_holds(m, n, k):
    """Few rows and a long contraction: the scales of a workgroup's rows of W come in parts.  The first and the last of W's rows against 64 bits."""
    dev = need_gpu()
    g = torch.Generator(device=dev).manual_seed(k)
    W = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, device=dev).to(torch.uint8)
    S = torch.randint(124, 131, (n, -(-k // 32)), generator=g, device=dev).to(torch.uint8)
    X = randn(m, m, k).bfloat16().to(dev)
    Y = B.brsvd_linear_e2m1(X, W.view(torch.float4_e2m1fn_x2), S.view(torch.float8_e8m0fnu))
    for at in (slice(0, 20), slice(max(n - 90, 0), n)):
        b = W[at].long().cpu()
        w = values(torch.stack([b & 15, b >> 4], dim=2).view(b.shape[0], -1)[:, :k], S[at].long().cpu())
        check_product(Y[:, at], X.double().cpu(), w.t())


@pytest.mark.parametrize("m", [1, 3, 20, 100, 300])
@pytest.mark.parametrize("n,k", [(5, 1), (40, 2), (33, 9), (70, 29), (70, 30), (70, 31), (70, 33), (300, 61), (300, 95), (40, 127), (40, 129), (40, 135), (300, 257), (300, 259), (20, 286), (20, 287), (64, 2001)])
def test_rows_that_end_anywhere(m, n, k):
    """The last piece of a row comes from in front of its end where the row has so much; nothing in front of a short row is read (NaN there would show)."""
    dev = need_gpu()
    store = torch.full((n * ((k + 1) // 2) + 64,), 0xff, dtype=torch.uint8, device=dev)
    W, S, w = four_bits(m + n + k, n, k, dev)
    flat = store[48:48 + n * ((k + 1) // 2)].view(n, (k + 1) // 2)
    flat.copy_(W.view(torch.uint8))
    x = torch.full((m * k + 64,), float("nan"), dtype=torch.bfloat16, device=dev)
    X = x[24:24 + m * k].view(m, k)
    X.copy_(randn(k + m, m, k))
    check_product(B.brsvd_linear_e2m1(X, flat.view(torch.float4_e2m1fn_x2), S), X.double().cpu(), w.t())
    dY = randn(m, m, n).bfloat16().to(dev)
    check_product(B.brsvd_linear_e2m1_backward(dY, flat.view(torch.float4_e2m1fn_x2), S, cols=k), dY.double().cpu(), w)
