"""The calls on a model's matrices where numbers or sizes leave the usual range."""
import math

import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e4m3 import cast_by_definition, codes, placed, randn
from tests.test_gpu_head import FINEST, HALF, ROUND, Reference, problem, teacher_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cast_of_more_than_2_to_the_31_columns(dtype):
    """One row: its last blocks are cast as they are alone."""
    dev = need_gpu()
    cols = 2 ** 31 + 300
    X = torch.zeros(1, cols, dtype=dtype, device=dev)
    tail = randn(5, 1, 556).to(dtype).to(dev)
    X[:, -556:] = tail                     # from a multiple of 128 on
    Q, S = B.brsvd_quantize_e4m3(X)
    del X
    q, s = B.brsvd_quantize_e4m3(tail)
    assert torch.equal(codes(Q[:, -556:]), codes(q)) and torch.equal(S[:, -5:], s)
    assert bool((S[:, :-5] == 1).all())
    for i in range(0, cols - 556, 2 ** 28):
        assert not bool(Q[:, i:min(i + 2 ** 28, cols - 556)].view(torch.uint8).any()), i


MANY = 2 ** 24 + 77            # workgroups of 256 threads that are more than the 2^32 threads of a launch


def test_gradients_of_more_tokens_than_a_launch_has_workgroups():
    """2^24 + 77 tokens, whose rows repeat after 2^16: each part has the bits of the first."""
    dev = need_gpu()
    vocab, dim, period = 40, 8, 2 ** 16
    H, W, y, g = problem(period, vocab, dim, torch.bfloat16, dev)
    y[1::5] = -1
    each = torch.rand(period, generator=g) + 0.5
    where = torch.arange(MANY, device=dev) % period
    big, labels, grad = H[where], y.to(dev)[where], each.to(dev)[where]
    loss, lse = B.brsvd_xent_forward(big, W, labels)
    dH, dW = B.brsvd_xent_backward(big, W, labels, lse, grad)
    loss1, lse1 = B.brsvd_xent_forward(H, W, y.to(dev))
    dH1, dW1 = B.brsvd_xent_backward(H, W, y.to(dev), lse1, each.to(dev))
    for i in range(0, MANY, period):
        n = min(period, MANY - i)
        assert torch.equal(loss[i:i + n], loss1[:n]) and torch.equal(lse[i:i + n], lse1[:n]) and torch.equal(dH[i:i + n], dH1[:n]), i
    # dW: 256 of the first part's and 77 tokens; 2^19 additions a sum (32 tokens an instruction) that lose at most a step each, of the sum of |terms|, and 2^-9 of bf16
    h = H.double().cpu()
    p = torch.softmax(h @ W.double().cpu().t(), dim=1)
    size = ((p + 1.0 * (torch.arange(vocab) == y[:, None])) * each.double()[:, None] * (y >= 0)[:, None]).t() @ h.abs()
    bound = 257 * size * (2.0 ** -4 + 2.0 ** -8) + 77 * 2 * 1.5 * float(h.abs().max())
    assert bool(((dW.double() - 256 * dW1.double()).abs().cpu() <= bound).all())


def test_distillation_of_more_tokens_than_a_launch_has_workgroups():
    dev = need_gpu()
    vocab, dim, period, top = 40, 8, 2 ** 16, 2
    H, W, _, g = problem(period, vocab, dim, torch.bfloat16, dev)
    ids = torch.randint(-1, vocab, (period, top), generator=g).to(dev)
    a = torch.randn(period, top, generator=g).to(dev)
    where = torch.arange(MANY, device=dev) % period
    one = torch.ones(1, device=dev)
    big, bids, ba = H[where], ids[where], a[where]
    loss, lse, z = B.brsvd_distill_forward(big, W, bids, ba, 2.0)
    dH, _ = B.brsvd_distill_backward(big, W, bids, ba, 2.0, lse, z, one, need_dW=False)
    loss1, lse1, z1 = B.brsvd_distill_forward(H, W, ids, a, 2.0)
    dH1, _ = B.brsvd_distill_backward(H, W, ids, a, 2.0, lse1, z1, one, need_dW=False)
    for i in range(0, MANY, period):
        n = min(period, MANY - i)
        assert torch.equal(loss[i:i + n], loss1[:n]) and torch.equal(z[i:i + n], z1[:n]) and torch.equal(dH[i:i + n], dH1[:n]), i


def test_no_tokens_of_more_words_than_a_launch_has_workgroups():
    dev = need_gpu()
    W = torch.ones(MANY, 1, dtype=torch.bfloat16, device=dev)
    none = torch.empty(0, device=dev)
    dW = B.brsvd_xent_backward(W[:0], W, none.long(), none, none)[1]
    assert dW.shape == W.shape and not bool(dW.any())


def test_casts_of_more_rows_than_a_launch_has_workgroups():
    """2^29 + 77 rows of one number, whose values repeat after 2^20."""
    dev = need_gpu()
    rows, period = 2 ** 29 + 77, 2 ** 20
    x = randn(11, period).float().to(dev)
    X = x.repeat(-(-rows // period))[:rows, None]
    Q, S = B.brsvd_quantize_e4m3(X)
    q, s = B.brsvd_quantize_e4m3(x[:, None])
    back = B.brsvd_dequantize_e4m3(Q, S)
    del X
    one = B.brsvd_dequantize_e4m3(q, s)
    for i in (0, period, 2 ** 28, rows // period * period - period, rows // period * period):
        n = min(period, rows - i)
        assert torch.equal(codes(Q[i:i + n]), codes(q[:n])) and torch.equal(S[i:i + n], s[:n]) and torch.equal(back[i:i + n], one[:n]), i


def test_casts_of_more_columns_than_a_launch_has_workgroups():
    """2^31 + 300 columns in all ways of a cast: the blocks at the end are those of the end alone."""
    dev = need_gpu()
    cols = 2 ** 31 + 300
    X = torch.zeros(1, cols, dtype=torch.bfloat16, device=dev)
    tail = randn(5, 1, 556).to(torch.bfloat16).to(dev)
    X[:, -556:] = tail                     # from a multiple of 128 on
    Q, S, Qt, St = B.brsvd_quantize_e4m3(X, transpose=True)
    q, s, qt, st = B.brsvd_quantize_e4m3(tail, transpose=True)
    assert torch.equal(codes(Q[:, -556:]), codes(q)) and torch.equal(S[:, -5:], s)
    assert torch.equal(codes(Qt[-556:]), codes(qt)) and torch.equal(St[-556:], st)
    assert not bool(Qt[:2 ** 20].view(torch.uint8).any()) and bool((St[:-556] == 1).all())
    del Qt, St
    back = B.brsvd_dequantize_e4m3(Q, S)
    assert torch.equal(back[:, -556:], B.brsvd_dequantize_e4m3(q, s)) and not bool(back[:, :2 ** 20].any())
    del back
    Q, S = B.brsvd_quantize_e4m3(X, block_rows=128)
    assert torch.equal(codes(Q[:, -556:]), codes(q)) and torch.equal(S[:, -5:], s) and not bool(Q[:, :2 ** 20].view(torch.uint8).any())


@pytest.mark.parametrize("need_dH,need_dW", [(True, False), (False, True), (True, True)])
def test_one_gradient_of_no_tokens(need_dH, need_dW):
    dev = need_gpu()
    H, W, y, _ = problem(3, 300, 40, torch.float16, dev)
    none, ids = torch.empty(0, device=dev), torch.empty(0, 4, dtype=torch.int64, device=dev)
    for dH, dW in (B.brsvd_xent_backward(H[:0], W, y[:0].to(dev), none, none, need_dH=need_dH, need_dW=need_dW),
                   B.brsvd_distill_backward(H[:0], W, ids, ids.float(), 2.0, none, ids.float(), none, need_dH=need_dH, need_dW=need_dW)):
        assert dH.shape == (0, 40) if need_dH else dH is None
        assert (dW.shape == W.shape and not bool(dW.any())) if need_dW else dW is None


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("tokens,vocab", [(10, 600), (66, 600), (300, 512), (300, 700)])
def test_rows_of_infinite_logits(tokens, vocab, dtype):
    """A logit of +inf makes lse +inf, a row of -inf makes it -inf; the loss is the difference, and no other row changes a bit."""
    dev = need_gpu()
    H, W, y, _ = problem(tokens, vocab, 64, dtype, dev)
    W[:, 0] = -1.0
    W[:, 5] = torch.where(torch.arange(vocab, device=dev) % 3 == 0, -0.5, 0.25)
    want = B.brsvd_xent_forward(H, W, y.to(dev))
    grad = torch.ones(tokens, device=dev)
    dH_want = B.brsvd_xent_backward(H, W, y.to(dev), want[1], grad, need_dW=False)[0]
    H[3, 5] = math.inf             # +inf and -inf
    H[4, 0] = math.inf             # -inf everywhere
    H[6, 0] = -math.inf            # +inf everywhere
    H[7, 9] = math.nan
    y[3] = 3                       # a logit of -inf: the loss is +inf
    z = H.double().cpu() @ W.double().cpu().t()
    ref = torch.logsumexp(z, dim=1)
    loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
    odd = torch.tensor([3, 4, 6, 7])
    assert ref[odd][:3].tolist() == [math.inf, -math.inf, math.inf]
    torch.testing.assert_close(lse.double().cpu()[odd], ref[odd], rtol=0, atol=0, equal_nan=True)
    torch.testing.assert_close(loss.double().cpu()[odd], (ref - z.gather(1, y[:, None])[:, 0])[odd], rtol=0, atol=0, equal_nan=True)
    keep = torch.ones(tokens, dtype=torch.bool, device=dev)
    keep[odd] = False
    dH = B.brsvd_xent_backward(H, W, y.to(dev), lse, grad, need_dW=False)[0]
    for a, b in ((loss, want[0]), (lse, want[1]), (dH, dH_want)):
        assert torch.equal(a[keep], b[keep])
    ids, a = y[:, None].to(dev).contiguous(), torch.zeros(tokens, 1, device=dev)
    assert torch.equal(B.brsvd_distill_forward(H, W, ids, a)[1].nan_to_num(7.0, 8.0, 9.0), lse.nan_to_num(7.0, 8.0, 9.0))


@pytest.mark.parametrize("tau", [1.0, 0.5, 0.25])
def test_teacher_logits_of_the_lowest_value(tau):
    """Masked with the lowest fp32 number instead of -inf: such an entry is listed and has no part, unless a token has no others: then they are alike."""
    dev = need_gpu()
    H, W, _, g = problem(70, 500, 40, torch.bfloat16, dev)
    ids = torch.randint(0, 500, (70, 6), generator=g)
    a = torch.randn(70, 6, generator=g) * 3
    low = torch.finfo(torch.float32).min
    a[::3, 2:] = low
    a[5], a[6, 1:] = low, -math.inf
    a[6, 0] = low
    a[7] = torch.tensor([3e38, low, 0.0, 3e38, -1.0, 1.0])
    ref = Reference(H, W, tau)
    want, target, counted, zs, off = teacher_reference(ref, ids, a, tau, 500)
    assert bool(torch.isfinite(want).all() and counted.all())
    loss, lse, z = B.brsvd_distill_forward(H, W, ids.to(dev), a.to(dev), tau)
    ref.check("loss", loss, want, off)
    grad = torch.ones(1, device=dev)
    dH, dW = B.brsvd_distill_backward(H, W, ids.to(dev), a.to(dev), tau, lse, z, grad)
    ref.check_gradients(dH, dW, target, tau * counted.double())


@pytest.mark.parametrize("tokens", [10, 66, 300])
@pytest.mark.parametrize("power", [10, 14, 20, 30])
def test_finite_logits_of_any_size(tokens, power):
    """Logits of up to 2^62, finite in fp32: lse is theirs to within their rounding, not an infinity."""
    dev = need_gpu()
    H, W, y, _ = problem(tokens, 600, 64, torch.bfloat16, dev, scale=2.0 ** power)
    W *= 2.0 ** power
    ref = Reference(H, W)
    loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
    ref.check_lse(lse)
    zy = ref.z.gather(1, y[:, None])[:, 0]
    ref.check("loss", loss, ref.lse - zy, ref.dlse + ref.dz.amax(dim=1) + 2.0 ** -22 * (ref.lse - zy).abs())


@pytest.mark.parametrize("power", [-70, -40, 40])
def test_temperatures_whose_square_leaves_fp32(power):
    """tau^2 and 1 / tau^2 need not be numbers of fp32: the loss does where it is one."""
    dev = need_gpu()
    tau = 2.0 ** power
    H, W, _, g = problem(66, 300, 32, torch.bfloat16, dev)
    ids = torch.randint(0, 300, (66, 3), generator=g)
    a = torch.randn(66, 3, generator=g) * 3
    ref = Reference(H, W, tau)
    want, _, _, _, off = teacher_reference(ref, ids, a, tau, 300)
    loss, _, _ = B.brsvd_distill_forward(H, W, ids.to(dev), a.to(dev), tau)
    ref.check("loss", loss, want, off)
    if power < 0:
        assert float((off / want.abs().clamp(min=1e-300)).median()) < 2.0 ** -8


def test_fp16_gradients_keep_probabilities_down_to_2_to_the_minus_28():
    """Two words, the second with a probability p of 2^-28 to 2^-27 and a row of W that lets its gradient show in fp16: G = g p is rounded by half a step of
    eleven bits, dH is that times a power of two and rounds nothing; beside that exp and lse in fp32 (z up to 20: 2^-17 is 16 of their steps)."""
    dev = need_gpu()
    tokens = 600
    H = torch.zeros(tokens, 3, dtype=torch.float16)
    H[:, 0] = 18.75
    H[:, 1] = torch.linspace(0.0, 0.656, tokens)
    W = torch.tensor([[1.0, 1.0, 0.0], [0.0, 0.0, 256.0]], dtype=torch.float16)
    z = H.double() @ W.double().t()
    p = torch.softmax(z, dim=1)[:, 1]
    assert 2.0 ** -28 <= float(p.min()) and float(p.max()) < 2.0 ** -26.9
    y = torch.zeros(tokens, dtype=torch.int64, device=dev)
    H, W = H.to(dev), W.to(dev)
    loss, lse = B.brsvd_xent_forward(H, W, y)
    dH, _ = B.brsvd_xent_backward(H, W, y, lse, torch.full((1,), 1024.0, device=dev), need_dW=False)
    want = 1024.0 * p * 256.0
    err = (dH[:, 2].double().cpu() - want).abs() / want
    assert float(err.max()) <= (1 + 2.0 ** -11) * (1 + 2.0 ** -17) - 1


def test_fp16_gradients_of_factors_that_differ_by_orders_of_magnitude():
    """One power of two serves all tokens: an entry of G is off by half a step of its eleven bits, or where it is small by max|g| 2^-39 (half of fp16's finest
    step, 2^-25, over 2^14 / max|g|), whatever the token's own factor.  Each row of dH is held to that."""
    dev = need_gpu()
    tokens, vocab, dim = 300, 700, 64
    H, W, y, _ = problem(tokens, vocab, dim, torch.float16, dev)
    ref = Reference(H, W)
    loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
    factor = 2.0 ** (10 - torch.arange(tokens, dtype=torch.float64) % 25)
    dH, _ = B.brsvd_xent_backward(H, W, y.to(dev), lse, factor.float().to(dev), need_dW=False)
    target = torch.zeros_like(ref.z).scatter_(1, y[:, None], 1.0)
    p = torch.exp(ref.z - ref.lse[:, None])
    G = factor[:, None] * (p - target)
    off = factor[:, None] * (p * (ref.dz + ref.dlse[:, None]) * 1.01 + 2.0 ** -20 * (p + target))
    u = ROUND[torch.float16]
    off = off + u * (G.abs() + off) + 2.0 ** 10 * 2.0 ** -39
    want = G @ ref.w
    bound = off @ ref.w.abs() + (G.abs() + off) @ ref.w.abs() * 2.0 ** -23 * (vocab + 70)
    ref.check("dH", dH, want, bound + u * (want.abs() + bound) + FINEST[torch.float16])


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 127, 1, 0), (128, 128, 0, 0), (129, 257, 0, 1), (260, 8, 8, 0)])
def test_cast_of_the_transpose_alone(rows, cols, pad, shift, dtype, block):
    """Q and S may be left out: Qt and St are the cast of X^T, and nothing beside them is written."""
    dev = need_gpu()
    X = placed(randn(rows * 1000 + cols, rows, cols), dtype, dev, pad, shift)
    qt = torch.full((cols, rows + 3), 99, dtype=torch.uint8, device=dev)
    st = torch.full((cols + 1 if block == 1 else -(-cols // 128) + 1, -(-rows // 128)), 9.0, device=dev)
    kind = {torch.float32: B.BRSVD_DTYPE_F32, torch.bfloat16: B.BRSVD_DTYPE_BF16, torch.float16: B.BRSVD_DTYPE_F16}[dtype]
    status = B.lib().brsvd_quantize_e4m3(X.data_ptr(), cols + pad, rows, cols, kind, block, None, 0, None, qt.data_ptr(), rows + 3, st.data_ptr(),
                                         torch.cuda.current_stream().cuda_stream or None)
    torch.cuda.synchronize()
    q, s = cast_by_definition(X.double().cpu().t().contiguous(), block)
    assert status == B.BRSVD_OK and torch.equal(codes(qt[:, :rows].view(torch.float8_e4m3fn)), q) and torch.equal(st[:-1].double().cpu(), s)
    assert bool((qt[:, rows:] == 99).all() and (st[-1] == 9).all())


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
def test_same_bits_whatever_torchs_default_type(default):
    dev = need_gpu()
    H, W, y, g = problem(70, 500, 40, torch.bfloat16, dev)
    ids, a = torch.randint(0, 500, (70, 3), generator=g).to(dev), torch.randn(70, 3, generator=g).to(dev)
    grad = torch.ones(70, device=dev)

    def all_calls():
        Q, S, Qt, St = B.brsvd_quantize_e4m3(H, transpose=True)
        loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
        distilled = B.brsvd_distill_forward(H, W, ids, a, 2.0)
        q, s = B.brsvd_quantize_e4m3(W, block_rows=128)
        return (codes(Q), S, codes(Qt), St, loss, lse, *B.brsvd_xent_backward(H, W, y.to(dev), lse, grad), *distilled,
                *B.brsvd_distill_backward(H, W, ids, a, 2.0, distilled[1], distilled[2], grad), B.brsvd_dequantize_e4m3(Q, S), B.brsvd_linear_e4m3(H, q, s))
    want = all_calls()
    torch.set_default_dtype(default)
    try:
        got = all_calls()
    finally:
        torch.set_default_dtype(torch.float32)
    assert all(x.dtype == w.dtype and torch.equal(x, w) for x, w in zip(got, want))
