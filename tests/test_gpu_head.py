"""Cross entropy and distillation over a vocabulary without the logits, against plain formulas in 64 bits and against differences: sizes at the
edges of tiles and pieces, tokens that do not count, rows at any alignment, large logits, duplicate and missing teacher entries."""
import math

import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
# unit roundoff of a 16-bit number, and half its finest step
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FINEST = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
SIZES = [(1, 1, 1), (1, 7, 5), (3, 256, 8), (5, 300, 16), (64, 257, 24), (65, 1000, 33), (128, 512, 64), (130, 513, 100), (257, 2000, 64), (300, 700, 272)]


def randn(seed, *shape):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def placed(x, dtype, dev, pad, shift):
    rows, cols = x.shape
    flat = torch.full((rows * (cols + pad) + shift + 8,), 7.0, device=dev).to(dtype)
    view = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x.to(dtype))
    return view


class Reference:
    """The formulas in 64 bits, and what each result may be off by: bounds that hold for any order of the sums.
    z: 64 products a step, exact in fp32, their additions and those of the steps lose at most a step of fp32 each.  lse: the same, as it moves no more than
    its largest z, and about 1e-6 of the exponent's size for exp, log and sums in fp32.  G: one rounding to 16 bits.  Gradients: additions in fp32
    over the contraction, one rounding at the end."""

    def __init__(self, H, W, tau=1.0):
        self.h, self.w, self.tau, self.dtype = H.double().cpu(), W.double().cpu(), tau, H.dtype
        self.z = self.h @ self.w.t()
        d = self.h.shape[1]
        self.dz = (self.h.abs() @ self.w.abs().t()) * 2.0 ** -23 * (min(d, 64) + -(-d // 64) + 2)
        self.lse = torch.logsumexp(self.z / tau, dim=1)
        span = (self.z / tau).abs().amax(dim=1)
        self.dlse = self.dz.amax(dim=1) / tau + 2.0 ** -20 * (4 + span + self.lse.abs())

    def check(self, name, got, want, bound):
        err = (got.double().cpu() - want).abs()
        assert bool((err <= bound).all()), (name, float((err / bound.clamp(min=1e-300)).max()), float(err.max()))

    def check_lse(self, lse):
        self.check("lse", lse, self.lse, self.dlse)

    def check_gradients(self, dH, dW, target, factor):
        """target: the distribution subtracted; factor: of each token, 0 for those that do not count."""
        p = torch.exp(self.z / self.tau - self.lse[:, None])
        G = factor[:, None] * (p - target)
        off = factor.abs()[:, None] * p * (self.dz / self.tau + self.dlse[:, None]) * 1.01 + factor.abs()[:, None] * 2.0 ** -20 * (p + target)
        u = ROUND[self.dtype]
        off = off + u * (G.abs() + off) + float(factor.abs().max()) * 2.0 ** -37      # the rounding of G and what fp16 cannot hold of it
        size = G.abs() + off
        for name, got, A, Am, O, X in (("dH", dH, G, size, off, self.w), ("dW", dW, G.t(), size.t(), off.t(), self.h.where(factor[:, None] != 0, torch.zeros(())))):
            if got is None:
                continue
            want = A @ X
            bound = O @ X.abs() + (Am @ X.abs()) * 2.0 ** -23 * (A.shape[1] + 70)
            self.check(name, got, want, bound + u * (want.abs() + bound) + FINEST[self.dtype])


def problem(tokens, vocab, dim, dtype, dev, pad=0, shift=0, scale=1.0):
    H = placed(randn(tokens * 7 + dim, tokens, dim) * scale, dtype, dev, pad, shift)
    W = placed(randn(vocab * 3 + dim, vocab, dim) * 2 / math.sqrt(dim), dtype, dev, pad, shift)
    g = torch.Generator().manual_seed(tokens + vocab)
    return H, W, torch.randint(0, vocab, (tokens,), generator=g), g


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("tokens,vocab,dim", SIZES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_xent(tokens, vocab, dim, dtype, pad, shift):
    dev = need_gpu()
    H, W, y, g = problem(tokens, vocab, dim, dtype, dev, pad, shift)
    if tokens > 2:
        y[1], y[2] = -1, vocab                        # neither counts
    counted = (y >= 0) & (y < vocab)
    ref = Reference(H, W)
    loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
    ref.check_lse(lse)
    zy = ref.z.gather(1, y.clamp(0, vocab - 1)[:, None])[:, 0]
    ref.check("loss", loss, torch.where(counted, ref.lse - zy, 0.0), torch.where(counted, ref.dlse + ref.dz.amax(dim=1) + 2.0 ** -22 * (ref.lse - zy).abs(), 0.0))
    target = torch.zeros_like(ref.z)
    target[torch.nonzero(counted)[:, 0], y[counted]] = 1.0
    each = (torch.rand(tokens, generator=g) + 0.5).to(dev)
    for grad, piece in ((each, 0), (torch.full((1,), 0.25, device=dev), 256), (torch.full((1,), -3.0, device=dev).expand(tokens), 512)):
        dH, dW = B.brsvd_xent_backward(H, W, y.to(dev), lse, grad, piece=piece)
        factor = grad.double().cpu().expand(tokens) * counted
        ref.check_gradients(dH, dW, target, factor)
        assert not bool(dH[~counted.to(dev)].any())
    only, none = B.brsvd_xent_backward(H, W, y.to(dev), lse, each, need_dW=False)
    assert none is None and torch.equal(only, B.brsvd_xent_backward(H, W, y.to(dev), lse, each)[0])
    none, only = B.brsvd_xent_backward(H, W, y.to(dev), lse, each, need_dH=False)
    assert none is None and torch.equal(only, B.brsvd_xent_backward(H, W, y.to(dev), lse, each)[1])


@pytest.mark.parametrize("tokens,vocab,dim,pad", [(300, 70001, 24, 0), (300, 70001, 17, 0), (70, 40000, 136, 0), (20, 5000, 40, 8), (33, 5000, 1000, 0)])
def test_xent_of_many_tiles(tokens, vocab, dim, pad):
    """More tiles than workgroups at once, aligned and not, and the tiles for few tokens."""
    dev = need_gpu()
    H, W, y, g = problem(tokens, vocab, dim, torch.bfloat16, dev, pad)
    y[0], y[1] = vocab - 1, -1
    ref = Reference(H, W)
    loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
    ref.check_lse(lse)
    counted = y >= 0
    target = torch.zeros_like(ref.z)
    target[torch.nonzero(counted)[:, 0], y[counted]] = 1.0
    ref.check("loss", loss, torch.where(counted, ref.lse - (target * ref.z).sum(dim=1), 0.0), torch.where(counted, ref.dlse + ref.dz.amax(dim=1) + 2.0 ** -22 * (ref.lse + 9), 0.0))
    grad = (torch.rand(tokens, generator=g) + 0.5).to(dev)
    for piece in (0, 20000):
        dH, dW = B.brsvd_xent_backward(H, W, y.to(dev), lse, grad, piece=piece)
        ref.check_gradients(dH, dW, target, grad.double().cpu() * counted)


def test_xent_whose_last_round_of_tiles_is_cut():
    """1000 x 22433 logits are 352 tiles of 256 x 256, dW 264: most of them as they are, the others in halves, by a launch of their own.  Labels on both sides
    of the cut and at its edge."""
    dev = need_gpu()
    tokens, vocab, dim = 1000, 22433, 750
    H, W, y, g = problem(tokens, vocab, dim, torch.bfloat16, dev, 2)
    y[0], y[1], y[2], y[3], y[4] = vocab - 1, -1, 64 * 256 - 1, 64 * 256, 85 * 256
    ref = Reference(H, W)
    loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
    ref.check_lse(lse)
    counted = y >= 0
    target = torch.zeros_like(ref.z)
    target[torch.nonzero(counted)[:, 0], y[counted]] = 1.0
    zy = (target * ref.z).sum(dim=1)
    ref.check("loss", loss, torch.where(counted, ref.lse - zy, 0.0), torch.where(counted, ref.dlse + ref.dz.amax(dim=1) + 2.0 ** -22 * (ref.lse - zy).abs(), 0.0))
    grad = (torch.rand(tokens, generator=g) + 0.5).to(dev)
    dH, dW = B.brsvd_xent_backward(H, W, y.to(dev), lse, grad)
    ref.check_gradients(dH, dW, target, grad.double().cpu() * counted)


@pytest.mark.parametrize("dtype", HALF)
def test_what_does_not_count_reaches_nothing(dtype):
    """NaN and infinities in the hidden states of padding, half of the tokens: gradients are those of the others alone."""
    dev = need_gpu()
    H, W, y, g = problem(300, 700, 64, dtype, dev)
    y[::2] = -1
    H[::4], H[2::4] = float("nan"), float("inf")
    grad = torch.rand(300, generator=g).to(dev)
    yd = y.to(dev)
    loss, lse = B.brsvd_xent_forward(H, W, yd)
    assert not bool(loss[::2].any()) and bool(torch.isfinite(loss).all())
    dH, dW = B.brsvd_xent_backward(H, W, yd, lse, grad)
    yo = yd[1::2].contiguous()
    loss1, lse1 = B.brsvd_xent_forward(H[1::2], W, yo)
    dH1, dW1 = B.brsvd_xent_backward(H[1::2], W, yo, lse1, grad[1::2])
    assert torch.equal(loss[1::2], loss1) and torch.equal(dH[1::2], dH1) and torch.equal(dW, dW1)
    assert not bool(dH[::2].any()) and bool(torch.isfinite(dW).all())


def test_no_token_counts():
    dev = need_gpu()
    H, W, y, _ = problem(70, 300, 40, torch.bfloat16, dev)
    y = torch.full_like(y, -100).to(dev)
    loss, lse = B.brsvd_xent_forward(H, W, y)
    dH, dW = B.brsvd_xent_backward(H, W, y, lse, torch.ones(70, device=dev))
    assert not bool(loss.any()) and not bool(dH.any()) and not bool(dW.any())
    ids, a = torch.full((70, 3), -1, device=dev), torch.zeros(70, 3, device=dev)
    loss, lse, z = B.brsvd_distill_forward(H, W, ids, a)
    dH, dW = B.brsvd_distill_backward(H, W, ids, a, 1.0, lse, z, torch.ones(70, device=dev))
    assert not bool(loss.any()) and not bool(dH.any()) and not bool(dW.any()) and not bool(z.any())


def test_no_tokens():
    dev = need_gpu()
    H, W, y, _ = problem(3, 300, 40, torch.float16, dev)
    none = torch.empty(0, device=dev)
    loss, lse = B.brsvd_xent_forward(H[:0], W, y[:0].to(dev))
    dH, dW = B.brsvd_xent_backward(H[:0], W, y[:0].to(dev), none, none)
    assert loss.numel() == 0 and dH.shape == (0, 40) and dW.shape == W.shape and not bool(dW.any())
    ids = torch.empty(0, 4, dtype=torch.int64, device=dev)
    loss, lse, z = B.brsvd_distill_forward(H[:0], W, ids, ids.float())
    dH, dW = B.brsvd_distill_backward(H[:0], W, ids, ids.float(), 2.0, lse, z, none)
    assert dH.shape == (0, 40) and not bool(dW.any())


def test_logits_of_every_size():
    """Logits of thousands: the largest is taken off before any exponential; one word that has all the probability leaves a gradient of zero."""
    dev = need_gpu()
    H, W, y, _ = problem(66, 600, 64, torch.bfloat16, dev, scale=300.0)
    ref = Reference(H, W)
    assert float(ref.z.abs().max()) > 1000
    y = ref.z.argmax(dim=1)
    loss, lse = B.brsvd_xent_forward(H, W, y.to(dev))
    ref.check_lse(lse)
    grad = torch.ones(66, device=dev)
    dH, dW = B.brsvd_xent_backward(H, W, y.to(dev), lse, grad)
    assert bool(torch.isfinite(dH).all() and torch.isfinite(dW).all())
    sure = (ref.lse - ref.z.amax(dim=1)) < 1e-9
    assert bool(sure.any())
    # p is one up to the error of z - lse
    worst = float((ref.dz.amax(dim=1) + ref.dlse)[sure].max())
    assert float(dH[sure.to(dev)].abs().max()) <= 1.1 * worst * float(ref.w.abs().max()) + 1e-6


def test_infinite_logits():
    dev = need_gpu()
    H, W, y, _ = problem(66, 600, 64, torch.bfloat16, dev)
    want = B.brsvd_xent_forward(H, W, y.to(dev))[1]
    H[3, 5] = float("nan")
    lse = B.brsvd_xent_forward(H, W, y.to(dev))[1]
    keep = torch.arange(66, device=dev) != 3
    assert bool(torch.isnan(lse[3])) and torch.equal(lse[keep], want[keep])


def test_xent_gradient_against_differences():
    """(L(H + e D) - L(H - e D)) / 2e on numbers that bf16 holds exactly.  The third derivative of log sum exp along a direction with logits in [-c, c] is
    at most 6 c^3 (its third cumulant), so the difference is off by e^2 c^3, and by the losses' fp32 error over e."""
    dev = need_gpu()
    tokens, vocab, dim = 40, 300, 32
    g = torch.Generator().manual_seed(3)
    H = torch.randint(-8, 9, (tokens, dim), generator=g).double() / 8
    W = torch.randint(-8, 9, (vocab, dim), generator=g).double() / 32
    y = torch.randint(0, vocab, (tokens,), generator=g).to(dev)
    e = 2.0 ** -4
    put = lambda x: x.to(torch.bfloat16).to(dev)  # noqa: E731
    L = lambda h, w: B.brsvd_xent_forward(put(h), put(w), y)[0].double().cpu()  # noqa: E731
    lse = B.brsvd_xent_forward(put(H), put(W), y)[1]
    dH, dW = (x.double().cpu() for x in B.brsvd_xent_backward(put(H), put(W), y, lse, torch.ones(1, device=dev)))
    for i in range(3):
        D = torch.randint(-1, 2, (tokens, dim), generator=g).double()
        c = (D @ W.t()).abs().amax(dim=1)
        diff = (L(H + e * D, W) - L(H - e * D, W)) / (2 * e)
        got = (dH * D).sum(dim=1)
        bound = e * e * c ** 3 + 2e-5 / e + 2.0 ** -8 * 2 * (dH * D).abs().sum(dim=1) + 2.0 ** -8 * 2 * D.abs().sum(dim=1) * float(W.abs().max())
        assert bool(((diff - got).abs() <= bound).all())
        assert float(bound.max()) < 0.25 * float(got.abs().max())
        D = torch.randint(-1, 2, (vocab, dim), generator=g).double() / 4
        c = (H @ D.t()).abs().amax(dim=1)
        diff = ((L(H, W + e * D) - L(H, W - e * D)) / (2 * e)).sum()
        got = (dW * D).sum()
        bound = (e * e * c ** 3 + 2e-5 / e).sum() + 2.0 ** -8 * 2 * (dW * D).norm() * 4
        assert abs(float(diff - got)) <= float(bound)


def teacher_reference(ref, ids, a, tau, vocab):
    """(loss, q as a distribution over the vocabulary, counted, and what the loss may be off by)"""
    listed = (ids >= 0) & (ids < vocab) & (a > -math.inf)
    counted = listed.any(dim=1)
    logq = torch.log_softmax((a.double() / tau).masked_fill(~listed, -math.inf), dim=1)
    q = logq.exp().nan_to_num(0.0).masked_fill(~listed, 0.0)
    zs = ref.z.gather(1, ids.clamp(0, vocab - 1))
    terms = torch.where(listed, q * (logq.nan_to_num(0.0, 0.0, 0.0) - zs / tau + ref.lse[:, None]), torch.zeros((), dtype=torch.float64))
    target = torch.zeros_like(ref.z).scatter_add_(1, ids.clamp(0, vocab - 1), q)
    size = torch.where(listed, q * (logq.nan_to_num(0.0, 0.0, 0.0).abs() + (zs / tau).abs() + ref.lse.abs()[:, None]), torch.zeros((), dtype=torch.float64)).sum(dim=1)
    # the student's listed logits are summed in another order over all of dim
    dz = (ref.h.abs() @ ref.w.abs().t()).amax(dim=1) * 2.0 ** -23 * (ref.h.shape[1] + 8) / tau
    off = tau * tau * (ref.dlse + dz + size * 2.0 ** -18) * counted
    return terms.sum(dim=1) * tau * tau, target, counted, zs.masked_fill(~listed, 0.0), off


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("top,tau", [(1, 1.0), (3, 2.0), (70, 0.5), (130, 4.0)])
@pytest.mark.parametrize("tokens,vocab,dim,pad,shift", [(1, 200, 5, 0, 0), (5, 300, 16, 8, 0), (65, 1000, 33, 0, 1), (300, 700, 264, 0, 0)])
def test_distill(tokens, vocab, dim, pad, shift, top, tau, dtype):
    dev = need_gpu()
    H, W, _, g = problem(tokens, vocab, dim, dtype, dev, pad, shift)
    ids = torch.randint(0, vocab, (tokens, top), generator=g)         # the same word twice here and there
    a = torch.randn(tokens, top, generator=g) * 3
    if tokens > 4:
        ids[1, 0], ids[2], a[3] = vocab, -1, -math.inf
        a[4, top // 2:] = -math.inf
        if top > 1:
            ids[0, 1] = ids[0, 0]
    ref = Reference(H, W, tau)
    want, target, counted, zs, off = teacher_reference(ref, ids, a, tau, vocab)
    loss, lse, z = B.brsvd_distill_forward(H, W, ids.to(dev), a.to(dev), tau)
    ref.check_lse(lse)
    ref.check("z", z, zs, (ref.h.abs() @ ref.w.abs().t()).amax(dim=1, keepdim=True) * 2.0 ** -23 * (dim + 8))
    ref.check("loss", loss, want, off)
    for grad, piece in (((torch.rand(tokens, generator=g) + 0.5).to(dev), 0), (torch.full((1,), 0.1, device=dev), 256)):
        dH, dW = B.brsvd_distill_backward(H, W, ids.to(dev), a.to(dev), tau, lse, z, grad, piece=piece)
        ref.check_gradients(dH, dW, target, grad.double().cpu().expand(tokens) * tau * counted)


def test_distill_towards_one_word_is_cross_entropy():
    dev = need_gpu()
    H, W, y, _ = problem(100, 500, 48, torch.bfloat16, dev)
    yd = y.to(dev)
    loss, lse = B.brsvd_xent_forward(H, W, yd)
    loss1, lse1, z = B.brsvd_distill_forward(H, W, yd[:, None].contiguous(), torch.zeros(100, 1, device=dev), 1.0)
    assert torch.equal(lse, lse1) and float((loss - loss1).abs().max()) <= 2e-5
    g = torch.ones(1, device=dev)
    a, b = B.brsvd_xent_backward(H, W, yd, lse, g), B.brsvd_distill_backward(H, W, yd[:, None].contiguous(), torch.zeros(100, 1, device=dev), 1.0, lse1, z, g)
    for x, w in zip(a, b):
        assert float((x.double() - w.double()).norm()) <= 2.0 ** -8 * float(x.double().norm())


def test_offsets_beyond_32_bits():
    """An output matrix of more than 2^32 bytes whose last rows hold the words that matter."""
    dev = need_gpu()
    vocab, dim = 300000, 8192
    W = torch.zeros(vocab, dim, dtype=torch.bfloat16, device=dev)
    tail = (randn(1, 300, dim) * 0.02).to(torch.bfloat16).to(dev)
    W[-300:] = tail
    H = (randn(2, 70, dim)).to(torch.bfloat16).to(dev)
    y = vocab - 1 - torch.arange(70, device=dev)
    loss, lse = B.brsvd_xent_forward(H, W, y)
    z = H.double().cpu() @ tail.double().cpu().t()
    want = torch.logaddexp(torch.logsumexp(z, dim=1), torch.tensor(math.log(vocab - 300.0), dtype=torch.float64))
    assert float((lse.double().cpu() - want).abs().max()) <= 1e-4
    assert float((loss.double().cpu() - (want - z[torch.arange(70), 299 - torch.arange(70)])).abs().max()) <= 1e-4
    dH, dW = B.brsvd_xent_backward(H, W, y, lse, torch.ones(1, device=dev))
    p = torch.exp(z - want[:, None])
    p[torch.arange(70), 299 - torch.arange(70)] -= 1
    expect = p.t() @ H.double().cpu()
    assert float((dW[-300:].double().cpu() - expect).norm()) <= 0.01 * float(expect.norm())
    expect = p @ tail.double().cpu()
    assert float((dH.double().cpu() - expect).norm()) <= 0.01 * float(expect.norm())
    other = (torch.exp(-want)[:, None] * H.double().cpu()).sum(dim=0)
    assert float((dW[1000].double().cpu() - other).norm()) <= 0.01 * float(other.norm())


def test_repeats_itself_in_graphs_on_other_streams_and_in_any_workspace():
    dev = need_gpu()
    H, W, y, g = problem(300, 1500, 100, torch.bfloat16, dev)
    yd, grad = y.to(dev), torch.rand(300, generator=g).to(dev)

    def step(h, **kw):
        loss, lse = B.brsvd_xent_forward(h, W, yd, **kw)
        return (loss, lse, *B.brsvd_xent_backward(h, W, yd, lse, grad, **kw))
    want, minus = step(H), step(-H)
    assert all(torch.equal(a, b) for a, b in zip(want, step(H)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(H, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    h, graph = H.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(h)
    for i in range(4):
        h.copy_(H if i % 2 == 0 else -H)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want if i % 2 == 0 else minus, got))
        torch.randn(1000, 1000, device=dev).sum().item()
    # a workspace full of NaN, and gradients into rows that are further apart
    sizes = (300, 1500, 100)
    nbytes = B.lib().brsvd_head_workspace_bytes(*sizes, 512, 0, 1)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device=dev)
    dH, dW = torch.full((300, 104), 9.0, device=dev).bfloat16(), torch.full((1500, 101), 9.0, device=dev).bfloat16()
    status = B.lib().brsvd_xent_backward(H.data_ptr(), 100, W.data_ptr(), 100, yd.data_ptr(), want[1].data_ptr(), grad.data_ptr(), 1, *sizes, 512, B.BRSVD_DTYPE_BF16,
                                         dH.data_ptr(), 104, dW.data_ptr(), 101, ws.data_ptr(), nbytes, None)
    torch.cuda.synchronize()
    a, b = B.brsvd_xent_backward(H, W, yd, want[1], grad, piece=512)
    assert status == B.BRSVD_OK and torch.equal(dH[:, :100], a) and torch.equal(dW[:, :100], b)
    assert bool((dH[:, 100:] == 9).all() and (dW[:, 100:] == 9).all())


def test_refusals():
    dev = need_gpu()
    H, W, y, _ = problem(4, 50, 16, torch.bfloat16, dev)
    y = y.to(dev)
    loss, lse = B.brsvd_xent_forward(H, W, y)
    one = torch.ones(1, device=dev)
    ids, a = torch.zeros(4, 3, dtype=torch.int64, device=dev), torch.zeros(4, 3, device=dev)
    for call in (lambda: B.brsvd_xent_forward(H.float(), W.float(), y), lambda: B.brsvd_xent_forward(H, W.half(), y), lambda: B.brsvd_xent_forward(H, W, y.int()),
                 lambda: B.brsvd_xent_forward(H, W, y[:3]), lambda: B.brsvd_xent_forward(H, W[:, :8], y), lambda: B.brsvd_xent_forward(H.cpu(), W, y),
                 lambda: B.brsvd_xent_forward(H.t(), W, y), lambda: B.brsvd_xent_backward(H, W, y, lse.double(), one),
                 lambda: B.brsvd_xent_backward(H, W, y, lse, torch.ones(3, device=dev)), lambda: B.brsvd_xent_backward(H, W, y, lse, 1.0),
                 lambda: B.brsvd_distill_forward(H, W, ids, a[:, :2]), lambda: B.brsvd_distill_forward(H, W, ids.int(), a),
                 lambda: B.brsvd_distill_forward(H, W, ids, a.double()), lambda: B.brsvd_distill_forward(H, W, ids[:3], a[:3])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        B.brsvd_xent_backward(H, W, y, lse, one, need_dH=False, need_dW=False)
    for tau in (0.0, -1.0, math.nan, math.inf, 1e-45):
        with pytest.raises(B.BrsvdError):
            B.brsvd_distill_forward(H, W, ids, a, tau)
    with pytest.raises(B.BrsvdError):
        B.brsvd_xent_backward(H, W, y, lse, one, piece=-1)
