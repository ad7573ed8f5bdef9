"""The gated feed-forward block's first half and its gradients against the formulas in 64 bits, each result within a bound that its roundings allow; at the ends of
chunks, tiles and parts, for rows at any alignment."""
import math

import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e2m1 import FINEST, HALF, ROUND
from tests.test_gpu_e4m3 import placed, randn

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "gelu_tanh"]
STEP = 2.0 ** -23           # what an addition in fp32 loses at most, cut off and not rounded


def act_of(g, act):
    """a(g), a'(g) and how large the argument of its exponential is (fp64)."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * torch.sigmoid(-g)), g.abs()
    if act == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi), g * g
    z = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    p = torch.sigmoid(z)
    return g * p, p * (1 + g * torch.sigmoid(-z) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)), z.abs()


def rounded(want, off, dtype):
    """The bound `off` on a number in fp32, once it is rounded to dtype."""
    return off + ROUND[dtype] * (want.abs() + off) + FINEST[dtype]


def held(name, got, want, bound):
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), (name, float((err / bound.clamp(min=1e-300)).max()))


def off_of_act(a, g, size):
    """a(g) = g p(g): exp and the reciprocal are good to 2^-22, the argument of size `size` to two steps of 2^-24; p below 2^-125 is cut off."""
    return a.abs() * 2.0 ** -20 * (1 + size) + 2.0 ** -125 * g.abs()


def problem(t, d, f, dtype, dev, pad=0, shift=0, seed=0):
    X = placed(randn(seed + t + d, t, d), dtype, dev, pad, shift)
    Wg, Wu = (placed(randn(seed + s + f + d, f, d) * 1.5 / math.sqrt(d), dtype, dev, pad, shift) for s in (1, 2))
    return X, Wg, Wu


def check_forward(X, Wg, Wu, act, H, G, U):
    x, wg, wu = (a.double().cpu() for a in (X, Wg, Wu))
    d, dtype = X.shape[1], X.dtype
    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = (STEP * (d + 32) * (x.abs() @ w.abs().t()) for w in (wg, wu))
    a, _, size = act_of(g, act)
    # no activation's slope is above 1.13
    ea = 1.13 * eg + off_of_act(a, g, size + 1.13 * eg)
    held("H", H, a * u, rounded(a * u, ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -23 * (a * u).abs(), dtype))
    if G is not None:
        held("G", G, g, rounded(g, eg, dtype))
        held("U", U, u, rounded(u, eu, dtype))


def check_gradients(X, Wg, Wu, G, U, dH, act, dX, dWg, dWu):
    x, wg, wu, g, u, dh = (a.double().cpu() for a in (X, Wg, Wu, G, U, dH))
    t, f, dtype = X.shape[0], Wg.shape[0], X.dtype
    a, slope, size = act_of(g, act)
    dg, du = dh * u * slope, dh * a
    # the slope, at most 1.13: 1 - p is off by a step, times up to 34 where p is not 1 yet
    eg = (dh * u).abs() * 2.0 ** -17 + 2.0 ** -22 * dg.abs()
    eu = dh.abs() * off_of_act(a, g, size) + 2.0 ** -23 * du.abs()
    # 16 bits, in fp16 times a power of two that takes the largest to 2^14 or beyond
    top = max(float(dg.abs().max()), float(du.abs().max())) * 1.01 if dg.numel() else 0.0
    least = FINEST[dtype] if dtype == torch.bfloat16 else top * 2.0 ** -39
    eg, eu = (e + ROUND[dtype] * (v.abs() + e) + least for e, v in ((eg, dg), (eu, du)))
    dg_, du_ = dg.abs() + eg, du.abs() + eu
    if dX is not None:
        want = dg @ wg + du @ wu
        off = eg @ wg.abs() + eu @ wu.abs() + STEP * (2 * f + 64) * (dg_ @ wg.abs() + du_ @ wu.abs())
        held("dX", dX, want, rounded(want, off, dtype))
    if dWg is not None:
        for name, got, v, e, v_ in (("dWg", dWg, dg, eg, dg_), ("dWu", dWu, du, eu, du_)):
            want = v.t() @ x
            held(name, got, want, rounded(want, e.t() @ x.abs() + STEP * (t + 32) * (v_.t() @ x.abs()), dtype))


SIZES = [(1, 1, 1, 0, 0), (1, 64, 16, 0, 0), (2, 129, 3, 1, 0), (15, 128, 130, 0, 0), (16, 127, 300, 1, 1), (17, 300, 257, 0, 0), (33, 1000, 64, 8, 0), (64, 2000, 129, 0, 3),
         (65, 256, 128, 0, 0), (66, 15, 257, 1, 1), (100, 4001, 300, 0, 0), (128, 144, 512, 0, 0), (129, 640, 256, 8, 0), (257, 130, 513, 0, 0), (300, 1001, 70, 7, 0), (513, 1008, 300, 8, 0),
         (200, 63, 1, 0, 0), (70, 64, 65, 0, 0), (600, 60, 700, 4, 0), (1030, 72, 40, 0, 0)]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("t,d,f,pad,shift", SIZES)
def test_forward_and_backward(t, d, f, pad, shift, dtype):
    dev = need_gpu()
    act = ACTS[(t + d + f) % 3]
    X, Wg, Wu = problem(t, d, f, dtype, dev, pad, shift)
    H, G, U = B.brsvd_glu_forward(X, Wg, Wu, act=act, keep=True)
    check_forward(X, Wg, Wu, act, H, G, U)
    assert torch.equal(B.brsvd_glu_forward(X, Wg, Wu, act=act), H)
    G, U, dH = (placed(v.double().cpu(), dtype, dev, pad, shift) for v in (G, U, randn(t + f, t, f)))
    dX, dWg, dWu = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH, act=act)
    check_gradients(X, Wg, Wu, G, U, dH, act, dX, dWg, dWu)
    x1, none, _ = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH, act=act, need_dW=False)
    none_x, wg1, wu1 = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH, act=act, need_dX=False)
    assert none is None and none_x is None and torch.equal(x1, dX) and torch.equal(wg1, dWg) and torch.equal(wu1, dWu)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t,d,f", [(5, 200, 3000), (70, 4096, 1500), (700, 300, 17000), (1000, 600, 4500), (2100, 264, 520)])
def test_ways_of_large_sizes(t, d, f, act):
    """Tiles of both sizes, most of them in large ones and the last round in small ones, contractions that are cut."""
    dev = need_gpu()
    X, Wg, Wu = problem(t, d, f, torch.bfloat16, dev)
    H, G, U = B.brsvd_glu_forward(X, Wg, Wu, act=act, keep=True)
    check_forward(X, Wg, Wu, act, H, G, U)
    dH = randn(t + f, t, f).bfloat16().to(dev)
    check_gradients(X, Wg, Wu, G, U, dH, act, *B.brsvd_glu_backward(X, Wg, Wu, G, U, dH, act=act))


def test_halves_of_one_matrix():
    dev = need_gpu()
    X, Wg, Wu = problem(90, 128, 200, torch.bfloat16, dev)
    both = torch.cat([Wg, Wu])
    want = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    got = B.brsvd_glu_forward(X, both[:200], both[200:], keep=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dH = randn(3, 90, 200).bfloat16().to(dev)
    dX, dWg, dWu = B.brsvd_glu_backward(X, both[:200], both[200:], *want[1:], dH)
    assert dWu.data_ptr() == dWg.data_ptr() + 2 * 200 * 128
    # rows of the two as far from each other as they like
    wide = torch.zeros(200, 256, dtype=torch.bfloat16, device=dev)
    wide[:, :128] = Wu
    for a, b in zip(B.brsvd_glu_forward(X, Wg, wide[:, :128], keep=True), want):
        assert torch.equal(a, b)
    for a, b in zip(B.brsvd_glu_backward(X, Wg, wide[:, :128], *want[1:], dH), (dX, dWg, dWu)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_whole_range(act, dtype):
    """G by way of a unit X: numbers from the type's finest to its largest, both signs; U and dH are one."""
    dev = need_gpu()
    g = torch.cat([torch.linspace(-30, 30, 2001), torch.logspace(-30, 4.8, 500) if dtype == torch.bfloat16 else torch.logspace(-7, 4.8, 500), torch.tensor([0.0])]).to(dtype)
    if dtype == torch.bfloat16:
        g = torch.cat([g, torch.tensor([1e20, 1e30, 3e38], dtype=dtype)])
    g = torch.cat([g, -g])[:, None].to(dev)
    one = torch.ones(1, 1, dtype=dtype, device=dev)
    for t in (1, 100):
        X = one.expand(t, 1).contiguous()
        H = B.brsvd_glu_forward(X, g, torch.ones_like(g), act=act)
        a, slope, size = act_of(g[:, 0].double().cpu(), act)
        assert bool(torch.isfinite(slope[g[:, 0].abs().cpu() < 1e10]).all())
        off = off_of_act(a, g[:, 0].double().cpu(), torch.where(torch.isfinite(size), size, 0.0))
        held(act, H, a.expand(t, -1), rounded(a, off, dtype).expand(t, -1))
    # backward with unit weights: dX = dG + dU over a width of one
    n = g.shape[0]
    ones = torch.ones(n, 1, dtype=dtype, device=dev)
    dX, dWg, dWu = B.brsvd_glu_backward(ones, one, one * 0, g, ones, ones, act=act)
    limit = torch.where(g[:, 0].cpu() > 0, 1.0, 0.0).double()
    slope = torch.where(torch.isfinite(slope), slope, limit)
    least = 0.0 if dtype == torch.bfloat16 else max(1.13, float(a.abs().max())) * 1.01 * 2.0 ** -39
    off = 2.0 ** -17 + ROUND[dtype] * (slope.abs() + 2.0 ** -17) + least + 66 * STEP * 1.2
    held("slope", dX[:, 0], slope, rounded(slope, off, dtype))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("t", [3, 40, 90, 300])
def test_nan_and_infinity_stay_in_their_rows(t, dtype):
    dev = need_gpu()
    X, Wg, Wu = problem(t, 200, 300, dtype, dev)
    want = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    dH = randn(4, t, 300).to(dtype).to(dev)
    dX = B.brsvd_glu_backward(X, Wg, Wu, *want[1:], dH, need_dW=False)[0]
    X[1, 7], Wu[299, 3] = float("nan"), float("inf")
    H, G, U = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    keep = torch.arange(t, device=dev) != 1
    assert bool(torch.isnan(H[1]).all() and torch.isnan(G[1]).all()) and torch.equal(G[keep], want[1][keep])
    assert torch.equal(H[keep][:, :299], want[0][keep][:, :299]) and not bool(torch.isfinite(U[:, 299]).any())
    Wu[299, 3] = 0.0
    dH[2, 5], G = float("nan"), want[1].clone()
    G[0, 9] = float("nan")
    got = B.brsvd_glu_backward(X, Wg, Wu, G, want[2], dH, need_dW=False)[0]
    keep = torch.arange(t, device=dev) > 2
    assert bool(torch.isnan(got[2]).all() and torch.isnan(got[0]).all())
    Wu[299, 3] = randn(0, 1, 1).item()           # back to any number: the rows' dX has to agree where the weights do
    clean = B.brsvd_glu_backward(X, Wg, Wu, want[1], want[2], torch.where(torch.isnan(dH), 0.0, dH), need_dW=False)[0]
    got = B.brsvd_glu_backward(X, Wg, Wu, G, want[2], dH, need_dW=False)[0]
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("act", ACTS)
def test_infinite_gates(act, dtype):
    """G that was rounded to an infinity: a and its slope have limits there, a(-inf) = 0, a'(inf) = 1, a'(-inf) = 0, and gradients are finite where those are."""
    dev = need_gpu()
    inf = float("inf")
    G = torch.tensor([[inf, -inf, -inf, 1.0, float("nan")]], dtype=dtype, device=dev).t().contiguous()
    U, dH = torch.tensor([[2.0, 3.0, -1.0, 0.0, 1.0]], dtype=dtype, device=dev).t().contiguous(), torch.full((5, 1), 0.5, dtype=dtype, device=dev)
    X, one = torch.ones(5, 1, dtype=dtype, device=dev), torch.ones(1, 1, dtype=dtype, device=dev)
    by_gate = B.brsvd_glu_backward(X, one, one * 0, G, U, dH, act=act, need_dW=False)[0][:, 0]        # dG, and 0 dU
    assert by_gate[1:3].tolist() == [0.0, 0.0] and bool(torch.isnan(by_gate[4])) and by_gate[3] == 0.0
    dWg, dWu = B.brsvd_glu_backward(X[:1], one, one, G[:1], U[:1], dH[:1], act=act, need_dX=False)[1:]
    assert dWg.item() == 1.0 and dWu.item() == inf                                                     # dH U a'(inf), dH a(inf)
    dWg, dWu = B.brsvd_glu_backward(X[1:4], one, one, G[1:4], U[1:4], dH[1:4], act=act, need_dX=False)[1:]
    a = float(act_of(torch.tensor(1.0).double(), act)[0])
    assert dWg.item() == 0.0 and abs(dWu.item() - 0.5 * a) <= (3 * ROUND[dtype] + 2.0 ** -20) * a      # dU and dWu rounded
    X = torch.tensor([[1.0, 1.0]], dtype=dtype, device=dev).t().contiguous()
    H = B.brsvd_glu_forward(X, torch.full((3, 1), -inf, dtype=dtype, device=dev), torch.full((3, 1), 2.0, dtype=dtype, device=dev), act=act)
    assert bool((H == 0).all())


@pytest.mark.parametrize("scale", [2.0 ** -24, 2.0 ** -12, 1.0, 2.0 ** 8])
def test_fp16_gradients_of_any_size(scale):
    """dH from fp16's finest numbers to large ones: dG and dU keep eleven bits, as one power of two takes them into fp16's range."""
    dev = need_gpu()
    t, d, f = 120, 80, 200
    X, Wg, Wu = problem(t, d, f, torch.float16, dev)
    _, G, U = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    U = U * 0.01
    dH = (torch.randint(1, 4, (t, f), generator=torch.Generator().manual_seed(1)) * scale).half().to(dev)
    grads = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH)
    check_gradients(X, Wg, Wu, G, U, dH, "silu", *grads)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """Along a direction V of all three operands: sum dH (H(+e V) - H(-e V)) / 2 e = <dX, Vx> + <dWg, Vg> + <dWu, Vu>, with H in 64 bits.  Each gradient is off by
    four roundings at most (G, U, dG or dU, its own) of 2^-11 of the terms it is a sum of, taken as independent: 2^-6 of the root of the sum of squares is 32 times that."""
    dev = need_gpu()
    t, d, f, e = 150, 100, 170, 1e-4
    ops = problem(t, d, f, torch.float16, dev)
    _, G, U = B.brsvd_glu_forward(*ops, act=act, keep=True)
    dH = randn(9, t, f).half().to(dev)
    grads = [v.double().cpu() for v in B.brsvd_glu_backward(*ops, G, U, dH, act=act)]
    x, wg, wu = (v.double().cpu() for v in ops)

    def total(s, v):
        return float((dH.double().cpu() * act_of((x + s * v[0]) @ (wg + s * v[1]).t(), act)[0] * ((x + s * v[0]) @ (wu + s * v[2]).t())).sum())
    for only in range(3):
        v = [randn(20 + i, *a.shape) * (i == only) for i, a in enumerate((x, wg, wu))]
        want = (total(e, v) - total(-e, v)) / (2 * e)
        got = sum(float((g * w).sum()) for g, w in zip(grads, v))
        size = math.sqrt(sum(float(((g * w) ** 2).sum()) for g, w in zip(grads, v)))
        assert abs(got - want) <= 2.0 ** -6 * size, (only, got, want, size)


def test_sizes_of_zero():
    dev = need_gpu()
    e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    for t, d, f in ((0, 8, 6), (4, 0, 6), (4, 8, 0), (0, 0, 0)):
        H, G, U = B.brsvd_glu_forward(e(t, d), e(f, d), e(f, d), keep=True)
        assert all(v.shape == (t, f) and not bool(v.any()) for v in (H, G, U))
        dX, dWg, dWu = B.brsvd_glu_backward(e(t, d), e(f, d), e(f, d), G, U, e(t, f))
        assert dX.shape == (t, d) and not bool(dX.any()) and all(v.shape == (f, d) and not bool(v.any()) for v in (dWg, dWu))


def test_rows_behind_the_results_are_left():
    """Results in rows of their own pitch: what stands beside them stays."""
    dev = need_gpu()
    t, d, f = 130, 72, 150
    X, Wg, Wu = problem(t, d, f, torch.bfloat16, dev)
    want = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    dH = randn(4, t, f).bfloat16().to(dev)
    grads = B.brsvd_glu_backward(X, Wg, Wu, *want[1:], dH)
    L, s = B.lib(), torch.cuda.current_stream().cuda_stream or None
    ws = torch.empty(L.brsvd_glu_workspace_bytes(t, d, f, 0, 1), dtype=torch.uint8, device=dev)
    H, G, U = (torch.full((t + 1, f + 5), 3.0, dtype=torch.bfloat16, device=dev) for _ in range(3))
    for rows in (t, 30):
        for v in (H, G, U):
            v.fill_(3.0)
        assert L.brsvd_glu_forward(X.data_ptr(), d, Wg.data_ptr(), d, Wu.data_ptr(), d, rows, d, f, B.BRSVD_DTYPE_BF16, 0, H.data_ptr(), f + 5, G.data_ptr(), f + 5, U.data_ptr(),
                                   f + 5, ws.data_ptr(), ws.numel(), s) == 0
        for got, w in zip((H, G, U), want):
            assert (torch.equal(got[:rows, :f], w[:rows]) if rows == t else got[0, 0] != 3) and bool((got[:, f:] == 3).all() and (got[rows:] == 3).all())
    outs = [torch.full((n + 1, d + 3), 3.0, dtype=torch.bfloat16, device=dev) for n in (t, f, f)]
    assert L.brsvd_glu_backward(X.data_ptr(), d, Wg.data_ptr(), d, Wu.data_ptr(), d, want[1].data_ptr(), f, want[2].data_ptr(), f, dH.data_ptr(), f, t, d, f, B.BRSVD_DTYPE_BF16, 0,
                                outs[0].data_ptr(), d + 3, outs[1].data_ptr(), d + 3, outs[2].data_ptr(), d + 3, ws.data_ptr(), ws.numel(), s) == 0
    for got, w in zip(outs, grads):
        assert torch.equal(got[:-1, :d], w) and bool((got[:, d:] == 3).all() and (got[-1] == 3).all())


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("t", [5, 100, 300])
def test_repeats_itself_in_graphs_and_on_other_streams(t, dtype):
    dev = need_gpu()
    X, Wg, Wu = problem(t, 301, 400, dtype, dev)
    dH = randn(2, t, 400).to(dtype).to(dev)

    def both(x, dh, **kw):
        H, G, U = B.brsvd_glu_forward(x, Wg, Wu, keep=True, **kw)
        return (H, G, U) + B.brsvd_glu_backward(x, Wg, Wu, G, U, dh, **kw)
    want, other = both(X, dH), both(-X, 2 * dH)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(X, dH, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x, dh = X.clone(), dH.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(x, dh)
    for i in range(4):
        x.copy_(-X if i % 2 else X)
        dh.copy_(2 * dH if i % 2 else dH)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, other if i % 2 else want)), i
        torch.randn(1000, 1000, device=dev).sum().item()


def test_refusals():
    dev = need_gpu()
    X, Wg, Wu = problem(4, 32, 20, torch.bfloat16, dev)
    H, G, U = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    for call in (lambda: B.brsvd_glu_forward(X.float(), Wg.float(), Wu.float()), lambda: B.brsvd_glu_forward(X, Wg, Wu.half()), lambda: B.brsvd_glu_forward(X, Wg, Wu[:19]),
                 lambda: B.brsvd_glu_forward(X, Wg[:, :31], Wu), lambda: B.brsvd_glu_forward(X.cpu(), Wg, Wu), lambda: B.brsvd_glu_forward(X, Wg.t(), Wu), lambda: B.brsvd_glu_forward(X[0], Wg, Wu),
                 lambda: B.brsvd_glu_backward(X, Wg, Wu, G, U, H[:3]), lambda: B.brsvd_glu_backward(X, Wg, Wu, G, U[:, :19], H), lambda: B.brsvd_glu_backward(X, Wg, Wu, G.float(), U, H)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.brsvd_glu_forward(X, Wg, Wu, act="relu"), lambda: B.brsvd_glu_backward(X, Wg, Wu, G, U, H, need_dX=False, need_dW=False)):
        with pytest.raises(ValueError):
            call()


def test_more_than_4_gib():
    """X, G, U, H, dG and dU whose bytes and numbers pass 32 bits: rows at both ends and where they pass; the tokens repeat, so that the weights' gradients are known."""
    dev = need_gpu()
    t, d, f, period = 140000, 64, 16008, 1000
    X, Wg, Wu = problem(period, d, f, torch.bfloat16, dev)
    dH = randn(8, period, f).bfloat16().to(dev)
    some = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    some_back = B.brsvd_glu_backward(X, Wg, Wu, *some[1:], dH)
    many = X.repeat(t // period, 1)
    H, G, U = B.brsvd_glu_forward(many, Wg, Wu, keep=True)
    dX, dWg, dWu = B.brsvd_glu_backward(many, Wg, Wu, G, U, dH.repeat(t // period, 1))
    for first in (0, 2 ** 31 // (2 * f) // period * period, 2 ** 31 // f // period * period, t - period):
        at = slice(first, first + period)
        for a, b in ((H, some[0]), (G, some[1]), (U, some[2])):
            assert torch.equal(a[at], b)                      # a contraction of one step, in whatever tiles
        # 16 bits of the same sum in other parts
        assert float((dX[at].double() - some_back[0].double()).norm() / some_back[0].double().norm()) <= 2 * ROUND[torch.bfloat16]
    # the sum over a period comes back t / period times, so that what is added up to is the result at most, and each of t additions cuts off a step of that
    for a, b in ((dWg, some_back[1]), (dWu, some_back[2])):
        b = b.double() * (t // period)
        assert float((a.double() - b).norm() / b.norm()) <= 2 * ROUND[torch.bfloat16] + 2 * STEP * t
