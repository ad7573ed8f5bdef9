"""The norm over many tensors and clipping by it against sums in 64 bits: mixed types, odd sizes and alignments, strided rows, lists longer than a launch takes."""
import math

import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e4m3 import randn

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FINEST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def drawn(seed, shapes, dev, types=TYPES, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g, dtype=torch.float64) * scale).to(types[i % len(types)]).to(dev) for i, s in enumerate(shapes)]


def norm_of(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def check_norm(got, tensors, scale=1.0):
    """Sums of squares in fp64 in any order are good to 2^-40 here; the result is rounded to fp32."""
    want = norm_of(tensors) * abs(scale)
    assert got.shape == (1,) and got.dtype == torch.float32 and abs(float(got) - want) <= want * (2.0 ** -24 + 2.0 ** -38) + 2.0 ** -150, (float(got), want)
    return want


def check_clipped(got, tensors, norm, max_norm, scale=1.0):
    """norm: the fp32 number that was handed over.  The factor is rounded to fp32, so is the product, then the result to its type."""
    f = scale * (max_norm / norm if max_norm < norm < math.inf else 1.0)
    for y, x in zip(got, tensors):
        want = x.double() * f
        bound = want.abs() * (2.0 ** -23 + 2.0 ** -46) + 2.0 ** -149
        bound = bound + ROUND[y.dtype] * (want.abs() + bound) + FINEST[y.dtype]
        inside = want.abs() * (1 + 2.0 ** -20) < torch.finfo(y.dtype).max
        assert y.shape == x.shape and bool(((y.double() - want).abs() <= bound)[inside].all())


SHAPES = [(1,), (7,), (8, 9), (3, 1, 5), (1000,), (257, 129), (32768,), (32769,), (70001,), (), (300, 8), (2, 40000)]


@pytest.mark.parametrize("out_type", [None] + TYPES)
@pytest.mark.parametrize("max_norm", [0.0, 1.0, 1e9])
def test_mixed_lists(max_norm, out_type):
    dev = need_gpu()
    tensors = drawn(1, SHAPES, dev)
    norm = B.brsvd_grad_norm(tensors)
    check_norm(norm, tensors)
    before = [t.clone() for t in tensors]
    out = None if out_type is None else [torch.full(t.shape, 9.0, dtype=out_type, device=dev) for t in tensors]
    got = B.brsvd_grad_clip(tensors, norm, max_norm, out=out)
    assert got is (tensors if out is None else out)
    check_clipped(got, before, float(norm), max_norm)
    if out is not None or max_norm > 1e6:
        assert all(torch.equal(a, b) for a, b in zip(tensors, before))


@pytest.mark.parametrize("dtype", TYPES)
def test_one_buffer_cut_at_any_number(dtype):
    """Tensors one behind the other in memory, at any alignment: what lies before, between and behind them is left."""
    dev = need_gpu()
    sizes = [1, 3, 8, 64, 101, 1000, 7, 32768, 40001, 5]
    flat = torch.randn(sum(sizes) + 20, generator=torch.Generator().manual_seed(3)).to(dtype).to(dev)
    for shift in range(0, 8, 3):
        views, gaps, at = [], [flat[:shift]], shift
        for n in sizes:
            views.append(flat[at:at + n])
            gaps.append(flat[at + n:at + n + 1])
            at += n + 1
        gaps.append(flat[at:])
        before, kept = [v.clone() for v in views], [v.clone() for v in gaps]
        norm = B.brsvd_grad_norm(views)
        check_norm(norm, before)
        B.brsvd_grad_clip(views, norm, 1.0)
        check_clipped(views, before, float(norm), 1.0)
        assert all(torch.equal(a, b) for a, b in zip(gaps, kept))


def test_strided_rows_and_dense_orders():
    dev = need_gpu()
    base = torch.randn(500, 400, generator=torch.Generator().manual_seed(4)).to(dev)
    keep = base.clone()
    wide = torch.randn(3, 200000, generator=torch.Generator().manual_seed(5)).to(dev)
    tensors = [base[:, :100], base[:, 100:101], base[:, 107:399], wide[:, 3:150000], torch.randn(40, 30, device=dev).t(), torch.randn(5, 6, 7, device=dev).permute(2, 0, 1)]
    before = [t.clone() for t in tensors]
    norm = B.brsvd_grad_norm(tensors)
    check_norm(norm, before)
    out = [torch.empty_strided(t.shape, t.stride(), dtype=torch.bfloat16, device=dev) for t in tensors]
    out[0] = torch.empty(500, 100, dtype=torch.bfloat16, device=dev)
    B.brsvd_grad_clip(tensors, norm, 2.0, out=out)
    check_clipped(out, before, float(norm), 2.0)
    B.brsvd_grad_clip(tensors, norm, 2.0)
    check_clipped(tensors, before, float(norm), 2.0)
    assert torch.equal(base[:, 101:107], keep[:, 101:107]) and torch.equal(base[:, 399:], keep[:, 399:])


@pytest.mark.parametrize("count", [1, 63, 64, 65, 129, 1000])
def test_lists_of_any_length(count):
    dev = need_gpu()
    tensors = drawn(count, [((i * 37) % 300,) for i in range(count)], dev)
    norm = B.brsvd_grad_norm(tensors, scale=-0.5)
    check_norm(norm, tensors, 0.5)
    out = [torch.empty(t.shape, device=dev) for t in tensors]
    B.brsvd_grad_clip(tensors, norm, 0.25, scale=-0.5, out=out)
    check_clipped(out, tensors, float(norm), 0.25, -0.5)


@pytest.mark.parametrize("count", [63, 64, 65, 85, 86, 126, 127, 128, 129, 300])
@pytest.mark.parametrize("every", [1, 2, 3])
def test_matrices_with_strided_rows_at_any_place(count, every):
    """They take two places in a launch's list: the list ends before, between and behind them."""
    dev = need_gpu()
    tensors = drawn(count, [(2 + i % 5, 1 + i * 7 % 40) for i in range(count)], dev)
    for i in range(0, count, every):
        wide = torch.full((tensors[i].shape[0], tensors[i].shape[1] + 3), 7.0, dtype=tensors[i].dtype, device=dev)
        wide[:, 1:-2] = tensors[i]
        tensors[i] = wide[:, 1:-2]
    norm = B.brsvd_grad_norm(tensors)
    check_norm(norm, tensors, 1.0)
    out = [torch.full((t.shape[0], t.shape[1] + i % 2), 9.0, device=dev)[:, :t.shape[1]] for i, t in enumerate(tensors)]
    B.brsvd_grad_clip(tensors, norm, 0.25, out=out)
    check_clipped(out, tensors, float(norm), 0.25)
    assert all(bool((o._base[:, -1] == 9).all()) for i, o in enumerate(out) if i % 2)


def test_no_tensors_and_empty_ones():
    dev = need_gpu()
    assert float(B.brsvd_grad_norm([])) == 0
    empty = [torch.empty(0, device=dev), torch.empty(3, 0, dtype=torch.float16, device=dev)]
    norm = B.brsvd_grad_norm(empty)
    assert float(norm) == 0 and B.brsvd_grad_clip(empty, norm, 1.0) is empty and B.brsvd_grad_clip([], norm, 1.0) == []
    one = torch.full((1,), 5.0, device=dev)
    B.brsvd_grad_clip(empty + [one], torch.full((1,), 5.0, device=dev), 1.0)
    assert float(one) == 1


@pytest.mark.parametrize("power", [-140, -70, -20, 60, 100, 126])
def test_numbers_whose_squares_leave_fp32(power):
    """fp32 and bf16 numbers of any size: neither the norm nor the clipped numbers lose anything on the way."""
    dev = need_gpu()
    tensors = [(torch.randint(1, 8, (1000,), generator=torch.Generator().manual_seed(i)).double() / 8 * 2.0 ** power).to(t).to(dev) for i, t in enumerate((torch.float32, torch.bfloat16))]
    norm = B.brsvd_grad_norm(tensors)
    want = norm_of(tensors)
    if want < 3e38:
        check_norm(norm, tensors)
        out = [torch.empty_like(t, dtype=torch.float32) for t in tensors]
        B.brsvd_grad_clip(tensors, norm, want / 4, out=out)
        # beside the roundings above the norm and max_norm are rounded: 2^-24 of the factor each
        for y, x in zip(out, tensors):
            assert bool(((y.double() - x.double() / 4).abs() <= x.double() * 2.0 ** -22 / 4 + 2.0 ** -148 + x.double() * 2.0 ** -148 / want).all())
    else:
        assert float(norm) == math.inf
    # a norm of 2^120 and clipping to 2^-120
    big = torch.full((1,), 2.0 ** 120, device=dev)
    x = torch.full((40,), 2.0 ** 110, device=dev)
    assert bool((B.brsvd_grad_clip([x], big, 2.0 ** -20)[0] == 2.0 ** -30).all())
    x = torch.full((40,), 2.0 ** 125, device=dev)
    assert bool((B.brsvd_grad_clip([x], big, 2.0 ** -120)[0] == 2.0 ** -115).all())


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_norms_that_are_not_finite_clip_nothing(bad):
    dev = need_gpu()
    tensors = drawn(5, [(1000,), (40,)], dev)
    tensors[1][7] = bad
    before = [t.clone() for t in tensors]
    norm = B.brsvd_grad_norm(tensors)
    assert float(norm) == math.inf if math.isinf(bad) else math.isnan(float(norm))
    B.brsvd_grad_clip(tensors, norm, 1.0)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(tensors, before))
    B.brsvd_grad_clip(tensors, norm, 1.0, scale=0.5)
    assert torch.equal(tensors[0], before[0] * 0.5)
    assert float(B.brsvd_grad_norm([torch.full((4,), 2.0 ** 127, device=dev)])) == math.inf


def test_more_numbers_than_32_bits_count():
    dev = need_gpu()
    n = 2 ** 32 + 12345
    x = torch.zeros(n, dtype=torch.bfloat16, device=dev)
    x[-3:] = 2.0
    x[5] = 2.0
    norm = B.brsvd_grad_norm([x])
    assert float(norm) == 4.0
    B.brsvd_grad_clip([x], norm, 1.0)
    assert x[-4:].tolist() == [0.0, 0.5, 0.5, 0.5] and x[4:7].tolist() == [0.0, 0.5, 0.0]
    rows = x[:2 ** 32].view(2 ** 16, 2 ** 16)[:, 1:]
    rows[-1, -1] = 3.0
    assert float(B.brsvd_grad_norm([rows])) == float(torch.tensor(math.sqrt(0.25 + 9.0), dtype=torch.float32))      # rounded to fp32, once


def test_repeats_itself_in_graphs_and_on_other_streams():
    dev = need_gpu()
    tensors = drawn(6, SHAPES * 7, dev)
    out = [torch.empty(t.shape, device=dev) for t in tensors]
    norm = B.brsvd_grad_norm(tensors)
    want = [t.clone() for t in B.brsvd_grad_clip(tensors, norm, 1.0, out=out)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = B.brsvd_grad_norm(tensors, stream=side)
    B.brsvd_grad_clip(tensors, again, 1.0, out=out, stream=side)
    side.synchronize()
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.brsvd_grad_norm(tensors)
        B.brsvd_grad_clip(tensors, got, 1.0, out=out)
    for i in range(4):
        for t in tensors:
            t.mul_(2.0 if i % 2 else 0.5)
        graph.replay()
        torch.cuda.synchronize()
        eager = B.brsvd_grad_norm(tensors)
        fresh = B.brsvd_grad_clip(tensors, eager, 1.0, out=[torch.empty_like(o) for o in out])
        assert torch.equal(got, eager) and all(torch.equal(a, b) for a, b in zip(out, fresh))


def test_refusals():
    dev = need_gpu()
    x, y = torch.ones(8, device=dev), torch.ones(4, 4, device=dev)
    norm = B.brsvd_grad_norm([x, y])
    for call in (lambda: B.brsvd_grad_norm(x), lambda: B.brsvd_grad_norm([x, None]), lambda: B.brsvd_grad_norm([x.double()]), lambda: B.brsvd_grad_norm([x.cpu()]),
                 lambda: B.brsvd_grad_norm([x.expand(3, 8)]), lambda: B.brsvd_grad_norm([torch.ones(40, device=dev)[::2]]), lambda: B.brsvd_grad_clip([x], norm.double(), 1.0),
                 lambda: B.brsvd_grad_clip([x], 1.0, 1.0), lambda: B.brsvd_grad_clip([x], norm, 1.0, out=[y]), lambda: B.brsvd_grad_clip([y], norm, 1.0, out=[torch.ones(4, 4, device=dev).t()]),
                 lambda: B.brsvd_grad_norm([y.to_sparse()])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        B.brsvd_grad_clip([x, y], norm, 1.0, out=[x])
    # the same memory twice, in place or as results, another tensor's memory, its own in another layout
    for call in (lambda: B.brsvd_grad_clip([x, y, x], norm, 1.0), lambda: B.brsvd_grad_clip([x, x * 2], norm, 1.0, out=[y.view(16)[:8], y.view(16)[:8]]),
                 lambda: B.brsvd_grad_clip([x, y.view(16)[:8]], norm, 1.0, out=[y.view(16)[:8], x]), lambda: B.brsvd_grad_clip([x], norm, -1.0),
                 lambda: B.brsvd_grad_clip([x], norm, float("nan")), lambda: B.brsvd_grad_norm([x], scale=float("inf"))):
        with pytest.raises(B.BrsvdError):
            call()
    assert bool((x == 1).all() and (y == 1).all())
    assert float(B.brsvd_grad_norm([x, x])) == 4.0


def test_columns_of_one_matrix():
    """Tensors that lie between each other's rows share no number; in place, and one into the gaps of another."""
    dev = need_gpu()
    m = randn(3, 40, 300).float().to(dev)
    parts = [m[:, :100], m[:, 100:101], m[:, 101:290]]
    want, norm = m.clone(), B.brsvd_grad_norm(parts)
    exact = math.sqrt(float(m[:, :290].double().square().sum()))
    assert abs(float(norm) - exact) <= exact * 2.0 ** -23
    B.brsvd_grad_clip(parts, norm, float("inf"), scale=0.5)
    want[:, :290] *= 0.5
    assert torch.equal(m, want)
    B.brsvd_grad_clip([m[:, :100]], norm, float("inf"), out=[m[:, 150:250]])
    want[:, 150:250] = want[:, :100]
    assert torch.equal(m, want)
    for bad in ([m, m[:, 3:5]], [m[:, :100], m[:, 99:120]], [m.view(-1)[:1000], m.view(-1)[999:]]):
        with pytest.raises(B.BrsvdError):
            B.brsvd_grad_clip(bad, norm, 1.0)
    assert torch.equal(m, want)
