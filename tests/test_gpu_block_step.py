"""The operators of a compressed layer together, as a repair step and a server run them: a gated feed-forward block whose second matrix is factors and a remainder in 4 bits,
the loss of the output matrix behind it, gradients of everything that is not frozen, clipped by their norm; eagerly, as a captured graph, and token by token."""
import importlib.util
import math
import os

import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e4m3 import randn

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
T, D, F, V, R = 300, 136, 400, 1000, 24


def layer(dev, dtype):
    """Weights of the block (fp64, as the type holds them) and of the output matrix, and the second matrix as factors and a remainder in 4 bits."""
    X, Wg, Wu = (randn(i, *s).mul(c).to(dtype).to(dev) for i, s, c in ((1, (T, D), 1.0), (2, (F, D), 1.5 / math.sqrt(D)), (3, (F, D), 1.5 / math.sqrt(D))))
    Wo = (randn(4, V, D) * 2 / math.sqrt(D)).to(dtype).to(dev)
    Wd = ((randn(5, D, R) @ randn(6, R, F) + 0.5 * randn(7, D, F)) / math.sqrt(R * F)).float().to(dev)
    Omega = B.brsvd_philox_normal(3, F, R + 8, device=dev)
    handle = B.brsvd_create(B.make_params(D, F, R, 8, 1))
    try:
        U, S, Vt, _ = B.brsvd_run(handle, Wd, Omega)
    finally:
        B.brsvd_destroy(handle)
    left, right = (U[:, :R] * S[:R]).to(dtype).contiguous(), Vt[:R].to(dtype).contiguous()
    Q, scales = B.brsvd_quantize_e2m1(Wd - left.float() @ right.float())
    kept = left.float() @ right.float() + B.brsvd_dequantize_e2m1(Q, scales)
    # what the factors leave is the noise, 0.5 / sqrt(R), a tenth of the matrix; a number is off by a quarter of itself at most from 0.75 of a group's steps on, by a quarter of a step below
    assert float((kept - Wd).norm() / Wd.norm()) < 0.1 * 0.3
    y = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(8)).to(dev)
    y[::17] = -1
    return X, Wg, Wu, left, right, (Q, scales), Wo, y


def step(X, Wg, Wu, left, right, W4, Wo, y, scale, most, out):
    H, G, U = B.brsvd_glu_forward(X, Wg, Wu, keep=True)
    narrow = H @ right.t()
    Y = B.brsvd_linear_e2m1(H, *W4) + narrow @ left.t()
    loss, lse = B.brsvd_xent_forward(Y, Wo, y)
    dY, dWo = B.brsvd_xent_backward(Y, Wo, y, lse, torch.full((1,), scale / T, device=Y.device))
    dnarrow = dY @ left
    dH = B.brsvd_linear_e2m1_backward(dY, *W4, cols=F) + dnarrow @ right
    dX, dWg, dWu = B.brsvd_glu_backward(X, Wg, Wu, G, U, dH)
    grads = [dWg, dWu, dY.t() @ narrow, dnarrow.t() @ H, dWo]
    norm = B.brsvd_grad_norm(grads, scale=1 / scale)
    B.brsvd_grad_clip(grads, norm, most, scale=1 / scale, out=out)
    return loss, norm, dX


@pytest.mark.parametrize("dtype,scale", [(torch.bfloat16, 1.0), (torch.float16, 4096.0)])
def test_step_against_64_bits(dtype, scale):
    dev = need_gpu()
    ops = layer(dev, dtype)
    X, Wg, Wu, left, right, W4, Wo, y = ops
    out = [torch.empty(s, device=dev) for s in ((F, D), (F, D), (D, R), (R, F), (V, D))]
    most = 0.01
    loss, norm, dX = step(*ops, scale, most, out)
    # the same in 64 bits
    leaves = [v.double().cpu().requires_grad_() for v in (X, Wg, Wu, left, right, Wo)]
    x, wg, wu, l, r, wo = leaves
    W = B.brsvd_dequantize_e2m1(*W4, cols=F).double().cpu()
    h = torch.nn.functional.silu(x @ wg.t()) * (x @ wu.t())
    z = (h @ W.t() + h @ r.t() @ l.t()) @ wo.t()
    counted = (y >= 0).cpu()
    each = torch.logsumexp(z, dim=1) - z.gather(1, y.cpu().clamp(min=0)[:, None])[:, 0]
    (each * counted).sum().div(T).backward()
    want = [leaves[i].grad for i in (1, 2, 3, 4, 5)]
    n = math.sqrt(sum(float(g.square().sum()) for g in want))
    assert n > most
    # a dozen arrays between the operators are rounded, each by at most u of its norm, and no map that takes them on has a condition above two here
    u = torch.finfo(dtype).eps / 2
    assert float(((loss.double().cpu() - each.detach() * counted)).norm() / (each.detach() * counted).norm()) <= 12 * u
    assert abs(float(norm) - n) <= 24 * u * n
    for got, g in zip(out, want):
        g = g * most / n
        assert float((got.double().cpu() - g).norm() / g.norm()) <= 24 * u
    assert abs(math.sqrt(sum(float(v.double().square().sum()) for v in out)) - most) <= most * 2.0 ** -20
    assert float((dX.double().cpu() / scale - x.grad).norm() / x.grad.norm()) <= 24 * u


def test_step_as_a_graph():
    """Captured once and replayed on other inputs, with eager steps and other work between: every replay has the bits of the eager step."""
    dev = need_gpu()
    ops = layer(dev, torch.bfloat16)
    X, rest = ops[0], ops[1:]
    make = lambda: [torch.empty(s, device=dev) for s in ((F, D), (F, D), (D, R), (R, F), (V, D))]  # noqa: E731
    inputs = [X, torch.flip(X, (0,)).contiguous(), X * 0.5]
    eager = []
    for v in inputs:
        out = make()
        eager.append((*step(v, *rest, 1.0, 0.01, out), *out))
    x, out = X.clone(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, *rest, 1.0, 0.01, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (*step(x, *rest, 1.0, 0.01, out), *out)
    for i in (0, 1, 2, 1, 0):
        x.copy_(inputs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager[i])), i
        step(inputs[(i + 1) % 3], *rest, 1.0, 0.01, make())
        torch.randn(500, 500, device=dev).sum().item()


def test_two_streams_at_once():
    """Two steps on two streams that nothing orders: each has the bits that it has alone."""
    dev = need_gpu()
    ops = layer(dev, torch.bfloat16)
    make = lambda: [torch.empty(s, device=dev) for s in ((F, D), (F, D), (D, R), (R, F), (V, D))]  # noqa: E731
    inputs = [ops[0], ops[0] * 0.5]
    eager = []
    for v in inputs:
        out = make()
        eager.append((*step(v, *ops[1:], 1.0, 0.01, out), *out))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in inputs]
    for _ in range(5):
        got = []
        for s, v in zip(streams, inputs):
            with torch.cuda.stream(s):
                out = make()
                got.append((*step(v, *ops[1:], 1.0, 0.01, out), *out))
        torch.cuda.synchronize()
        for g, e in zip(got, eager):
            assert all(torch.equal(a, b) for a, b in zip(g, e))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_token_by_token(dtype):
    """Serving one token at a time gives what the batch gives, but for the order of the sums."""
    dev = need_gpu()
    X, Wg, Wu, _, _, W4, _, _ = layer(dev, dtype)
    whole = B.brsvd_linear_e2m1(B.brsvd_glu_forward(X, Wg, Wu), *W4)
    one = torch.cat([B.brsvd_linear_e2m1(B.brsvd_glu_forward(X[i:i + 1], Wg, Wu), *W4) for i in range(T)])
    some = torch.cat([B.brsvd_linear_e2m1(B.brsvd_glu_forward(x, Wg, Wu), *W4) for x in X.split(24)])
    # H may be rounded the other way where sums differ: each of them by a step, u of its size, at most
    u = torch.finfo(dtype).eps / 2
    H, W = B.brsvd_glu_forward(X, Wg, Wu).double(), B.brsvd_dequantize_e2m1(*W4, cols=F).double()
    bound = 2 * u * (H.abs() @ W.abs().t()) + 2 * u * whole.double().abs() + 2.0 ** -24
    for got in (one, some):
        assert bool(((got.double() - whole.double()).abs() <= bound).all())
        assert float((got != whole).float().mean()) < 0.2


def test_example_keeps_the_remainder_in_4_bits():
    need_gpu()
    spec = importlib.util.spec_from_file_location("compress_output_matrix", os.path.join(ROOT, "examples", "compress_output_matrix.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    said = example.main(["--vocab", "2000", "--dim", "151", "--rank", "30", "--tokens", "300", "--steps", "3"])
    assert all(math.isfinite(v) for v in said.values())
    assert 0 < said["4 bits: logits off by"] < 1 and said["factors and 4-bit remainder"] > 0
