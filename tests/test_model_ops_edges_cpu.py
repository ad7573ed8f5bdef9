"""Refusals of the calls on a model's matrices at the ends of what they take, before any GPU call, with addresses that are never followed."""
import os
import re

import pytest
import torch

import paper_1706_07191_amd as B
from tests.test_model_ops_cpu import ARG, AT, BF16, BUDGET, F32, OK, dequantize, gemm, linear, quantize, xent

LAUNCH = 2 ** 32               # threads that a launch has fewer of along a direction


def ceil_div(a, b):
    return -(-a // b)


def distill_backward(_, **kw):
    a = dict(H=AT, ldh=64, W=AT, ldw=64, ids=AT, logits=AT, top=5, tau=2.0, lse=AT, z=AT, grad=AT, stride=1, tokens=10, vocab=1000, dim=64, piece=0, dtype=BF16,
             dH=AT, lddh=64, dW=AT, lddw=64, ws=AT, bytes=1 << 50)
    a.update(kw)
    return B.lib().brsvd_distill_backward(*a.values(), None)


@pytest.mark.parametrize("tokens,vocab,dim,piece", [(2 ** 30 - 1024, 300, 1, 0), (2 ** 24 + 5, 300, 8, 0), (2 ** 20, 1000, 4096, 0), (600000, 1000, 8192, 0),
                                                    (2 ** 28, 1000, 8, 256), (2 ** 17, 2 ** 20, 64, 2 ** 20), (1, 2 ** 17, 2 ** 20, 0)])
def test_losses_take_what_launches_may_have(tokens, vocab, dim, piece):
    """Sizes whose tiles are fewer than 2^32 threads in all are accepted; the other kernels go in several launches."""
    assert B.lib().brsvd_head_workspace_bytes(tokens, vocab, dim, piece, 1, 1) > 0


@pytest.mark.parametrize("tokens,vocab,dim,piece", [(2 ** 30 - 127, 300, 1, 0), (2 ** 30 - 1, 300, 1, 0), (2 ** 20, 2 ** 20, 64, 2 ** 20), (2 ** 22, 1000, 2 ** 16, 0),
                                                    (1, 2 ** 18, 2 ** 20, 0)])
def test_losses_refuse_tiles_that_a_launch_may_not_have(tokens, vocab, dim, piece):
    """Logits of a piece, dH or dW in 2^23 tiles of 512 threads: of such a launch only a part would run."""
    rows = min(piece or max(256, 2 ** 27 // tokens // 256 * 256), 2 ** 20, ceil_div(vocab, 256) * 256)
    tiles = max(ceil_div(rows, 256) * ceil_div(tokens, 128), ceil_div(dim, 256) * ceil_div(tokens, 128), ceil_div(dim, 256) * ceil_div(rows, 128))
    assert tiles * 512 >= LAUNCH
    for backward in (0, 1):
        if piece == 0 or backward:
            assert B.lib().brsvd_head_workspace_bytes(tokens, vocab, dim, piece, 1, backward) == 0
    assert xent(True, tokens=tokens, vocab=vocab, dim=dim, ldh=dim, ldw=dim, lddh=dim, lddw=dim, piece=piece) == ARG


def test_products_refuse_what_a_launch_may_not_have():
    # up to 32 rows: 256 threads for 32 columns
    n = 2 ** 29
    assert gemm(m=1, n=n, k=128, lda=128, ldb=128, ldc=n) == ARG
    assert linear(m=20, n=n, k=128, ldx=128, ldw=128, ldy=n) == ARG
    assert linear(m=20, n=n - 32, k=128, ldx=128, ldw=128, ldy=n, bytes=0) == BUDGET          # accepted: the cast's scratch is missing
    # tiles of 128 rows and 256 columns, 512 threads each; of 256 rows for a 16-bit result of aligned rows
    m = 2 ** 30
    assert linear(m=m, n=100, k=128, ldx=128, ldw=128, ldy=100, dtype=F32, bytes=0) == ARG
    assert linear(m=m - 1024, n=100, k=128, ldx=128, ldw=128, ldy=100, dtype=F32, bytes=0) == BUDGET
    assert linear(m=m, n=100, k=128, ldx=128, ldw=130, ldy=100, dtype=BF16, bytes=0) == ARG
    assert linear(m=m, n=100, k=128, ldx=128, ldw=128, ldy=100, dtype=BF16, bytes=0) == BUDGET


@pytest.mark.parametrize("loss", [xent, distill_backward])
def test_no_tokens_have_any_of_the_gradients(loss):
    """An empty dH may be NULL, as an empty tensor's address is; with tokens one gradient has to be wanted."""
    none = dict(tokens=0, H=None, lse=None, grad=None, ws=None, bytes=0)
    for out in (dict(dH=None, dW=None), dict(dW=None)):
        assert loss(True, **none, **out) == OK
        assert loss(True, **dict(none, tokens=-1), **out) == ARG
    assert loss(True, dH=None, dW=None) == ARG


def test_inline_assembly_names_the_registers_that_it_writes():
    """m0 holds where a load into LDS goes: a statement that writes it says so, as the compiler may have a value of its own there."""
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    found = 0
    for name in sorted(os.listdir(csrc)):
        if name.endswith((".hip", ".h")):
            with open(os.path.join(csrc, name)) as f:
                for statement in re.findall(r"asm(?: volatile)?\((?:[^;]|;(?!\n))*;\n", f.read()):
                    if re.search(r"s_\w+ m0,", statement):
                        found += 1
                        assert re.search(r':\s*"memory",\s*"m0"\s*\)', statement), (name, statement)
    assert found >= 2


class Elsewhere(torch.Tensor):
    """A tensor that says that it lies on a CUDA device."""
    at = 0

    is_cuda = True
    device = property(lambda self: torch.device("cuda", self.at))

    def get_device(self):
        return self.at


def on(index, *shape, dtype=torch.bfloat16):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(Elsewhere)
    t.at = index
    return t


@pytest.fixture
def two_devices(monkeypatch):
    """Two devices, of which the first is current: what makes another current and when."""
    monkeypatch.setattr(B, "torch", torch)
    monkeypatch.setattr(B, "_devices", 2, raising=False)
    now = [0]

    class device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *_):
            now[0] = self.before
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    return now


def test_operands_on_several_devices_are_refused(two_devices):
    H, W, y = on(0, 4, 8), on(1, 6, 8), on(0, 4, dtype=torch.int64)
    q, s = on(1, 4, 16, dtype=torch.float8_e4m3fn), on(0, 4, 1, dtype=torch.float32)
    for call in (lambda: B.brsvd_xent_forward(H, W, y), lambda: B.brsvd_xent_forward(H=H, labels=on(1, 4, dtype=torch.int64), W=on(0, 6, 8)),
                 lambda: B.brsvd_dequantize_e4m3(q, s), lambda: B.brsvd_gemm_e4m3(q, s, q, s, block_rows=1),
                 lambda: B.brsvd_linear_e4m3(H, W, s), lambda: B.brsvd_gemm_e4m3(q, on(1, 4, 1, dtype=torch.float32), q, on(1, 4, 1, dtype=torch.float32), out=on(0, 4, 4))):
        with pytest.raises(TypeError, match="one device"):
            call()


def test_calls_run_with_the_operands_device_current(two_devices):
    seen = []
    call = B._scoped(lambda X, block_rows=1: seen.append(two_devices[0]))
    call(on(1, 2, 2))
    call(X=on(1, 2, 2), block_rows=128)
    call(on(0, 2, 2))
    assert seen == [1, 1, 0] and two_devices == [0]

    class stream:
        device_index = 0
    with pytest.raises(ValueError, match="stream"):
        call(on(1, 2, 2), stream=stream())
    assert seen == [1, 1, 0] and two_devices == [0]


@pytest.mark.parametrize("ld", [2 ** 61, 2 ** 62, 2 ** 63 - 1])
def test_leading_dimensions_whose_bytes_are_no_64_bit_number(ld):
    for dtype in (F32, BF16):
        if ld * (4 if dtype == F32 else 2) >= 2 ** 63:
            for m in (8, 100):
                assert linear(dtype=dtype, ldx=ld, m=m) == ARG
            assert quantize(dtype=dtype, ldx=ld) == ARG and dequantize(dtype=dtype, ldx=ld) == ARG


class NoLibrary:
    """In the library's place: every call succeeds, every size is a few KiB."""

    def __getattr__(self, name):
        return lambda *a: 4096 if name.endswith("_bytes") else 0


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_results_are_fp32_whatever_torchs_default_type(default, monkeypatch):
    """A model's code may set the default to 16 bits: memory that the library writes fp32 into must not become half as large."""
    monkeypatch.setattr(B, "torch", torch)
    monkeypatch.setattr(B, "lib", NoLibrary)
    monkeypatch.setattr(B, "_current", lambda device: None)
    for name in ("empty", "empty_strided"):
        monkeypatch.setattr(torch, name, lambda *a, real=getattr(torch, name), device=None, **kw: real(*a, **kw))
    H, W, y = on(0, 4, 8), on(0, 6, 8), on(0, 4, dtype=torch.int64)
    ids, a = on(0, 4, 3, dtype=torch.int64), on(0, 4, 3, dtype=torch.float32)
    torch.set_default_dtype(default)
    try:
        Q, S, Qt, St = B.brsvd_quantize_e4m3(H, transpose=True)
        fp32 = [S, St, *B.brsvd_xent_forward(H, W, y), *B.brsvd_distill_forward(H, W, ids, a), B.brsvd_dequantize_e4m3(on(0, 4, 16, dtype=torch.float8_e4m3fn), a[:, :1].contiguous())]
    finally:
        torch.set_default_dtype(torch.float32)
    assert [t.dtype for t in fp32] == [torch.float32] * 8
