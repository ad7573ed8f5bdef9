"""The calls on a model's matrices where numbers or sizes leave the usual range."""
import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_e4m3 import codes, randn

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
