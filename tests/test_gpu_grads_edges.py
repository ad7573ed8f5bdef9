"""Clipping at the ends of what it takes: a norm beside, in front of and behind the memory that is written."""
import pytest
import torch

import paper_1706_07191_amd as B
from tests.gpu_util import need_gpu
from tests.test_gpu_grads import check_clipped

pytestmark = pytest.mark.gpu


def test_norm_beside_what_is_written():
    """In the gaps of a matrix, in front of and behind a tensor, in one that is read only: taken, and none of them changes; inside a result: refused, and nothing is written."""
    dev = need_gpu()
    base = torch.full((10, 50), 4.0, device=dev)
    part = base[:, 5:25]
    flat = base.view(-1)
    for where in (0, 4, 25, 49, 9 * 50 + 25):
        base.fill_(4.0)
        flat[where] = 8.0
        assert B.brsvd_grad_clip([part], flat[where:where + 1], 2.0)[0] is part
        want = torch.full((10, 50), 4.0, device=dev)
        want[:, 5:25] = 1.0
        want.view(-1)[where] = 8.0
        assert torch.equal(base, want), where
    x, y = torch.full((100,), 4.0, device=dev), torch.zeros(100, device=dev)
    x[99] = 8.0
    B.brsvd_grad_clip([x], x[99:], 2.0, out=[y])
    assert bool((y[:99] == 1).all()) and y[99] == 2
    for where in (0, 50, 99):
        for kw in ({}, {"out": [x]}):
            with pytest.raises(B.BrsvdError):
                B.brsvd_grad_clip([y if kw else x], x[where:where + 1], 2.0, **kw)
    with pytest.raises(B.BrsvdError):
        B.brsvd_grad_clip([part], flat[5:6], 2.0)
    assert bool((x[:99] == 4).all()) and x[99] == 8


@pytest.mark.parametrize("power_scale,power_most", [(-126, -110), (-120, -100), (-100, -126), (-126, -126), (-140, -130), (-149, -149), (-99, 0), (-101, 0), (-100, -1), (110, 3), (0, -110)])
def test_factors_of_any_size(power_scale, power_most):
    """scale max_norm / norm from 2^-400 to 2^110, on numbers whose results are normal ones where there are such: the factor keeps its 24 bits."""
    dev = need_gpu()
    scale, most = 1.375 * 2.0 ** power_scale if power_scale > -149 else 2.0 ** -149, 1.5 * 2.0 ** power_most if power_most > -149 else 2.0 ** -149
    x = (1 + torch.rand(1000, generator=torch.Generator().manual_seed(1))) * 2.0 ** (-130 if power_scale > 0 else 110)
    x[::7] = 1.75 * 2.0 ** (-149 if power_scale > 0 else 127)
    tensors = [x.to(dev), x.bfloat16().to(dev)]
    out = [torch.empty(1000, device=dev) for _ in tensors]
    norm = B.brsvd_grad_norm(tensors, scale=scale)
    B.brsvd_grad_clip(tensors, norm, most, scale=scale, out=out)
    check_clipped(out, tensors, float(norm), most, scale)
    # and with a norm that has nothing to do with them
    for power in (-60, 0, 120):
        norm = torch.full((1,), 1.25 * 2.0 ** power, device=dev)
        B.brsvd_grad_clip(tensors, norm, most, scale=scale, out=out)
        check_clipped(out, tensors, float(norm), most, scale)
