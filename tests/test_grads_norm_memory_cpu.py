"""Clipping refuses a norm that lies in memory which it writes: every workgroup reads the norm while results are being written.  Checked without a GPU, with
addresses that are never followed."""
import ctypes as C

import pytest

import paper_1706_07191_amd as B
from tests.test_glu_grads_cpu import clip, tensor
from tests.test_model_ops_cpu import ARG, BF16


def at(address):
    return C.c_void_p(address)


@pytest.mark.parametrize("byte", [0, 4, 400, 796])
def test_norm_in_a_tensor_that_is_written(byte):
    """A tensor of 10 x 20 numbers in place, and as a result of another one: at its first number, inside, at its last."""
    mine, other = tensor(), tensor(data=65536)
    assert clip([mine], [mine], norm=at(4096 + byte)) == ARG
    assert clip([other], [mine], norm=at(4096 + byte)) == ARG
    far = tensor(data=131072)
    assert clip([far, other], [far, mine], norm=at(4096 + byte)) == ARG and clip([other, far], [mine, far], norm=at(4096 + byte)) == ARG


def test_norm_that_touches_a_result():
    """The last number of 16 bits, of which the norm takes more; the last row of a matrix with gaps."""
    other = tensor(data=65536, dtype=BF16)
    assert clip([other], [tensor(dtype=BF16)], norm=at(4096 + 396)) == ARG
    wide = tensor(ld=50)
    assert clip([wide], [wide], norm=at(4096 + 4 * (9 * 50 + 19))) == ARG
