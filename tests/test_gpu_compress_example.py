"""The example that runs the operators together: what it prints has to hang together."""
import importlib.util
import os

import pytest

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_compress_output_matrix():
    need_gpu()
    spec = importlib.util.spec_from_file_location("compress_output_matrix", os.path.join(ROOT, "examples", "compress_output_matrix.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    said = example.main(["--vocab", "3000", "--dim", "200", "--rank", "40", "--tokens", "600", "--steps", "20"])
    # factors lose, the 8-bit remainder brings almost all of it back, distillation repairs a part
    assert said["factors"] > said["whole"]
    assert abs(said["factors and 8-bit remainder"] - said["whole"]) < 0.1 * (said["factors"] - said["whole"])
    assert said["logits of four tokens off by"] < 0.05
    assert said["divergence after"] < 0.5 * said["divergence before"]
    assert said["factors, distilled"] < said["factors"]
