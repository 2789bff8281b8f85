"""8-bit floating-point codes, products and layers at the edges of what their definitions allow."""
import numpy as np
import pytest

from oracle import f8_oracle as F
from tests.test_gpu_f8 import host, rng

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_1805_11046_b200.binding as binding
    return binding


@pytest.mark.parametrize("shape", [(3, 0), (2, 3, 0), (2, 1, 5, 0), (0,)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_a_layer_of_no_inputs_puts_out_zeros(B, shape, dtype):
    """A sum of nothing, for activations of any number of dimensions."""
    import torch
    x = torch.empty(shape, dtype=getattr(torch, dtype), device="cuda")
    w, sw = torch.empty((48, 0), dtype=torch.uint8, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")
    y = torch.full((*shape[:-1], 48), 7.0, dtype=x.dtype, device="cuda")
    assert B.qbp_linear_f8(x, w, sw, y=y) is y and not y.any()
