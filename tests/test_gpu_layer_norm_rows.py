"""Layer norm backward on both sides of the number of rows at which rows of 65 to 128 chunks go from a block each to a warp
each (8192), with and without edges, to the tolerances of the other sizes."""
import pytest
import torch

from test_gpu_layer_norm import run_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [272, 300, 501, 512, 700, 768, 1000, 1024])
@pytest.mark.parametrize("T", [40, 8192, 8193, 9001])
def test_backward(cuda_device, T, D, dtype):
    run_backward(T, D, dtype, torch.float32, torch.float32)
    run_backward(T, D, dtype, torch.bfloat16, torch.bfloat16, pad=1)
