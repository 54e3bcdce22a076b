"""The dense operators at sizes that take every tile of their products, whole and with the depth split:
few rows against wide weights, deep and narrow ones, a last turn of smaller tiles."""
import pytest
import torch

import test_gpu_dense as dense

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.mark.parametrize("m,n,k", [(40, 130, 72), (40, 130, 2056), (70, 20000, 72), (70, 20000, 136), (1300, 130, 4104),
                                   (260, 20000, 72), (6100, 130, 8208), (6100, 2056, 72), (2600, 6008, 72)])
@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, F32)])
def test_int8_linear(m, n, k, dtype, out):
    dense.test_int8_linear(m, n, k, dtype, out)


@pytest.mark.parametrize("m,f,k", [(40, 130, 72), (40, 130, 2056), (70, 8200, 72), (40, 8200, 8208), (70, 8200, 136),
                                   (900, 130, 4104), (70, 20000, 136), (150, 3000, 8208), (2100, 3000, 72),
                                   (260, 20000, 72), (150, 8200, 8208)])
@pytest.mark.parametrize("out,act", [(BF16, 1), (F32, 0)])
def test_int8_gated_linear(m, f, k, out, act):
    dense.test_int8_gated_linear(m, f, k, BF16, out, act)


@pytest.mark.parametrize("m,f,k", [(40, 130, 72), (40, 130, 1096), (40, 20000, 72), (40, 8200, 4104), (70, 8200, 72),
                                   (200, 130, 8208), (70, 20000, 72), (150, 3000, 4104), (200, 20000, 72),
                                   (260, 20000, 72), (150, 8200, 4104)])
@pytest.mark.parametrize("dtype,act", [(F16, 1), (BF16, 0)])
def test_gated_linear(m, f, k, dtype, act):
    dense.test_gated_linear(m, f, k, dtype, act)


@pytest.mark.parametrize("m,f,k", [(40, 520, 72), (6100, 130, 264), (70, 4500, 520), (400, 130, 8208), (1300, 8200, 136),
                                   (900, 130, 8208), (4000, 130, 4104), (6100, 3000, 264), (70, 20000, 264),
                                   (2600, 6008, 72)])
def test_gated_backward(m, f, k):
    dense.test_gated_backward(m, f, k, BF16, 0)
