"""The gradient of 4-bit projections against bounds that a part of fp32 numbers, or the last outputs, gone missing does not keep (see gradient_cases.py;
tests/test_gradient_close_host.py shows which)."""
import pytest
import torch

import paper_2405_13053_amd as m
from tests import gradient_cases as gc
from tests.test_gpu_mx4 import TYPES, gen, operand

pytestmark = pytest.mark.gpu


def from_codes(T, d_in, dtype):
    """Whether the codes themselves are read: up to 256 tokens always, to 1024 in one round of workgroups (fp32: up to 65536)."""
    if dtype == torch.float32:
        return T <= 65536
    return T <= 256 or (T <= 1024 and -(-d_in // 128) * -(-T // 64) <= 256)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out", [(1, 32, 8), (1, 128, 264), (15, 160, 4096), (16, 4096, 512), (17, 608, 8200), (33, 2080, 1376), (64, 5120, 13824),
                                          (65, 96, 1160), (200, 544, 2056), (257, 4096, 4096), (1000, 1376, 2080), (1025, 256, 9000), (3, 131072, 64),
                                          (2, 64, 300000), (40, 32, 131072), (7, 96, 131080), (20, 96, 13816), (300, 96, 4096)])
def test_gradient(T, d_in, d_out, dtype):
    g = gen(T + d_in + d_out + 1)
    W, ws, V = operand(d_out, d_in, g)
    dy = torch.randn((T, d_out), generator=g, device="cuda").to(dtype)
    codes = from_codes(T, d_in, dtype)
    gc.close(m.base_gemm_mx4_backward(dy, W, ws), gc.reference(dy, V, dtype, codes))
    for numbers in (32, 8, 1):   # nothing but the last outputs
        last = dy.clone()
        last[:, :-numbers] = 0
        gc.close(m.base_gemm_mx4_backward(last, W, ws), gc.reference(last, V, dtype, codes, min(numbers, d_out)))
