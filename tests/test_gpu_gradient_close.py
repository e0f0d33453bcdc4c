"""The gradient of 4-bit projections against bounds that a part of fp32 numbers, or the last outputs, gone missing does not keep (see gradient_cases.py;
tests/test_gradient_close_host.py shows which)."""
import pytest
import torch

import paper_2405_13053_amd as m
from tests import gradient_cases as gc
from tests.test_gpu_mx4 import TYPES, gen, operand

pytestmark = pytest.mark.gpu


def from_codes(T, d_in, d_out, dtype):
    """Whether the codes themselves are read: up to 256 tokens always, to 1024 in one round of workgroups (fp32: where there are more than 192 outputs, or
    up to two rounds)."""
    if dtype == torch.float32:
        return d_out > 192 or -(-d_in // 128) * -(-T // 32) <= 512
    return T <= 256 or (T <= 1024 and -(-d_in // 128) * -(-T // 64) <= 256)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out", [(1, 32, 8), (1, 128, 264), (15, 160, 4096), (16, 4096, 512), (17, 608, 8200), (33, 2080, 1376), (64, 5120, 13824),
                                          (65, 96, 1160), (200, 544, 2056), (257, 4096, 4096), (1000, 1376, 2080), (1025, 256, 9000), (3, 131072, 64),
                                          (2, 64, 300000), (40, 32, 131072), (7, 96, 131080), (20, 96, 13816), (300, 96, 4096),
                                          (16384, 128, 192), (16385, 128, 192), (16385, 128, 200), (70000, 96, 264)])
def test_gradient(T, d_in, d_out, dtype):
    g = gen(T + d_in + d_out + 1)
    W, ws, V = operand(d_out, d_in, g)
    dy = torch.randn((T, d_out), generator=g, device="cuda").to(dtype)
    codes = from_codes(T, d_in, d_out, dtype)
    gc.close(m.base_gemm_mx4_backward(dy, W, ws), gc.reference(dy, V, dtype, codes))
    for numbers in (32, 8, 1):   # nothing but the last outputs
        last = dy.clone()
        last[:, :-numbers] = 0
        gc.close(m.base_gemm_mx4_backward(last, W, ws), gc.reference(last, V, dtype, codes, min(numbers, d_out)))


def test_fp32_rows_do_not_depend_on_how_many_there_are():
    """Beyond 65536 tokens the same sums as for fewer."""
    g = gen(31)
    W, ws, _ = operand(264, 96, g)
    dy = torch.randn((70000, 264), generator=g, device="cuda")
    dx = m.base_gemm_mx4_backward(dy, W, ws)
    assert torch.equal(dx[:40000], m.base_gemm_mx4_backward(dy[:40000], W, ws)) and torch.equal(dx[40000:], m.base_gemm_mx4_backward(dy[40000:], W, ws))


def test_fp32_batches():
    """131072 inputs go in batches of 8192 tokens; the results are 4.3 GB."""
    g = gen(32)
    T, d_in, d_out = 8192 + 40, 131072, 200
    W, ws, V = operand(d_out, d_in, g)
    dy = torch.randn((T, d_out), generator=g, device="cuda")
    dx = torch.full((T + 1, d_in), 7.0, device="cuda")
    m.base_gemm_mx4_backward(dy, W, ws, out=dx[:T])
    at = torch.tensor([0, 33, 4095, 8159, 8191, 8192, 8193, T - 1], device="cuda")
    gc.close(dx[at], gc.reference(dy[at], V, torch.float32, True))
    assert (dx[T] == 7).all() and (dx[:T:40] != 0).any(1).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_groups_one_by_one(dtype):
    """The gradient of a product over groups with respect to its rows: a call for every group that has some."""
    g = gen(33)
    bounds, d_in, d_out = [0, 7, 7, 300, 333], 352, 136
    parts = [operand(d_out, d_in, g) for _ in range(4)]
    W, ws = torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])
    dy = torch.randn((340, d_out), generator=g, device="cuda").to(dtype)
    dx = torch.full((340, d_in), 7.0, device="cuda", dtype=dtype)
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        if b > a:
            m.base_gemm_mx4_backward(dy[a:b], W[e], ws[e], out=dx[a:b])
            codes = from_codes(b - a, d_in, d_out, dtype)
            gc.close(dx[a:b], gc.reference(dy[a:b], parts[e][2], dtype, codes))
    assert (dx[bounds[-1]:] == 7).all()
