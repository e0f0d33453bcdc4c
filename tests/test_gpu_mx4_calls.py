"""Calls of the 4-bit operators and the experts that programs make: rows without a number through every way, a routed token without one, the least workspace of
the fp32 gradient, and that gradient in a graph."""
import pytest
import torch

import paper_2405_13053_amd as m
from tests.test_gpu_experts import Layer, randn
from tests.test_gpu_mx4 import TYPES, gen, operand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out", [(2, 4096, 4096), (4, 1056, 264), (16, 1024, 4104), (17, 96, 72), (40, 2080, 1376), (64, 4096, 520), (300, 1056, 4096),
                                          (1100, 544, 4096), (2100, 4096, 4096)])
def test_rows_and_blocks_without_a_number(T, d_in, d_out, dtype):
    g = gen(T + d_in)
    x = torch.randn((T, d_in), generator=g, device="cuda").to(dtype)
    W, ws, _ = operand(d_out, d_in, g)
    clean = m.base_gemm_mx4(x, W, ws)
    assert torch.isfinite(clean).all()
    x[1, d_in - 1] = float("nan")
    x[T - 1, 7] = float("-inf")
    out = m.base_gemm_mx4(x, W, ws)
    hit = torch.zeros(T, dtype=torch.bool, device="cuda")
    hit[[1, T - 1]] = True
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], clean[~hit])
    ws[(d_in - 1) // 512, d_out - 1, (d_in // 32 - 1) % 4 * 4 + (d_in // 32 - 1) % 16 // 4] = 255   # the last block of the last channel
    out = m.base_gemm_mx4(x, W, ws)
    assert torch.isnan(out[:, -1]).all() and torch.equal(out[~hit, :-1], clean[~hit, :-1])


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T,N,k,d,f", [(1, 8, 2, 512, 256), (1, 28, 4, 4096, 64), (3, 8, 2, 512, 256), (5, 28, 4, 288, 96), (16, 8, 8, 1056, 96), (40, 64, 2, 288, 96)])
def test_a_gated_token_without_a_number_keeps_it(T, N, k, d, f, mx4):
    g = gen(T + N + d)
    layer, x, Wg = Layer(N, d, f, mx4, g), randn((T, d), g), randn((d, N), g, d ** -0.5, torch.float32)
    clean, idx, w = m.moe_forward(x, Wg, None, *layer.weights, k, **layer.scales, return_routing=True)
    t = T // 2
    x[t, d - 3] = float("nan")
    out, i, v = m.moe_forward(x, Wg, None, *layer.weights, k, **layer.scales, return_routing=True)
    rest = torch.arange(T, device="cuda") != t
    assert torch.equal(out[rest], clean[rest]) and torch.equal(i[rest], idx[rest]) and torch.equal(v[rest], w[rest])
    assert torch.isnan(out[t]).all() and ((i[t] >= 0) & (i[t] < N)).all() and i[t].unique().numel() == k


@pytest.mark.parametrize("T,d_in,d_out", [(1, 512, 14336), (64, 4096, 14336), (5000, 32, 4096), (30000, 32, 13824), (20000, 4096, 8)])
def test_least_workspace_of_the_fp32_gradient(T, d_in, d_out):
    g = gen(T + d_out)
    W, ws = m.quantize_mx4(torch.randn((d_out, d_in), generator=g, device="cuda"))
    dy = torch.randn((T, d_out), generator=g, device="cuda")
    need = m.base_gemm_mx4_backward_workspace_bytes(d_in, d_out, torch.float32) - 256
    room = torch.full((need + (1 << 20),), 9, dtype=torch.uint8, device="cuda")
    dx = m.base_gemm_mx4_backward(dy, W, ws, ws=room[:need])
    assert (room[need:] == 9).all() and torch.equal(dx, m.base_gemm_mx4_backward(dy, W, ws))
    with pytest.raises(m.MeteoraError):
        m.base_gemm_mx4_backward(dy, W, ws, ws=room[:need - 256])


def test_fp32_gradients_in_graphs_that_share_a_workspace():
    g = gen(51)
    m.init()
    W, ws = m.quantize_mx4(torch.randn((1032, 544), generator=g, device="cuda"))
    room = torch.empty(m.base_gemm_mx4_backward_workspace_bytes(544, 1032, torch.float32), dtype=torch.uint8, device="cuda")
    cases = []
    for T in (1, 70, 3000):
        dy, dx = torch.randn((T, 1032), generator=g, device="cuda"), torch.empty((T, 544), device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.base_gemm_mx4_backward(dy, W, ws, out=dx, ws=room)
        cases.append((dy, dx, graph))
    for i in range(3):
        for dy, dx, graph in cases:
            dy.copy_(torch.randn(dy.shape, generator=g, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dx, m.base_gemm_mx4_backward(dy, W, ws)), f"replay {i}"
