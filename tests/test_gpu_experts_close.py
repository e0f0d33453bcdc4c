"""The experts' operators at the sizes of tests/test_gpu_experts.py, against bounds that a few inputs, channels or weights gone wrong do not keep (see
experts_cases.py; tests/test_experts_close_host.py shows which)."""
import pytest
import torch

import paper_2405_13053_amd as m
from tests import experts_cases as ex
from tests import mx4_cases as mx
from tests import test_gpu_experts as te
from tests.test_gpu_experts import Layer, gen, randn, routing

pytestmark = pytest.mark.gpu


def close(out, layer, x, idx, w, **more):
    ex.close(out, ex.reference(x, idx, w, layer.V1, layer.V2, **more))


def only(layer, mx4, channels):
    """The same layer with nothing but its last channels."""
    (W1, W2), f = layer.weights, layer.f
    kept = torch.arange(f, device="cuda") >= f - channels
    W1 = torch.where(torch.cat([kept, kept])[:, None], W1, torch.zeros_like(W1))
    V1 = [torch.where(torch.cat([kept, kept])[:, None], v, 0.0) for v in layer.V1]
    new = Layer.__new__(Layer)
    new.N, new.d, new.f, new.weights, new.scales, new.V1, new.V2 = layer.N, layer.d, f, (W1, W2), layer.scales, V1, layer.V2
    return new


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T,N,k,d,f", te.CASES)
def test_experts_forward(T, N, k, d, f, mx4):
    g = gen(T * 100 + N + d + f + 1)
    layer, x = Layer(N, d, f, mx4, g), randn((T, d), g)
    idx, w = routing(T, N, k, g, padded=T % 4 == 0, zipf=T % 2 == 1)
    close(m.experts_forward(x, idx, w, *layer.weights, **layer.scales), layer, x, idx, w)
    base = randn((T, d), g)
    close(m.experts_forward(x, idx, w, *layer.weights, **layer.scales, scale=2.0, base=base), layer, x, idx, w, scale=2.0, base=base)


@pytest.mark.parametrize("T,N,k,d,f", [(1, 4, 2, 40, 24), (3, 5, 2, 1000, 72), (7, 5, 2, 200, 1016), (30, 4, 3, 72, 136)])
def test_bf16_widths_that_are_no_multiple_of_32(T, N, k, d, f):
    g = gen(T + d + 1)
    layer, x = Layer(N, d, f, False, g), randn((T, d), g)
    idx, w = routing(T, N, k, g)
    close(m.experts_forward(x, idx, w, *layer.weights), layer, x, idx, w)


WIDEST = [(8, 8, False), (8, 131072, False), (131072, 8, False), (32, 131072, True), (131072, 32, True), (2080, 1376, True), (4096, 4104, False), (4104, 4096, False),
          (992, 4000, True), (5120, 1056, True)]


@pytest.mark.parametrize("T", [1, 4, 13, 64])
@pytest.mark.parametrize("d,f,mx4", WIDEST)
def test_what_stands_last_is_there(d, f, mx4, T):
    """Rows of nothing but their last 8 inputs, and experts of nothing but their last 8 channels."""
    g = gen(T + d + f)
    layer, x = Layer(3, d, f, mx4, g), randn((T, d), g)
    idx, w = routing(T, 3, 2, g)
    close(m.experts_forward(x, idx, w, *layer.weights, **layer.scales), layer, x, idx, w)
    last = torch.zeros_like(x)
    last[:, -8:] = x[:, -8:]
    close(m.experts_forward(last, idx, w, *layer.weights, **layer.scales), layer, last, idx, w)
    tail = only(layer, mx4, 8)
    out = m.experts_forward(x, idx, w, *tail.weights, **tail.scales)
    close(out, tail, x, idx, w)
    assert (out != 0).float().mean() > 0.99
    Wg = randn((d, 3), g, d ** -0.5, torch.float32)
    out, idx, w = m.moe_forward(last, Wg, None, *tail.weights, 2, **tail.scales, return_routing=True)
    close(out, tail, last, idx, w)
    assert (out != 0).float().mean() > 0.99


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T,N,k,d,f", [(1, 8, 2, 512, 256), (1, 64, 8, 1024, 96), (5, 8, 2, 512, 256), (17, 12, 3, 1056, 96), (64, 28, 4, 2080, 1376)])
def test_moe_forward(T, N, k, d, f, mx4):
    g = gen(T * 9 + N + d + 1)
    layer, x, base = Layer(N, d, f, mx4, g), randn((T, d), g), randn((T, d), g)
    Wg = randn((d, N), g, d ** -0.5, torch.float32)
    out, idx, w = m.moe_forward(x, Wg, None, *layer.weights, k, **layer.scales, scale=0.5, base=base, return_routing=True)
    close(out, layer, x, idx, w, scale=0.5, base=base)


@pytest.mark.parametrize("T", [1, 4, 16, 64])
@pytest.mark.parametrize("d,N", [(64, 6), (1000, 28), (8192, 8), (8200, 64)])
def test_equal_columns_go_to_the_lowest_index(T, d, N):
    """Of columns of the gate that are equal the first ones are chosen, whatever order a batch's sums are in."""
    g = gen(T + d)
    layer, x = Layer(N, d, 32, False, g), randn((T, d), g)
    Wg = randn((d, 2), g, d ** -0.5, torch.float32)[:, torch.arange(N, device="cuda") % 2].contiguous()
    _, idx, w = m.moe_forward(x, Wg, None, *layer.weights, 2, return_routing=True)
    assert (idx == idx[:, :1] % 2 + torch.tensor([0, 2], device="cuda")).all() and (idx[:, 0] < 2).all() and (w == 0.5).all()
