"""Mixture of experts for a few tokens against the definition in fp64.

Tolerances, element by element.  Products of bf16 numbers are exact in fp32, and sums of n of them are off by at most n * 2^-23 * the sum of
magnitudes (each addition cut, or rounded): dg, du for the two halves of the first product.  silu has a slope of at most 1.1 and
|silu(g)| <= |g|, so h is off by 1.1 dg |u| + |g| du + 1.1 dg du, 8 * 2^-24 of itself (exp, quotient, product) and its rounding to bf16, 2^-8.  The
second product adds |W2| dh and f * 2^-23 of its magnitudes; the weighted sum of k experts and the base k + 2 roundings; the output half a step."""
import pytest
import torch

import paper_2405_13053_amd as m
from tests import mx4_cases as mx

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
BF = torch.bfloat16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(shape, g, std=1.0, dtype=BF):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


class Layer:
    """Weights of N experts, and their values in fp64."""

    def __init__(self, N, d, f, mx4, g):
        W1, W2 = randn((N, 2 * f, d), g, d ** -0.5), randn((N, d, f), g, f ** -0.5)
        if mx4:
            a, b = [m.quantize_mx4(w) for w in W1], [m.quantize_mx4(w) for w in W2]
            self.V1, self.V2 = [mx.values(*q) for q in a], [mx.values(*q) for q in b]
            self.weights = (torch.stack([q for q, _ in a]), torch.stack([q for q, _ in b]))
            self.scales = dict(w1_scale=torch.stack([s for _, s in a]), w2_scale=torch.stack([s for _, s in b]))
        else:
            self.V1, self.V2 = W1.double(), W2.double()
            self.weights, self.scales = (W1, W2), {}
        self.N, self.d, self.f = N, d, f

    def reference(self, x, idx, w, scale=1.0, base=None):
        """(out, how far off it may be)"""
        T, k = idx.shape
        x, f = x.double(), self.f
        out, tol, size = (torch.zeros((T, self.d), dtype=torch.float64, device="cuda") for _ in range(3))
        for e in range(self.N):
            share = (w.double() * (idx == e)).sum(1)
            most = (w.double().abs() * (idx == e)).sum(1)
            rows = (idx == e).any(1).nonzero().flatten()
            if rows.numel() == 0:
                continue
            V1, V2 = self.V1[e], self.V2[e]
            both, off = x[rows] @ V1.t(), (x[rows].abs() @ V1.abs().t()) * self.d * U
            g, u, dg, du = both[:, :f], both[:, f:], off[:, :f], off[:, f:]
            h = g / (1 + torch.exp(-g)) * u
            dh = 1.1 * dg * u.abs() + g.abs() * du + 1.1 * dg * du + h.abs() * (4 * U + 2.0 ** -8)
            y, dy = h @ V2.t(), (dh + (h.abs() + dh) * f * U) @ V2.abs().t()
            out[rows] += share[rows, None] * y
            tol[rows] += most[rows, None] * dy
            size[rows] += most[rows, None] * (y.abs() + dy)
        out, tol, size = scale * out, abs(scale) * tol, abs(scale) * size
        if base is not None:
            out, size = out + base.double(), size + base.double().abs()
        tol = tol + (k + 2) * U * size
        return out, tol + 2.0 ** -8 * (out.abs() + tol)


def close(out, ref):
    ref, tol = ref
    bad = ~((out.double() - ref).abs() <= tol * 1.001)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, worst {float(((out.double() - ref).abs() / tol.clamp_min(1e-300)).max()):.3f}"


def routing(T, N, k, g, padded=False, zipf=False):
    u = torch.rand((T, N), generator=g, device="cuda")
    if zipf:
        u = u ** (torch.arange(1, N + 1, device="cuda") ** 1.5)
    idx = torch.topk(u, min(k, N), 1).indices.to(torch.int32)
    if k > N:   # ids that stand twice
        idx = torch.cat([idx, idx[:, :1].expand(T, k - N)], 1)
    if padded:
        idx[torch.rand(T, generator=g, device="cuda") < 0.4] = -1
        idx[torch.rand((T, k), generator=g, device="cuda") < 0.1] = N
    return idx.contiguous(), torch.softmax(randn((T, k), g, 1.0, torch.float32), 1).contiguous()


# T, N, k, d, f: one token to the most; channels past the last tile, K tiles that end in parts, more tokens to an expert than a block takes
CASES = [(1, 8, 2, 512, 256), (1, 1, 1, 32, 32), (1, 64, 8, 1024, 96), (2, 4, 2, 544, 1056), (3, 3, 3, 96, 4128), (4, 7, 2, 1056, 288),
         (4, 2, 8, 256, 64), (5, 8, 2, 512, 256), (9, 28, 4, 2080, 160), (16, 4, 1, 288, 544), (16, 8, 8, 64, 1024), (17, 8, 2, 512, 96),
         (33, 28, 4, 1056, 352), (64, 2, 2, 320, 288), (64, 64, 8, 128, 64), (63, 3, 2, 4096, 512), (40, 1, 1, 96, 2048), (1, 2, 2, 2048, 16384),
         (4, 5, 3, 64, 8192), (1, 7, 4, 992, 4000), (2, 64, 8, 544, 2048), (4, 16, 2, 4096, 320), (2, 3, 2, 12288, 64), (4, 3, 2, 8192, 96)]


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T,N,k,d,f", CASES)
def test_experts_forward(T, N, k, d, f, mx4):
    g = gen(T * 100 + N + d + f)
    layer, x = Layer(N, d, f, mx4, g), randn((T, d), g)
    idx, w = routing(T, N, k, g, zipf=T % 2 == 1)
    out = torch.full((T + 1, d), 7.0, dtype=BF, device="cuda")
    m.experts_forward(x, idx, w, *layer.weights, **layer.scales, out=out[:T])
    close(out[:T], layer.reference(x, idx, w))
    assert (out[T] == 7).all()
    base = randn((T, d), g)
    ref = layer.reference(x, idx, w, 2.0, base)
    close(m.experts_forward(x, idx, w, *layer.weights, **layer.scales, scale=2.0, base=base), ref)
    again = base.clone()   # base and out are one
    m.experts_forward(x, idx, w, *layer.weights, **layer.scales, scale=2.0, base=again, out=again)
    close(again, ref)


@pytest.mark.parametrize("T,N,k,d,f", [(1, 4, 2, 40, 24), (3, 5, 2, 1000, 72), (7, 5, 2, 200, 1016), (30, 4, 3, 72, 136)])
def test_bf16_widths_that_are_no_multiple_of_32(T, N, k, d, f):
    g = gen(T + d)
    layer, x = Layer(N, d, f, False, g), randn((T, d), g)
    idx, w = routing(T, N, k, g)
    close(m.experts_forward(x, idx, w, *layer.weights), layer.reference(x, idx, w))


@pytest.mark.parametrize("T", [1, 4, 64])
@pytest.mark.parametrize("d,f,mx4", [(8, 8, False), (8, 131072, False), (131072, 8, False), (32, 131072, True), (131072, 32, True)])
def test_least_and_largest_widths(T, d, f, mx4):
    g = gen(T + d)
    layer, x = Layer(3, d, f, mx4, g), randn((T, d), g)
    Wg = randn((d, 3), g, d ** -0.5, torch.float32)
    out, idx, w = m.moe_forward(x, Wg, None, *layer.weights, 2, **layer.scales, return_routing=True)
    close(out, layer.reference(x, idx, w))
    assert torch.equal(out, m.experts_forward(x, idx, w, *layer.weights, **layer.scales))


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T", [1, 4, 13, 64])
def test_padding_and_ids_outside(T, mx4):
    g = gen(T)
    layer, x = Layer(6, 256, 320, mx4, g), randn((T, 256), g)
    idx, w = routing(T, 6, 3, g, padded=True)
    base = randn((T, 256), g)
    out = m.experts_forward(x, idx, w, *layer.weights, **layer.scales, base=base)
    close(out, layer.reference(x, idx, w, 1.0, base))
    idx[:] = -1
    x[:] = float("nan")
    assert torch.equal(m.experts_forward(x, idx, w, *layer.weights, **layer.scales, base=base), base)
    assert (m.experts_forward(x, idx, w, *layer.weights, **layer.scales) == 0).all()


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T", [3, 4, 16, 40])
def test_what_is_not_finite_stays_with_its_token_and_its_expert(T, mx4):
    g = gen(T + 50)
    layer, x = Layer(4, 288, 160, mx4, g), randn((T, 288), g)
    idx = torch.stack([torch.arange(T, device="cuda") % 3, torch.full((T,), 2, device="cuda")], 1).to(torch.int32)
    idx[:, 1] = torch.where(idx[:, 0] == 2, 0, 1)
    idx[idx[:, 0] == 1, 1] = 0
    w = torch.full((T, 2), 0.5, device="cuda")
    clean = m.experts_forward(x, idx, w, *layer.weights, **layer.scales)
    x2 = x.clone()
    x2[1, 7] = float("nan")
    out = m.experts_forward(x2, idx, w, *layer.weights, **layer.scales)
    rest = torch.arange(T, device="cuda") != 1
    assert torch.isnan(out[1]).all() and torch.equal(out[rest], clean[rest])
    W = [t.clone() for t in layer.weights]
    scales = {n: s.clone() for n, s in layer.scales.items()}
    if mx4:   # expert 3 is nobody's, expert 2 some tokens'
        scales["w2_scale"][2:] = 255
        scales["w1_scale"][3] = 255
    else:
        W[1][2:] = float("nan")
        W[0][3] = float("inf")
    out = m.experts_forward(x, idx, w, *W, **scales)
    hit = (idx == 2).any(1)
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], clean[~hit])


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T,N,k,d,f,inv", [(1, 8, 2, 512, 256, 1.0), (2, 28, 4, 4096, 64, 0.05), (1, 64, 8, 1000, 64, 1.0), (17, 12, 3, 1056, 96, 1.0),
                                           (64, 28, 1, 256, 128, 0.5), (5, 1, 1, 96, 64, 1.0), (64, 5, 5, 64, 32, 1.0)])
def test_moe_forward(T, N, k, d, f, inv, mx4):
    if mx4 and d % 32:
        pytest.skip("4 bits come in blocks of 32")
    g = gen(T * 9 + N + d)
    layer, x = Layer(N, d, f, mx4, g), randn((T, d), g)
    Wg, bias = randn((d, N), g, d ** -0.5, torch.float32), randn((N,), g, 0.5, torch.float32)
    for b in (bias, None):
        logits = x.double() @ Wg.double() + (0 if b is None else b.double())
        # an element's way through the sum: d / 16 rows at most in a lane, then less than 32 partial sums
        off = ((x.double().abs() @ Wg.double().abs()) * (d / 16 + 32) * 2.0 ** -24).amax(1) + 2.0 ** -24 * logits.abs().amax(1)
        top, order = torch.sort(logits, dim=1, descending=True, stable=True)
        n = min(k, N - 1)
        clear = (top[:, :n] - top[:, 1:n + 1]).amin(1) > 2 * off if N > 1 else torch.ones(T, dtype=torch.bool, device="cuda")
        assert clear.sum() >= 0.75 * T   # the others may rank either way
        out, idx, w = m.moe_forward(x, Wg, b, *layer.weights, k, **layer.scales, inv_temperature=inv, return_routing=True)
        assert torch.equal(idx[clear].long(), order[clear, :k])
        want = torch.softmax(torch.gather(logits, 1, idx.long()) * inv, 1)
        assert ((w.double() - want).abs() <= 1e-6 + inv * off[:, None]).all()
        close(out, layer.reference(x, idx, w))
        assert torch.equal(out, m.moe_forward(x, Wg, b, *layer.weights, k, **layer.scales, inv_temperature=inv))
        assert torch.equal(out, m.experts_forward(x, idx, w, *layer.weights, **layer.scales))


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("N,k,d", [(64, 8, 512), (28, 4, 1024), (28, 3, 1056), (8, 2, 4096), (8, 2, 4128), (3, 2, 64), (16, 1, 1376), (1, 1, 32),
                                   (64, 8, 1024), (28, 4, 2048), (28, 4, 2080), (5, 2, 8192), (5, 2, 8224)])
def test_moe_forward_of_one_token(N, k, d, mx4):
    """Up to 65536 columns times rows of the gate in the first product's workgroups, beyond that a launch in front."""
    test_moe_forward(1, N, k, d, 96, 1.0, mx4)


def test_equal_logits_go_to_the_lowest_index():
    g = gen(5)
    layer, x = Layer(6, 64, 32, False, g), randn((9, 64), g)
    Wg = randn((64, 1), g, 0.1, torch.float32).expand(64, 6).contiguous()
    _, idx, w = m.moe_forward(x, Wg, None, *layer.weights, 3, return_routing=True)
    assert (idx == torch.arange(3, device="cuda")).all() and ((w - 1 / 3).abs() <= 1e-6).all()


# ---- calls that programs make -----------------------------------------------------------------------------------------------------
def moe(layer, x, Wg, k, **more):
    return m.moe_forward(x, Wg, None, *layer.weights, k, **layer.scales, **more)


def test_without_tokens():
    layer = Layer(4, 64, 32, True, gen(1))
    x, idx, w = torch.empty((0, 64), dtype=BF, device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda")
    assert m.experts_forward(x, idx, w, *layer.weights, **layer.scales).shape == (0, 64)
    out, i, v = moe(layer, x, torch.zeros((64, 4), device="cuda"), 2, return_routing=True)
    assert out.shape == (0, 64) and i.shape == v.shape == (0, 2)


def test_refusals_of_the_binding():
    g = gen(2)
    a, b = Layer(4, 64, 96, True, g), Layer(4, 64, 96, False, g)
    x, (idx, w) = randn((8, 64), g), routing(8, 4, 2, g)
    call = lambda layer=a, x=x, idx=idx, w=w, W1=None, W2=None, **more: m.experts_forward(
        x, idx, w, W1 if W1 is not None else layer.weights[0], W2 if W2 is not None else layer.weights[1], **{**layer.scales, **more})
    Wg = torch.zeros((64, 4), device="cuda")
    wrong = [lambda: call(x=x[:4]), lambda: call(idx=idx[:4]), lambda: call(w=w[:, :1]), lambda: call(W1=a.weights[0][:2]), lambda: call(W2=a.weights[1][:, :32]),
             lambda: call(w1_scale=None), lambda: call(w2_scale=a.scales["w2_scale"][:, :, :8]), lambda: call(layer=b, W1=b.weights[0][:, :96]),
             lambda: call(base=x[:4]), lambda: call(out=x[:, :32]), lambda: call(x=x.t()), lambda: call(idx=idx.t()),
             lambda: moe(a, x, Wg.t().contiguous(), 2), lambda: m.moe_forward(x, Wg, torch.zeros(3, device="cuda"), *a.weights, 2, **a.scales)]
    for f in wrong:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: call(idx=idx.long()), lambda: call(w=w.double()), lambda: call(layer=b, x=x.float()), lambda: call(W1=a.weights[0].view(torch.int8)),
              lambda: call(base=x.float())):
        with pytest.raises(TypeError):
            f()
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    f32 = [t.float() for t in b.weights]
    for f, status in ((lambda: call(ws=small), 3), (lambda: call(layer=b, x=x.float(), W1=f32[0], W2=f32[1]), 2), (lambda: call(scale=float("nan")), 1),
                      (lambda: moe(a, x, Wg, 5), 1), (lambda: moe(a, x, Wg, 2, ws=small), 3),
                      (lambda: m.experts_forward(randn((65, 64), g), *routing(65, 4, 2, g), *a.weights, **a.scales), 2)):
        with pytest.raises(m.MeteoraError) as e:
            f()
        assert e.value.status == status


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("T,N,k,d,f", [(1, 8, 2, 512, 256), (3, 16, 4, 64, 8192), (4, 3, 2, 8192, 96), (13, 8, 2, 1056, 352), (64, 6, 3, 96, 2080)])
def test_what_a_workspace_holds_does_not_matter(T, N, k, d, f, mx4):
    g = gen(T + d)
    layer, x, Wg = Layer(N, d, f, mx4, g), randn((T, d), g), randn((d, N), g, d ** -0.5, torch.float32)
    idx, w = routing(T, N, k, g)
    for call in (lambda ws: m.experts_forward(x, idx, w, *layer.weights, **layer.scales, ws=ws), lambda ws: moe(layer, x, Wg, k, ws=ws)):
        got = [call(torch.full((m.experts_workspace_bytes(64, d, f, N, k),), fill, dtype=torch.uint8, device="cuda")) for fill in (0, 255, 255)]
        assert torch.equal(got[0], got[1]) and torch.equal(got[1], got[2])


@pytest.mark.parametrize("mx4", [True, False])
def test_graphs_that_share_a_workspace_and_another_stream(mx4):
    g = gen(61)
    N, k, d, f = 6, 2, 288, 352
    layer, Wg = Layer(N, d, f, mx4, g), randn((d, N), g, d ** -0.5, torch.float32)
    m.init()
    ws = torch.empty(m.experts_workspace_bytes(64, d, f, N, k), dtype=torch.uint8, device="cuda")

    def step(x, idx, w, ws):   # a gated layer, and one with its routing given onto it
        y, i, v = moe(layer, x, Wg, k, ws=ws, return_routing=True)
        return m.experts_forward(y, idx, w, *layer.weights, **layer.scales, base=x, scale=0.5, ws=ws), i, v

    cases = []
    for T in (64, 1, 20, 4):
        x, (idx, w) = randn((T, d), g), routing(T, N, k, g)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(x, idx, w, ws)
        cases.append((x, idx, w, got, graph))
    for i in range(3):
        for x, idx, w, got, graph in cases:
            x.copy_(randn(x.shape, g))
            idx.copy_(routing(x.shape[0], N, k, g, padded=i == 2)[0])
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, step(x, idx, w, None))), f"replay {i}"
    x, idx, w, got, _ = cases[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step(x, idx, w, None)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, other))


def test_two_streams_at_once():
    g = gen(63)
    layer, Wg = Layer(8, 512, 768, True, g), randn((512, 8), g, 512 ** -0.5, torch.float32)
    xs = [randn((T, 512), g) for T in (64, 2)]
    want = [moe(layer, x, Wg, 2) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(moe(layer, xs[i], Wg, 2))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in (0, 1) for y in got[i])


@pytest.mark.parametrize("T", [2, 24])
def test_weights_past_four_gigabytes(T):
    """The last of 48 experts of 57 + 29 MB in 4 bits; the first product's weights are 4.8 GB, their scales 0.3."""
    g = gen(70 + T)
    N, d, f = 48, 4096, 24576
    W1 = torch.zeros((N, 2 * f, d // 2), dtype=torch.uint8, device="cuda")
    W2 = torch.zeros((N, d, f // 2), dtype=torch.uint8, device="cuda")
    s1, s2 = (torch.zeros((N, *m.mx4_scale_shape(*shape)), dtype=torch.uint8, device="cuda") for shape in ((2 * f, d), (d, f)))
    W1[-1], s1[-1] = m.quantize_mx4(randn((2 * f, d), g, d ** -0.5))
    W2[-1], s2[-1] = m.quantize_mx4(randn((d, f), g, f ** -0.5))
    x = randn((T, d), g)
    idx = torch.full((T, 1), N - 1, dtype=torch.int32, device="cuda")
    w = torch.ones((T, 1), device="cuda")
    out = m.experts_forward(x, idx, w, W1, W2, w1_scale=s1, w2_scale=s2)
    one = Layer.__new__(Layer)
    one.N, one.d, one.f, one.V1, one.V2 = 1, d, f, [mx.values(W1[-1], s1[-1])], [mx.values(W2[-1], s2[-1])]
    close(out, one.reference(x, idx * 0, w))


# ---- run together -----------------------------------------------------------------------------------------------------------------
def test_a_block_with_4_bit_experts_from_its_own_quantisation():
    """A decode step of a block: a 4-bit projection, then the experts onto the residual stream, then the same through sorted rows."""
    g = gen(80)
    T, N, k, d, f = 24, 6, 2, 512, 352
    x, Wo = randn((T, d), g), m.quantize_mx4(randn((d, d), g, d ** -0.5))
    layer, Wg = Layer(N, d, f, True, g), randn((d, N), g, d ** -0.5, torch.float32)
    y = m.base_gemm_mx4(x, *Wo)
    out, idx, w = moe(layer, y, Wg, k, base=x, return_routing=True)
    close(out, layer.reference(y, idx, w, 1.0, x))
    # the experts' products over sorted rows, with x and h in 4 bits too: the same but for their rounding
    ys, pos, offsets = m.sort_tokens(y, idx, N)
    both = m.gemm_mx4(*m.quantize_mx4(ys), layer.weights[0], layer.scales["w1_scale"], offsets=offsets).float()
    h = (torch.nn.functional.silu(both[:, :f]) * both[:, f:]).bfloat16()
    sorted_out = m.unsort_tokens(m.gemm_mx4(*m.quantize_mx4(h.contiguous()), layer.weights[1], layer.scales["w2_scale"], offsets=offsets), pos, w, base=x)
    moved = (out.double() - x.double()).norm()
    # a normal row rounded to 4 bits is off by some 0.12 of its norm: y's rounding acts on gate and up (0.17), h's adds its own: 0.21 together
    assert (sorted_out.double() - out.double()).norm() <= 0.35 * moved
