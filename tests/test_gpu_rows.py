"""Rows sorted by adapter and back, with gradients, against plain fp64 on the CPU; and the 8-bit layer that they make together.

Tolerances.  Places, offsets and moved rows are equal.  unsort: k products and sums, the scale and the base in fp32, each off by at
most 2^-24 of the sum of magnitudes, then one rounding of the output.  dys: two products and one rounding.  dw: a thread adds
4 or 8 elements of every 256th piece of a row, then at most 10 sums across threads and the scale."""
import pytest
import torch

import paper_2405_13053_amd as m
from tests.test_gpu_i8 import U32, close, dense_ref, gen, half_step, rows_ref

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def places(idx, N):
    """pos, offsets by counting, on the CPU."""
    flat = idx.flatten().tolist()
    pos, offsets, at = [-1] * len(flat), [0], 0
    for e in range(N):
        for p, v in enumerate(flat):
            if v == e:
                pos[p] = at
                at += 1
        offsets.append(at)
    return torch.tensor(pos, dtype=torch.int32).view_as(idx), torch.tensor(offsets, dtype=torch.int32)


def routing(T, N, k, kind, g):
    idx = torch.randint(0, N, (T, k), generator=g, device="cuda", dtype=torch.int32)   # an id may stand twice
    if kind == "one":
        idx[:] = N - 1
    elif kind == "padded":
        idx[T // 3:T // 2 + 1] = -1
        idx[:, k // 2] = torch.where(torch.rand(T, generator=g, device="cuda") < 0.3, N + 5, idx[:, k // 2])
    elif kind == "none":
        idx[:] = -1
    elif kind == "junk":
        idx[::2] = 2 ** 31 - 1
        idx[1::3] = -2 ** 31
    return idx


SORTS = [(1, 4, 1), (1, 1, 8), (3, 28, 2), (64, 28, 2), (100, 5, 3), (129, 64, 8), (512, 7, 1), (777, 28, 2), (2050, 4, 4)]


@pytest.mark.parametrize("kind", ["uniform", "one", "padded", "none", "junk"])
@pytest.mark.parametrize("T,N,k", SORTS)
def test_sort_and_its_order(T, N, k, kind):
    g = gen(T + 17 * k)
    idx = routing(T, N, k, kind, g)
    pos, off = places(idx.cpu(), N)
    for dtype, d in ((torch.bfloat16, 8), (torch.float32, 136), (torch.bfloat16, 4104)):
        x = torch.randn((T, d), generator=g, device="cuda").to(dtype)
        xs = torch.full((T * k + 1, d), 7.0, device="cuda", dtype=dtype)
        _, gpos, goff = m.sort_tokens(x, idx, N, out=xs[:T * k])
        assert torch.equal(gpos.cpu(), pos) and torch.equal(goff.cpu(), off)
        want = torch.full((T * k + 1, d), 7.0, dtype=dtype)
        for j in range(k):
            there = pos[:, j] >= 0
            want[pos[there, j].long()] = x.cpu()[there]
        assert torch.equal(xs.cpu(), want)   # rows behind the last place as they were


@pytest.mark.parametrize("kind", ["uniform", "padded", "none"])
@pytest.mark.parametrize("T,N,k", SORTS)
def test_sort_quantised(T, N, k, kind):
    g = gen(T + 19 * k)
    idx = routing(T, N, k, kind, g)
    pos, off = places(idx.cpu(), N)
    for dtype, d in ((torch.bfloat16, 16), (torch.float32, 520), (torch.bfloat16, 4096), (torch.float32, 16400)):
        if T * d > 4e6:
            continue
        x = torch.randn((T, d), generator=g, device="cuda").to(dtype)
        xs = torch.full((T * k, d), 7, device="cuda", dtype=torch.int8)
        _, sc, gpos, goff = m.sort_tokens(x, idx, N, quantize=True, out=xs)
        assert torch.equal(gpos.cpu(), pos) and torch.equal(goff.cpu(), off)
        q, s = rows_ref(x.cpu())
        want = torch.full((T * k, d), 7, dtype=torch.int8)
        for j in range(k):
            there = pos[:, j] >= 0
            want[pos[there, j].long()] = q[there]
            assert torch.equal(sc.cpu()[pos[there, j].long()], s[there])
        assert torch.equal(xs.cpu(), want)


@pytest.mark.parametrize("T,N,k", [(4096, 28, 2), (9001, 64, 8), (70000, 28, 2), (70000, 64, 8), (33000, 1, 1)])
def test_long_batches_agree_with_the_bucket_lists(T, N, k):
    g = gen(T)
    idx = routing(T, N, k, "uniform", g)
    x = torch.randn((T, 8), generator=g, device="cuda").bfloat16()
    xs, pos, off = m.sort_tokens(x, idx, N)
    _, boff, tok, slot = m.bucket_tokens(idx, N)
    assert torch.equal(off, boff)
    assert torch.equal(pos.flatten()[(tok * k + slot).long()], torch.arange(T * k, device="cuda", dtype=torch.int32))
    assert torch.equal(xs, x[tok.long()])
    ws = torch.empty(m.sort_workspace_bytes(T, k, N), dtype=torch.uint8, device="cuda")
    m.sort_tokens(x, idx, N, ws=ws)
    few = m.sort_tokens(x[:50], idx[:50].contiguous(), N, ws=ws)   # a smaller batch in the same workspace
    want = m.sort_tokens(x[:50], idx[:50].contiguous(), N)
    assert all(torch.equal(a, b) for a, b in zip(few, want))


@pytest.mark.parametrize("kind", ["uniform", "one", "padded"])
def test_many_pairs_to_a_workgroup_again_and_again(kind):
    T, N, k = 150000, 64, 8   # 4688 pairs to each of 256 workgroups, 256 at a time
    g = gen(len(kind))
    idx = routing(T, N, k, kind, g)
    x = torch.zeros((T, 8), device="cuda", dtype=torch.bfloat16)
    flat = idx.flatten()
    order = torch.argsort(torch.where((flat >= 0) & (flat < N), flat, N).long(), stable=True)
    want = torch.empty(T * k, device="cuda", dtype=torch.int32)
    want[order] = torch.arange(T * k, device="cuda", dtype=torch.int32)
    want[(flat < 0) | (flat >= N)] = -1
    xs = torch.empty((T * k, 8), device="cuda", dtype=torch.bfloat16)
    for _ in range(10):
        _, pos, _ = m.sort_tokens(x, idx, N, out=xs)
        assert torch.equal(pos.flatten(), want)


# ---- back ----------------------------------------------------------------------------------------------------------------------
def unsort_ref(ys, pos, w, scale, base):
    """(result, sum of magnitudes) in fp64."""
    T, k = pos.shape
    out = torch.zeros((T, ys.shape[1]), dtype=torch.float64) if base is None else base.double().clone()
    mag = out.abs()
    for j in range(k):
        there = (pos[:, j] >= 0) & (pos[:, j] < ys.shape[0])
        part = scale * (1.0 if w is None else w[there, j, None].double()) * ys[pos[there, j].long()].double()
        out[there] += part
        mag[there] += part.abs()
    return out, mag


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weights,with_base", [(True, False), (True, True), (False, False), (False, True)])
@pytest.mark.parametrize("T,N,k,d,kind", [(1, 4, 1, 8, "uniform"), (3, 28, 2, 4096, "uniform"), (64, 28, 8, 136, "padded"),
                                          (257, 7, 3, 24, "padded"), (50, 4, 2, 5128, "one"), (40, 4, 2, 64, "none"),
                                          (333, 64, 4, 1032, "junk")])
def test_unsort(T, N, k, d, kind, weights, with_base, dtype):
    g = gen(T + d)
    pos, _ = places(routing(T, N, k, kind, g).cpu(), N)
    ys = torch.randn((T * k, d), generator=g, device="cuda").to(dtype)
    w = torch.randn((T, k), generator=g, device="cuda") if weights else None
    base = torch.randn((T, d), generator=g, device="cuda").to(dtype) if with_base else None
    ref, mag = unsort_ref(ys.cpu(), pos, None if w is None else w.cpu(), 1.75, None if base is None else base.cpu())
    out = m.unsort_tokens(ys, pos.cuda(), w, 1.75, base=base)
    tol = (k + 3) * U32 * mag + half_step(dtype) * 1.001 * ref.abs()
    assert ((out.cpu().double() - ref).abs() <= tol).all()
    if with_base:   # in place
        assert m.unsort_tokens(ys, pos.cuda(), w, 1.75, base=base, out=base) is base and torch.equal(base, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,k,d,kind", [(1, 4, 1, 8, "uniform"), (3, 28, 2, 4096, "uniform"), (64, 28, 8, 136, "padded"),
                                          (257, 7, 3, 24, "padded"), (50, 4, 2, 5128, "uniform"), (40, 4, 2, 64, "none"),
                                          (333, 64, 4, 1032, "junk"), (9, 4, 5, 14336, "padded")])
def test_unsort_backward(T, N, k, d, kind, dtype):
    g = gen(T + 3 * d)
    pos, _ = places(routing(T, N, k, kind, g).cpu(), N)
    ys = torch.randn((T * k, d), generator=g, device="cuda").to(dtype)
    dy = torch.randn((T, d), generator=g, device="cuda").to(dtype)
    for w in (torch.randn((T, k), generator=g, device="cuda"), None):
        dys = torch.full((T * k, d), 7.0, device="cuda", dtype=dtype)
        _, dw = m.unsort_backward(dy, ys, pos.cuda(), w, -0.5, out=dys)
        want = torch.full((T * k, d), 7.0, dtype=torch.float64)
        rw, mag = torch.zeros((T, k), dtype=torch.float64), torch.zeros((T, k), dtype=torch.float64)
        cy, cys = dy.cpu().double(), ys.cpu().double()
        for j in range(k):
            there = pos[:, j] >= 0
            at = pos[there, j].long()
            want[at] = -0.5 * (1.0 if w is None else w.cpu()[there, j, None].double()) * cy[there]
            rw[there, j] = -0.5 * (cy[there] * cys[at]).sum(1)
            mag[there, j] = 0.5 * (cy[there] * cys[at]).abs().sum(1)
        close(dys.cpu(), want, 2)
        n = 8 if dtype == torch.bfloat16 else 4
        chain = n * (d // n // 256 + 1) + 12
        assert ((dw.cpu().double() - rw).abs() <= chain * U32 * mag).all()
        only, none = m.unsort_backward(dy, ys, pos.cuda(), w, -0.5, out=torch.full_like(dys, 7.0), want_dw=False)
        assert none is None and torch.equal(only, dys)


def test_gradients_against_differences():
    """unsort is linear in w and in ys, sort in x: a difference over a power of two is the gradient itself up to fp32 rounding."""
    g = gen(21)
    T, N, k, d = 37, 5, 3, 72
    idx = routing(T, N, k, "padded", g)
    x = torch.randn((T, d), generator=g, device="cuda")
    xs, pos, off = m.sort_tokens(x, idx, N, out=torch.zeros((T * k, d), device="cuda"))
    w = torch.rand((T, k), generator=g, device="cuda")
    dy = torch.randn((T, d), generator=g, device="cuda")
    loss = lambda xs, w: (m.unsort_tokens(xs, pos, w, 1.5).double() * dy.double()).sum()
    dxs, dw = m.unsort_backward(dy, xs, pos, w, 1.5)
    dx = m.unsort_tokens(dxs, pos)
    size = float((1.5 * w.sum(1, keepdim=True) * dy.abs()).max() * x.abs().max()) * d * k
    for t, j in ((0, 0), (5, 1), (T - 1, 2), (T // 3, 0)):
        e = torch.zeros_like(w)
        e[t, j] = 4.0
        diff = float(loss(xs, w + e) - loss(xs, w)) / 4
        assert abs(diff - float(dw[t, j])) <= 8 * k * U32 * size
    for t, c in ((0, 0), (7, 71), (T - 1, 5), (T // 3, 1)):
        e = torch.zeros_like(x)
        e[t, c] = 4.0
        moved = m.sort_tokens(x + e, idx, N, out=torch.zeros_like(xs))[0]
        diff = float(loss(moved, w) - loss(xs, w)) / 4
        assert abs(diff - float(dx[t, c])) <= 8 * k * U32 * size
    assert (dx[T // 3] == 0).all() and (dw[T // 3] == 0).all()   # a padding token


def test_places_outside_ys_give_nothing():
    ys = torch.ones((4, 64), device="cuda")
    pos = torch.tensor([[0, 4], [-7, 2 ** 31 - 1], [3, -2 ** 31]], dtype=torch.int32, device="cuda")
    out = m.unsort_tokens(ys, pos)
    assert torch.equal(out[:, 0].cpu(), torch.tensor([1.0, 0.0, 1.0]))
    buf = torch.full((12, 64), 7.0, device="cuda")
    dys, dw = m.unsort_backward(torch.ones((3, 64), device="cuda"), ys, pos, out=buf[4:8])
    assert (buf[[0, 1, 2, 3, 5, 6, 8, 9, 10, 11]] == 7).all() and (buf[[4, 7]] == 1).all()
    assert torch.equal(dw.cpu(), torch.tensor([[64.0, 0], [0, 0], [64.0, 0]]))


def test_nan_in_rows_that_no_place_names():
    """Rows behind the last place hold anything: they reach no output."""
    g = gen(4)
    idx = routing(60, 4, 2, "padded", g)
    pos, off = places(idx.cpu(), 4)
    ys = torch.randn((120, 64), generator=g, device="cuda")
    ys[int(off[-1]):] = float("nan")
    w = torch.rand((60, 2), generator=g, device="cuda")
    w[pos.cuda() < 0] = float("inf")
    out = m.unsort_tokens(ys, pos.cuda(), w)
    dys, dw = m.unsort_backward(torch.ones((60, 64), device="cuda"), ys, pos.cuda(), w)
    assert torch.isfinite(out).all() and torch.isfinite(dw).all() and torch.isfinite(dys).all()


def test_rows_beyond_32_bit_offsets():
    g = gen(8)
    T, N, k, d = 140000, 8, 2, 8192   # xs: 4.6 GB
    idx = routing(T, N, k, "uniform", g)
    x = torch.randint(-100, 100, (T, d), generator=g, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    xs, pos, off = m.sort_tokens(x, idx, N)
    rows = torch.cat([torch.arange(0, T, 1999), torch.arange(T - 40, T)]).cuda()
    for j in range(k):
        assert torch.equal(xs[pos[rows, j].long()], x[rows])
    out = m.unsort_tokens(xs, pos, None, 0.5)
    assert torch.equal(out[rows], x[rows])
    dys, dw = m.unsort_backward(x, xs, pos, None, 2.0)
    assert torch.equal(dys[pos[rows, 1].long()], 2 * x[rows])


# ---- together ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,N,k,d_in,d_out,padded", [(1, 4, 2, 512, 264, False), (40, 8, 2, 1024, 512, True),
                                                     (300, 28, 2, 528, 776, True), (1100, 4, 1, 256, 1032, False)])
def test_a_layer_in_8_bits(T, N, k, d_in, d_out, padded):
    """Gate, rows by adapter, a product per adapter and the weighted sum onto the base projection, all weights in 8 bits."""
    g = gen(T)
    x = torch.randn((T, d_in), generator=g, device="cuda").bfloat16()
    Wg = torch.randn((d_in, N), generator=g, device="cuda") * d_in ** -0.5
    W, wsc = m.quantize_rows(torch.randn((d_out, d_in), generator=g, device="cuda") * d_in ** -0.5)
    E, esc = m.quantize_rows(torch.randn((N * d_out, d_in), generator=g, device="cuda") * d_in ** -0.5)
    E, esc = E.view(N, d_out, d_in), esc.view(N, d_out)
    idx, w, _ = m.gate_topk(x, Wg, None, k)
    if padded:
        idx[T - T // 4:] = -1
    out = m.base_gemm_i8(x, W, wsc)
    q, s = rows_ref(x.cpu())
    s = x.cpu().abs().amax(1).double() / 127
    ref = dense_ref(q, s, W.cpu(), wsc.cpu())
    close(out.cpu(), ref, 4)
    base = out.cpu().double()
    xs, xsc, pos, off = m.sort_tokens(x, idx, N, quantize=True)
    ys = m.gemm_i8(xs, xsc, E, esc, offsets=off)
    m.unsort_tokens(ys, pos, w, 2.0, base=out, out=out)
    want, mag = base.clone(), base.abs()
    for t in range(T):
        for j in range(k):
            e = int(idx[t, j])
            if 0 <= e < N:
                part = 2.0 * float(w[t, j]) * dense_ref(q[t:t + 1], s[t:t + 1], E[e].cpu(), esc[e].cpu())[0]
                want[t] += part
                mag[t] += part.abs()
    u = half_step(torch.bfloat16)   # the rows of ys and the output are rounded to bf16
    tol = (u * 1.01 + (k + 8) * U32) * mag + u * 1.01 * want.abs()
    assert ((out.cpu().double() - want).abs() <= tol).all()


def test_graphs_that_share_a_workspace_and_another_stream():
    g = gen(31)
    N, k, d_in, d_out = 8, 2, 512, 256
    E, esc = m.quantize_rows(torch.randn((N * d_out, d_in), generator=g, device="cuda"))
    E, esc = E.view(N, d_out, d_in), esc.view(N, d_out)
    m.init()

    def layer(x, idx, w, out, ws):
        xs, xsc, pos, off = m.sort_tokens(x, idx, N, quantize=True, ws=ws)
        return m.unsort_tokens(m.gemm_i8(xs, xsc, E, esc, offsets=off), pos, w, out=out)

    ws = torch.empty(m.sort_workspace_bytes(900, k, N), dtype=torch.uint8, device="cuda")
    cases = []
    for T in (900, 33):
        x = torch.randn((T, d_in), generator=g, device="cuda").bfloat16()
        idx, w = routing(T, N, k, "padded", g), torch.rand((T, k), generator=g, device="cuda")
        out = torch.empty((T, d_out), device="cuda", dtype=torch.bfloat16)
        layer(x, idx, w, out, ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(x, idx, w, out, ws)
        cases.append((x, idx, w, out, graph))
    for i in range(3):
        for x, idx, w, out, graph in cases:
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            idx.copy_(routing(x.shape[0], N, k, "padded" if i else "uniform", g))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, layer(x, idx, w, torch.empty_like(out), None)), f"replay {i}"
    x, idx, w, out, _ = cases[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer(x, idx, w, None, None)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, out)


def test_two_streams_at_once():
    g = gen(37)
    N, k, d_in, d_out = 8, 2, 1024, 520
    E, esc = m.quantize_rows(torch.randn((N * d_out, d_in), generator=g, device="cuda"))
    E, esc = E.view(N, d_out, d_in), esc.view(N, d_out)

    def layer(x, idx, w, out):
        xs, xsc, pos, off = m.sort_tokens(x, idx, N, quantize=True)
        base = m.base_gemm_i8(x, E[0], esc[0])
        return m.unsort_tokens(m.gemm_i8(xs, xsc, E, esc, offsets=off), pos, w, base=base, out=out)

    work = []
    for T in (2, 64, 777, 9000):
        x = torch.randn((T, d_in), generator=g, device="cuda").bfloat16()
        idx, w = routing(T, N, k, "padded", g), torch.rand((T, k), generator=g, device="cuda")
        work.append((x, idx, w, layer(x, idx, w, None)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(4):
        for a, b in zip(work, reversed(work)):
            for stream, (x, idx, w, want) in zip(streams, (a, b)):
                with torch.cuda.stream(stream):
                    got.append((layer(x, idx, w, None), want))
    torch.cuda.synchronize()
    for y, want in got:
        assert torch.equal(y, want)


def test_gradients_inside_a_graph():
    g = gen(41)
    T, N, k, d = 200, 8, 2, 264
    m.init()
    idx = routing(T, N, k, "padded", g)
    dy, w = torch.randn((T, d), generator=g, device="cuda").bfloat16(), torch.rand((T, k), generator=g, device="cuda")
    xs, pos, _ = m.sort_tokens(dy, idx, N)
    ys = torch.randn((T * k, d), generator=g, device="cuda").bfloat16()
    dys = torch.zeros_like(ys)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, dw = m.unsort_backward(dy, ys, pos, w, 2.0, out=dys)
        dx = m.unsort_tokens(dys, pos)
    for _ in range(3):
        dy.copy_(torch.randn((T, d), generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        e_dys, e_dw = m.unsort_backward(dy, ys, pos, w, 2.0)
        assert torch.equal(dys, e_dys) and torch.equal(dw, e_dw) and torch.equal(dx, m.unsort_tokens(e_dys, pos))


def test_binding_checks():
    x = torch.zeros((4, 64), device="cuda", dtype=torch.bfloat16)
    idx = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        m.sort_tokens(x, idx.long(), 4)
    with pytest.raises(ValueError):
        m.sort_tokens(x, idx[:3], 4)
    with pytest.raises(ValueError):
        m.sort_tokens(x[:, ::2], idx, 4)
    with pytest.raises(m.MeteoraError) as e:
        m.sort_tokens(x, idx, 65)
    assert e.value.status == 2
    with pytest.raises(m.MeteoraError) as e:
        m.sort_tokens(x, idx, 4, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    with pytest.raises(TypeError):
        m.unsort_tokens(x, idx, base=x.float())
    with pytest.raises(ValueError):
        m.unsort_backward(x[:3], x, idx)
    assert m.unsort_tokens(x[:0], idx).abs().sum() == 0    # no rows: every place is outside


@pytest.mark.parametrize("dtype", TYPES)
def test_no_tokens(dtype):
    """T = 0 (a step in which no sequence takes part): empty results, and no place taken."""
    N, k, d, n = 4, 2, 64, 24
    new = lambda *shape, dt=dtype: torch.empty(shape, device="cuda", dtype=dt)
    x, idx, w = new(0, d), new(0, k, dt=torch.int32), new(0, k, dt=torch.float32)
    W, ws = m.quantize_rows(torch.randn((N * n, d), device="cuda"))
    W, ws = W.view(N, n, d), ws.view(N, n)
    junk = torch.full((64,), 77, device="cuda", dtype=torch.int32)   # what the allocator may hand out for offsets
    del junk
    xs, pos, off = m.sort_tokens(x, idx, N)
    assert xs.shape == (0, d) and pos.shape == (0, k) and torch.equal(off.cpu(), torch.zeros(N + 1, dtype=torch.int32))
    xs, xsc, pos, off = m.sort_tokens(x, idx, N, quantize=True)
    assert xs.shape == (0, d) and xsc.shape == (0,) and not off.cpu().any()
    ys = m.gemm_i8(xs, xsc, W, ws, offsets=off, dtype=dtype)
    assert ys.shape == (0, n) and m.gemm_i8(xs, xsc, W[0], ws[0], dtype=dtype).shape == (0, n)
    base = m.base_gemm_i8(x, W[0], ws[0])
    assert base.shape == (0, n)
    assert m.unsort_tokens(ys, pos, w, 2.0, base=base, out=base) is base
    dys, dw = m.unsort_backward(base, ys, pos, w, 2.0)
    assert dys.shape == (0, n) and dw.shape == (0, k)
    q, s = m.quantize_rows(x)
    assert q.shape == (0, d) and s.shape == (0,)
    # rows that no token asks for
    ys = torch.randn((5, n), device="cuda").to(dtype)
    kept = torch.full_like(ys, 7.0)
    assert m.unsort_tokens(ys, pos, w).shape == (0, n)
    _, dw = m.unsort_backward(base, ys, pos, w, out=kept)
    assert dw.shape == (0, k) and (kept == 7).all()
    # limits hold all the same
    with pytest.raises(m.MeteoraError) as e:
        m.sort_tokens(new(0, 12), idx, N)
    assert e.value.status == 2
    with pytest.raises(m.MeteoraError) as e:
        m.quantize_rows(new(0, 12))
    assert e.value.status == 2


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,d", [(1, 1, 8), (37, 3, 136), (40, 2, 5128), (600, 2, 4104)])
def test_unsort_backward_without_the_rows(T, k, d, dtype):
    """Frozen weights of the slots: no dw, and then the rows ys are not read and need not be there."""
    g = gen(T + d)
    pos, _ = places(routing(T, 5, k, "padded", g).cpu(), 5)
    dy, w = torch.randn((T, d), generator=g, device="cuda").to(dtype), torch.randn((T, k), generator=g, device="cuda")
    ys = torch.randn((T * k, d), generator=g, device="cuda").to(dtype)
    want, _ = m.unsort_backward(dy, ys, pos.cuda(), w, 1.5, out=torch.full_like(ys, 7.0))
    out = torch.full_like(ys, 7.0)
    dys, dw = m.unsort_backward(dy, None, pos.cuda(), w, 1.5, out=out, want_dw=False)
    assert dys is out and dw is None and torch.equal(dys, want)
    with pytest.raises(ValueError):
        m.unsort_backward(dy, None, pos.cuda(), w, 1.5, out=out)            # dw is a product with ys
    with pytest.raises(ValueError):
        m.unsort_backward(dy, None, pos.cuda(), w, 1.5, want_dw=False)      # nothing says how many rows there are
    with pytest.raises(TypeError):
        m.unsort_backward(dy, None, pos.cuda(), w, 1.5, out=out.double(), want_dw=False)
    with pytest.raises(ValueError):
        m.unsort_backward(dy, None, pos.cuda(), w, 1.5, out=out[:, :d - 1], want_dw=False)


def places_sorted(idx, N):
    """pos, offsets by a stable sort, on the GPU."""
    flat = idx.flatten()
    valid = (flat >= 0) & (flat < N)
    key = torch.where(valid, flat, N).long()
    pos = torch.empty_like(flat)
    pos[torch.argsort(key, stable=True)] = torch.arange(flat.numel(), device=idx.device, dtype=torch.int32)
    counts = torch.bincount(key, minlength=N + 1)[:N]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    return torch.where(valid, pos, -1).view_as(idx), offsets


# as many pairs as the one launch takes with the most to a workgroup (21 of them with k = 7), and one token more
BORDER = [(2340, 64, 7), (2341, 64, 7), (3276, 28, 5), (3277, 28, 5), (16384, 28, 1), (16385, 28, 1), (2048, 64, 8), (2049, 64, 8), (8192, 4, 2)]


@pytest.mark.parametrize("kind", ["uniform", "one", "padded"])
@pytest.mark.parametrize("T,N,k", BORDER)
def test_sort_either_side_of_the_one_launch(T, N, k, kind):
    g = gen(T + 23 * k)
    idx = routing(T, N, k, kind, g)
    pos, off = places_sorted(idx, N)
    for dtype, d in ((torch.bfloat16, 8), (torch.float32, 72), (torch.bfloat16, 2056)):
        x = torch.randn((T, d), generator=g, device="cuda").to(dtype)
        xs = torch.full((T * k + 1, d), 7.0, device="cuda", dtype=dtype)
        _, gpos, goff = m.sort_tokens(x, idx, N, out=xs[:T * k])
        assert torch.equal(gpos, pos) and torch.equal(goff, off)
        want = torch.full_like(xs, 7.0)
        for j in range(k):
            there = pos[:, j] >= 0
            want[pos[there, j].long()] = x[there]
        assert torch.equal(xs, want)


# rows in a launch of their own: every width at which a wavefront or a workgroup holds another number of pieces, and rows that are read
# twice; the last ones have few pairs and more than 2^24 elements
MOVED = [(2049, 64, 8, 16), (2049, 64, 8, 512), (2341, 64, 7, 520), (8200, 28, 2, 2048), (2049, 5, 8, 2056), (16385, 28, 1, 1032),
         (2060, 64, 8, 4096), (2050, 7, 8, 4104), (2049, 4, 8, 8200), (2049, 4, 8, 16392), (1030, 4, 2, 16400), (5000, 28, 2, 4096)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["uniform", "padded"])
@pytest.mark.parametrize("T,N,k,d", MOVED)
def test_sort_quantised_with_the_rows_in_a_launch_of_their_own(T, N, k, d, kind, dtype):
    g = gen(T + d)
    idx = routing(T, N, k, kind, g)
    pos, off = places_sorted(idx, N)
    x = torch.randn((T, d), generator=g, device="cuda").to(dtype)
    x[T // 2] = 0
    x[1, d - 1], x[T - 1, 0], x[T - 1, d // 2] = float("nan"), float("inf"), -float("inf")
    good = torch.isfinite(x).all(1)
    finite = torch.where(good[:, None], x, torch.zeros_like(x))
    q, _ = rows_ref(finite)
    # by a tensor: fp32 tensors of a GPU are divided by a number by its reciprocal, which is an ulp off
    s = finite.abs().amax(1).float() / torch.full((T,), 127.0, device="cuda")
    s[1], s[T - 1] = float("nan"), float("inf")
    xs = torch.full((T * k + 1, d), 7, device="cuda", dtype=torch.int8)
    _, sc, gpos, goff = m.sort_tokens(x, idx, N, quantize=True, out=xs[:T * k])
    assert torch.equal(gpos, pos) and torch.equal(goff, off)
    want = torch.full_like(xs, 7)
    for j in range(k):
        there = pos[:, j] >= 0
        at = pos[there, j].long()
        want[at] = q[there]
        assert torch.equal(torch.nan_to_num(sc[at], nan=-1.0), torch.nan_to_num(s[there], nan=-1.0))
    assert torch.equal(xs, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out,N,r,k", [(1, 512, 264, 4, 8, 2), (4, 1024, 1032, 28, 8, 2), (40, 528, 776, 8, 16, 2),
                                                (300, 1040, 512, 28, 8, 1), (1100, 512, 1032, 28, 8, 2)])
def test_a_layer_on_an_8_bit_base(T, d_in, d_out, N, r, k, dtype):
    """The frozen base projection in 8 bits and the layer's own adapters on it: base_gemm_i8, gate_topk, lora_forward onto its output.
    Rounded: the base's scales and scalings (4 * 2^-24) and its output; s w h, in bf16 as the operand of the expand; fp32 sums over d_in and
    over the k r products; the sum of the two as the output."""
    g = gen(T + d_out)
    x = torch.randn((T, d_in), generator=g, device="cuda").to(dtype)
    W, wsc = m.quantize_rows(torch.randn((d_out, d_in), generator=g, device="cuda") * d_in ** -0.5)
    Wg = torch.randn((d_in, N), generator=g, device="cuda") * d_in ** -0.5
    A = (torch.randn((N, d_in, r), generator=g, device="cuda") * d_in ** -0.5).to(dtype)
    B = (torch.randn((N, r, d_out), generator=g, device="cuda") * r ** -0.5).to(dtype)
    out = m.base_gemm_i8(x, W, wsc)
    idx, w, _ = m.gate_topk(x, Wg, None, k)
    assert m.lora_forward(x, A, B, idx, w, 2.0, out=out, accumulate=True) is out
    q, _ = rows_ref(x.cpu())
    base = dense_ref(q, x.cpu().abs().amax(1).double() / 127, W.cpu(), wsc.cpu())
    xd, A, B, idx, w = x.cpu().double(), A.cpu().double(), B.cpu().double(), idx.cpu().long(), w.cpu().double()
    logits = xd @ Wg.cpu().double()
    top = logits.topk(k, 1).values[:, -1:]
    assert (logits.gather(1, idx) >= top - 1e-4).all()
    want, mag = base.clone(), torch.zeros_like(base)
    for j in range(k):
        for e in range(N):
            t = idx[:, j] == e
            want[t] += 2.0 * w[t, j, None] * ((xd[t] @ A[e]) @ B[e])
            mag[t] += 2.0 * w[t, j, None] * ((xd[t].abs() @ A[e].abs()) @ B[e].abs())
            if dtype == torch.bfloat16:
                half = 2.0 * w[t, j, None] * ((xd[t] @ A[e]).abs() @ B[e].abs())
                mag[t] += half * half_step(dtype) / ((d_in + k * r + 8) * U32)
    u = half_step(dtype) * 1.01
    tol = (u + 4 * U32) * base.abs() + 1.01 * (d_in + k * r + 8) * U32 * mag
    tol = tol + (u + U32) * (want.abs() + tol)
    assert ((out.cpu().double() - want).abs() <= tol).all()
