"""8-bit rows and products against plain fp64 on the CPU or GPU.

Tolerances.  Whole numbers are equal.  out = fl(fl(fl(sum) * q_scale) * w_scale): the sum is exact, so three roundings of 2^-24
each, and one of eps/2 where the output is bf16; base_gemm_i8's scale a / 127 is rounded once more."""
import pytest
import torch

import paper_2405_13053_amd as m
from tests import i8_kernels

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float32]


def half_step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def close(out, ref, roundings=3):
    """|out - ref| within `roundings` of fp32 and the output's own, element by element."""
    tol = (roundings * U32 + half_step(out.dtype)) * 1.001
    err = (out.double() - ref).abs()
    bad = err > tol * ref.abs()
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, worst {float((err / ref.abs().clamp_min(1e-300)).max()):.3e} > {tol:.3e}"


def rows_ref(x):
    """Definition: q = rne(127 x / a) of the exact quotient, in fp64 (exact to 2^-46; see the kernel), scale = a / 127 in fp32."""
    a = x.abs().amax(1, keepdim=True).double() if x.shape[1] else x.double()
    q = torch.round(x.double() * 127 / torch.where(a > 0, a, torch.ones_like(a)))
    return q.to(torch.int8), (a[:, 0].float() / 127)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def int8(shape, g, lo=-127, hi=128):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int8)


def scales(shape, g):
    return torch.rand(shape, generator=g, device="cuda") * 0.02 + 1e-3


# ---- quantize_rows -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 8), (3, 24), (5, 136), (64, 2048), (7, 2056), (2, 4104), (33, 5120), (4, 8200), (2, 16384),
                                    (3, 16392), (2, 40000), (513, 64)])
def test_quantize_rows(rows, d, dtype):
    g = gen(rows * 131 + d)
    x = torch.randn((rows, d), generator=g, device="cuda").to(dtype)
    x[:, 0] *= 9
    q, s = m.quantize_rows(x)
    rq, rs = rows_ref(x.cpu())
    assert torch.equal(q.cpu(), rq) and torch.equal(s.cpu(), rs)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_rows_rounds_the_exact_quotient(dtype):
    """Halves: every odd multiple of a / 254 that the type holds, for maxima of all mantissas; and what lies next to them."""
    g = gen(5)
    a = (torch.arange(128, 256, device="cuda").float() * 2.0 ** -7)[:, None]
    n = torch.arange(-127, 127, device="cuda").float()[None, :] + 0.5
    x = a * n / 127
    if dtype == torch.float32:   # any mantissa
        a = torch.rand((128, 1), generator=g, device="cuda") + 1
        x = (a.double() * n.double() / 127).float()
        x = torch.cat([x, torch.nextafter(x, x * 2), torch.nextafter(x, x * 0)], 1)
    else:
        x = x.to(dtype).float()
        x = torch.cat([x, x * (1 + 2.0 ** -7), x * (1 - 2.0 ** -7)], 1)
    x = torch.cat([a, a / 2, -a / 2, x.clamp(-a, a)], 1)
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % 8)).to(dtype).contiguous()
    q, s = m.quantize_rows(x)
    rq, rs = rows_ref(x.cpu())
    assert torch.equal(q.cpu(), rq) and torch.equal(s.cpu(), rs)
    assert (q[:, 1] == 64).all() and (q[:, 2] == -64).all()   # 63.5 goes to the even number


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_rows_of_zeros_and_of_the_smallest_and_largest(dtype):
    x = torch.zeros((6, 64), device="cuda", dtype=dtype)
    x[1, 5] = torch.finfo(dtype).max
    x[1, 6] = -torch.finfo(dtype).max / 2
    x[2, 0] = torch.finfo(dtype).tiny
    x[3, 63] = -1.0
    x[4, 7], x[4, 8] = 2.0 ** -120, -(2.0 ** -121)
    x[5, 1] = -0.0
    q, s = m.quantize_rows(x)
    rq, rs = rows_ref(x.cpu())
    assert torch.equal(q.cpu()[[0, 2, 3, 4, 5]], rq[[0, 2, 3, 4, 5]]) and torch.equal(s.cpu()[[0, 1, 3, 5]], rs[[0, 1, 3, 5]])
    assert q[1, 5] == 127


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [16, 512, 1024, 2048, 4096, 8192, 16384, 20480])
def test_infinities_and_nan_stay_visible_and_in_their_row(d, dtype):
    for T in (3, 9, 2100) if d <= 4096 else (3, 9):
        g = gen(d + T)
        x = torch.randn((T, d), generator=g, device="cuda").to(dtype)
        clean = m.quantize_rows(x)
        x[0, d - 1], x[1, 0], x[1, d // 2] = float("nan"), float("inf"), -float("inf")
        q, s = m.quantize_rows(x)
        assert torch.isnan(s[0]) and s[1] == float("inf") and not q[:2].any()
        assert torch.equal(q[2:], clean[0][2:]) and torch.equal(s[2:], clean[1][2:])
        idx = torch.zeros((T, 1), device="cuda", dtype=torch.int32)
        xs, xsc, _, _ = m.sort_tokens(x, idx, 1, quantize=True)
        assert torch.equal(xs, q) and torch.equal(xsc[1:], s[1:]) and torch.isnan(xsc[0])
        W, ws = m.quantize_rows(torch.randn((24, d), generator=g, device="cuda"))
        y = m.base_gemm_i8(x, W, ws)
        assert torch.isnan(y[:2]).all() and torch.equal(y[2:], m.gemm_i8(q, s, W, ws, dtype=dtype)[2:])
        assert torch.isfinite(y[2:]).all()
        one = m.base_gemm_i8(x[:1], W, ws)
        assert torch.isnan(one).all()


# ---- gemm_i8 -----------------------------------------------------------------------------------------------------------------
def dense_ref(q, qs, W, ws):
    return (q.double() @ W.double().t()) * qs.double()[:, None] * ws.double()


T_SMALL = [1, 2, 15, 16, 17, 33, 64, 65, 100, 128, 130, 257, 300]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_in,d_out", [(16, 8), (48, 24), (112, 64), (128, 136), (144, 72), (1024, 520), (1040, 264), (4096, 256),
                                        (2064, 1032)])
def test_dense(d_in, d_out, dtype):
    for T in T_SMALL:
        g = gen(T * 7919 + d_in + d_out)
        q, W = int8((T, d_in), g, -128), int8((d_out, d_in), g, -128)
        qs, ws = scales((T,), g), scales((d_out,), g)
        out = torch.full((T + 1, d_out), 7.0, device="cuda", dtype=dtype)
        m.gemm_i8(q, qs, W, ws, out=out[:T])
        close(out[:T], dense_ref(q, qs, W, ws))
        assert (out[T] == 7).all(), f"T={T}: written behind the last row"


@pytest.mark.parametrize("T,d_in,d_out", [(640, 4096, 4096), (1000, 1040, 2056), (2048, 4096, 1024), (4096, 512, 4096),
                                          (1531, 4096, 4096), (4097, 272, 4104), (700, 14336, 1024), (3000, 2048, 13824),
                                          (8192, 64, 1024), (5000, 4096, 64), (16384, 128, 264)])
def test_dense_large(T, d_in, d_out):
    g = gen(T + d_in)
    q, W = int8((T, d_in), g), int8((d_out, d_in), g)
    qs, ws = scales((T,), g), scales((d_out,), g)
    ref = dense_ref(q, qs, W, ws)
    for dtype in TYPES:
        close(m.gemm_i8(q, qs, W, ws, dtype=dtype), ref)


@pytest.mark.parametrize("T,d_in,d_out", [(4300, 4096, 4096), (4600, 4112, 4096), (5000, 4096, 4104), (6001, 4096, 4096), (9000, 2064, 4096),
                                          (1025, 4096, 16640), (20000, 512, 2040)])
def test_dense_with_a_last_round_of_few_tiles(T, d_in, d_out):
    """272, 288, 340, 384, 576, 325 and 632 tiles of 256 x 256: what lies behind whole rounds of 256 is done in smaller ones."""
    g = gen(T + d_in)
    q, W = int8((T, d_in), g), int8((d_out, d_in), g)
    qs, ws = scales((T,), g), scales((d_out,), g)
    ref = dense_ref(q, qs, W, ws)
    for dtype in TYPES:
        out = torch.full((T + 1, d_out), 7.0, device="cuda", dtype=dtype)
        m.gemm_i8(q, qs, W, ws, out=out[:T])
        close(out[:T], ref)
        assert (out[T] == 7).all()


@pytest.mark.parametrize("T,N,counts", [(4002, 8, [2624, 655, 291, 164, 105, 73, 53, 30]), (8192, 8, [5368, 1340, 595, 335, 214, 149, 100, 91]),
                                        (4300, 3, [4296, 0, 1]), (9001, 28, [300] * 28), (4096, 8, [512] * 8)])
def test_groups_with_a_last_round_of_few_tiles(T, N, counts):
    g = gen(T + N)
    d_in, d_out = 4096, 4096
    q, qs, W, ws, off = grouped_case(T, N, d_in, d_out, counts, g)
    out = torch.full((T, d_out), 7.0, device="cuda", dtype=torch.bfloat16)
    m.gemm_i8(q, qs, W, ws, offsets=off.cuda(), out=out)
    for e in range(N):
        a, b = int(off[e]), int(off[e + 1])
        close(out[a:b], dense_ref(q[a:b], qs[a:b], W[e], ws[e]))
    assert (out[int(off[-1]):] == 7).all()


@pytest.mark.parametrize("T", [1, 40, 300, 700])
def test_the_largest_sums(T):
    """131056 inputs of -128 on both sides add up to just below 2^31; of -128 and 127 to the other end."""
    K = 131056
    q = torch.full((T, K), -128, device="cuda", dtype=torch.int8)
    W = torch.full((264, K), -128, device="cuda", dtype=torch.int8)
    W[1::2] = 127
    one = torch.ones
    out = m.gemm_i8(q, one(T, device="cuda"), W, one(264, device="cuda"), dtype=torch.float32)
    sums = torch.tensor([K * 16384.0, -K * 127 * 128.0], device="cuda", dtype=torch.float64).repeat(132).expand(T, 264)
    close(out, sums, 1)


def grouped_case(T, N, d_in, d_out, counts, g):
    q, W = int8((T, d_in), g), int8((N, d_out, d_in), g)
    qs, ws = scales((T,), g), scales((N, d_out), g)
    off = torch.tensor([0] + counts, dtype=torch.int64).cumsum(0).to(torch.int32)
    return q, qs, W, ws, off


GROUPS = [
    (1, 1, [1]), (1, 4, [0, 0, 1, 0]), (5, 3, [0, 0, 0]), (40, 3, [13, 0, 27]), (64, 4, [16, 16, 16, 16]), (130, 5, [0, 1, 128, 1, 0]),
    (300, 7, [70, 0, 3, 64, 65, 40, 20]), (300, 2, [299, 0]), (700, 3, [257, 300, 143]), (1000, 64, [15] * 64),
    (2000, 28, [0] * 27 + [1999]), (1200, 2, [513, 600]), (4096, 8, [512] * 8), (2048, 3, [1100, 20, 900]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_in,d_out", [(64, 512), (528, 64), (1024, 8), (16, 1032), (1040, 776)])
@pytest.mark.parametrize("T,N,counts", GROUPS, ids=lambda v: str(v)[:20])
def test_groups(T, N, counts, d_in, d_out, dtype):
    g = gen(T + N + d_in)
    q, qs, W, ws, off = grouped_case(T, N, d_in, d_out, counts, g)
    out = torch.full((T, d_out), 7.0, device="cuda", dtype=dtype)
    m.gemm_i8(q, qs, W, ws, offsets=off.cuda(), out=out)
    for e in range(N):
        a, b = int(off[e]), int(off[e + 1])
        close(out[a:b], dense_ref(q[a:b], qs[a:b], W[e], ws[e]))
    assert (out[int(off[-1]):] == 7).all()   # rows of no group


@pytest.mark.parametrize("d_in,dtype", [(4096, torch.bfloat16), (4112, torch.float32)])
@pytest.mark.parametrize("T,counts", [(4002, [1389, 778, 367, 201, 134, 104, 73, 58]), (4002, [1500, 800, 300, 300, 100, 100, 100, 100]),
                                      (4050, [0, 1500, 513, 513, 513, 300, 257, 257]), (4200, [513] * 8), (4500, [4353, 0, 0, 0, 0, 0, 0, 1])],
                         ids=lambda v: str(v)[:20])
def test_tails_of_groups_of_every_size(T, counts, d_in, dtype):
    """17, 18, 21, 24 and 19 row tiles of 256: 16, 32, 80, 128 and 48 tiles of 256 x 256 behind the first 256."""
    g = gen(T + d_in)
    q, qs, W, ws, off = grouped_case(T, 8, d_in, 4096, counts, g)
    out = torch.full((T, 4096), 7.0, device="cuda", dtype=dtype)
    m.gemm_i8(q, qs, W, ws, offsets=off.cuda(), out=out)
    for e in range(8):
        a, b = int(off[e]), int(off[e + 1])
        close(out[a:b], dense_ref(q[a:b], qs[a:b], W[e], ws[e]))
    assert (out[int(off[-1]):] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,d_in,d_out,most", [(8, 4096, 4096, 24), (8, 4096, 4096, 60), (8, 4096, 4096, 120), (8, 4096, 4096, 190),
                                               (26, 1040, 4000, 64), (26, 1040, 4000, 130), (3, 6160, 5704, 100)])
def test_groups_whose_weights_are_past_the_caches(N, d_in, d_out, most, dtype):
    """Groups of one row tile, of several and of none beside each other; 134, 108 and 105 MB of weights."""
    g = gen(N + d_in + most)
    counts = [most - (e * 7) % most if e % 5 else (most * 2 + 3 if e % 2 else 0) for e in range(N)]
    T = sum(counts) + 3
    q, qs, W, ws, off = grouped_case(T, N, d_in, d_out, counts, g)
    out = torch.full((T, d_out), 7.0, device="cuda", dtype=dtype)
    m.gemm_i8(q, qs, W, ws, offsets=off.cuda(), out=out)
    for e in range(N):
        a, b = int(off[e]), int(off[e + 1])
        close(out[a:b], dense_ref(q[a:b], qs[a:b], W[e], ws[e]))
    assert (out[int(off[-1]):] == 7).all()


@pytest.mark.parametrize("T", [1, 20, 64, 90, 128, 200, 300])
def test_a_matrix_past_the_caches(T):
    g = gen(T)
    q, W = int8((T, 8208), g, -128), int8((12808, 8208), g, -128)
    qs, ws = scales((T,), g), scales((12808,), g)
    ref = dense_ref(q, qs, W, ws)
    for dtype in TYPES:
        close(m.gemm_i8(q, qs, W, ws, dtype=dtype), ref)


def test_offsets_outside_the_rows_write_nothing_outside():
    g = gen(3)
    q, qs, W, ws, _ = grouped_case(100, 4, 64, 64, [25] * 4, g)
    for bad in ([0, 50, 40, 200, 1 << 30], [-5, -1, 20, 100, 100], [2 ** 31 - 1] * 5, [-2 ** 31, 2 ** 31 - 1, 0, 3, 9]):
        buf = torch.full((300, 64), 7.0, device="cuda", dtype=torch.float32)
        m.gemm_i8(q, qs, W, ws, offsets=torch.tensor(bad, dtype=torch.int32, device="cuda"), out=buf[100:200])
        assert (buf[:100] == 7).all() and (buf[200:] == 7).all()


def test_operands_and_outputs_beyond_32_bit_offsets():
    g = gen(9)
    T, K, n = 270000, 16384, 64   # q: 4.4 GB
    q, W, qs, ws = int8((T, K), g), int8((n, K), g), scales((T,), g), scales((n,), g)
    out = m.gemm_i8(q, qs, W, ws, dtype=torch.float32)
    rows = torch.cat([torch.arange(0, T, 1777), torch.arange(T - 70, T)]).cuda()
    close(out[rows], dense_ref(q[rows], qs[rows], W, ws))
    N, n, K = 64, 8192, 8208      # W: 4.3 GB
    q, W, qs, ws = int8((200, K), g), int8((N, n, K), g), scales((200,), g), scales((N, n), g)
    off = torch.tensor([0] * 62 + [3, 90, 200], dtype=torch.int32)
    out = m.gemm_i8(q, qs, W, ws, offsets=off.cuda(), dtype=torch.float32)
    for e in (61, 62, 63):
        a, b = int(off[e]), int(off[e + 1])
        close(out[a:b], dense_ref(q[a:b], qs[a:b], W[e], ws[e]))
    T, K, n = 150000, 16, 16384   # out: 9.8 GB in fp32
    q, W, qs, ws = int8((T, K), g), int8((n, K), g), scales((T,), g), scales((n,), g)
    out = m.gemm_i8(q, qs, W, ws, dtype=torch.float32)
    rows = torch.cat([torch.arange(0, T, 3001), torch.arange(T - 70, T)]).cuda()
    close(out[rows], dense_ref(q[rows], qs[rows], W, ws))


# ---- base_gemm_i8 --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out", [(1, 4096, 4096), (1, 16, 8), (2, 5120, 520), (4, 4096, 1024), (7, 1040, 264), (16, 512, 512),
                                          (64, 4096, 4096), (65, 528, 1032), (300, 4096, 1024), (1000, 1024, 4096), (2, 16400, 64)])
def test_base_gemm_i8(T, d_in, d_out, dtype):
    g = gen(T + d_out)
    x = torch.randn((T, d_in), generator=g, device="cuda").to(dtype)
    W, ws = m.quantize_rows(torch.randn((d_out, d_in), generator=g, device="cuda"))
    ws_buf = torch.empty(m.base_gemm_i8_workspace_bytes(T + 3, d_in), dtype=torch.uint8, device="cuda")
    out = m.base_gemm_i8(x, W, ws, ws=ws_buf)
    q, _ = rows_ref(x)
    s = x.abs().amax(1).double() / 127
    close(out, dense_ref(q, s, W, ws), 4)
    again = m.base_gemm_i8(x, W, ws)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out", [(1, 16384, 24), (1, 4112, 5000), (1, 144, 4104), (2, 8192, 264), (2, 8176, 4120), (3, 5456, 40),
                                          (3, 48, 8200), (4, 4096, 8200), (4, 4080, 16), (4, 4112, 64), (5, 3264, 64), (1, 16400, 64)])
def test_base_gemm_i8_of_a_few_tokens(T, d_in, d_out, dtype):
    """Either side of what quantises inside the product, against the two calls, which it equals."""
    g = gen(T * 3 + d_in)
    x = torch.randn((T, d_in), generator=g, device="cuda").to(dtype)
    x[0, d_in - 1] = 7.0   # the largest in the last place
    W, ws = m.quantize_rows(torch.randn((d_out, d_in), generator=g, device="cuda"))
    out = torch.full((T + 1, d_out), 7.0, device="cuda", dtype=dtype)
    m.base_gemm_i8(x, W, ws, out=out[:T])
    q, s = m.quantize_rows(x)
    assert torch.equal(out[:T], m.gemm_i8(q, s, W, ws, dtype=dtype)) and (out[T] == 7).all()
    close(out[:T], dense_ref(q, x.abs().amax(1).double() / 127, W, ws), 4)


@pytest.mark.parametrize("T", [1, 4, 64, 500])
def test_base_gemm_i8_rows_of_zeros(T):
    x = torch.zeros((T, 256), device="cuda", dtype=torch.bfloat16)
    x[::2] = 1.0
    W, ws = m.quantize_rows(torch.randn((64, 256), device="cuda"))
    out = m.base_gemm_i8(x, W, ws)
    assert (out[1::2] == 0).all() and torch.isfinite(out).all()


def test_another_stream_and_a_graph_replayed_between_eager_calls():
    g = gen(11)
    for T, d_in, d_out in ((1, 4096, 1024), (64, 1024, 1024), (300, 1024, 512), (2048, 512, 2048)):
        x = torch.randn((T, d_in), generator=g, device="cuda").bfloat16()
        W, ws = m.quantize_rows(torch.randn((d_out, d_in), generator=g, device="cuda"))
        wsb = torch.empty(m.base_gemm_i8_workspace_bytes(T, d_in), dtype=torch.uint8, device="cuda")
        m.init()
        want = m.base_gemm_i8(x, W, ws)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = m.base_gemm_i8(x, W, ws, ws=wsb)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
        xin, out = x.clone(), torch.empty_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.base_gemm_i8(xin, W, ws, out=out, ws=wsb)
        for i in range(3):
            xin.copy_(torch.randn((T, d_in), generator=g, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, m.base_gemm_i8(xin, W, ws)), f"replay {i}"


def test_binding_checks():
    q, s = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    with pytest.raises(ValueError):
        m.gemm_i8(q, s, q[:, ::2], s)                      # not contiguous
    with pytest.raises(ValueError):
        m.gemm_i8(q, s[:3], q, s)
    with pytest.raises(TypeError):
        m.gemm_i8(q.float(), s, q, s)
    with pytest.raises(TypeError):
        m.gemm_i8(q, s, q, s, dtype=torch.float16)
    with pytest.raises(m.MeteoraError) as e:
        m.quantize_rows(torch.zeros((4, 12), device="cuda"))
    assert e.value.status == 2
    with pytest.raises(TypeError):
        m.quantize_rows(torch.zeros((4, 16), device="cuda", dtype=torch.float16))
    with pytest.raises(m.MeteoraError) as e:
        m.base_gemm_i8(torch.zeros((4, 64), device="cuda"), torch.zeros((8, 64), dtype=torch.int8, device="cuda"),
                       torch.zeros(8, device="cuda"), ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out", [(1, 64, 16), (33, 272, 528), (300, 1024, 1040), (1000, 528, 256)])
def test_gradient_of_the_rows(T, d_in, d_out, dtype):
    """dx = dy V with V[c,i] = w_scale[c] W[c,i], as an 8-bit product of dy and V^T quantised anew: each element of dy is off by half a step,
    a / 254, each of V by b / 254, and the product by what the two add up to.  Rounded beyond that: V and both scales (2^-24 each), the two
    scalings, and the output.  And as a bf16 product on V rounded to bf16: 2^-8 of each product, and fp32 sums."""
    g = gen(T + d_in)
    W, ws = m.quantize_rows(torch.randn((d_out, d_in), generator=g, device="cuda") * d_in ** -0.5)
    dy = torch.randn((T, d_out), generator=g, device="cuda").to(dtype)
    V = (W.float() * ws[:, None]).t().contiguous()      # [d_in, d_out]
    exact = dy.double() @ (W.double() * ws.double()[:, None])
    Vq, vs = m.quantize_rows(V)
    q, s = m.quantize_rows(dy)
    dx = m.gemm_i8(q, s, Vq, vs, dtype=dtype)
    a, b = dy.double().abs().amax(1)[:, None], V.double().abs().amax(1)[None, :]
    size = dy.double().abs() @ V.double().abs().t()
    off = (V.double().abs().sum(1)[None, :] * a + dy.double().abs().sum(1)[:, None] * b + d_out * a * b / 254) / 254
    tol = off * (1 + 8 * U32) + 8 * U32 * (size + off)
    tol = tol + half_step(dtype) * 1.001 * (exact.abs() + tol)
    assert ((dx.double() - exact).abs() <= tol).all()
    if dtype == torch.bfloat16:
        dx = m.base_gemm(dy, V.bfloat16())
        tol = (2.0 ** -8 * 1.001 + (d_out + 2) * U32) * size
        assert ((dx.double() - exact).abs() <= tol + half_step(dtype) * 1.001 * (exact.abs() + tol)).all()
    # against differences: the product is linear in its rows, and a row of the identity gives a column of V
    eye, es = m.quantize_rows(torch.eye(d_in, device="cuda")[:16].contiguous())
    col = m.gemm_i8(eye, es, W, ws, dtype=torch.float32)    # [16, d_out]: V's first rows
    assert ((col - V[:16]).abs() <= 4 * U32 * V[:16].abs()).all()
    part = dy.double() @ col.double().t()
    assert ((part - exact[:, :16]).abs() <= 5 * U32 * size[:, :16]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out,N", i8_kernels.PRODUCTS)
def test_every_kernel_of_the_product(T, d_in, d_out, N, dtype):
    """Sizes that lead to each tile shape and copy of its loop, dense and over groups, with whole K tiles and with a partial one."""
    g = gen(T + d_in + d_out)
    out = torch.full((T + 1, d_out), 7.0, device="cuda", dtype=dtype)
    if N is None:
        q, W = int8((T, d_in), g, -128), int8((d_out, d_in), g, -128)
        qs, ws = scales((T,), g), scales((d_out,), g)
        m.gemm_i8(q, qs, W, ws, out=out[:T])
        close(out[:T], dense_ref(q, qs, W, ws))
        assert (out[T] == 7).all()
        return
    counts = i8_kernels.deal(T, N)
    q, qs, W, ws, off = grouped_case(T, N, d_in, d_out, counts, g)
    m.gemm_i8(q, qs, W, ws, offsets=off.cuda(), out=out[:T])
    for e in range(N):
        a, b = int(off[e]), int(off[e + 1])
        close(out[a:b], dense_ref(q[a:b], qs[a:b], W[e], ws[e]))
    assert (out[int(off[-1]):] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d_in,d_out", [case for cases in i8_kernels.TAILS.values() for case in cases])
def test_tails_of_a_dense_product_at_their_borders(T, d_in, d_out, dtype):
    """1, 16, 17, 32, 33 and 128 tiles of 256 x 256 behind a whole round, which the largest tiles then leave to smaller ones."""
    g = gen(T + d_in)
    q, W = int8((T, d_in), g), int8((d_out, d_in), g)
    qs, ws = scales((T,), g), scales((d_out,), g)
    out = torch.full((T + 1, d_out), 7.0, device="cuda", dtype=dtype)
    m.gemm_i8(q, qs, W, ws, out=out[:T])
    close(out[:T], dense_ref(q, qs, W, ws))
    assert (out[T] == 7).all()
