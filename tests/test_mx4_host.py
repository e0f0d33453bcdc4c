"""Host-side checks of the 4-bit rows and products and of the experts: sizes, the kernels that sizes lead to, and refusals before any launch."""
import ctypes
import math
import random

import pytest
import torch

import paper_2405_13053_amd as m
from tests.i8_kernels import deal
from tests.mx4_kernels import PRODUCTS, code_of

OK, INVALID, UNSUPPORTED, WORKSPACE, HIP = range(5)
F32, BF16 = 0, 1
P = ctypes.c_void_p(0x10000)       # aligned, never read
ODD = ctypes.c_void_p(0x10008)     # not aligned to 16
ODDER = ctypes.c_void_p(0x10002)   # not aligned to 4
WS = ctypes.c_void_p(0x100000)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return m.load_library()


def test_scale_bytes(lib):
    size = lib.meteora_mx4_scale_bytes
    for rows, d in ((1, 32), (3, 512), (7, 544), (64, 4096), (5, 131072)):
        a, b, c = m.mx4_scale_shape(rows, d)
        assert size(rows, d) == a * b * c == -(-d // 512) * rows * 16
    assert size(0, 64) == 0 and size(-1, 64) == 0 and size(4, 0) == 0 and size(4, 48) == 0 and size(4, 131072 + 32) == 0
    assert size(1 << 24, 32) == 0 and size((1 << 24) - 1, 32) > 0 and size(1 << 20, 65536) == 0   # 2^36 values


def test_rows_refuse(lib):
    def quantize(x=P, rows=8, d=64, dt=BF16, q=P, s=P, out=None):
        return lib.meteora_quantize_mx4(x, rows, d, dt, q, s, None)

    def back(x=None, rows=8, d=64, dt=BF16, q=P, s=P, out=P, turn=0):
        return lib.meteora_dequantize_mx4(q, s, rows, d, dt, turn, out, None)

    for f, names in ((quantize, ("x", "q", "s")), (back, ("q", "s", "out"))):
        for name in names:
            assert f(**{name: None}) == INVALID and f(**{name: ODD}) == UNSUPPORTED, name
        assert f(rows=-1) == INVALID and f(d=0) == INVALID and f(d=-32) == INVALID
        assert f(dt=2) == UNSUPPORTED and f(dt=-1) == UNSUPPORTED and f(d=48) == UNSUPPORTED and f(d=131072 + 32) == UNSUPPORTED
        assert f(rows=1 << 24) == UNSUPPORTED and f(rows=1 << 20, d=65536) == UNSUPPORTED
        assert f(rows=0) == OK
    assert back(rows=12, turn=1) == UNSUPPORTED and back(rows=0, turn=1) == OK


def test_gemm_mx4_refuses(lib):
    def call(q=P, qs=P, W=P, ws=P, off=P, T=64, di=64, do=64, N=4, dt=BF16, out=P):
        return lib.meteora_gemm_mx4(q, qs, W, ws, off, T, di, do, N, dt, out, None)

    for name in ("q", "qs", "W", "ws", "out"):
        assert call(**{name: None}) == INVALID, name
        assert call(**{name: ODD}) == UNSUPPORTED, name
    assert call(off=None) == INVALID            # several matrices and no groups
    assert call(off=None, N=1, T=0) == OK
    assert call(off=ODDER) == UNSUPPORTED
    assert call(N=0) == INVALID and call(T=-1) == INVALID and call(di=0) == INVALID and call(do=0) == INVALID
    assert call(N=65) == UNSUPPORTED and call(dt=2) == UNSUPPORTED
    assert call(di=48) == UNSUPPORTED and call(di=131072 + 32) == UNSUPPORTED and call(do=12) == UNSUPPORTED
    assert call(do=(1 << 20) + 8) == UNSUPPORTED and call(T=1 << 24) == UNSUPPORTED
    assert call(T=1 << 23, do=1024) == UNSUPPORTED   # 2^33 outputs
    assert call(T=0) == OK and call(T=0, di=131072) == OK


def test_base_gemm_mx4_and_its_gradient_refuse(lib):
    need = m.base_gemm_mx4_workspace_bytes(64, 4096)
    assert need >= 64 * 2048 + 64 * 128 and m.base_gemm_mx4_workspace_bytes(0, 64) > 0
    assert m.base_gemm_mx4_workspace_bytes(64, 4112) == 0 and m.base_gemm_mx4_workspace_bytes(-1, 64) == 0
    assert m.base_gemm_mx4_workspace_bytes(64, 131072 + 32) == 0 and m.base_gemm_mx4_workspace_bytes(1 << 24, 64) == 0
    back = m.base_gemm_mx4_backward_workspace_bytes
    assert back(64, 128, "bf16") >= 64 * 128 * 2 and back(64, 128, F32) >= 64 * 128 * 4
    assert back(48, 128, "bf16") == 0 and back(64, 12, "bf16") == 0 and back(0, 64, "bf16") == 0
    assert lib.meteora_base_gemm_mx4_backward_workspace_bytes(64, 64, 2) == 0

    def fwd(x=P, W=P, sc=P, T=64, di=64, do=64, dt=BF16, out=P, ws=WS, wsb=BIG):
        return lib.meteora_base_gemm_mx4(x, W, sc, T, di, do, dt, out, ws, wsb, None)

    def bwd(x=P, W=P, sc=P, T=64, di=64, do=64, dt=BF16, out=P, ws=WS, wsb=BIG):
        return lib.meteora_base_gemm_mx4_backward(x, W, sc, T, di, do, dt, out, ws, wsb, None)

    for call in (fwd, bwd):
        for name in ("x", "W", "sc", "out"):
            assert call(**{name: None}) == INVALID, name
            assert call(**{name: ODD}) == UNSUPPORTED, name
        assert call(T=-1) == INVALID and call(dt=2) == UNSUPPORTED and call(di=16) == UNSUPPORTED and call(do=4) == UNSUPPORTED
        assert call(ws=None) == WORKSPACE and call(ws=ODD) == WORKSPACE and call(wsb=64 * 32) == WORKSPACE
        assert call(T=0) == OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused must not reach a GPU: its addresses are made up")
@pytest.mark.parametrize("di,do", [(32, 8), (4096, 14336), (14336, 4096), (672, 12336), (1024, 131072), (96, 1 << 20), (64, 8192)])
def test_no_batch_needs_more_than_the_query_of_the_gradient_says(lib, di, do):
    most = m.base_gemm_mx4_backward_workspace_bytes(di, do, "bf16") - 256
    for T in [*range(1, 200), *range(200, 3000, 97), 5000, 100000]:
        if T * do < 1 << 33:
            assert lib.meteora_base_gemm_mx4_backward(P, P, P, T, di, do, BF16, P, WS, most, None) == HIP, T
    assert lib.meteora_base_gemm_mx4_backward(P, P, P, 1, di, do, BF16, P, WS, 2 * di * do - 1, None) == WORKSPACE


def test_experts_refuse(lib):
    size = m.experts_workspace_bytes
    assert size(64, 4096, 14336, 8, 2) > 0 and size(0, 64, 64, 4, 2) > 0
    for bad in ((65, 64, 64, 4, 2), (-1, 64, 64, 4, 2), (4, 60, 64, 4, 2), (4, 64, 60, 4, 2), (4, 64, 64, 65, 2), (4, 64, 64, 4, 9), (4, 64, 64, 0, 2),
                (4, 64, 64, 4, 0), (4, 131080, 64, 4, 2), (4, 64, 131080, 4, 2)):
        assert size(*bad) == 0, bad
    for d, f, N, k in ((64, 64, 4, 2), (4096, 512, 64, 8), (131072, 8, 1, 1)):
        sizes = [size(T, d, f, N, k) for T in range(65)]
        assert sizes == sorted(sizes)

    def experts(x=P, idx=P, w=P, W1=P, s1=P, W2=P, s2=P, T=8, d=64, f=96, N=4, k=2, scale=1.0, dt=BF16, base=None, out=P, ws=WS, wsb=BIG):
        return lib.meteora_experts_forward(x, idx, w, W1, s1, W2, s2, T, d, f, N, k, scale, dt, base, out, ws, wsb, None)

    def moe(x=P, idx=P, w=P, W1=P, s1=P, W2=P, s2=P, T=8, d=64, f=96, N=4, k=2, scale=1.0, dt=BF16, base=None, out=P, ws=WS, wsb=BIG, Wg=P, bias=None,
            inv=1.0, io=None, wo=None):
        return lib.meteora_moe_forward(x, Wg, bias, W1, s1, W2, s2, T, d, f, N, k, scale, inv, dt, base, out, io, wo, ws, wsb, None)

    for call in (experts, moe):
        for name in ("x", "W1", "W2", "out"):
            assert call(**{name: None}) == INVALID, name
            assert call(**{name: ODD}) == UNSUPPORTED, name
        assert call(s1=None) == INVALID and call(s2=None) == INVALID      # one of the two in 4 bits
        assert call(s1=ODD) == UNSUPPORTED and call(base=ODD) == UNSUPPORTED
        assert call(scale=float("nan")) == INVALID and call(scale=float("inf")) == INVALID
        assert call(T=-1) == INVALID and call(d=0) == INVALID and call(f=0) == INVALID and call(N=0) == INVALID and call(k=0) == INVALID
        assert call(T=65) == UNSUPPORTED and call(N=65) == UNSUPPORTED and call(dt=F32) == UNSUPPORTED and call(dt=2) == UNSUPPORTED
        assert call(d=40) == UNSUPPORTED and call(f=40) == UNSUPPORTED    # blocks of 32
        assert call(d=40, f=72, s1=None, s2=None, T=0) == OK              # bf16: whole eights
        assert call(d=36, s1=None, s2=None) == UNSUPPORTED
        assert call(ws=None) == WORKSPACE and call(ws=ODD) == WORKSPACE and call(wsb=64) == WORKSPACE
        assert call(T=0) == OK
    assert experts(k=9) == UNSUPPORTED and experts(idx=None) == INVALID and experts(w=None) == INVALID
    assert experts(idx=ODDER) == UNSUPPORTED and experts(w=ODDER) == UNSUPPORTED and experts(k=8, T=0) == OK
    assert moe(Wg=None) == INVALID and moe(Wg=ODD) == UNSUPPORTED and moe(bias=ODDER) == UNSUPPORTED and moe(k=5) == INVALID
    assert moe(inv=float("nan")) == INVALID and moe(io=ODDER) == UNSUPPORTED and moe(wo=ODDER) == UNSUPPORTED


def test_every_kernel_that_sizes_lead_to_is_covered():
    """The products of tests.mx4_kernels reach every kernel, and every copy of its loop, that gemm_mx4 starts for any size."""
    code = lambda T, half, d_out, N: code_of(T, half, d_out, None if N is None else deal(T, N))
    covered = set().union(*(code(*case) for case in PRODUCTS))
    rng, seen = random.Random(7), {}
    spread = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    for _ in range(400000):
        T, half, d_out, N = spread(1, 12000), 16 * spread(9, 900), 8 * spread(1, 2000), rng.choice([None, 2, 3, 5, 8])
        if rng.random() < 0.5:
            half = max(half // 128, 2) * 128
        if T * d_out <= 2e8 and (rng.random() < 0.5 or half * d_out * (N or 1) >= 1e8):
            for c in code(T, half, d_out, N):
                seen.setdefault(c, (T, half, d_out, N))
    missing = {c: case for c, case in seen.items() if c not in covered}
    assert not missing, missing
    assert len(covered) >= 100 and len({c[:4] for c in covered}) == 13   # tile shapes


def test_up_to_256_inputs_take_one_kernel():
    for d_in in range(32, 257, 32):
        for T in (1, 64, 5000):
            assert m.gemm_mx4_kernel(T, d_in, 4096)[0] == m.gemm_mx4_kernel(T, d_in, 4096, 28)[0] == "one"


def test_the_query_refuses_what_the_product_refuses():
    for args in ((0, 64, 64), (64, 48, 64), (64, 64, 12), (1 << 24, 64, 64), (64, 131072 + 32, 64), (64, 64, (1 << 20) + 8), (1 << 23, 64, 1024),
                 (64, 64, 64, 65), (64, 64, 64, 0), (-1, 64, 64), (64, 0, 64)):
        assert m.gemm_mx4_kernel(*args) is None, args
    lib = m.load_library()
    assert lib.meteora_gemm_mx4_kernel(64, 512, 64, 2, 0, *[None] * 6) == -1     # several matrices and no groups
    assert lib.meteora_gemm_mx4_kernel(64, 512, 64, 2, 1, *[None] * 6) == 0


def test_binding_refuses_host_tensors():
    x, q, s = torch.zeros(8, 64), torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(1, 8, 16, dtype=torch.uint8)
    idx, w = torch.zeros(8, 2, dtype=torch.int32), torch.zeros(8, 2)
    W1, W2 = torch.zeros(4, 128, 64), torch.zeros(4, 64, 64)
    for call in (lambda: m.quantize_mx4(x), lambda: m.dequantize_mx4(q, s), lambda: m.gemm_mx4(q, s, q, s), lambda: m.base_gemm_mx4(x, q, s),
                 lambda: m.base_gemm_mx4_backward(x, q, s), lambda: m.experts_forward(x, idx, w, W1, W2),
                 lambda: m.moe_forward(x, torch.zeros(64, 4), None, W1, W2, 2), lambda: m.gemm_mx4(q, s, q[None], s[None]),
                 lambda: m.experts_forward(x, idx, w, W1, W2, w1_scale=s)):
        with pytest.raises(ValueError):
            call()
