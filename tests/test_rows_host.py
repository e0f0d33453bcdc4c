"""Host-side checks of the 8-bit products and of the rows sorted by adapter: sizes, and refusals before any launch."""
import ctypes

import pytest

import paper_2405_13053_amd as m

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


def test_quantize_rows_refuses(lib):
    def call(x=P, rows=4, d=64, dt=BF16, q=P, scale=P):
        return lib.meteora_quantize_rows(x, rows, d, dt, q, scale, None)

    assert call(x=None) == INVALID and call(q=None) == INVALID and call(scale=None) == INVALID
    assert call(rows=-1) == INVALID and call(d=0) == INVALID
    assert call(dt=2) == UNSUPPORTED and call(dt=-1) == UNSUPPORTED
    assert call(d=12) == UNSUPPORTED and call(rows=1 << 24) == UNSUPPORTED
    assert call(x=ODD) == UNSUPPORTED and call(q=ODD) == UNSUPPORTED and call(scale=ODD) == UNSUPPORTED
    assert call(rows=0) == OK


def test_gemm_i8_refuses(lib):
    def call(q=P, qs=P, W=P, ws=P, off=P, T=64, di=64, do=64, N=4, dt=BF16, out=P):
        return lib.meteora_gemm_i8(q, qs, W, ws, off, T, di, do, N, dt, out, None)

    for name in ("q", "qs", "W", "ws", "out"):
        assert call(**{name: None}) == INVALID, name
        assert call(**{name: ODD}) == UNSUPPORTED, name
    assert call(off=None) == INVALID            # several matrices and no groups
    assert call(off=None, N=1, T=0) == OK
    assert call(off=ODDER) == UNSUPPORTED
    assert call(N=0) == INVALID and call(T=-1) == INVALID and call(di=0) == INVALID and call(do=0) == INVALID
    assert call(N=65) == UNSUPPORTED and call(dt=2) == UNSUPPORTED
    assert call(di=24) == UNSUPPORTED and call(di=131072) == UNSUPPORTED and call(do=12) == UNSUPPORTED
    assert call(do=(1 << 20) + 8) == UNSUPPORTED and call(T=1 << 24) == UNSUPPORTED
    assert call(T=1 << 23, do=1024) == UNSUPPORTED   # 2^33 outputs
    assert call(T=0) == OK and call(T=0, di=131056) == OK


def test_base_gemm_i8_refuses(lib):
    need = m.base_gemm_i8_workspace_bytes(64, 4096)
    assert need >= 64 * 4096 + 64 * 4
    assert m.base_gemm_i8_workspace_bytes(0, 64) > 0
    assert m.base_gemm_i8_workspace_bytes(64, 4104) == 0 and m.base_gemm_i8_workspace_bytes(-1, 64) == 0
    assert m.base_gemm_i8_workspace_bytes(64, 131072) == 0 and m.base_gemm_i8_workspace_bytes(1 << 24, 64) == 0

    def call(x=P, W=P, sc=P, T=64, di=64, do=64, dt=BF16, out=P, ws=WS, wsb=BIG):
        return lib.meteora_base_gemm_i8(x, W, sc, T, di, do, dt, out, ws, wsb, None)

    for name in ("x", "W", "sc", "out"):
        assert call(**{name: None}) == INVALID, name
        assert call(**{name: ODD}) == UNSUPPORTED, name
    assert call(T=-1) == INVALID and call(dt=2) == UNSUPPORTED and call(di=8) == UNSUPPORTED and call(do=4) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(ws=ODD) == WORKSPACE and call(wsb=64 * 64) == WORKSPACE
    assert call(T=0) == OK and call(T=0, wsb=0) == OK


def test_sort_tokens_refuses(lib):
    def call(x=P, idx=P, T=64, k=2, N=4, d=64, dt=BF16, xs=P, xsc=None, pos=P, off=P, ws=WS, wsb=BIG):
        return lib.meteora_sort_tokens(x, idx, T, k, N, d, dt, xs, xsc, pos, off, ws, wsb, None)

    for name in ("x", "idx", "xs", "pos", "off"):
        assert call(**{name: None}) == INVALID, name
    for name in ("x", "xs"):
        assert call(**{name: ODD}) == UNSUPPORTED, name
    for name in ("idx", "xsc", "pos", "off"):
        assert call(**{name: ODDER}) == UNSUPPORTED, name
    assert call(T=-1) == INVALID and call(k=0) == INVALID and call(N=0) == INVALID and call(d=0) == INVALID
    assert call(k=9) == UNSUPPORTED and call(N=65) == UNSUPPORTED and call(d=12) == UNSUPPORTED and call(dt=2) == UNSUPPORTED
    assert call(T=1 << 24) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(ws=ODD) == WORKSPACE and call(wsb=16) == WORKSPACE
    assert call(T=0) == OK and call(T=0, k=8, N=4, wsb=0) == OK
    assert m.sort_workspace_bytes(64, 9, 4) == 0 and m.sort_workspace_bytes(64, 2, 65) == 0
    assert m.sort_workspace_bytes(-1, 2, 4) == 0 and m.sort_workspace_bytes(1 << 24, 2, 4) == 0


@pytest.mark.parametrize("k,N", [(1, 1), (1, 64), (2, 28), (8, 64), (7, 5)])
def test_a_sort_workspace_for_more_tokens_holds_fewer(k, N):
    sizes = [m.sort_workspace_bytes(T, k, N) for T in [*range(0, 4500), *range(4500, 300000, 777), (1 << 24) - 1]]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_unsort_refuses(lib):
    def fwd(ys=P, rows=128, pos=P, w=P, T=64, k=2, d=64, s=1.0, dt=BF16, base=None, out=P):
        return lib.meteora_unsort_tokens(ys, rows, pos, w, T, k, d, s, dt, base, out, None)

    def bwd(dy=P, ys=P, rows=128, pos=P, w=P, T=64, k=2, d=64, s=1.0, dt=BF16, dys=P, dw=P):
        return lib.meteora_unsort_backward(dy, ys, rows, pos, w, T, k, d, s, dt, dys, dw, None)

    for f in (fwd, bwd):
        assert f(ys=None) == INVALID and f(pos=None) == INVALID and f(T=-1) == INVALID and f(rows=-1) == INVALID
        assert f(k=0) == INVALID and f(d=0) == INVALID and f(s=float("nan")) == INVALID and f(s=float("inf")) == INVALID
        assert f(k=9) == UNSUPPORTED and f(d=12) == UNSUPPORTED and f(dt=2) == UNSUPPORTED
        assert f(T=1 << 24) == UNSUPPORTED and f(rows=1 << 31) == UNSUPPORTED
        assert f(ys=ODD) == UNSUPPORTED and f(pos=ODDER) == UNSUPPORTED and f(w=ODDER) == UNSUPPORTED
        assert f(T=0) == OK and f(T=0, w=None) == OK and f(T=0, rows=0) == OK
    assert fwd(out=None) == INVALID and fwd(out=ODD) == UNSUPPORTED and fwd(base=ODD) == UNSUPPORTED
    assert bwd(dy=None) == INVALID and bwd(dys=None) == INVALID and bwd(dy=ODD) == UNSUPPORTED and bwd(dys=ODD) == UNSUPPORTED
    assert bwd(dw=ODDER) == UNSUPPORTED and bwd(ys=None, dw=None, T=0) == OK


def test_binding_refuses_host_tensors():
    import torch
    x, q, s = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    idx = torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: m.quantize_rows(x), lambda: m.gemm_i8(q, s, q, s), lambda: m.base_gemm_i8(x, q, s),
                 lambda: m.sort_tokens(x, idx, 4), lambda: m.unsort_tokens(x, idx), lambda: m.unsort_backward(x, x, idx)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        m.gemm_i8(q, s, q[None], s[None])        # one matrix per group and no groups
