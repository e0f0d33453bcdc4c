"""The workspace of the gradient of a 4-bit projection in fp32: its size, and that no batch asks for more."""
import pytest
import torch

import paper_2405_13053_amd as m

P, WS = 0x100000, 0x200000          # aligned addresses that nothing reads before a launch
F32, WORKSPACE, HIP = 0, 3, 4


def test_fp32_asks_for_no_values_where_it_reads_the_codes():
    need = lambda d_in, d_out: m.base_gemm_mx4_backward_workspace_bytes(d_in, d_out, torch.float32)
    for d_in, d_out in ((4096, 14336), (14336, 4096), (5120, 13824), (131072, 200)):
        assert need(d_in, d_out) <= (32 << 20) + 256
    assert need(131072, 192) >= 131072 * 192 * 4 and need(64, 200) >= 64 * 200 * 4


@pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused must not reach a GPU: its addresses are made up")
@pytest.mark.parametrize("d_in,d_out", [(32, 8), (4096, 14336), (131072, 192), (131072, 200), (32, 1 << 20)])
def test_no_batch_needs_more_than_the_query_says(d_in, d_out):
    lib = m.load_library()
    most = m.base_gemm_mx4_backward_workspace_bytes(d_in, d_out, torch.float32) - 256
    for T in (1, 2, 33, 1000, 8192, 65536, 65537, 1 << 20, (1 << 24) - 1):
        if T * d_out < 1 << 33 and T * d_in < 1 << 36:
            assert lib.meteora_base_gemm_mx4_backward(P, P, P, T, d_in, d_out, F32, P, WS, most, None) == HIP, T
            assert lib.meteora_base_gemm_mx4_backward(P, P, P, T, d_in, d_out, F32, P, WS, most - 1, None) == WORKSPACE, T
