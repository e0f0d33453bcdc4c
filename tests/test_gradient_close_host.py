"""The bounds of tests/gradient_cases.py let a right gradient pass and none of these: nothing, outputs left out at the end, scales of a block one step off,
fp32 rows of two parts instead of three.  The gradients are made on the CPU in fp32, the mistakes in them."""
import pytest
import torch

from tests import gradient_cases as gc
from tests import mx4_cases as mx


def case(T, d_in, d_out, dtype):
    g = torch.Generator().manual_seed(T + d_in + d_out)
    q = torch.randint(0, 256, (d_out, d_in // 2), generator=g, dtype=torch.uint8)
    E = torch.randint(121, 133, (d_out, d_in // 32), generator=g, dtype=torch.uint8)
    return torch.randn((T, d_out), generator=g).to(dtype), mx.values(q, mx.place(E))


def parts(dy, n):
    """The first n parts of fp32 numbers, added: cut to 8 bits each time."""
    out, rest = torch.zeros_like(dy), dy.clone()
    for _ in range(n):
        top = (rest.view(torch.int32) & -65536).view(torch.float32)
        out, rest = out + top, rest - top
    return out


def fails(dx, ref, dtype):
    return gc.misses(dx.to(dtype), ref)[0] > 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d_in,d_out", [(3, 96, 520), (2, 64, 4096), (2, 64, 13824), (3, 32, 131072), (1, 32, 300000), (4, 32, 8)])
def test_mistakes_fail(T, d_in, d_out, dtype):
    dy, V = case(T, d_in, d_out, dtype)
    ref = gc.reference(dy, V, dtype, True)
    right = dy.float() @ V.float()
    assert gc.misses(right.to(dtype), ref)[0] == 0
    assert fails(torch.zeros_like(right), ref, dtype) and fails(right * 1.01, ref, dtype)
    if d_out <= 13824:   # of more, 8 are too little to be seen
        assert fails(right - dy[:, -8:].float() @ V[-8:].float(), ref, dtype)
    if dtype == torch.float32:
        assert fails(dy.bfloat16().float() @ V.float(), ref, dtype) and fails(parts(dy, 1) @ V.float(), ref, dtype)
    for numbers in (8, 1):
        last = dy.clone()
        last[:, :-numbers] = 0
        ref = gc.reference(last, V, dtype, True, numbers)
        right = last.float() @ V.float()
        assert gc.misses(right.to(dtype), ref)[0] == 0
        assert fails(right * 1.01, ref, dtype) and fails(right - last[:, -1:].float() @ V[-1:].float(), ref, dtype)
        if dtype == torch.float32:
            assert fails(parts(last, 2) @ V.float(), ref, dtype)
        W = V.clone()
        W[-1] *= 2
        assert fails(last.float() @ W.float(), ref, dtype)
