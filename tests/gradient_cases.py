"""How far the gradient of a 4-bit projection may be off: dx = dy V, V the weight's values, in fp64.

Products of bf16 numbers and values of two bits are exact.  A row of fp32 numbers is three rows of bf16 numbers (two of 8 bits and the rest) that go through one sum, or
is taken as it is with a rounding to a product.  A matrix instruction adds 32 products in four additions at most, each off by at most 2^-23 of a partial
sum, and partial sums are about as large as the root of the sum of squares of the terms or as the result where that is larger (together: R).  Where the codes
themselves are read, a wavefront has every eighth 32 outputs; eight wavefronts and up to 32 parts are added.  So n additions are off by (n + 8 sqrt(n)) * 2^-23 * R, as if
all cuts went one way and 8 deviations of what goes either way; a product of fp32 numbers adds 2^-24 of its own, half a step of bf16 where dx is that.  Additions of zeros lose nothing: rows with few numbers in them have
as many additions as those have parts."""
import torch

U = 2.0 ** -23


def additions(d_out, dtype, codes, numbers=None):
    """codes: whether the codes themselves are read, or the values through a product of matrices of dx's type; numbers: in a row of dy, if few."""
    parts = 3 if dtype == torch.float32 else 1
    if numbers is not None:
        return parts * numbers
    if codes:
        return 4 * parts * -(-d_out // 256) + 8 + 32
    return d_out / 8 + 8 if dtype == torch.bfloat16 else d_out


def reference(dy, V, dtype, codes, numbers=None):
    """(dx, how far off an element may be)"""
    dy, V = dy.double(), V.contiguous()
    dx, R = dy @ V, ((dy * dy) @ (V * V)).sqrt()
    n = additions(dy.shape[1], dtype, codes, numbers)
    tol = (n + 8 * n ** 0.5 + 1) * U * (R + dx.abs())
    return dx, tol if dtype == torch.float32 else tol + 2.0 ** -8 * (dx.abs() + tol)


def misses(dx, ref):
    ref, tol = ref
    err = (dx.double() - ref).abs()
    return int((~(err <= tol * 1.001 + 1e-37)).sum()), float((err / tol.clamp_min(1e-300)).max())


def close(dx, ref):
    bad, worst = misses(dx, ref)
    assert bad == 0, f"{bad} of {tuple(dx.shape)}, worst {worst:.3f}"
