"""The bounds of tests/experts_cases.py let a right result pass and none of these: nothing, inputs or channels left out at the end of a row, weights that
are a percent wrong (a tenth where there is little else to see), h in three bits less.  The results are made on the CPU in fp32, the mistakes in them."""
import pytest
import torch

from tests import experts_cases as ex

BF = torch.bfloat16


def layer(N, d, f, g):
    return ((torch.randn((N, *shape), generator=g) * shape[1] ** -0.5).to(BF) for shape in ((2 * f, d), (d, f)))


def result(x, idx, w, W1, W2, inputs=None, channels=None, factor=1.0, bits=8):
    """inputs, channels: those that take part, the first ones; bits: of h."""
    f = W2.shape[2]
    out = torch.zeros(x.shape)
    for t, j in ((t, j) for t in range(x.shape[0]) for j in range(idx.shape[1])):
        e = int(idx[t, j])
        both = W1[e, :, :inputs].float() @ x[t, :inputs].float()
        h = both[:f] / (1 + torch.exp(-both[:f])) * both[f:]
        m, at = torch.frexp(h)
        h = torch.ldexp(torch.round(m * 2.0 ** bits) * 2.0 ** -bits, at)
        out[t] += factor * w[t, j] * (W2[e, :, :channels].float() @ h[:channels])
    return out.to(BF)


def case(T, N, k, d, f):
    g = torch.Generator().manual_seed(T + d + f)
    W1, W2 = layer(N, d, f, g)
    x = torch.randn((T, d), generator=g).to(BF)
    idx = torch.topk(torch.rand((T, N), generator=g), k, 1).indices
    return x, idx, torch.softmax(torch.randn((T, k), generator=g), 1), W1, W2


def fails(operands, ref, **mistake):
    return ex.misses(result(*operands, **mistake), ref)[0] > 0


@pytest.mark.parametrize("T,N,k,d,f", [(1, 8, 2, 512, 256), (3, 2, 2, 4096, 512), (1, 7, 4, 992, 4000), (1, 2, 2, 2048, 16384), (3, 5, 2, 1000, 72),
                                       (8, 3, 2, 96, 4128)])
def test_mistakes_fail(T, N, k, d, f):
    operands = case(T, N, k, d, f)
    ref = ex.reference(*operands[:3], *(W.double() for W in operands[3:]))
    assert ex.misses(result(*operands), ref)[0] == 0
    for mistake in (dict(factor=0.0), dict(factor=1.01), dict(inputs=d - 8), dict(channels=f - 8)):
        assert fails(operands, ref, **mistake), mistake
    if f >= 256:
        assert fails(operands, ref, bits=5)


@pytest.mark.parametrize("d,f", [(131072, 8), (131072, 32), (8192, 96)])
def test_mistakes_of_long_rows_fail(d, f):
    """8 of 131072 inputs are too little of a sum to be seen in it, so that the rows that the GPU's tests take have nothing else."""
    operands = case(2, 3, 2, d, f)
    ref = ex.reference(*operands[:3], *(W.double() for W in operands[3:]))
    assert ex.misses(result(*operands), ref)[0] == 0
    assert fails(operands, ref, factor=0.0) and fails(operands, ref, channels=f - 8)
    operands[0][:, :-8] = 0
    ref = ex.reference(*operands[:3], *(W.double() for W in operands[3:]))
    assert ex.misses(result(*operands), ref)[0] == 0
    for mistake in (dict(inputs=d - 8), dict(inputs=d - 1), dict(factor=0.9), dict(channels=f - 8)):
        assert fails(operands, ref, **mistake), mistake


@pytest.mark.parametrize("d,f", [(8, 131072), (32, 131072), (96, 16384)])
def test_mistakes_of_many_channels_fail(d, f):
    operands = case(2, 3, 2, d, f)
    ref = ex.reference(*operands[:3], *(W.double() for W in operands[3:]))
    assert ex.misses(result(*operands), ref)[0] == 0
    assert fails(operands, ref, factor=0.0) and fails(operands, ref, inputs=d - 4)
    operands[3][:, torch.arange(2 * f) % f < f - 8] = 0
    ref = ex.reference(*operands[:3], *(W.double() for W in operands[3:]))
    assert ex.misses(result(*operands), ref)[0] == 0
    for mistake in (dict(channels=f - 8), dict(channels=f - 1), dict(factor=0.9), dict(inputs=d - 4)):
        assert fails(operands, ref, **mistake), mistake
