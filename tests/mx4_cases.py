"""The 4-bit format in fp64, written from its definition, and the sizes of products that reach every kernel."""
import torch

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def place(E):
    """E[rows, blocks] in the operators' order: [chunk of 16 blocks][row][(b % 4) * 4 + b % 16 / 4]."""
    rows, blocks = E.shape
    out = torch.zeros(((blocks + 15) // 16, rows, 16), dtype=torch.uint8, device=E.device)
    for b in range(blocks):
        out[b // 16, :, (b % 4) * 4 + b % 16 // 4] = E[:, b]
    return out


def quantize(x):
    """(q, scale) by looking for the nearest value, of two as near the one with the even code."""
    rows, d = x.shape
    b = x.double().view(rows, d // 32, 32)
    top = b.abs().amax(2)
    finite = torch.isfinite(top)
    _, e = torch.frexp(torch.where(finite & (top > 0), top, torch.ones_like(top)))
    E = torch.where(top > 0, (e - 1 - 2 + 127).clamp_min(0), torch.zeros_like(e))
    E = torch.where(finite, E, torch.full_like(E, 255))
    t = torch.where(finite[..., None], b, torch.zeros_like(b)) / torch.exp2(torch.where(finite, E, 0).double() - 127)[..., None]
    code, best = torch.zeros_like(t, dtype=torch.int64), torch.full_like(t, 1e300)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):
        away = (t.abs() - VALUES[c]).abs()
        code = torch.where(away < best, c, code)
        best = torch.minimum(best, away)
    code = (code + 8 * (torch.signbit(t) & finite[..., None])).view(rows, d)
    return (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8), place(E.to(torch.uint8))


def values(q, scale):
    rows, half = q.shape
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float64, device=q.device)
    v = torch.empty((rows, half * 2), dtype=torch.float64, device=q.device)
    v[:, 0::2], v[:, 1::2] = table[(q & 15).long()], table[(q >> 4).long()]
    for b in range(half // 16):
        E = scale[b // 16, :, (b % 4) * 4 + b % 16 // 4].double()
        v[:, b * 32:(b + 1) * 32] *= torch.where(E == 255, float("nan"), torch.exp2(E - 127))[:, None]
    return v


def product(a, b):
    return torch.matmul(a, b.t().contiguous())


# T, d_in, d_out: one token to many, K tiles and chunks that end in parts, rows and columns past the last tile
DENSE = [(1, 32, 8), (3, 64, 40), (65, 256, 264), (200, 224, 136), (16, 288, 16), (1, 512, 64), (5, 544, 72), (16, 4096, 4096), (1, 4128, 96),
         (33, 2080, 5120), (64, 5120, 1376), (7, 131072, 24), (100, 1056, 1000), (130, 2048, 776), (257, 4096, 1032), (300, 4096, 4096),
         (513, 1312, 4096), (700, 1024, 6144), (1000, 608, 4104), (1100, 4096, 4096), (1531, 2080, 4096), (2000, 768, 4096), (2100, 4096, 8192),
         (3000, 544, 5128), (4300, 1024, 4096), (4600, 800, 4096), (5000, 4096, 4104), (4096, 512, 4096), (8200, 288, 2048)]
# T, d_in, d_out, N
GROUPED = [(1, 64, 16, 4), (16, 288, 72, 3), (64, 4096, 512, 8), (300, 544, 264, 7), (777, 1024, 1032, 4), (2001, 2048, 1376, 8), (64, 256, 4096, 28),
           (5, 1056, 40, 64), (4002, 800, 4096, 8), (500, 16384, 1544, 8)]
