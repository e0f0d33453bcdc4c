"""What the experts' operators return, in fp64 with h rounded to bf16 as the definition has it, and how far off an element may be.

Operands are random, so what n additions lose is counted from the partial sums that there are, not from the sum of magnitudes: those are about as large
as the root of the sum of squares of the terms, or as the result where that is larger (together: R).  A matrix instruction adds 32 products in four
additions at most, each cut or rounded, 2^-23 of a partial sum at most: n / 8 * 2^-23 * R if all cuts went one way, and 8 sqrt(n) * 2^-23 * R (8
deviations) for what goes either way, which also covers the few additions of wavefronts and parts.  silu has a slope of at most 1.1 and |silu(g)| <= |g|;
exp, quotient and products are 8 * 2^-24 of h.  So h is known to dh, and its rounding to bf16 where both h - dh and h + dh round to one number; an h in whose
dh there is a border may be either neighbour, which reaches the output as the root of the sum of squares of these steps, 8 deviations.  The weighted sum
of k experts and the base: k + 2 roundings; the output half a step.  Over a token's d channels the steps of h reach the norm of the error as the norm of those
roots, with 8 deviations of a mean over d (1 + 8 / sqrt(2 d)), and everything else as its norm at most."""
import torch

U = 2.0 ** -23


def lost(n):
    """Of R by a sum of n products."""
    return (n / 8 + 8 * n ** 0.5) * U


def dots(a, V):
    """(a V^T, R)"""
    y, squares = a @ V.t().contiguous(), (a * a) @ (V * V).t().contiguous()
    return y, squares.sqrt() + y.abs()


def rounded(h):
    return h.to(torch.bfloat16).double()


def reference(x, idx, w, V1, V2, scale=1.0, base=None):
    """(out, how far off an element may be, how far a token's row in its norm); V1[e], V2[e] in fp64."""
    T, k = idx.shape
    x, f, d = x.double(), V2[0].shape[1], V2[0].shape[0]
    out, sums, size, steps = (torch.zeros((T, d), dtype=torch.float64, device=x.device) for _ in range(4))
    for e in range(len(V1)):
        here = idx == e
        rows = here.any(1).nonzero().flatten()
        if rows.numel() == 0:
            continue
        share, most = (w.double() * here).sum(1)[rows, None], (w.double().abs() * here).sum(1)[rows, None]
        both, R = dots(x[rows], V1[e])
        off = lost(d) * R
        g, u, dg, du = both[:, :f], both[:, f:], off[:, :f], off[:, f:]
        h = g / (1 + torch.exp(-g)) * u
        dh = 1.1 * dg * u.abs() + g.abs() * du + 1.1 * dg * du + 8 * 2.0 ** -24 * h.abs()
        mid = rounded(h)
        step = torch.maximum((rounded(h + dh) - mid).abs(), (mid - rounded(h - dh)).abs())
        y, R = dots(mid, V2[e])
        out[rows] += share * y
        sums[rows] += most * lost(f) * R
        steps[rows] += most * ((step * step) @ (V2[e] * V2[e]).t().contiguous()).sqrt()
        size[rows] += most * R
    out, sums, size, steps = scale * out, abs(scale) * sums, abs(scale) * size, abs(scale) * steps
    if base is not None:
        out, size = out + base.double(), size + base.double().abs()
    sums = sums + (k + 2) * U * size
    tol = sums + 8 * steps
    norm = (sums + 2.0 ** -8 * (out.abs() + sums)).norm(dim=1) + (1 + 2.0 ** -8) * (1 + 8 / (2 * d) ** 0.5) * steps.norm(dim=1)
    return out, tol + 2.0 ** -8 * (out.abs() + tol), norm


def misses(out, ref):
    """Elements and rows that are further off than they may be, and how far the worst of either is in units of what it may be."""
    ref, tol, norm = ref
    err = (out.double() - ref).abs()
    far = err.norm(dim=1)
    return (int((~(err <= tol * 1.001)).sum() + (~(far <= norm * 1.001)).sum()),
            max(float((err / tol.clamp_min(1e-300)).max()), float((far / norm.clamp_min(1e-300)).max())))


def close(out, ref):
    bad, worst = misses(out, ref)
    assert bad == 0, f"{bad} elements and rows of {tuple(out.shape)}, worst {worst:.3f}"
