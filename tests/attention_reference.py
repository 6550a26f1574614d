"""Attention and the rotation by positions in 64 bits, from their definitions, with the sizes of the terms that roundings act on -- TEST
INFRASTRUCTURE ONLY.  Torch on whatever device the inputs are on.

Bounds.  A rounding to bf16 moves a value by at most 2^-8 of it.  The kernels round the outputs, and as operands the probabilities and
dS; the scores are fp32 sums of bf16 products, whose error (about hd 2^-24 of the sum of the products' magnitudes, a few thousandths of a unit at the
scores used here) moves a probability by 2^-11 at most, the approximate power of two by 2^-22.  So
    |O^ - O|   <= 2^-8 |O| + (2^-8 + 2^-11) P |V|
    |dV^ - dV| <= 2^-8 |dV| + (2^-8 + 2^-11) P^T |dO|
    |dQ^ - dQ| <= 2^-8 |dQ| + scale (2^-8 + 2^-11) |dS| |K| + scale 2^-14 (P (|dO| |V|^T + |dO| |O|)) |K|
and dK like dQ: the last term is fp32's error in the difference dO V^T - D, whose terms may be far larger than itself.
"""
import math

import torch

HALF, SCORE, DIFF = 2.0 ** -8, 2.0 ** -11, 2.0 ** -14


def visible(n, causal, window, device):
    i = torch.arange(n, device=device)
    back = i[:, None] - i[None, :]
    seen = torch.ones(n, n, dtype=torch.bool, device=device)
    if causal:
        seen &= back >= 0
    if window:
        seen &= back < window
    return seen


def heads_of(x, hd):
    return x.double().reshape(x.shape[0], -1, hd).permute(1, 0, 2)


def attention(Q, K, V, hd, sequences, causal, window=0, scale=None, dO=None, O=None, lse=None):
    """{name: (value, bound)} as [b x columns] ([heads x b] for lse), rows of no sequence NaN.  With dO the gradients, from O and lse as they
    were stored."""
    scale = hd ** -0.5 if scale is None else scale
    b, heads, kv = Q.shape[0], Q.shape[1] // hd, K.shape[1] // hd
    out = {}

    def put(name, like, h, rows, value, bound):
        if name not in out:
            shape = (heads, b) if name == "lse" else like.shape
            out[name] = tuple(torch.full(shape, math.nan, dtype=torch.float64, device=Q.device) for _ in range(2))
        for t, v in zip(out[name], (value, bound)):
            if name == "lse":
                t[h, rows] = v
            else:
                t[rows, h * hd:(h + 1) * hd] = v

    for first, n in sequences:
        rows = slice(first, first + n)
        if n == 0:
            continue
        seen = visible(n, causal, window, Q.device)
        q, k, v = (heads_of(x[rows], hd) for x in (Q, K, V))
        if dO is not None:
            g, o = heads_of(dO[rows], hd), heads_of(O[rows], hd)
            sums = {}
        for h in range(heads):
            kh = h // (heads // kv)
            S = (q[h] @ k[kh].T * scale).masked_fill(~seen, -math.inf)
            if dO is None:
                l = torch.logsumexp(S, dim=1)
                P = torch.exp(S - l[:, None])
                value, size = P @ v[kh], P @ v[kh].abs()
                put("O", Q, h, rows, value, HALF * value.abs() + (HALF + SCORE) * size)
                most = (q[h].abs() @ k[kh].abs().T * scale).masked_fill(~seen, 0).amax(1)
                put("lse", None, h, rows, l, 2.0 ** -18 * (1 + most))
                continue
            P = torch.exp(S - lse[h, rows].double()[:, None])
            dS = P * (g[h] @ v[kh].T - (g[h] * o[h]).sum(1, keepdim=True))
            loose = P * (g[h].abs() @ v[kh].abs().T + (g[h].abs() * o[h].abs()).sum(1, keepdim=True))
            dq = scale * (dS @ k[kh])
            put("dQ", Q, h, rows, dq, HALF * dq.abs() + scale * ((HALF + SCORE) * dS.abs() + DIFF * loose) @ k[kh].abs())
            part = (P.T @ g[h], (HALF + SCORE) * (P.T @ g[h].abs()), scale * (dS.T @ q[h]),
                    scale * (((HALF + SCORE) * dS.abs() + DIFF * loose).T @ q[h].abs()))
            sums[kh] = part if kh not in sums else tuple(x + y for x, y in zip(sums[kh], part))
        if dO is not None:
            for kh, (dv, dv_b, dk, dk_b) in sums.items():
                put("dV", K, kh, rows, dv, HALF * dv.abs() + dv_b)
                put("dK", K, kh, rows, dk, HALF * dk.abs() + dk_b)
    return out


def check(got, want, name):
    """`got` within the bound of `want` wherever that is a number."""
    value, bound = want
    inside = ~value.isnan()
    off = (got.double() - value).abs()[inside]
    bad = ~(off <= bound[inside] + 1e-30)
    assert not bad.any(), (name, int(bad.sum()), "of", bad.numel(), float((off / (bound[inside] + 1e-30)).nan_to_num(1e30).max()))


def rotary(X, positions, frequencies, hd, factor=1.0, interleaved=False, backward=False):
    """Pairs as complex numbers, in 64 bits."""
    n = frequencies.numel()
    x = X.double().reshape(X.shape[0], -1, hd)
    u, v = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    angle = positions.double()[:, None] * frequencies.double()
    z = torch.complex(u, v) * (factor * torch.exp(1j * (-angle if backward else angle)))[:, None]
    y = x.clone()
    if interleaved:
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = z.real, z.imag
    else:
        y[..., :n], y[..., n:2 * n] = z.real, z.imag
    return y.reshape(X.shape)


def rotary_bound(X, want, hd, n, factor, interleaved, half):
    """Bound of a rotated matrix: one rounding of the result, and an angle known to 2^-20 plus fp32's roundings, relative to the pair."""
    x = X.double().reshape(X.shape[0], -1, hd)
    size = torch.zeros_like(x)
    u, v = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    r = abs(factor) * (u * u + v * v).sqrt()
    if interleaved:
        size[..., 0:2 * n:2], size[..., 1:2 * n:2] = r, r
    else:
        size[..., :n], size[..., n:2 * n] = r, r
    return half * want.abs() + 2.0 ** -20 * size.reshape(X.shape)
