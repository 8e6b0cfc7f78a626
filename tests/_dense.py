"""Plain 64-bit forms of the dense attention operators, with bounds on how far
16-bit results may be off, for the tests.

Bounds are per element.  u is half a step of the result's type relative to the
value (bf16 2^-8, fp16 2^-11); fp16 values below 2^-14 are multiples of 2^-24, so
that half a step there is 2^-25 (``tiny``).  A result is rounded once (u |result|); the
probabilities (and score gradients) are rounded to 16 bits before their
product (u times the sum of the magnitudes); 32-bit sums add N * 2^-24 of the
sum of magnitudes for N terms in a row."""
import math

import torch

F32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(u):
    """Half a step between the smallest values of the type whose half step is u."""
    return 2.0 ** -25 if u < 2.0 ** -10 else 2.0 ** -134


def attention(Q, K, V, scale, u, up=None, seen=None, floor=None):
    """One head: Q [n, d], K, V [m, d] in 64 bits.  Returns a dict with O, lse
    and P and the bounds O_tol and lse_tol.  up: half a step of the
    probabilities' type; seen [n, m]; floor [m, d]: what a probability too small
    for its type may lose of a value."""
    up = u if up is None else up
    n, d = Q.shape
    m = K.shape[0]
    x = Q @ K.T * scale
    # 32-bit sums of d products, and the scaled score's own rounding; two ulp
    # of the exponential
    dx = (d + 4) * F32 * abs(scale) * (Q.abs() @ K.abs().T) + 4 * F32 * x.abs()
    if seen is not None:
        x = torch.where(seen, x, -math.inf)
        dx = torch.where(seen, dx, 0.0)
    lse = torch.logsumexp(x, 1) if m else torch.full((n,), -math.inf, dtype=x.dtype)
    P = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    worst = dx.amax(1) if m else torch.zeros(n, dtype=x.dtype)
    terms = m / 64 + 64  # of a lane's running sum, and of the joining
    ep = 2 * worst + (terms + 8) * F32
    absO = P @ V.abs()
    O = P @ V
    O_tol = (up + ep[:, None]) * absO + u * O.abs() + tiny(u) + tiny(up) * V.abs().sum(0)
    if floor is not None:
        O_tol = O_tol + floor.sum(0)
    lse_tol = worst + (terms + 8) * F32 + 4 * F32 * torch.where(lse == -math.inf, 0.0, lse.abs())
    return dict(O=O, lse=lse, P=P, ep=ep, O_tol=O_tol, lse_tol=lse_tol)


def gradients(Q, K, V, G, scale, u, f):
    """One head's gradients from f = attention(...): dict of dQ, dK, dV and
    their bounds (without the results' own rounding, which the caller adds
    after summing heads)."""
    d = Q.shape[1]
    P = f["P"]
    dP = G @ V.T
    delta = (G * f["O"]).sum(1, keepdim=True)
    dS = P * (dP - delta)
    # P from lse (which is off as O's normaliser is), dP's and delta's 32-bit
    # sums, delta from a rounded O
    eP = P * (2 * f["ep"][:, None] + f["lse_tol"].nan_to_num(0)[:, None])
    edP = (d + 4) * F32 * (G.abs() @ V.abs().T)
    ed = (G.abs() * f["O_tol"]).sum(1, keepdim=True) \
        + (d + 4) * F32 * (G.abs() * f["O"].abs()).sum(1, keepdim=True)
    edS = u * dS.abs() + P * (edP + ed) + eP * (dP - delta).abs() + tiny(u)
    n, m = P.shape
    sums_q, sums_k = (m / 32 + 64) * F32, (n / 32 + 64) * F32
    s = abs(scale)
    return dict(
        dQ=scale * dS @ K, dK=scale * dS.T @ Q, dV=P.T @ G,
        dQ_tol=s * ((edS + sums_q * dS.abs()) @ K.abs()),
        dK_tol=s * ((edS + sums_k * dS.abs()).T @ Q.abs()),
        dV_tol=(u * P + eP + sums_k * P + tiny(u)).T @ G.abs())


def close(got, want, tol, what):
    """Every element within its bound; equal infinities count as equal."""
    got = got.double().cpu()
    same = got == want
    off = torch.where(same, 0.0, (got - want).abs())
    worst = (off / tol.clamp(min=1e-300)).nan_to_num(math.inf)
    worst = torch.where(same, 0.0, worst)
    assert got.shape == want.shape, what
    assert bool((worst <= 1).all()), (what, float(worst.max()), int((worst > 1).sum()),
                                      got.numel())


# ---- the cache's format ------------------------------------------------------

def code_values():
    b = torch.arange(256, dtype=torch.float64)
    sign, e, f = 1 - 2 * (b // 128), b % 128 // 8, b % 8
    v = torch.where(e > 0, (1 + f / 8) * 2.0 ** (e - 7), f / 8 * 2.0 ** -6)
    return sign * torch.where(b % 128 == 127, math.nan, v)


def two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantised(x):
    """(values, exponent bytes) that the cache keeps of rows of x, from the
    format's definition: the nearest code of the row's power of two, the even
    one in the middle."""
    x = x.double()
    finite = torch.isfinite(x)
    top = torch.where(finite, x, 0.0).abs().amax(-1)
    e = torch.full(top.shape, -127)
    for k in range(-127, 128):  # the smallest power that keeps the row within 448
        e = torch.where((top > 448 * two_to(torch.tensor(k - 1))) & (k > -127), k, e)
    y = x * two_to(-e)[..., None]
    grid = code_values()[:127]
    a = torch.where(finite, y, 0.0).abs()
    hi = torch.searchsorted(grid, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    v = torch.copysign(grid[pick], y) * two_to(e)[..., None]
    return torch.where(finite, v, math.nan), (e + 127).to(torch.uint8)
