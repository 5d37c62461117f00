"""The 4-bit cache and the attention over it from their definitions, in 64 bits on the CPU, and the bounds that the kernels' results are held to."""
import math

import torch


def steps(x, g):
    """(s, m, codes) of x [tokens, heads, dim]: binary32 where the definition says so, each quotient correctly rounded"""
    y = x.double().unflatten(-1, (-1, g))
    lo, hi = y.amin(-1), y.amax(-1)
    fifteen = torch.tensor(15.0, dtype=torch.float64)
    m = lo.half()
    s = ((hi - lo).float().double() / fifteen).float().clamp_min(2.0 ** -24).half()
    bad = ~torch.isfinite(y.half()).all(-1)                  # not finite, or beyond binary16
    s, m = s.masked_fill(bad, math.nan), m.masked_fill(bad, math.nan)
    c = ((y - m.double().unsqueeze(-1)).float().double() / s.double().unsqueeze(-1)).float().double().round().clamp(0, 15)
    return s.double(), m.double(), c


def held(x, g):
    """the values that the cache stands for, exactly"""
    s, m, c = steps(x, g)
    return (m.unsqueeze(-1) + s.unsqueeze(-1) * c).flatten(-2)


def attention(q, k, v, g, scale=None, causal=True, window=0, gone=None):
    """One sequence: q [n, Hq, D] stand at its last n positions, k and v [L, H, D] as they were written; gone: positions that are not there.
    Returns out, lse, and bounds on their errors (apart from the rounding of out to its type): the scores are binary32 sums of |q| (|m| + s c) terms,
    and the weights of the sums over codes are rounded to 11 bits (bf16) or 22 (fp32).  A bf16 sequence of more than 64 rows (query, head that shares a head of the
    cache) may have its keys and values rebuilt as binary16, its queries held so with the scale in them, and sums its rounded p: 2^-11 of every |q| |k^| in a score,
    2^-12 of a value, and of the sum in lse."""
    n, Hq, D = q.shape
    L, H = k.shape[:2]
    R = Hq // H
    rebuilt = q.dtype == torch.bfloat16 and n * R > 64
    scale = scale or 1 / math.sqrt(D)
    ks, km, kc = steps(k, g)
    kh = held(k, g)
    vh = held(v, g)
    vs, vm, vc = steps(v, g)
    pos = torch.arange(L - n, L)[:, None]
    j = torch.arange(L)[None]
    seen = torch.ones(n, L, dtype=torch.bool)
    if causal:
        seen &= j <= pos
    if window:
        seen &= j > pos - window
    if gone is not None:
        seen &= ~gone[None]
    if (pos < 0).any():
        seen &= pos >= 0
    out, lse = torch.zeros(n, Hq, D, dtype=torch.float64), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    r = 2.0 ** -11 if q.dtype == torch.bfloat16 else 2.0 ** -21
    size = (km.abs().unsqueeze(-1) + ks.unsqueeze(-1) * kc).flatten(-2)                # |m| + s c
    span = (vm.abs().unsqueeze(-1) + vs.unsqueeze(-1) * vc).flatten(-2)
    for h in range(Hq):
        Q, K, V = q[:, h].double(), kh[:, h // R], vh[:, h // R]
        for i in range(n):
            at = seen[i].nonzero()[:, 0]
            if len(at) == 0:
                continue
            S = scale * (K[at] @ Q[i])
            lse[i, h] = torch.logsumexp(S, 0)
            p = torch.exp(S - lse[i, h])
            out[i, h] = p @ V[at]
            eps = 2.0 ** -21 * float((size[at, h // R] @ Q[i].abs()).max()) * scale       # of a score: 2^-22 for either of its two sums
            if rebuilt:
                eps += 2.0 ** -11 * float((K[at].abs() @ Q[i].abs()).max()) * scale + 2.0 ** -24
            weights = p @ span[at, h // R]
            tol_o[i, h] = weights * (r + 2 * eps + 2.0 ** -19)
            tol_l[i, h] = eps + 2.0 ** -20 * (1 + lse[i, h].abs()) + (2.0 ** -12 if rebuilt else 0.0)
    return out, lse, tol_o, tol_l
