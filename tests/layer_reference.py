"""Plain implementations, in 64 bits, of the norm, the rotary positions and the gated feed-forward, and the bounds that follow from the kernels' roundings."""
import math

import torch

F32 = 2.0 ** -24                        # a binary32 rounding, relative


def half(dtype):
    """A rounding to `dtype`, relative."""
    return torch.finfo(dtype).eps / 2


def norm(X, W, eps, R=None):
    """(S, rstd, Y in 64 bits)"""
    S = X if R is None else (X.float() + R.float()).to(X.dtype)
    s = S.double()
    rstd = 1.0 / (s.square().mean(-1, keepdim=True) + eps).sqrt()
    return S, rstd, s * rstd * (1.0 if W is None else W.double())


# A row's sum of squares: up to 32 elements one after the other in a lane, six meetings of lanes, 16 of waves: 54 roundings; half of that in rstd; some six more behind it.
NORM_ROUNDINGS = 54 // 2 + 6


def norm_back(S, W, eps, dY, dS=None):
    """(dX, dW, bound of dX, terms of dW)"""
    s, e = S.double(), dY.double() * (1.0 if W is None else W.double())
    rstd = 1.0 / (s.square().mean(-1, keepdim=True) + eps).sqrt()
    dX = rstd * (e - s * rstd ** 2 * (e * s).mean(-1, keepdim=True)) + (0.0 if dS is None else dS.double())
    terms = dY.double() * s * rstd
    # what the three terms can be off by: 54 roundings of the sums, twice rstd's, and some ten
    loose = rstd * e.abs() + rstd ** 3 * s.abs() * (e * s).abs().mean(-1, keepdim=True) + (0.0 if dS is None else dS.double().abs())
    return dX, terms.sum(0), half(S.dtype) * dX.abs() + (54 + 2 * NORM_ROUNDINGS + 10) * F32 * loose, terms


def e4m3_step(v):
    """the distance of neighbouring e4m3 numbers around v"""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3.0)


def turned(x, pos, freq, interleaved=False, amplitude=1.0, inverse=False):
    """(value, bound of the result of x's type)"""
    n = freq.numel()
    angle = (pos.double()[:, None] * freq.double()[None])[:, None]
    c, s = angle.cos() * amplitude, angle.sin() * (-amplitude if inverse else amplitude)
    y = x.double().clone()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = x.double()[..., first], x.double()[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    # cosine and sine: the angle's quarter rounded (2^-25 of at most pi / 4), the polynomials' first terms left out (2.5e-8) and three roundings of theirs; the amplitude's, a product's and
    # a sum's: 8 roundings of |a| + |b|
    bound = half(x.dtype) * y.abs()
    both = (a.abs() + b.abs()) * 8 * F32 * abs(amplitude)
    bound[..., first] += both
    bound[..., second] += both
    return y, bound


def codes_of(packed, count, bits):
    b = ((packed.unsqueeze(-1) >> torch.arange(8, dtype=torch.uint8, device=packed.device)) & 1).flatten(1)[:, :count * bits].unflatten(1, (count, bits))
    return (b.int() << torch.arange(bits, dtype=torch.int32, device=packed.device)).sum(-1)


def what(Wpacked, s, zpacked, I, bits, rounded):
    """the weights that a packed layer stands for; `rounded`: as the bf16 kernels hold them (q s - z s by one multiply-add, then bf16)"""
    G = s.shape[1]
    q = codes_of(Wpacked, I, bits).double().unflatten(1, (G, -1))
    z, s = codes_of(zpacked, G, bits).double().unsqueeze(-1), s.double().unsqueeze(-1)
    if not rounded:
        return ((q - z) * s).flatten(1)
    return (q * s - (z * s).float().double()).float().bfloat16().double().flatten(1)


def act(kind, g):
    """value and derivative; kind 0: silu, 1: gelu (tanh)"""
    if kind == 0:
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    k = math.sqrt(2 / math.pi)
    p = torch.sigmoid(2 * k * (g + 0.044715 * g ** 3))       # (1 + tanh(x)) / 2 without the difference, which leaves nothing for x below -19
    return g * p, p + 2 * g * p * (1 - p) * k * (1 + 3 * 0.044715 * g * g)


def gate(kind, g, u, dH, dtype, dg=0.0, du=0.0, near=False):
    """{name: (value, bound)} of H and dY from G and U that are good to dg and du (absolute).  act(x) = x p(t), act'(x) = p + x p q t', q = 1 - p; the derivative of either activation
    is below 1.13, its own derivative below 1.1 (silu 0.5).  p and q are good to eight roundings each; gelu's t = 2 k x (1 + 0.044715 x^2) has four roundings of its own, each of which moves p
    by q |t| of them and q by p |t|.  t', the products and the sum behind act': six more of x p q t'.
    `near`, as the kernels with bf16 results have it: exp(-t) by a product that is rounded once (t and log2 e: 2 |t| roundings, of which p has q's share), and q = 1 - p, off by what p is.
    Where 1 + exp(-t) is 2^126 or more, p <= 2^-126 is no normal binary32 number and may be 0: act is off by |x| 2^-126 there, and act' by 2^-126 (1 + |x| t'), t' <= 1 for silu and below
    2 x^2 for the |x| > 5 where gelu's p is so small."""
    a, slope = act(kind, g)
    h = half(dtype)
    k = math.sqrt(2 / math.pi)
    t = g if kind == 0 else 2 * k * (g + 0.044715 * g ** 3)
    t1 = 1.0 if kind == 0 else 2 * k * (1 + 3 * 0.044715 * g * g)
    p, q, far = torch.sigmoid(t), torch.sigmoid(-t), 4 * t.abs() if kind == 1 else 0.0
    gone = 2.0 ** -126 * g.abs()
    da = 1.13 * dg + (8 + far * q) * F32 * a.abs() + gone
    rp, rq = 8 + far * q, 8 + far * p                        # roundings of p and q
    if near:
        rp = rp + 2 * t.abs() * q
        rq = rp * p / q.clamp_min(2.0 ** -60) + 1
        da = da + 2 * t.abs() * q * F32 * a.abs()
    ds = 1.1 * dg + F32 * (p * rp + g.abs() * p * q * t1 * (rp + rq + 6)) + 2.0 ** -126 + gone * (1 if kind == 0 else 2 * g.square() + 1)
    out = {"H": (a * u, h * (a * u).abs() + da * u.abs() + a.abs() * du + da * du + 2 * F32 * (a * u).abs())}
    if dH is not None:
        d = dH.double()
        dG, dU = d * u * slope, d * a
        bG = h * dG.abs() + d.abs() * (u.abs() * ds + slope.abs() * du + ds * du) + 4 * F32 * dG.abs()
        bU = h * dU.abs() + d.abs() * da + 2 * F32 * dU.abs()
        out["dY"] = (torch.cat((dG, dU), 1), torch.cat((bG, bU), 1))
    return out


def within(got, ref, bound, tiny=1e-37):
    """Asserts that got is ref to the bound, and says by how much of it the worst element is off."""
    got = got.double()
    assert got.shape == ref.shape
    off = (got - ref).abs()
    bad = ~(off <= bound + tiny)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((off / (bound + tiny)).nan_to_num(1e30).max()):.3g} of the bound"
