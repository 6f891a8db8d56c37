"""8-bit matrices, their product and the 8-bit expert FFN from their definitions in 64 bits."""
import numpy as np
import torch

EPS = 2.0 ** -24


def quantize(v):
    """(q, scale) of the rows of v, both in float64: scale the fp32 product with 1 / 127, q the nearest integer to v / scale."""
    v = v.double()
    scale = (v.abs().amax(1).float() * torch.tensor(np.float32(1) / np.float32(127), device=v.device)).double()
    return torch.round(v / torch.where(scale > 0, scale, 1.0)[:, None]).clamp(-127, 127), scale


def product(q, scale, w, w_scale):
    return (q @ w.double().t()) * scale[:, None] * w_scale.double()


# What fp32 may be off in an element of h = silu(g) u, relative to it, for |g| <= 20: g and u are a rounded sum times a rounded
# product of scales (3 roundings each); the exponential's argument, |g| log2 e, is rounded twice, which is |g| 2^-23 of its
# value, 20 * 2 * EPS; the exponential, the reciprocal and what joins them are within 1 ulp (2 EPS) each, 6 of them.
H_ERROR = (3 + 3 * 21 + 2 * 20 + 2 * 6) * EPS


def swiglu(x, gate, up, down):
    """(y, how far fp32 sums of it may be off) of one expert's rows; gate, up, down: (int8 [n, k], scale [n])."""
    q, scale = quantize(x)
    g, u = product(q, scale, *gate), product(q, scale, *up)
    assert float(g.abs().max()) <= 20.0
    h = g / (1 + torch.exp(-g)) * u
    hq, hs = quantize(h)
    y = product(hq, hs, *down)
    # an element whose quotient is so near to a half that fp32's error (its own and its row's scale's) may turn it
    t = h / torch.where(hs > 0, hs, 1.0)[:, None]
    near = ((t - torch.floor(t) - 0.5).abs() <= 2 * H_ERROR * t.abs() + 1e-12).double()
    w = down[0].double().abs()
    turned = (near @ w.t()) * hs[:, None] * down[1].double()
    # the scale, and 4 roundings of each of at most 8 parts of the sum
    sums = (hq.abs() @ w.t()) * hs[:, None] * down[1].double()
    return y, turned + H_ERROR * y.abs() + 12 * EPS * sums
