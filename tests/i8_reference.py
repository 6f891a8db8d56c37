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


# Layers of the expert FFN's tests.
SHAPES = [
    # H, F, E, k, S, T, hosted: every path of ffn_paths.h, ragged tiles, one token, experts with no row
    (64, 64, 4, 1, 0, 1, range(4)), (64, 64, 8, 2, 1, 65, range(0, 8, 2)), (128, 192, 8, 2, 2, 33, range(5)), (192, 448, 8, 2, 0, 64, range(8)),
    (512, 2048, 8, 2, 0, 1, range(8)), (512, 2048, 8, 2, 1, 37, (0, 3, 4)), (512, 2048, 8, 2, 0, 66, range(8)), (512, 2048, 8, 2, 0, 200, (1,)),
    (512, 2048, 8, 2, 0, 256, range(5)), (512, 2048, 8, 2, 1, 300, range(5)), (2880, 2048, 8, 2, 0, 500, range(3)), (1024, 1408, 60, 4, 2, 90, range(0, 60, 2)),
    (1024, 1408, 60, 4, 2, 333, range(30)), (384, 384, 64, 6, 0, 100, range(64)), (256, 320, 8, 2, 1, 700, range(4)),
    (320, 8192, 4, 2, 0, 600, range(3)), (256, 8256, 8, 2, 0, 400, (7,)), (1024, 512, 8, 2, 0, 1500, range(8)), (64, 1024, 4, 4, 0, 300, range(4)),
    (384, 1024, 8, 2, 0, 20, range(8)), (1024, 8192, 4, 2, 1, 900, range(4)),
]
