"""8-bit products in every tile and split, quantisation and schedules by every number of lanes, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2508_12851_amd as P
import i8_reference as R
from matmul_plans import PRODUCTS
from test_gpu_i8 import Layer, _check_quantized, _rows, _weights

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,n,k,tile,splits", PRODUCTS)
def test_products_of_every_tile_and_split(m, n, k, tile, splits, dtype):
    v = _rows(m, k, BF16, m + n)
    q, scale = R.quantize(v)
    w, ws = _weights(n, k, k)
    buf = P.alloc_matmul_i8_workspace(m, n, k)
    buf.fill_(255)
    a, b = P.prism_quantize_i8(v), P.prism_pack_i8(w, ws)
    got = P.prism_matmul_i8(a, b, buf, dtype=dtype)
    want = R.product(q, scale, w, ws)
    # the conversion of a part's sum and its two products, then the additions of the parts: of the magnitudes of the terms; the output's
    sums = (q.abs() @ w.double().abs().t()) * scale[:, None] * ws.double()
    tol = (3 + splits - 1) * R.EPS * sums * (1 + 2.0 ** -20)
    tol = tol + (0 if dtype == F32 else 2.0 ** -8) * (want.abs() + tol)
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    buf.fill_(0)
    assert torch.equal(P.prism_matmul_i8(a, b, buf, dtype=dtype), got)


# by the lanes that take a row: 64 (many short rows), 256, 512 (many long rows), 1024 (few); rows that are read twice beyond 16384
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(4097, 1408), (5001, 2047), (4100, 7), (4096, 2048), (33, 2049), (513, 4097), (700, 14335), (520, 16384),
                                       (515, 16393), (257, 4100), (257, 16385), (256, 4100), (256, 16385), (9, 130944)])
def test_quantisation_by_every_number_of_lanes(rows, cols, dtype):
    v = _rows(rows, cols, dtype, rows + cols)
    v[rows // 2] = 0
    v[:, cols // 2] = v.abs().amax(1) / 2       # 63.5 where the scale is what it would be without rounding
    _check_quantized(P.prism_quantize_i8(v), v)


def test_the_scale_is_the_product_with_the_reciprocal_of_127():
    """Not the quotient by 127, which is another fp32 number for one maximum in twenty."""
    top = np.random.default_rng(0).uniform(1, 2, 4000).astype(np.float32)
    product, quotient = top * (np.float32(1) / np.float32(127)), top / np.float32(127)
    top = top[product != quotient]
    assert len(top) > 100
    v = torch.from_numpy(top)[:, None].repeat(1, 5).cuda()
    v[:, 1:] *= torch.tensor([0.5, -0.5, 1.0, 0.25], device="cuda")
    m = P.prism_quantize_i8(v)
    assert np.array_equal(m.values()[1].cpu().numpy(), top * (np.float32(1) / np.float32(127)))
    _check_quantized(m, v)


# hidden sizes beyond 4096: the launch that quantises the tokens and builds the schedules has workgroups of 1024 and 512 threads
WIDE_LAYERS = [(4160, 2048, 4, 2, 0, 1, range(4)), (4160, 2048, 4, 2, 1, 40, range(3)), (4160, 2048, 4, 2, 0, 100, range(4)),
               (4160, 2048, 4, 2, 0, 300, range(3)), (4160, 512, 40, 4, 1, 90, range(0, 40, 2)), (4160, 512, 4, 2, 1, 513, range(4)),
               (4160, 512, 4, 2, 0, 1100, (1, 2)), (4160, 8256, 4, 2, 0, 600, range(4)), (4224, 8256, 4, 2, 0, 520, (2,))]


@pytest.mark.parametrize("H,F,E,k,S,T,hosted", WIDE_LAYERS)
def test_layers_wider_than_4096(H, F, E, k, S, T, hosted):
    layer = Layer(H, F, E, k, S, T, hosted, seed=T)
    r, s = layer.route()
    layer.ws.fill_(255)
    y = P.prism_expert_ffn(layer.desc, layer.x, layer.table, s.local_src, s.local_offsets, layer.ws)
    layer.check_rows(y, s.local_src, s.local_offsets)
    out = P.prism_combine(layer.desc, y, s.local_src, s.local_offsets, r.topk_gate, layer.ws)
    layer.ws.fill_(255)
    assert torch.equal(P.prism_moe_layer(layer.desc, layer.x, layer.router, layer.bias, layer.table, layer.mask, layer.ws).out, out)


def test_a_decode_sweep_with_8_bit_experts_counts_a_byte_per_weight():
    from paper_2508_12851_amd.decode_sweep import sweep
    args = dict(n_layers=1, T=16, H=256, F=512, E=8, k=2, steps=1, warmup=1, seed=4)      # (one layer: the same tokens, the same picks)
    bf16, i8 = sweep(**args), sweep(**args, weights="int8")
    assert [r["weight_bytes_streamed_per_step"] for r in bf16] == [2 * r["weight_bytes_streamed_per_step"] for r in i8]
    assert i8[-1]["weight_bytes_streamed_per_step"] > 0
