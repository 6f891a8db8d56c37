"""Tables whose matrices do not fit a layer are refused by every call that reads them, before any launch."""
import pytest
import torch

import paper_2508_12851_amd as P
from paper_2508_12851_amd.migration import Migrator

pytestmark = pytest.mark.gpu

T, H, F, E, k = 40, 256, 512, 8, 2


def _normal(*shape):
    return (torch.randn(shape, device="cuda") / 16).to(torch.bfloat16)


def _triple():
    return tuple(_normal(*s) for s in ((F, H), (F, H), (H, F)))


def _calls(layout):
    """The calls that take a table."""
    desc = P.make_desc(H, F, E, k, weight_layout=layout)
    x, router, mask, ws = _normal(T, H), _normal(E, H), torch.ones(E, dtype=torch.uint8, device="cuda"), P.alloc_workspace(desc, T)
    r = P.prism_route(desc, x, router, None)
    d = P.prism_dispatch(desc, r.topk_idx, mask, ws)
    out = P.alloc_layer_out(desc, T)
    return [lambda t: P.prism_expert_ffn(desc, x, t, d.local_src, d.local_offsets, ws),
            lambda t: P.prism_moe_layer(desc, x, router, None, t, mask, ws),
            lambda t: P.prism_moe_layer_static(desc, x, router, None, t, mask, out),
            lambda t: P.prism_debug_check_weights(desc, t, mask)]


def test_tables_of_another_layout_are_refused():
    bf16 = [_triple() for _ in range(E)]
    i8 = [tuple(P.prism_quantize_i8(w) for w in t) for t in bf16]
    raw = [tuple(m.data for m in t) for t in i8]
    for layout, good, bad in (("int8", (i8, raw, i8[:5] + raw[5:]), (bf16, i8[:7] + bf16[7:])), ("row_major", (bf16,), (i8, raw, bf16[:7] + raw[7:]))):
        for call in _calls(layout):
            for experts in good:
                call(P.WeightTable(experts))
            for experts in bad:
                with pytest.raises(P.PrismError, match="w_gate"):
                    call(P.WeightTable(experts))
    # the same table in another layer
    table = P.WeightTable(i8)
    _calls("int8")[0](table)
    wide = P.make_desc(H, 2 * F, E, k, weight_layout="int8")
    with pytest.raises(P.PrismError, match="w_gate"):
        P.prism_moe_layer(wide, _normal(T, H), _normal(E, H), None, table, torch.ones(E, dtype=torch.uint8, device="cuda"), P.alloc_workspace(wide, T))
    _calls("int8")[1](table)


def test_a_table_of_8_bit_matrices_is_a_table_of_their_bytes():
    i8 = [tuple(P.prism_quantize_i8(w) for w in _triple()) for _ in range(E)]
    a, b = P.WeightTable(i8, i8[:1]), P.WeightTable([tuple(m.data for m in t) for t in i8], [tuple(m.data for m in t) for t in i8[:1]])
    assert all(torch.equal(s, t) for s, t in zip(a.tables, b.tables))


def test_migrated_8_bit_experts():
    """Experts admitted as 8-bit matrices in pinned memory; one that does not fit is refused by the next call."""
    experts = [tuple(P.prism_quantize_i8(w) for w in _triple()) for _ in range(E)]
    desc = P.make_desc(H, F, E, k, weight_layout="int8")
    x, router, ws = _normal(T, H), _normal(E, H), P.alloc_workspace(desc, T)
    mask = torch.ones(E, dtype=torch.uint8, device="cuda")
    want = P.prism_moe_layer(desc, x, router, None, P.WeightTable(experts), mask, ws).out
    table = P.WeightTable(experts[:4] + [None] * 4)
    mask[4:] = 0
    P.prism_moe_layer(desc, x, router, None, table, mask, ws)
    host = {e: tuple(P.I8Matrix(m.data.cpu().pin_memory(), m.rows, m.cols) for m in experts[e]) for e in range(4, E)}
    mig = Migrator()
    mig.start(table, host, torch.ones(E, dtype=torch.uint8).numpy())
    mig.commit(mask)
    got = P.prism_moe_layer(desc, x, router, None, table, mask, ws).out
    assert torch.equal(got, want) and mig.bytes == sum(m.data.numel() for t in experts[4:] for m in t)
    torch.cuda.synchronize()
    mig.start(table, {7: tuple(torch.zeros(1024, dtype=torch.uint8).pin_memory() for _ in range(3))}, torch.ones(E, dtype=torch.uint8).numpy())
    with pytest.raises(P.PrismError, match="w_gate"):
        P.prism_moe_layer(desc, x, router, None, table, mask, ws)
    torch.cuda.synchronize()
