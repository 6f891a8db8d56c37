"""Calls on another stream than the current one: whose memory their outputs are, and on which stream they are filled."""
import pytest
import torch

import paper_2508_12851_amd as P

pytestmark = pytest.mark.gpu

T, H, F, E, k = 768, 512, 256, 64, 4


def _setup(layout):
    gen = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    desc = P.make_desc(H, F, E, k, weight_layout=layout)
    load = {"row_major": lambda w: w, "int8": lambda w: P.prism_quantize_i8(w).data}[layout]
    mask = torch.ones(E, dtype=torch.uint8, device="cuda")
    mask[E // 2:] = 0
    experts = [tuple(load(normal(*s) / 16) for s in ((F, H), (F, H), (H, F))) if e < E // 2 else None for e in range(E)]
    return desc, normal(T, H), normal(E, H) / 16, P.WeightTable(experts), mask, P.alloc_workspace(desc, T)


def _tensors(out):
    return [out] if isinstance(out, torch.Tensor) else [t for t in vars(out).values() if t is not None]


# call -> (its outputs, the bytes of one of them)
CALLS = {
    "route": T * E * 4, "dispatch": 2 * T * k * 4, "ffn": T * k * H * 2, "combine": T * H * 2, "layer": T * H * 2,
    "permutation": T * k * 4, "pack_remote": T * k * H * 2, "pack_weights": 1024 * 1024 * 2,
}


@pytest.mark.parametrize("layout", ["row_major", "int8"])
@pytest.mark.parametrize("call", CALLS)
def test_outputs_of_a_call_on_another_stream_are_of_its_memory(call, layout):
    desc, x, router, table, mask, ws = _setup(layout)
    r = P.prism_route(desc, x, router, None)
    d = P.prism_dispatch(desc, r.topk_idx, mask, ws)
    y = P.prism_expert_ffn(desc, x, table, d.local_src, d.local_offsets, ws)
    layer_ws = P.alloc_workspace(desc, T)
    P.prism_moe_layer(desc, x, router, None, table, mask, layer_ws)
    w = torch.zeros((1024, 1024), dtype=torch.bfloat16, device="cuda").normal_()
    run = {"route": lambda s: P.prism_route(desc, x, router, None, stream=s),
           "dispatch": lambda s: P.prism_dispatch(desc, r.topk_idx, mask, ws, stream=s),
           "ffn": lambda s: P.prism_expert_ffn(desc, x, table, d.local_src, d.local_offsets, ws, stream=s),
           "combine": lambda s: P.prism_combine(desc, y, d.local_src, d.local_offsets, r.topk_gate, ws, stream=s),
           "layer": lambda s: P.prism_moe_layer(desc, x, router, None, table, mask, ws, stream=s),
           "permutation": lambda s: P.prism_layer_permutation(desc, T, layer_ws, stream=s),
           "pack_remote": lambda s: P.prism_pack_remote(desc, x, d.remote_src, d.remote_offsets, stream=s),
           "pack_weights": lambda s: P.prism_pack_weights(w, stream=s)}[call]
    if call == "permutation":       # what the list does not reach is what the workspace held: the list itself is compared
        n = int(d.local_offsets[-1])
        parts = lambda out: [out.local_src[:n], out.local_offsets, out.inv]
    else:
        parts = _tensors
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = [t.clone() for t in parts(run(None))]
    nbytes = CALLS[call]
    old = [torch.full((nbytes,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
    kept = [torch.empty_like(o) for o in old]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for a, o in zip(kept, old):
        a.copy_(o)
    del old, o                       # freed here, read later by this stream
    got = run(side)
    torch.cuda.synchronize()
    assert all(bool((a == 77).all()) for a in kept)
    assert all(torch.equal(a, b) for a, b in zip(parts(got), want))     # (no fill of this stream came after the call)
