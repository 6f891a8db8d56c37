"""8-bit layers beyond what 32-bit offsets reach are refused before anything is launched (no GPU here: a launch would fail)."""
import ctypes

import pytest

import paper_2508_12851_amd as P

P0 = ctypes.c_void_p(0x10000)       # never dereferenced
UNSUPPORTED = 2


# rows of h, rows of tokens, a weight matrix, of 4 GiB and more
@pytest.mark.parametrize("H,F,k,S,T", [(256, 14336, 2, 0, 150000), (14336, 256, 2, 0, 150000), (256, 14336, 1, 1, 150000), (65536, 65536, 2, 0, 32)])
def test_refused_before_any_launch(H, F, k, S, T):
    lib = P.load_library()
    desc = P.make_desc(H, F, 8, k, S, "bf16", weight_layout="int8")
    size = ctypes.c_size_t(0)
    assert lib.prism_workspace_bytes(ctypes.byref(desc), T, ctypes.byref(size)) == 0
    weights = P.binding.ExpertWeights(*[0x10000] * 6)
    assert lib.prism_expert_ffn(ctypes.byref(desc), P0, ctypes.byref(weights), P0, P0, T, P0, P0, size, None) == UNSUPPORTED
    layer = (ctypes.byref(desc), P0, P0, None, ctypes.byref(weights), P0, T, P0, P0, P0, P0, None, P0, P0, P0, P0, P0, size, None)
    assert lib.prism_moe_layer(*layer) == UNSUPPORTED
    assert lib.prism_moe_layer_traced(*layer, None) == UNSUPPORTED
