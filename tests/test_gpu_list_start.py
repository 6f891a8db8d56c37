"""A caller's own list of assignments that starts behind row 0: the rows before it are left as they were."""
import numpy as np
import pytest
import torch

import paper_2508_12851_amd as P
from prism_inputs import make_config, make_inputs

from gpu_util import desc_of, to_dev, weight_table

pytestmark = pytest.mark.gpu


# decode, streamed and split tiles; prefill tiles with the copy of the token rows
@pytest.mark.parametrize("T,H,F", [(20, 256, 1024), (200, 256, 1024), (300, 256, 1024), (700, 4096, 4096)])
def test_rows_before_the_first_segment(T, H, F):
    cfg = make_config("cfg3_mixtral_decode", T=T, H=H, F=F, E=4, n_local=4)
    inp = make_inputs(cfg)
    desc, x, wt = desc_of(cfg, weight_layout="tiled"), to_dev(inp.x), weight_table(inp, all_experts=True, tiled=True)
    A, first = 2 * T, T // 3
    ws = P.alloc_workspace(desc, T)

    def rows(start):
        src = torch.zeros(A, dtype=torch.int32, device="cuda")
        src[start:start + T] = torch.arange(T, dtype=torch.int32, device="cuda") * 2
        offsets = torch.tensor([start, start + T // 2, start + T // 2, start + T, start + T], dtype=torch.int32, device="cuda")
        y = torch.full((A, H), 5.0, dtype=torch.bfloat16, device="cuda")
        ws.fill_(255)
        P.prism_expert_ffn(desc, x, wt, src, offsets, ws, y=y)
        return y
    want, got = rows(0), rows(first)
    assert bool((got[:first] == 5.0).all()) and bool((got[first + T:] == 5.0).all())
    err = (got[first:first + T].float() - want[:T].float()).abs()
    # the same products in other row tiles: sums in another order, rounded to bf16
    assert bool((err <= 2.0 ** -7 * want[:T].float().abs() + 2.0 ** -8 * want[:T].float().abs().max()).all())
