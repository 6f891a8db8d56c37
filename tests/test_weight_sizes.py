"""Which expert matrices a layer's calls take: the sizes they would read, without a GPU."""
import pytest
import torch

import paper_2508_12851_amd as P
from paper_2508_12851_amd import binding as B

H, F = 128, 192
BF16, F32 = torch.bfloat16, torch.float32


def _triple(dtype=BF16, shapes=((F, H), (F, H), (H, F))):
    return tuple(torch.empty(s, dtype=dtype) for s in shapes)


def _i8(rows, cols, wrap=True, short=0):
    data = torch.empty(B._i8_bytes(rows, cols) - short, dtype=torch.uint8)
    return P.I8Matrix(data, rows, cols) if wrap else data


def _i8_triple(wrap=True, shapes=((F, H), (F, H), (H, F))):
    return tuple(_i8(*s, wrap) for s in shapes)


def _check(triples, layout="row_major", dtype="bf16"):
    B._check_sizes(B._sizes_of(triples), P.make_desc(H, F, 8, 2, 0, dtype, weight_layout=layout))


def test_matrices_that_fit():
    _check([_triple(), None, _triple(torch.int16)])                     # (bf16 bits)
    _check([_triple()], "tiled")
    _check([_triple(F32)], dtype="f32")
    _check([None, _i8_triple(), _i8_triple(wrap=False)], "int8")
    _check([tuple(_i8(*s, wrap=False).view(torch.int8) for s in ((F, H), (F, H), (H, F)))], "int8")
    _check([None, None])
    _check([])


@pytest.mark.parametrize("layout,dtype,triple", [
    ("int8", "bf16", _triple()),                                        # bf16 matrices in a layer with 8-bit ones
    ("int8", "bf16", _triple(torch.uint8)),                             # their bytes without the scales
    ("int8", "bf16", (_i8(F, H, False), _i8(F, H, False), _i8(H, F, False, short=1))),
    ("int8", "bf16", _i8_triple(shapes=((H, F), (F, H), (H, F)))),      # of another shape, if with bytes enough
    ("int8", "bf16", _i8_triple(shapes=((F, H), (F, H), (H + 16, F)))),
    ("row_major", "bf16", _i8_triple()), ("tiled", "bf16", _i8_triple(wrap=False)), ("row_major", "f32", _triple()),
    ("row_major", "bf16", _triple(shapes=((F, H), (F - 1, H), (H, F)))),
])
def test_matrices_that_would_be_read_beyond_their_end_or_as_something_else(layout, dtype, triple):
    good = {"int8": _i8_triple(), "f32": _triple(F32)}.get(layout if layout == "int8" else dtype, _triple())
    for triples in ([triple], [good, triple], [None, triple, good]):
        with pytest.raises(P.PrismError, match="w_(gate|up|down)"):
            _check(triples, layout, dtype)
