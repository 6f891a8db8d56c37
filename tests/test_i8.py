"""8-bit matrices without a GPU: sizes, refusals, tile rules."""
import ctypes

import pytest

import paper_2508_12851_amd as P
import i8_reference as R
from ffn_paths import cuts_last_round, ffn_path, packs_rows

P0 = ctypes.c_void_p(0x10000)       # never dereferenced


def _bytes(rows, cols):
    n = ctypes.c_size_t(0)
    return P.load_library().prism_i8_bytes(rows, cols, ctypes.byref(n)), n.value


@pytest.mark.parametrize("rows,cols,elements", [(1, 1, 16 * 128), (16, 128, 16 * 128), (17, 129, 32 * 256), (14336, 4096, 14336 * 4096)])
def test_size(rows, cols, elements):
    status, n = _bytes(rows, cols)
    from paper_2508_12851_amd import binding
    assert binding._i8_bytes(rows, cols) == n
    assert status == 0 and n == -(-(elements + 4 * (-(-rows // 16) * 16)) // 256) * 256


def test_size_refusals():
    assert _bytes(0, 4)[0] == 1 and _bytes(4, 0)[0] == 1 and _bytes(4, 130945)[0] == 2 and _bytes(4, 130944)[0] == 0
    assert P.load_library().prism_i8_bytes(4, 4, None) == 1


def test_quantize_refusals_before_any_launch():
    def call(src=P0, dtype=1, ld=64, rows=4, cols=64, dst=P0):
        return P.load_library().prism_quantize_i8(src, dtype, ld, rows, cols, dst, None)
    assert call(src=None) == 1 and call(dst=None) == 1 and call(dst=ctypes.c_void_p(0x10008)) == 1
    assert call(src=ctypes.c_void_p(0x10001)) == 1 and call(dtype=0, src=ctypes.c_void_p(0x10002)) == 1
    assert call(dtype=2) == 1 and call(ld=63) == 1 and call(rows=-1) == 1 and call(cols=0) == 1
    assert call(cols=130945, ld=130945) == 2
    assert call(rows=0, src=None, dst=None) == 0


def test_pack_refusals_before_any_launch():
    def call(src=P0, ld=64, scale=P0, rows=4, cols=64, dst=P0):
        return P.load_library().prism_pack_i8(src, ld, scale, rows, cols, dst, None)
    assert call(src=None) == 1 and call(scale=None) == 1 and call(dst=None) == 1 and call(dst=ctypes.c_void_p(0x10004)) == 1
    assert call(ld=63) == 1 and call(rows=0) == 1 and call(cols=0) == 1 and call(cols=130945, ld=130945) == 2


def test_matmul_refusals_before_any_launch():
    lib = P.load_library()
    n = ctypes.c_size_t(0)
    assert lib.prism_matmul_i8_workspace_bytes(100, 64, 64, ctypes.byref(n)) == 0
    size = n.value

    def call(a=P0, b=P0, m=4, n=64, k=64, out=P0, ldo=64, dtype=1, ws=P0, size=size):
        return lib.prism_matmul_i8(a, b, m, n, k, out, ldo, dtype, ws, size, None)
    for name in ("a", "b", "out", "ws"):
        assert call(**{name: None}) == 1, name
    assert call(a=ctypes.c_void_p(0x10008)) == 1 and call(b=ctypes.c_void_p(0x10008)) == 1
    assert call(ws=ctypes.c_void_p(0x10010)) == 1 and call(out=ctypes.c_void_p(0x10001)) == 1
    assert call(out=ctypes.c_void_p(0x10002), dtype=0) == 1
    assert call(m=-1) == 1 and call(n=0) == 1 and call(k=0) == 1 and call(ldo=63) == 1 and call(dtype=3) == 1
    assert call(k=130945) == 2
    assert call(size=0) == 3
    big = ctypes.c_size_t(0)
    assert lib.prism_matmul_i8_workspace_bytes(40_000_000, 64, 64, ctypes.byref(big)) == 0
    assert call(m=40_000_000, size=big.value) == 2          # 4 GiB and more of one operand
    assert call(m=0, a=None, b=None, out=None, ws=None) == 0
    for args in ((-1, 4, 4), (4, 0, 4), (4, 4, 0)):
        assert lib.prism_matmul_i8_workspace_bytes(*args, ctypes.byref(n)) == 1
    assert lib.prism_matmul_i8_workspace_bytes(4, 4, 4, None) == 1
    assert lib.prism_matmul_i8_workspace_bytes(4, 4, 130945, ctypes.byref(n)) == 2


def test_workspace_for_most_rows_serves_fewer():
    lib, n, sizes = P.load_library(), ctypes.c_size_t(0), []
    for m in (*range(0, 300), 512, 1000, 5000, 100000):
        assert lib.prism_matmul_i8_workspace_bytes(m, 1411, 4096, ctypes.byref(n)) == 0
        sizes.append(n.value)
    assert sizes == sorted(sizes)


def test_layer_description():
    lib, n = P.load_library(), ctypes.c_size_t(0)

    def status(hidden=128, ffn=192, dtype="bf16"):
        d = P.make_desc(hidden, ffn, 8, 2, 1, dtype, weight_layout="int8")
        return lib.prism_workspace_bytes(ctypes.byref(d), 16, ctypes.byref(n))
    assert status() == 0 and status(dtype="f32") == 2 and status(hidden=100) == 2 and status(ffn=32) == 2
    assert status(ffn=130944 + 64) == 2 and status(hidden=64, ffn=64) == 0
    d = P.make_desc(2048, 1408, 60, 4, 4, "bf16", weight_layout="int8")
    sizes = [P.workspace_bytes(d, t) for t in (*range(0, 700), 1000, 4096)]
    assert sizes == sorted(sizes)
    row_major = P.make_desc(2048, 1408, 60, 4, 4, "bf16")
    assert P.workspace_bytes(d, 64) > P.workspace_bytes(row_major, 64)


@pytest.mark.parametrize("T", [1, 64, 65, 200, 300, 512, 513, 700, 4096])
def test_tile_rules_count_bytes(T):
    """A ring of tiles is never longer than the contraction, which is counted in bytes: 64 a k-tile, rows padded to 128."""
    need = {"kDecodeTiled": 7, "kDecode": 6, "kDecodeShort": 2, "kStream": 6, "kSplitSquare": 6, "kSplitWide": 4,
            "kFewRows64": 6, "kFewRows128": 6, "kPrefill": 3, "kPrefillShort": 2}
    for H, F in ((64, 64), (128, 192), (192, 448), (256, 256), (320, 8192), (384, 384), (512, 2048), (2048, 1408), (4096, 14336)):
        for E, k, S in ((8, 2, 0), (64, 6, 2), (4, 1, 0)):
            path = ffn_path(H, F, E, k, S, T, 2)
            assert min(-(-H // 128), -(-F // 128)) * 2 >= need[path], (H, F, path)


def test_tile_rules_of_the_usual_sizes():
    assert ffn_path(4096, 14336, 8, 2, 0, 32, 2) == "kDecodeTiled"
    assert ffn_path(4096, 14336, 8, 2, 0, 200, 2) == "kStream"
    assert ffn_path(4096, 14336, 8, 2, 0, 300, 2) == "kSplitWide"
    assert ffn_path(2048, 1408, 60, 4, 4, 333, 2) == "kFewRows128"
    assert ffn_path(4096, 14336, 8, 2, 0, 4096, 2) == "kPrefill"
    assert ffn_path(64, 64, 8, 2, 0, 65, 2) == "kPrefillShort"


def test_the_layers_of_the_tests_reach_every_path():
    at = [(H, F, E, k, S, T, 2) for H, F, E, k, S, T, _ in R.SHAPES]
    assert {ffn_path(*a) for a in at} == {"kDecodeTiled", "kDecode", "kDecodeShort", "kStream", "kSplitSquare", "kSplitWide",
                                          "kFewRows64", "kFewRows128", "kPrefill", "kPrefillShort"}
    assert any(packs_rows(*a) for a in at) and any(cuts_last_round(*a) for a in at)
