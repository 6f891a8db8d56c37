"""8-bit matrices, their product and layers with 8-bit expert weights on the GPU, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2508_12851_amd as P
import i8_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(rows, cols, dtype, seed, std=1.0):
    return (torch.randn((rows, cols), generator=_gen(seed), device="cuda") * std).to(dtype)


def _check_quantized(m, v):
    q, scale = m.values()
    want, want_scale = R.quantize(v)
    assert torch.equal(scale.double(), want_scale)
    assert torch.equal(q.double(), want)


# ---- quantisation ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (16, 64), (17, 65), (5, 127), (33, 128), (2, 129), (1, 1408), (77, 1411), (1000, 256),
                                       (3, 4096), (2, 14336), (2, 16384), (3, 16391), (2, 40000)])
def test_quantize(rows, cols, dtype):
    v = _rows(rows, cols, dtype, rows * 7 + cols)
    m = P.prism_quantize_i8(v)
    _check_quantized(m, v)
    # zeros behind the columns, as far as the library multiplies
    R16, C = -(-rows // 16) * 16, -(-cols // 128) * 128
    tiles = m.data[:R16 * C].view(R16 // 16, C // 64, 16, 64).permute(0, 2, 1, 3).reshape(R16, C)
    assert int(tiles[:rows, cols:].abs().sum() if cols < C else 0) == 0


def test_quantize_halves_are_ties_to_even():
    """bf16 rows with elements at every multiple of half a step."""
    steps = torch.arange(-254, 255, device="cuda").float() / 2
    for top in (127.0, 127.0 * 2 ** -40, 127.0 * 2 ** 60):
        v = (steps * (top / 127.0)).to(BF16)[None].contiguous()
        assert torch.equal(v.float()[0] * (127.0 / top), steps)
        m = P.prism_quantize_i8(v)
        _check_quantized(m, v)
    v = _rows(2000, 512, BF16, 3)               # and wherever rows have an element of half the largest's digits
    v[:, 7] = v.abs().amax(1) / 2
    _check_quantized(P.prism_quantize_i8(v), v)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantize_of_all_magnitudes(dtype):
    """Rows from the smallest subnormal to the largest finite value, rows of zeros among them."""
    v = _rows(64, 300, F32, 5).clamp(-3, 3) / 3
    exps = torch.linspace(-149, 127, 64, device="cuda").round()
    v = (v.double() * torch.pow(2.0, exps.double())[:, None]).to(dtype)
    v[10] = 0.0
    v[11] = -0.0
    v[12, 1:] = 0.0
    v[13] = torch.finfo(dtype).max
    v[14] = torch.finfo(dtype).min
    v[15] = 0.0
    v[15, 3] = 2.0 ** -149 if dtype == F32 else 2.0 ** -133
    _check_quantized(P.prism_quantize_i8(v), v)


def test_quantize_says_by_the_scale_that_a_row_is_not_finite():
    v = _rows(4, 100, F32, 6)
    v[1, 50] = float("nan")
    v[2, 99] = float("-inf")
    q, scale = P.prism_quantize_i8(v).values()
    assert torch.isnan(scale[1]) and torch.isinf(scale[2]) and torch.isfinite(scale[[0, 3]]).all()
    _check_quantized(P.prism_quantize_i8(v[[0, 3]].contiguous()), v[[0, 3]])
    out = P.prism_matmul_i8(P.prism_quantize_i8(v), P.prism_quantize_i8(_rows(5, 100, F32, 7)), P.alloc_matmul_i8_workspace(4, 5, 100))
    assert not torch.isfinite(out[[1, 2]]).any() and torch.isfinite(out[[0, 3]]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset,ld", [(0, 520), (1, 515), (8, 513), (3, 600)])
def test_quantize_strides_and_addresses(dtype, offset, ld):
    buf = _rows(1, 40 * ld + offset, dtype, offset + ld)[0]
    v = torch.as_strided(buf, (40, 513), (ld, 1), offset)
    _check_quantized(P.prism_quantize_i8(v), v)


def test_pack_keeps_bytes_and_scales():
    for rows, cols, ld in ((1, 1, 1), (33, 130, 130), (16, 128, 144), (7, 1411, 1411), (50, 4096, 4097)):
        buf = torch.randint(-128, 128, (rows, ld), generator=_gen(rows), device="cuda", dtype=torch.int8)
        scale = torch.rand(rows, generator=_gen(rows), device="cuda")
        q, s = P.prism_pack_i8(buf[:, :cols], scale).values()
        assert torch.equal(q, buf[:, :cols]) and torch.equal(s, scale)


# ---- the product ----------------------------------------------------------------------------
def _weights(n, k, seed):
    q = torch.randint(-127, 128, (n, k), generator=_gen(seed), device="cuda", dtype=torch.int8)
    return q, torch.rand(n, generator=_gen(seed + 1), device="cuda") / 100 + 1e-3


def _check_product(m, n, k, dtype=F32, out=None, seed=0):
    v = _rows(m, k, BF16, seed + m)
    q, scale = R.quantize(v)
    w, ws = _weights(n, k, seed)
    ws_buf = P.alloc_matmul_i8_workspace(m, n, k)
    ws_buf.fill_(255)
    got = P.prism_matmul_i8(P.prism_quantize_i8(v), P.prism_pack_i8(w, ws), ws_buf, out=out, dtype=dtype)
    want = R.product(q, scale, w, ws)
    # at most 8 parts: the conversion of a sum, the product of the scales, theirs and the addition, 4 roundings of each
    sums = (q.abs() @ w.double().abs().t()) * scale[:, None] * ws.double()
    tol = 4 * R.EPS * sums + (R.EPS if dtype == F32 else 2.0 ** -8) * want.abs() * (1 + 2.0 ** -8)
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 64), (1, 4096, 4096), (2, 77, 129), (15, 1000, 333), (64, 128, 8192), (64, 130, 500),
                                   (65, 129, 100), (77, 2053, 1411), (100, 100, 4096), (128, 128, 128), (129, 257, 383), (200, 3000, 4096),
                                   (600, 4096, 2048), (1000, 999, 1000), (2048, 8192, 512), (4100, 4099, 130), (4097, 4352, 64)])
def test_product(m, n, k, dtype):
    _check_product(m, n, k, dtype)


@pytest.mark.parametrize("m", [1, 3, 16, 17, 31, 33, 48, 63, 64, 65, 96, 127, 128, 255, 256, 257, 300])
def test_product_row_counts(m):
    _check_product(m, 320, 704, BF16)
    _check_product(m, 14336, 256, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset,ldo", [(0, 144), (1, 133), (2, 134), (4, 131)])
def test_product_into_a_part_of_a_wider_matrix(dtype, offset, ldo):
    for m in (5, 70):
        for k in (100, 4096):                   # without and with contractions that are shared
            buf = torch.full((m * ldo + offset + 8,), 7.0, dtype=dtype, device="cuda")
            out = torch.as_strided(buf, (m, 131), (ldo, 1), offset)
            _check_product(m, 131, k, dtype, out=out)
            rest = torch.ones_like(buf, dtype=torch.bool)
            torch.as_strided(rest, (m, 131), (ldo, 1), offset).fill_(False)
            assert bool((buf[rest] == 7.0).all())


@pytest.mark.parametrize("value", [127, -128])
def test_product_of_the_largest_sums(value):
    k = 130944
    a = torch.full((3, k), value, dtype=torch.int8, device="cuda")
    b = torch.full((70, k), value, dtype=torch.int8, device="cuda")
    b[1] = 127 if value < 0 else -127
    one = torch.ones(70, device="cuda")
    got = P.prism_matmul_i8(P.prism_pack_i8(a, one[:3]), P.prism_pack_i8(b, one), P.alloc_matmul_i8_workspace(3, 70, k), dtype=F32)
    want = a.double() @ b.double().t()
    assert bool(((got.double() - want).abs() <= 4 * R.EPS * want.abs()).all())


def test_product_with_no_rows_and_of_zero_rows():
    w, s = _weights(70, 100, 1)
    b = P.prism_pack_i8(w, s)
    empty = P.prism_quantize_i8(torch.empty((0, 100), device="cuda"))
    assert P.prism_matmul_i8(empty, b, P.alloc_matmul_i8_workspace(0, 70, 100)).shape == (0, 70)
    zero = P.prism_quantize_i8(torch.zeros((3, 100), device="cuda"))
    assert int(P.prism_matmul_i8(zero, b, P.alloc_matmul_i8_workspace(3, 70, 100)).abs().sum()) == 0


def test_product_in_a_graph_and_on_another_stream():
    m, n, k = 20, 1000, 4096
    w, s = _weights(n, k, 4)
    b, ws = P.prism_pack_i8(w, s), P.alloc_matmul_i8_workspace(m, n, k)
    v, a = _rows(m, k, BF16, 1), P.prism_quantize_i8(_rows(m, k, BF16, 9))
    out = torch.empty((m, n), dtype=BF16, device="cuda")

    def step(stream=None):
        P.prism_matmul_i8(P.prism_quantize_i8(v, out=a, stream=stream), b, ws, out=out, stream=stream)
    step()
    want = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for i in range(3):
        v.copy_(_rows(m, k, BF16, 20 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        assert torch.equal(out, got)


# ---- experts --------------------------------------------------------------------------------
class Layer:
    """A server's layer with 8-bit expert weights, its tokens and the 64-bit reference of its rows."""

    def __init__(self, H, F, E, k, S, T, hosted, seed=0, gates="renormalized"):
        self.H, self.F, self.E, self.k, self.S, self.T = H, F, E, k, S, T
        self.desc = P.make_desc(H, F, E, k, S, "bf16", gate_mode=gates, weight_layout="int8")
        gen = _gen(seed)
        self.x = torch.randn((T, H), generator=gen, device="cuda").to(BF16)
        self.router = (torch.randn((E, H), generator=gen, device="cuda") / H ** 0.5).to(BF16)
        self.bias = torch.randn((1, E), generator=gen, device="cuda")
        self.mask = torch.zeros(E, dtype=torch.uint8)
        self.mask[list(hosted)] = 1
        self.mask = self.mask.cuda()

        def triple():
            out = []
            for n, kk in ((F, H), (F, H), (H, F)):
                w = torch.randn((n, kk), generator=gen, device="cuda") / kk ** 0.5
                out.append(P.prism_quantize_i8(w))
            return out
        self.experts = {e: triple() for e in hosted}
        self.shared = [triple() for _ in range(S)]
        self.table = P.WeightTable([tuple(m.data for m in self.experts[e]) if e in self.experts else None for e in range(E)],
                                   [tuple(m.data for m in t) for t in self.shared])
        self.ws = P.alloc_workspace(self.desc, T)
        self.ws.fill_(255)

    def route(self):
        r = P.prism_route(self.desc, self.x, self.router, self.bias)
        return r, P.prism_dispatch(self.desc, r.topk_idx, self.mask, self.ws)

    def check_rows(self, y, local_src, local_offsets):
        at, T = local_offsets.tolist(), self.T
        pieces = [(at[e], at[e + 1], local_src[at[e]:at[e + 1]].long() // self.k, t) for e, t in self.experts.items()]
        pieces += [(T * self.k + s * T, T * self.k + (s + 1) * T, torch.arange(T, device="cuda"), t) for s, t in enumerate(self.shared)]
        for first, last, tokens, t in pieces:
            if first == last:
                continue
            want, off = R.swiglu(self.x[tokens], *(m.values() for m in t))
            err = (y[first:last].double() - want).abs()
            tol = 2.0 ** -8 * (want.abs() + off) + off
            assert bool((err <= tol).all()), (first, float((err / (tol + 1e-30)).max()))
        assert bool((y[at[-1]:T * self.k] == 0).all())


SHAPES = R.SHAPES


@pytest.mark.parametrize("H,F,E,k,S,T,hosted", SHAPES)
def test_expert_ffn(H, F, E, k, S, T, hosted):
    layer = Layer(H, F, E, k, S, T, hosted, seed=H + T)
    _, s = layer.route()
    layer.ws.fill_(255)
    y = P.prism_expert_ffn(layer.desc, layer.x, layer.table, s.local_src, s.local_offsets, layer.ws)
    layer.check_rows(y, s.local_src, s.local_offsets)
    again = P.prism_expert_ffn(layer.desc, layer.x, layer.table, s.local_src, s.local_offsets, layer.ws)
    assert torch.equal(y, again)
    # a caller's y: rows that hold no assignment stay as they are
    mine = torch.full_like(y, 5.0)
    P.prism_expert_ffn(layer.desc, layer.x, layer.table, s.local_src, s.local_offsets, layer.ws, y=mine)
    n = int(s.local_offsets[-1])
    assert torch.equal(mine[:n], y[:n]) and torch.equal(mine[T * k:], y[T * k:]) and bool((mine[n:T * k] == 5.0).all())


@pytest.mark.parametrize("T", [1, 40, 200, 333, 700])
def test_nothing_hosted_and_uneven_lists(T):
    layer = Layer(512, 1024, 8, 2, 0, T, (2, 5), seed=T)
    none = torch.zeros(9, dtype=torch.int32, device="cuda")
    src = torch.full((2 * T,), -1, dtype=torch.int32, device="cuda")
    y = torch.full((2 * T, 512), 5.0, dtype=BF16, device="cuda")
    P.prism_expert_ffn(layer.desc, layer.x, layer.table, src, none, layer.ws, y=y)
    assert bool((y == 5.0).all())
    # a caller's own list: it starts behind row 0, and one expert has all of it
    first = T // 3
    src[first:2 * T] = torch.arange(2 * T - first, dtype=torch.int32, device="cuda").flip(0)
    offsets = torch.tensor([first] * 6 + [2 * T] * 3, dtype=torch.int32, device="cuda")
    y = P.prism_expert_ffn(layer.desc, layer.x, layer.table, src, offsets, layer.ws)
    assert bool((y[:first] == 0).all())
    layer.check_rows(y, src, offsets)


@pytest.mark.parametrize("gates", ["renormalized", "softmax_all"])
@pytest.mark.parametrize("H,F,E,k,S,T,hosted", [SHAPES[i] for i in (0, 1, 5, 7, 9, 12, 13, 15, 17)])
def test_layer_is_its_steps(H, F, E, k, S, T, hosted, gates):
    """Whole layer: routing and lists of the bf16 layer, the sum of the expert rows of the separate call, bit for bit."""
    layer = Layer(H, F, E, k, S, T, hosted, seed=H + T, gates=gates)
    r, s = layer.route()
    y = P.prism_expert_ffn(layer.desc, layer.x, layer.table, s.local_src, s.local_offsets, layer.ws)
    out = P.prism_combine(layer.desc, y, s.local_src, s.local_offsets, r.topk_gate, layer.ws)
    layer.ws.fill_(255)
    o = P.prism_moe_layer(layer.desc, layer.x, layer.router, layer.bias, layer.table, layer.mask, layer.ws)
    assert torch.equal(o.topk_idx, r.topk_idx) and torch.equal(o.counts, r.counts)
    assert torch.equal(o.n_local_remote, s.n_local_remote) and torch.equal(o.remote_offsets, s.remote_offsets)
    assert torch.equal(o.out, out)
    P.prism_debug_check_weights(layer.desc, layer.table, layer.mask)
    if P.workspace_bytes(layer.desc, T) <= P.STATIC_SCRATCH_BYTES:
        got = P.alloc_layer_out(layer.desc, T)
        P.prism_moe_layer_static(layer.desc, layer.x, layer.router, layer.bias, layer.table, layer.mask, got)
        assert torch.equal(got.out, out)


def test_remote_call_with_8_bit_experts():
    """Two servers that host half of the experts each: local part, rows shipped, served by the other, added."""
    T, H, F, E, k = 150, 256, 512, 8, 2
    whole = Layer(H, F, E, k, 1, T, range(E), seed=1)
    r, s = whole.route()
    y = P.prism_expert_ffn(whole.desc, whole.x, whole.table, s.local_src, s.local_offsets, whole.ws)
    want = P.prism_combine(whole.desc, y, s.local_src, s.local_offsets, r.topk_gate, whole.ws)
    mask = whole.mask.clone()
    mask[4:] = 0
    s = P.prism_dispatch(whole.desc, r.topk_idx, mask, whole.ws)
    y = P.prism_expert_ffn(whole.desc, whole.x, whole.table, s.local_src, s.local_offsets, whole.ws)
    out = P.prism_combine(whole.desc, y, s.local_src, s.local_offsets, r.topk_gate, whole.ws)
    packed = P.prism_pack_remote(whole.desc, whole.x, s.remote_src, s.remote_offsets)
    n = int(s.n_local_remote[1])
    peer = P.make_desc(H, F, E, 1, 0, "bf16", weight_layout="int8")
    rows = torch.arange(n, dtype=torch.int32, device="cuda")
    served = P.prism_expert_ffn(peer, packed[:n].contiguous(), whole.table, rows, s.remote_offsets, P.alloc_workspace(peer, n))
    P.prism_combine_remote(whole.desc, served, s.remote_src, s.remote_offsets, r.topk_gate, out, whole.ws)
    # the sum is rounded to bf16 once more
    err = (out.double() - want.double()).abs()
    assert bool((err <= 2.0 ** -7 * (want.double().abs() + out.double().abs()) + 2.0 ** -7 * want.double().abs().max()).all())


@pytest.mark.parametrize("T", [1, 32, 200, 600])
def test_layer_in_a_graph_and_on_two_streams(T):
    layer = Layer(512, 2048, 8, 2, 1, T, range(5), seed=3)
    out = P.alloc_layer_out(layer.desc, T)

    def step(o, ws, stream=None):
        P.prism_moe_layer(layer.desc, layer.x, layer.router, layer.bias, layer.table, layer.mask, ws, outputs=o, stream=stream)
    step(out, layer.ws)
    want = out.out.clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [P.alloc_layer_out(layer.desc, T) for _ in range(2)]
    wss = [P.alloc_workspace(layer.desc, T) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for o, ws, st in zip(outs, wss, streams):
            step(o, ws, st)
    torch.cuda.synchronize()
    assert all(torch.equal(o.out, want) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, layer.ws, torch.cuda.current_stream())
    for i in range(3):
        layer.x.copy_(_rows(T, 512, BF16, 30 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = out.out.clone()
        step(outs[0], wss[0])
        assert torch.equal(outs[0].out, got)


def test_no_tokens():
    layer = Layer(256, 512, 8, 2, 1, 0, range(8))
    o = P.prism_moe_layer(layer.desc, layer.x, layer.router, layer.bias, layer.table, layer.mask, layer.ws)
    assert o.out.shape == (0, 256) and int(o.counts.sum()) == 0


def test_layer_with_stage_events():
    import ctypes
    layer = Layer(512, 2048, 8, 2, 1, 40, range(5), seed=3)
    want = P.prism_moe_layer(layer.desc, layer.x, layer.router, layer.bias, layer.table, layer.mask, layer.ws)
    events = [torch.cuda.Event(enable_timing=True) for _ in range(2 * len(P.STAGES))]
    for e in events:
        e.record()                                # (makes the handles)
    handles = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    got = P.prism_moe_layer(layer.desc, layer.x, layer.router, layer.bias, layer.table, layer.mask, layer.ws, stage_events=handles)
    torch.cuda.synchronize()
    assert torch.equal(got.out, want.out)
    assert all(events[2 * i].elapsed_time(events[2 * i + 1]) >= 0 for i in range(len(P.STAGES)))


def test_decode_loop_with_8_bit_experts():
    from paper_2508_12851_amd.decode_sweep import Stack, sweep
    st = Stack(n_layers=2, T=24, H=256, F=512, E=8, k=2, seed=5, weights="int8")
    ref = Stack(n_layers=2, T=24, H=256, F=512, E=8, k=2, seed=5)
    masks = st.masks_hosting(8)
    got, want = st.step(masks).double(), ref.step(masks).double()
    # Weights, tokens and h in 8 bits: a row's step is its largest value / 127, 3.5 rms / 127 in a normal row of 256 or 512, 8 rms / 127 in
    # one of h, and its rounding errors are 0.29 steps: 0.8 % of each of x and the weights, 1.8 % of h, together below 3 % of a
    # layer's output, which is no larger than the x it is added to.
    assert float((got - want).norm() / want.norm()) < 0.05
    rows = sweep(n_layers=2, T=16, H=256, F=512, E=8, k=2, steps=2, warmup=1, weights="int8")
    assert rows[-1]["weight_bytes_streamed_per_step"] % (3 * 256 * 512) == 0 and rows[-1]["weights"] == "int8"


# ---- beyond 32-bit offsets ---------------------------------------------------------------------
def test_h_beyond_4_gib():
    T, H, F, E, k = 40000, 256, 14336, 4, 2
    layer = Layer(H, F, E, k, 0, T, range(E), seed=4)
    _, s = layer.route()
    y = P.prism_expert_ffn(layer.desc, layer.x, layer.table, s.local_src, s.local_offsets, layer.ws)
    at = s.local_offsets.tolist()
    assert at[-1] * F * 4 > 1 << 32
    for e in range(E):                            # the first, the last and some rows of every expert
        rows = torch.unique(torch.cat([torch.tensor([at[e], at[e + 1] - 1]), torch.randint(at[e], at[e + 1], (60,), generator=torch.Generator().manual_seed(e))])).cuda()
        want, off = R.swiglu(layer.x[s.local_src[rows].long() // k], *(m.values() for m in layer.experts[e]))
        err = (y[rows].double() - want).abs()
        assert bool((err <= 2.0 ** -8 * (want.abs() + off) + off).all())


def test_product_and_quantisation_beyond_4_gib():
    m, n, k = 300001, 4096, 128
    v = _rows(m, k, BF16, 1)
    w, ws = _weights(n, k, 2)
    out = P.prism_matmul_i8(P.prism_quantize_i8(v), P.prism_pack_i8(w, ws), P.alloc_matmul_i8_workspace(m, n, k), dtype=F32)
    rows = torch.cat([torch.arange(0, m, 1009), torch.arange(m - 40, m)]).cuda()
    q, scale = R.quantize(v[rows])
    want = R.product(q, scale, w, ws)
    sums = (q.abs() @ w.double().abs().t()) * scale[:, None] * ws.double()
    assert bool(((out[rows].double() - want).abs() <= 4 * R.EPS * sums + R.EPS * want.abs() * (1 + 2.0 ** -8)).all())
    quantised = P.prism_quantize_i8(out)          # 4.9 GB in
    q, scale = quantised.values()
    want, want_scale = R.quantize(out[rows])
    assert torch.equal(q[rows].double(), want) and torch.equal(scale[rows].double(), want_scale)


def test_router_and_experts_of_a_training_step():
    """The layer's forward with 8-bit experts, and its router's gradient from the same logits."""
    layer = Layer(256, 512, 16, 4, 0, 300, range(16), seed=8, gates="softmax_all")
    r, s = layer.route()
    y = P.prism_expert_ffn(layer.desc, layer.x, layer.table, s.local_src, s.local_offsets, layer.ws)
    out = P.prism_combine(layer.desc, y, s.local_src, s.local_offsets, r.topk_gate, layer.ws)
    b = P.prism_balance_loss(layer.desc, r.logits, r.topk_idx, P.alloc_balance_workspace(layer.desc), group_tokens=100)
    assert torch.equal(b.counts.sum(0).int(), r.counts)
    # d(sum of out * t) / d gate[t, j] = the expert row of the pick, times t
    t = _rows(300, 256, BF16, 2)
    inv = torch.empty(300 * 4, dtype=torch.int64, device="cuda")
    inv[s.local_src.long()] = torch.arange(300 * 4, device="cuda")
    rows = y.float()[inv].view(300, 4, 256)
    d_gate = (rows * t.float()[:, None]).sum(2).contiguous()
    d = P.prism_route_backward(layer.desc, r.logits, r.topk_idx, b, torch.full((3,), 0.01, device="cuda"), d_gate, group_tokens=100)

    def value(logits):                          # in 64 bits, the picks and counts held
        p = torch.softmax(logits, 1)
        gate = p.gather(1, r.topk_idx.long())
        probs = p.view(3, 100, 16).mean(1)
        return (gate * d_gate.double()).sum() + 0.01 * (16 / (4 * 100) * (b.counts.double() * probs).sum())
    logits = r.logits.double()
    for e in range(3):
        direction = torch.randn(logits.shape, generator=_gen(e), device="cuda", dtype=torch.float64)
        slope = (value(logits + 1e-5 * direction) - value(logits - 1e-5 * direction)) / 2e-5
        want = (d.double() * direction).sum()
        assert abs(float(slope - want)) <= 1e-4 * float((d.double() * direction).abs().sum())
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("call", ["quantize", "pack", "matmul", "balance", "backward"])
def test_outputs_of_another_stream_do_not_take_memory_that_this_one_still_reads(call):
    desc = P.make_desc(64, 64, 256, 8)
    v = _rows(512, 512, F32, 1)
    q, scale = P.prism_quantize_i8(v).values()
    a, b, ws = P.prism_quantize_i8(v), P.prism_quantize_i8(v), P.alloc_matmul_i8_workspace(512, 512, 512)
    logits = _rows(1024, 256, F32, 2)
    idx, wsb = logits.topk(8, 1).indices.int(), P.alloc_balance_workspace(desc)
    d_gate = _rows(1024, 8, F32, 3)
    run, nbytes = {"quantize": (lambda s: P.prism_quantize_i8(v, stream=s).data, a.data.numel()),
                   "pack": (lambda s: P.prism_pack_i8(q, scale, stream=s).data, a.data.numel()),
                   "matmul": (lambda s: P.prism_matmul_i8(a, b, ws, dtype=F32, stream=s), 512 * 512 * 4),
                   "balance": (lambda s: P.prism_balance_loss(desc, logits, idx, wsb, group_tokens=1, stream=s).probs, 1024 * 256 * 4),
                   "backward": (lambda s: P.prism_route_backward(desc, logits, idx, d_gate=d_gate, stream=s), 1024 * 256 * 4)}[call]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = run(None).clone()
    old = [torch.full((nbytes,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
    kept = [torch.empty_like(o) for o in old]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for k, o in zip(kept, old):
        k.copy_(o)
    del old, o                       # freed here, read later by this stream
    got = run(side)
    torch.cuda.synchronize()
    assert all(bool((k == 77).all()) for k in kept)
    assert torch.equal(got, want)


def test_binding_refuses_what_does_not_fit():
    a, b = P.prism_quantize_i8(_rows(4, 64, BF16, 1)), P.prism_quantize_i8(_rows(5, 65, BF16, 1))
    ws = P.alloc_matmul_i8_workspace(4, 5, 65)
    with pytest.raises(P.PrismError):
        P.prism_matmul_i8(a, b, ws)
    with pytest.raises(P.PrismError):
        P.prism_quantize_i8(_rows(64, 4, BF16, 1).t())
    with pytest.raises(P.PrismError):
        P.prism_quantize_i8(_rows(4, 64, BF16, 1).half())
    with pytest.raises(P.PrismError):
        P.prism_pack_i8(torch.zeros((4, 4), device="cuda"), torch.ones(4, device="cuda"))
    with pytest.raises(P.PrismError):
        P.prism_matmul_i8(b, b, ws, out=torch.empty((5, 4), device="cuda"))
    with pytest.raises(P.PrismError):
        P.prism_matmul_i8(b, b, ws, out=torch.empty((5, 5), device="cuda", dtype=torch.float16))
    with pytest.raises(P.PrismError):
        P.prism_quantize_i8(_rows(4, 64, BF16, 1), out=b)
    with pytest.raises(P.PrismError):
        P.I8Matrix(a.data, 4, 129)
    with pytest.raises(P.PrismError):
        P.prism_quantize_i8(torch.as_strided(_rows(1, 200, BF16, 1)[0], (4, 64), (32, 1)))   # rows that overlap
