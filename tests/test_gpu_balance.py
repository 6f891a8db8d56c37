"""Balance loss, counts and router gradient on the GPU against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2508_12851_amd as P
import balance_reference as R

pytestmark = pytest.mark.gpu


def _inputs(T, E, k, group, masked, seed, spread=3.0):
    rng = np.random.default_rng(seed)
    logits = (rng.standard_normal((T, E)) * spread / 3).clip(-2 * spread, 2 * spread).astype(np.float32)
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :k].astype(np.int32)
    mask = None
    if masked:
        mask = (rng.random(T) > 0.4).astype(np.uint8)
        if group and T > 2 * group:
            mask[group:2 * group] = 0            # a group without tokens
        logits[mask == 0] = np.array([np.nan, np.inf, -np.inf])[rng.integers(0, 3, ((mask == 0).sum(), E))]
        idx[mask == 0] = rng.integers(-5, 3 * E, ((mask == 0).sum(), k))
    G = 1 if group == 0 else -(-T // group)
    d_loss = rng.standard_normal(G).astype(np.float32)
    d_gate = rng.standard_normal((T, k)).astype(np.float32)
    if masked:
        d_gate[mask == 0] = np.nan
    return logits, idx, mask, d_loss, d_gate


def _dev(a, offset=0):
    """On the device, `offset` elements behind an aligned address."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a))
    buf = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    buf[offset:].copy_(t.reshape(-1))
    return buf[offset:].view(t.shape)


def _check(E, k, group, mode, logits, idx, mask, d_loss, d_gate, offset=0, use_loss=True, use_gate=True, spread=6.0):
    desc = P.make_desc(64, 64, E, k, gate_mode=mode)
    ws = P.alloc_balance_workspace(desc)
    ws.fill_(255)
    dl, di, dm = _dev(logits, offset), _dev(idx), _dev(mask)
    b = P.prism_balance_loss(desc, dl, di, ws, dm, group)
    loss, counts, probs, n = R.balance(logits, idx, mask, group, E, k)
    assert np.array_equal(b.counts.cpu().numpy(), counts)
    assert np.array_equal(b.n_tokens.cpu().numpy(), n)
    # p as derived, the fp32 additions of a workgroup's rows (at most one per row a lane adds, 16 here, and 10 more), one rounding
    tol = R.relative_error_of_p(2 * spread) + (16 + 10 + 1) * R.EPS
    assert np.all(np.abs(b.probs.cpu().numpy() - probs) <= tol * probs + 1e-38)
    assert np.all(np.abs(b.loss.cpu().numpy() - loss) <= (tol + R.EPS) * np.abs(loss))
    got = P.prism_route_backward(desc, dl, di, b if use_loss else None, _dev(d_loss) if use_loss else None,
                                 _dev(d_gate) if use_gate else None, dm, group, d_logits=_dev(np.full(logits.shape, 7, np.float32), offset))
    d, size = R.backward(logits, idx, mask, group, E, k, d_loss if use_loss else None, d_gate if use_gate else None, mode)
    # every term of the sums has the errors of a p twice (its own and the mean's) and a few roundings
    tol = 2 * R.relative_error_of_p(2 * spread) + 12 * R.EPS
    err = np.abs(got.cpu().numpy() - d)
    assert np.all(err <= tol * size + 1e-38), float(np.max(err / (size + 1e-30)))
    return b, got


@pytest.mark.parametrize("E", [1, 2, 3, 4, 5, 8, 13, 16, 17, 32, 33, 60, 64, 100, 128, 129, 255, 256])
@pytest.mark.parametrize("T,group,masked", [(1, 0, False), (67, 0, True), (130, 33, True)])
def test_every_row_layout(E, T, group, masked):
    k = min(E, 1 + E % 8)
    for mode in ("renormalized", "softmax_all"):
        _check(E, k, group, mode, *_inputs(T, E, k, group, masked, E * 7 + T))


@pytest.mark.parametrize("T,E,k,group", [(2, 8, 2, 1), (63, 4, 4, 64), (4099, 8, 2, 0), (4099, 64, 6, 512), (2500, 256, 8, 0),
                                         (2049, 7, 3, 1000), (20011, 16, 2, 0), (9000, 33, 8, 1)])
@pytest.mark.parametrize("masked", [False, True])
def test_sizes_and_groups(T, E, k, group, masked):
    _check(E, k, group, "renormalized", *_inputs(T, E, k, group, masked, T + E))


def test_groups_that_several_workgroups_share():
    """Their sums are made by several and added by several, on one workspace, whatever it holds."""
    cases = [(3000, 200, 5, 700), (6000, 67, 3, 2500), (9001, 40, 6, 0), (2501, 256, 8, 1250)]
    ws = P.alloc_balance_workspace(P.make_desc(64, 64, 256, 8))
    for T, E, k, group in cases:
        inputs = _inputs(T, E, k, group, True, T)
        _check(E, k, group, "renormalized", *inputs)
        desc = P.make_desc(64, 64, E, k)
        logits, idx, mask = (_dev(a) for a in inputs[:3])
        first = P.prism_balance_loss(desc, logits, idx, ws, mask, group)
        for fill in (255, 0, 255):
            ws.fill_(fill)
            again = P.prism_balance_loss(desc, logits, idx, ws, mask, group)
            for name in ("loss", "counts", "probs", "n_tokens"):
                assert torch.equal(getattr(first, name), getattr(again, name)), name


@pytest.mark.parametrize("E", [8, 64, 256])
def test_addresses_that_are_not_16_byte_aligned(E):
    for offset in (1, 2, 3):
        _check(E, 2, 0, "softmax_all", *_inputs(301, E, 2, 0, True, offset), offset=offset)


@pytest.mark.parametrize("mode", ["renormalized", "softmax_all"])
def test_either_gradient_alone(mode):
    args = _inputs(300, 64, 6, 100, True, 5)
    _check(64, 6, 100, mode, *args, use_gate=False)
    _check(64, 6, 100, mode, *args, use_loss=False)


@pytest.mark.parametrize("mode", ["renormalized", "softmax_all"])
def test_picks_that_are_none_twice_or_not_the_best(mode):
    logits, idx, _, d_loss, d_gate = _inputs(200, 12, 4, 50, False, 3)
    rng = np.random.default_rng(1)
    idx = rng.integers(-3, 15, idx.shape).astype(np.int32)          # some outside, some twice
    idx[5] = -1
    idx[6] = 4
    idx[7] = 2 ** 31 - 1
    _check(12, 4, 50, mode, logits, idx, None, d_loss, d_gate)


@pytest.mark.parametrize("mode", ["renormalized", "softmax_all"])
@pytest.mark.parametrize("E", [6, 64])
def test_experts_at_minus_infinity_and_rows_of_nothing_else(mode, E):
    logits, idx, _, d_loss, d_gate = _inputs(90, E, 2, 30, False, 9)
    logits[:, 1] = -np.inf
    logits[10] = -np.inf
    logits[20] = np.finfo(np.float32).min                            # masks that write the lowest value
    logits[21, 2:] = np.finfo(np.float32).min
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :2].astype(np.int32)
    _check(E, 2, 30, mode, logits, idx, None, d_loss, d_gate)


@pytest.mark.parametrize("E", [4, 9, 20, 40, 128, 256])
def test_an_expert_picked_many_times_gives_the_same_bits(E):
    k = min(8, E)
    logits, idx, _, d_loss, d_gate = _inputs(500, E, k, 0, False, E)
    idx[:, 1:] = idx[:, :1]
    idx[::3, k // 2] = (idx[::3, 0] + 1) % E
    desc = P.make_desc(64, 64, E, k, gate_mode="softmax_all")
    args = (desc, _dev(logits), _dev(idx))
    first = P.prism_route_backward(*args, d_gate=_dev(d_gate))
    for _ in range(5):
        assert torch.equal(P.prism_route_backward(*args, d_gate=_dev(d_gate)), first)
    _check(E, k, 0, "softmax_all", logits, idx, None, d_loss, d_gate)


def test_near_even_spread_keeps_its_digits():
    """Counts that differ by one in 4096: the gradient is what the difference says, to fp32 precision."""
    T, E, k = 8192, 8, 4
    rng = np.random.default_rng(0)
    logits = rng.standard_normal((T, E)).astype(np.float32) * 0.1
    idx = (np.arange(T * k).reshape(T, k) % E).astype(np.int32)
    idx[0, 0] = 1
    _check(E, k, 0, "renormalized", logits, idx, None, np.array([3.0], np.float32), np.zeros((T, k), np.float32))


def test_no_tokens():
    desc = P.make_desc(64, 64, 8, 2)
    ws = P.alloc_balance_workspace(desc)
    logits, idx = torch.empty((0, 8), device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda")
    b = P.prism_balance_loss(desc, logits, idx, ws)
    assert b.loss.tolist() == [0.0] and b.n_tokens.tolist() == [0] and int(b.counts.abs().sum()) == 0
    assert float(b.probs.abs().sum()) == 0.0
    assert P.prism_balance_loss(desc, logits, idx, ws, group_tokens=4).loss.shape == (0,)
    assert P.prism_route_backward(desc, logits, idx, b, torch.ones(1, device="cuda")).shape == (0, 8)


def test_beyond_4_gib_of_logits():
    T, E, k = 4_500_001, 256, 2
    gen = torch.Generator(device="cuda").manual_seed(0)
    logits = torch.randn((T, E), generator=gen, device="cuda")
    idx = torch.randint(0, E, (T, k), generator=gen, device="cuda").int()
    desc = P.make_desc(64, 64, E, k)
    b = P.prism_balance_loss(desc, logits, idx, P.alloc_balance_workspace(desc), group_tokens=3_000_000)
    assert torch.equal(b.counts[0].long(), torch.bincount(idx[:3_000_000].reshape(-1), minlength=E))
    assert torch.equal(b.counts[1].long(), torch.bincount(idx[3_000_000:].reshape(-1), minlength=E))
    p = sum(torch.softmax(part.double(), 1).sum(0) for part in logits[3_000_000:].split(100_000)) / 1_500_001
    # the derived error of a p, and one addition per row of a lane in fp32 (each of half an ulp of the sum so far)
    lane_rows = -(-3_000_000 // 128) // 16 + 1
    assert bool(((b.probs[1].double() - p).abs() <= (R.relative_error_of_p(12.0) + lane_rows * R.EPS) * p).all())
    d = P.prism_route_backward(desc, logits, idx, b, torch.ones(2, device="cuda"), torch.ones((T, k), device="cuda"), group_tokens=3_000_000)
    rows = torch.cat([torch.arange(0, T, 40009), torch.arange(T - 50, T)])
    l, i = logits[rows.cuda()].cpu().numpy(), idx[rows.cuda()].cpu().numpy()
    group = (rows >= 3_000_000).long().numpy()
    n, c = np.array([3_000_000, 1_500_001]), b.counts.cpu().numpy().astype(np.float64)
    u = (E * (c - c.mean(1, keepdims=True)) / (k * n * n.astype(float))[:, None])[group]
    pr = R.softmax(l.astype(np.float64))
    want = pr * (u - (u * pr).sum(1, keepdims=True))
    size = pr * (np.abs(u) + (np.abs(u) * pr).sum(1, keepdims=True))
    for t in range(len(rows)):
        gate = R.softmax(l[t, i[t]][None].astype(np.float64))[0]
        np.add.at(want[t], i[t], gate * (1.0 - gate.sum()))
        np.add.at(size[t], i[t], 2 * gate)
    err = np.abs(d[rows.cuda()].cpu().numpy() - want)
    assert np.all(err <= (2 * R.relative_error_of_p(12.0) + 12 * R.EPS) * size + 1e-38)


def test_same_bits_every_time_on_streams_and_in_graphs():
    T, E, k = 30011, 64, 6
    logits, idx, mask, d_loss, d_gate = (_dev(a) for a in _inputs(T, E, k, 0, True, 2))
    desc = P.make_desc(64, 64, E, k)
    ws = P.alloc_balance_workspace(desc)
    out = P.BalanceOut(*(torch.empty(s, dtype=t, device="cuda") for s, t in
                         (((1,), torch.float32), ((1, E), torch.int32), ((1, E), torch.float32), ((1,), torch.int32))))
    grad = torch.empty((T, E), device="cuda")

    def step(stream=None):
        P.prism_balance_loss(desc, logits, idx, ws, mask, outputs=out, stream=stream)
        P.prism_route_backward(desc, logits, idx, out, d_loss, d_gate, mask, d_logits=grad, stream=stream)
        return [t.clone() for t in (out.loss, out.counts, out.probs, out.n_tokens, grad)] if stream is None else None

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for t in (out.loss, out.probs, grad):
        t.fill_(9)
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, (out.loss, out.counts, out.probs, out.n_tokens, grad)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for _ in range(3):
        for t in (out.loss, out.probs, grad):
            t.fill_(9)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out.loss, out.counts, out.probs, out.n_tokens, grad)))
        assert torch.equal(step()[4], want[4])


def test_after_the_router():
    """prism_route's own logits and picks: counts agree with the router's, and the loss of a skewed router is above 1."""
    T, H, E, k = 777, 256, 60, 4
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((T, H), generator=gen, device="cuda").to(torch.bfloat16)
    w = (torch.randn((E, H), generator=gen, device="cuda") / 16).to(torch.bfloat16)
    bias = (-1.2 * torch.log(torch.arange(E, device="cuda") + 1.0)).float()[None].contiguous()
    desc = P.make_desc(H, 128, E, k, gate_mode="softmax_all")
    r = P.prism_route(desc, x, w, bias)
    b = P.prism_balance_loss(desc, r.logits, r.topk_idx, P.alloc_balance_workspace(desc))
    assert torch.equal(b.counts[0], r.counts)
    assert float(b.loss) > 1.5
    # the gradient of the gates alone, in the router's own gates: sum over experts of d_logits is 0
    d = P.prism_route_backward(desc, r.logits, r.topk_idx, b, torch.ones(1, device="cuda"), torch.ones((T, k), device="cuda"))
    assert float(d.double().sum(1).abs().max()) < 64 * 2 ** -24


def test_binding_refuses_other_types_and_shapes():
    desc = P.make_desc(64, 64, 8, 2)
    ws = P.alloc_balance_workspace(desc)
    logits, idx = torch.zeros((5, 8), device="cuda"), torch.zeros((5, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(P.PrismError):
        P.prism_balance_loss(desc, logits.half(), idx, ws)
    with pytest.raises(P.PrismError):
        P.prism_balance_loss(desc, logits, idx.long(), ws)
    with pytest.raises(P.PrismError):
        P.prism_balance_loss(desc, logits, idx, ws, torch.ones(4, dtype=torch.uint8, device="cuda"))
    with pytest.raises(P.PrismError):
        P.prism_balance_loss(desc, torch.zeros((8, 5), device="cuda").t(), idx, ws)
    with pytest.raises(P.PrismError):
        P.prism_route_backward(desc, logits, idx, None, torch.ones(1, device="cuda"))
    with pytest.raises(P.PrismError):
        P.prism_route_backward(desc, logits, idx)
