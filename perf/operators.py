"""Operators of the layer beyond its bf16 and fp32 forward, measured against their plain forms.

Three operators, each in the sizes this repository's layers have (perf/cases.py, prism_inputs):

* balance: per-expert counts and the balance loss of a batch's routing, and the gradient of that loss and
  of the gates with respect to the router logits -- one training step of a router;
* linear: rows of activations quantised to 8 bits, one scale per token, times a weight matrix in 8 bits
  with one scale per output channel -- a dense layer of a served model;
* experts: the SwiGLU experts of one server with 8-bit weights -- the rows of prism_expert_ffn.

``run`` computes them from elementary torch operations, or, with ``own``, by the calls that a user of
the package makes.  ``exact`` computes the same from the definitions in 64 bits.

Definitions.  quantise(v): scale = fl32(max |v| / 127) of a row, q = the integer nearest to v / scale
(ties to even, at most 127 in magnitude; 0 in a row of zeros).  linear: out = (sum of q_x q_w) scale_x
scale_w.  experts: the same for gate, up and down; h = silu(gate) up is quantised by rows as well.
balance: n tokens that count in a group, c_e picks of expert e among them, p = softmax(logits),
P_e = mean of p_e over them, loss = E / (k n) sum_e c_e P_e.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

# The expert shapes of this repository's workloads.
WIDE = dict(H=4096, F=14336, E=8, k=2, S=0, n_local=5, zipf_s=1.0)
FINE = dict(H=2048, F=1408, E=60, k=4, S=4, n_local=36, zipf_s=1.2)
FINE2 = dict(H=2048, F=1408, E=64, k=6, S=2, n_local=32, zipf_s=1.0)
MANY = dict(H=1024, F=1024, E=256, k=8, S=0, n_local=128, zipf_s=1.0)


def _balance(name, T, E, k, group=0, padded=0.0, gates="renormalized"):
    return dict(({"name": name} if name else {}), op="balance", T=T, E=E, k=k, group=group, padded=padded, gates=gates)


def _linear(name, M, N, K, dtype="bf16"):
    return dict(({"name": name} if name else {}), op="linear", M=M, N=N, K=K, dtype=dtype)


def _experts(name, shape, T):
    return dict(({"name": name} if name else {}), op="experts", T=T, **shape)


def listed():
    return [
        # router of the wide layer on a decode batch: launches and host work
        _balance("balance_32", 32, 8, 2),
        # fine-tuning batch of 16 padded sequences of 512 tokens, a loss for each, narrow-expert router
        _balance("balance_seqs_8192", 8192, 64, 6, group=512, padded=0.3, gates="softmax_all"),
        # the largest batch and router, a ragged number of tokens
        _balance("balance_65531", 65531, 256, 8),
        # one token through a wide projection: the weights streamed once
        _linear("linear_1", 1, 14336, 4096),
        # a few dozen tokens, odd sizes throughout, fp32 activations
        _linear("linear_odd_77", 77, 2053, 1411, "f32"),
        # a short prompt through a middling projection
        _linear("linear_600", 600, 4096, 2048),
        # prefill through the widest contraction: bound by the matrix cores
        _linear("linear_4096", 4096, 4096, 14336),
        # one sequence generating on the wide layer
        _experts("experts_wide_1", WIDE, 1),
        # decode batch of the wide layer: every hosted expert's weights streamed once
        _experts("experts_wide_32", WIDE, 32),
        # short prompt on the narrow-expert layer: a dozen rows per expert, beside shared experts
        _experts("experts_fine_333", FINE, 333),
        # prefill of the variant, ragged
        _experts("experts_fine_5001", FINE2, 5001),
        # prefill of the wide layer: bound by the matrix cores
        _experts("experts_wide_4096", WIDE, 4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["balance", "linear", "experts"])
    if op == "balance":
        T, E = _log_int(rng, 1, 65536), rng.choice([_log_int(rng, 2, 256), 8, 64, 256])
        group = rng.choice([0, _log_int(rng, 16, 4096)])
        return _balance(None, T, E, rng.randint(1, min(8, E)), group, rng.choice([0.0, 0.1, 0.5]),
                        rng.choice(["renormalized", "softmax_all"]))
    if op == "linear":
        M, N, K = _log_int(rng, 1, 4096), _log_int(rng, 64, 14336), _log_int(rng, 64, 14336)
        if rng.random() < 0.5:      # as most layers are
            N, K = 64 * max(1, N // 64), 64 * max(1, K // 64)
        if M * N * K > 4096 * 4096 * 14336:
            M = max(1, 4096 * 4096 * 14336 // (N * K))
        return _linear(None, M, N, K, rng.choice(["bf16", "bf16", "f32"]))
    kind = rng.choice(["wide", "fine", "fine2", "many"])
    if kind == "wide":
        shape = dict(WIDE, H=64 * rng.randint(16, 64), F=64 * rng.randint(64, 224), n_local=rng.randint(2, 5))
        return _experts(None, shape, _log_int(rng, 1, 4000))
    if kind == "fine":
        return _experts(None, dict(FINE, n_local=rng.randint(12, 60), zipf_s=rng.choice([0.0, 1.0, 1.2])), _log_int(rng, 1, 4096))
    if kind == "fine2":
        return _experts(None, dict(FINE2, n_local=rng.randint(12, 64), F=64 * rng.randint(12, 32)), _log_int(rng, 1, 4096))
    shape = dict(MANY, E=rng.randint(65, 256), k=rng.randint(4, 8), F=64 * rng.randint(8, 24))
    return _experts(None, dict(shape, n_local=rng.randint(16, min(shape["E"], 160))), _log_int(rng, 1, 2000))


# ---- inputs ---------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _popularity(E, zipf_s, gen):
    """Router bias of a Zipf-skewed popularity: -s ln(rank)."""
    rank = torch.randperm(E, generator=gen, device="cuda") + 1
    return -zipf_s * torch.log(rank.float())


def _weights_i8(gen, n, rows, cols):
    """n matrices of 8-bit weights [rows, cols] as quantised normal ones are, and a scale per row."""
    q = torch.empty((n, rows, cols), dtype=torch.int8, device="cuda")
    for i in range(n):
        q[i] = torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.bfloat16).mul_(30).round_().clamp_(-127, 127)
    scale = (torch.rand((n, rows), generator=gen, device="cuda") * 0.5 + 0.75) / (30 * math.sqrt(cols))
    return q, scale


def prepare(case, seed):
    gen = _generator(seed)
    st = dict(case=case)
    if case["op"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        groups = -(-T // case["group"]) if case["group"] else 1
        logits = torch.randn((T, E), generator=gen, device="cuda") + _popularity(E, 1.0, gen)
        st["topk_idx"] = logits.topk(k, dim=1).indices.int()
        st["token_mask"] = (torch.rand(T, generator=gen, device="cuda") >= case["padded"]).to(torch.uint8) if case["padded"] else None
        if case["padded"]:          # what stands in padded places is nobody's value
            logits[st["token_mask"] == 0] = math.nan
        st["logits"] = logits
        st["d_loss"] = torch.rand(groups, generator=gen, device="cuda") * 0.02      # the loss's weight in a training loss
        st["d_gate"] = torch.randn((T, k), generator=gen, device="cuda") / T
        if own:
            import paper_2508_12851_amd as P
            st["desc"] = P.make_desc(64, 64, E, k, gate_mode=case["gates"])
            st["ws"] = P.alloc_balance_workspace(st["desc"])
        return st
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = torch.randn((M, K), generator=gen, device="cuda").to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        q, scale = _weights_i8(gen, 1, N, K)
        st["w"], st["w_scale"] = q[0], scale[0]
        if own:                     # the weights laid out once, as a model is loaded
            import paper_2508_12851_amd as P
            st["packed"] = P.prism_pack_i8(st["w"], st["w_scale"])
            st["ws"] = P.alloc_matmul_i8_workspace(M, N, K)
        return st
    T, H, F, E, k, S, L = (case[n] for n in ("T", "H", "F", "E", "k", "S", "n_local"))
    bias = _popularity(E, case["zipf_s"], gen)
    hosted = bias.topk(L).indices.sort().values if case["zipf_s"] else torch.arange(L, device="cuda")
    st["x"] = torch.randn((T, H), generator=gen, device="cuda").to(torch.bfloat16)
    picks = (torch.randn((T, E), generator=gen, device="cuda") + bias).topk(k, dim=1).indices.reshape(-1)
    # the placement split: hosted assignments, bucketed by expert, and where the buckets start
    mask = torch.zeros(E, dtype=torch.bool, device="cuda")
    mask[hosted] = True
    n_picks = torch.bincount(picks, minlength=E) * mask
    order = torch.sort(torch.where(mask[picks], picks, E), stable=True).indices
    st["local_src"] = order.int()
    st["local_offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), n_picks.cumsum(0)]).int()
    st["slot"] = mask.cumsum(0) - 1                         # of a hosted expert among the hosted ones
    st["n_rows"], st["most_rows"] = int(n_picks.sum()), int(n_picks.max())
    shapes = ((F, H), (F, H), (H, F))
    st["w"] = [_weights_i8(gen, L, *s) for s in shapes]     # gate, up, down of the hosted experts
    st["shared"] = [_weights_i8(gen, S, *s) for s in shapes]
    if own:
        import paper_2508_12851_amd as P
        st["desc"] = P.make_desc(H, F, E, k, S, "bf16", weight_layout="int8")
        packed = [tuple(P.prism_pack_i8(q[i], s[i]).data for q, s in st["w"]) for i in range(L)]
        of = dict(zip(hosted.tolist(), packed))
        st["table"] = P.WeightTable([of.get(e) for e in range(E)],
                                    [tuple(P.prism_pack_i8(q[i], s[i]).data for q, s in st["shared"]) for i in range(S)])
        st["ws"] = P.alloc_workspace(st["desc"], T)
    return st


# ---- the operators ----------------------------------------------------------------------------
def _quantise(v):
    """Rows of v as integers in fp32, and their scales; quotients next to a half need 64 bits."""
    scale = (v.float().abs().amax(-1, keepdim=True) / 127.0)
    q = torch.round(v.double() / torch.where(scale > 0, scale, 1.0).double()).clamp_(-127, 127).float()
    return q, scale


def _balance_plain(st):
    case, logits, idx = st["case"], st["logits"], st["topk_idx"].long()
    T, E, k = case["T"], case["E"], case["k"]
    size = case["group"] or T
    G = -(-T // size)
    live = torch.ones((T, 1), device=logits.device) if st["token_mask"] is None else (st["token_mask"] != 0).float()[:, None]

    def of_groups(rows):            # sums over the tokens of a group
        return torch.cat([rows, rows.new_zeros((G * size - T, rows.shape[1]))]).view(G, size, -1).sum(1, dtype=torch.float64)

    n = of_groups(live)
    counts = of_groups(torch.zeros((T, E), device=logits.device).scatter_add(1, idx, live.expand(T, k)))
    logits = torch.where(live > 0, logits, 0.0)
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    some = n.clamp(min=1.0)
    probs = of_groups(p * live) / some
    loss = (counts * probs).sum(1) * (E / k) / some[:, 0]
    # gradient: the balance loss, then the gates of the picks
    group = torch.arange(T, device=logits.device) // size
    c = (counts - counts.mean(1, keepdim=True)).float()[group]      # (a constant changes nothing: p sums to 1)
    d = p * (c - (c * p).sum(1, keepdim=True)) * (st["d_loss"][:, None] * (E / k) / (some * some)).float()[group]
    if case["gates"] == "renormalized":
        picked = logits.gather(1, idx)
        g = torch.exp(picked - picked.amax(1, keepdim=True))
        g = g / g.sum(1, keepdim=True)
        d = d.scatter_add(1, idx, g * (st["d_gate"] - (g * st["d_gate"]).sum(1, keepdim=True)))
    else:
        g = p.gather(1, idx) * st["d_gate"]
        d = (d - p * g.sum(1, keepdim=True)).scatter_add(1, idx, g)
    return dict(loss=loss.float(), counts=counts.int(), probs=probs.float(), n_tokens=n[:, 0].int(), d_logits=d * live)


def _linear_plain(st):
    q, scale = _quantise(st["x"])
    return (torch.mm(q, st["w"].float().t()) * scale * st["w_scale"]).to(st["x"].dtype)


def _swiglu_plain(q, scale, weights):
    """Experts as a batch: q [n, rows, H] integers, scale [n, rows, 1]."""
    (wg, sg), (wu, su), (wd, sd) = weights
    gate = torch.bmm(q, wg.float().transpose(1, 2)) * scale * sg[:, None]
    up = torch.bmm(q, wu.float().transpose(1, 2)) * scale * su[:, None]
    h, h_scale = _quantise(gate / (1.0 + torch.exp(-gate)) * up)
    return torch.bmm(h, wd.float().transpose(1, 2)) * h_scale * sd[:, None]


def _experts_plain(st):
    case, x = st["case"], st["x"]
    T, H, k, S = (case[n] for n in ("T", "H", "k", "S"))
    L, n, most = case["n_local"], st["n_rows"], st["most_rows"]
    q, scale = _quantise(x)
    y = torch.zeros((T * k + S * T, H), dtype=torch.bfloat16, device=x.device)
    if n:
        row = torch.arange(n, device=x.device)
        expert = torch.searchsorted(st["local_offsets"][1:].contiguous(), row.int(), right=True)
        place = st["slot"][expert] * most + row - st["local_offsets"][expert]      # rows of an expert side by side
        token = st["local_src"][:n].long() // k
        qs = torch.zeros((L * most, H), device=x.device).index_copy_(0, place, q[token])
        scales = torch.zeros((L * most, 1), device=x.device).index_copy_(0, place, scale[token])
        out = _swiglu_plain(qs.view(L, most, H), scales.view(L, most, 1), st["w"])
        y[:n] = out.view(L * most, H)[place].to(torch.bfloat16)
    if S:
        out = _swiglu_plain(q.expand(S, T, H), scale.expand(S, T, 1), st["shared"])
        y[T * k:] = out.reshape(S * T, H).to(torch.bfloat16)
    return y


def run(st):
    op = st["case"]["op"]
    if not own:
        return {"balance": _balance_plain, "linear": _linear_plain, "experts": _experts_plain}[op](st)
    import paper_2508_12851_amd as P
    if op == "balance":
        group = st["case"]["group"]
        b = P.prism_balance_loss(st["desc"], st["logits"], st["topk_idx"], st["ws"], st["token_mask"], group)
        d = P.prism_route_backward(st["desc"], st["logits"], st["topk_idx"], b, st["d_loss"], st["d_gate"], st["token_mask"], group)
        return dict(loss=b.loss, counts=b.counts, probs=b.probs, n_tokens=b.n_tokens, d_logits=d)
    if op == "linear":
        return P.prism_matmul_i8(P.prism_quantize_i8(st["x"]), st["packed"], st["ws"], dtype=st["x"].dtype)
    return P.prism_expert_ffn(st["desc"], st["x"], st["table"], st["local_src"], st["local_offsets"], st["ws"])


# ---- the definitions in 64 bits ---------------------------------------------------------------
def _exact_quantise(v):
    scale = (v.abs().max(1).values.float() / np.float32(127)).double()
    return torch.round(v / torch.where(scale > 0, scale, 1.0)[:, None]).clamp(-127, 127), scale


def _exact_balance(st):
    case = st["case"]
    T, E, k = case["T"], case["E"], case["k"]
    size = case["group"] or T
    G = -(-T // size)
    loss, probs, grad = torch.zeros(G), torch.zeros(G, E), torch.zeros(T, E, dtype=torch.float64)
    counts, n_tokens = torch.zeros(G, E, dtype=torch.int32), torch.zeros(G, dtype=torch.int32)
    mask = torch.ones(T, dtype=torch.bool) if st["token_mask"] is None else st["token_mask"].cpu() != 0
    logits, idx = st["logits"].cpu().double(), st["topk_idx"].cpu().long()
    d_loss, d_gate = st["d_loss"].cpu().double(), st["d_gate"].cpu().double()
    loss, probs = loss.double(), probs.double()
    for g in range(G):
        rows = torch.arange(g * size, min(T, (g + 1) * size))
        rows = rows[mask[rows]]
        n = len(rows)
        n_tokens[g] = n
        if not n:
            continue
        p = torch.softmax(logits[rows], 1)
        c = torch.bincount(idx[rows].reshape(-1), minlength=E)
        counts[g], probs[g] = c.int(), p.mean(0)
        loss[g] = E / (k * n) * (c.double() @ probs[g])
        u = d_loss[g] * E / (k * n * n) * c.double()            # d loss / d p of every counted row
        u = u.expand(n, E).clone()
        if case["gates"] == "softmax_all":
            u.scatter_add_(1, idx[rows], d_gate[rows])
        d = p * (u - (u * p).sum(1, keepdim=True))
        if case["gates"] == "renormalized":
            gate = torch.softmax(logits[rows].gather(1, idx[rows]), 1)
            d.scatter_add_(1, idx[rows], gate * (d_gate[rows] - (gate * d_gate[rows]).sum(1, keepdim=True)))
        grad[rows] = d
    return dict(loss=loss, counts=counts, probs=probs, n_tokens=n_tokens, d_logits=grad)


def _exact_swiglu(x, gate, up, down):
    def product(a, w):
        q, scale = a
        return (q @ w[0].double().t()) * scale[:, None] * w[1].double()
    a = _exact_quantise(x.double())
    g = product(a, gate)
    return product(_exact_quantise(g / (1 + torch.exp(-g)) * product(a, up)), down)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "balance":
        return _exact_balance(st)
    if case["op"] == "linear":
        q, scale = _exact_quantise(st["x"].double())
        return (q @ st["w"].double().t()) * scale[:, None] * st["w_scale"].double()
    T, H, k, S = (case[n] for n in ("T", "H", "k", "S"))
    y = torch.zeros((T * k + S * T, H), dtype=torch.float64, device="cuda")
    at = st["local_offsets"].tolist()
    for e in range(case["E"]):
        if at[e + 1] > at[e]:
            i = int(st["slot"][e])
            tokens = st["local_src"][at[e]:at[e + 1]].long() // k
            y[at[e]:at[e + 1]] = _exact_swiglu(st["x"][tokens], *((q[i], s[i]) for q, s in st["w"]))
    for s in range(S):
        y[T * k + s * T:T * k + (s + 1) * T] = _exact_swiglu(st["x"], *((q[s], z[s]) for q, z in st["shared"]))
    return y


# ---- what a pass cannot do without --------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _expected_picks(T, E, k, n_local, zipf_s):
    """(assignments to hosted experts, hosted experts with one) of a batch, from sampled routings."""
    rng = np.random.default_rng(0)
    local, touched, passes, n = 0.0, 0.0, max(1, min(64, 4096 // T)), min(T, 4096)
    bias = -zipf_s * np.log(np.arange(1, E + 1))
    for _ in range(passes):
        picks = np.argsort(-(rng.standard_normal((n, E)) + bias), axis=1)[:, :k]
        hits = np.bincount(picks.reshape(-1), minlength=E)[:n_local]
        local += hits.sum() * T / n / passes
        touched += (hits > 0).sum() / passes
    return float(local), float(touched)


def work(case):
    if case["op"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        groups = -(-T // case["group"]) if case["group"] else 1
        # logits, picks and gate gradients in; the logits' gradient, counts and probabilities out
        nbytes = 8.0 * T * E + 8.0 * T * k + (T if case["padded"] else 0) + groups * (8.0 * E + 12)
        return dict(bytes=nbytes, flops=12.0 * T * E)
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        es = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=1.0 * M * K * es + 1.0 * N * K + 4.0 * N + 1.0 * M * N * es, flops=2.0 * M * N * K)
    T, H, F, E, k, S = (case[n] for n in ("T", "H", "F", "E", "k", "S"))
    local, touched = _expected_picks(T, E, k, case["n_local"], case["zipf_s"])
    rows = local + S * T
    # tokens and lists, the experts that have rows with their scales, output rows
    nbytes = 2.0 * T * H + 4.0 * (local + E) + (touched + S) * (3.0 * H * F + 8.0 * F + 4.0 * H) + 2.0 * rows * H
    return dict(bytes=nbytes, flops=6.0 * H * F * rows)
