"""Balance loss and router gradient without a GPU: the reference against differences, refusals, sizes."""
import ctypes

import numpy as np
import pytest

import paper_2508_12851_amd as P
import balance_reference as R


@pytest.mark.parametrize("mode", ["renormalized", "softmax_all"])
@pytest.mark.parametrize("E,k,group", [(5, 2, 0), (4, 4, 3), (3, 1, 2)])
def test_reference_gradient_against_differences(mode, E, k, group):
    rng = np.random.default_rng(E)
    T = 7
    logits = rng.standard_normal((T, E))
    idx = np.argsort(-logits, axis=1)[:, :k].astype(np.int32)
    idx[2, 0] = idx[2, k - 1]                   # an expert twice
    idx[3, 0] = -1                              # no pick
    mask = np.array([1, 1, 1, 1, 0, 1, 1], np.uint8)
    G = 1 if group == 0 else -(-T // group)
    d_loss, d_gate = rng.standard_normal(G), rng.standard_normal((T, k))

    def value(l):
        loss = R.balance(l, idx, mask, group, E, k)[0]
        total = float(loss @ d_loss)
        p = R.softmax(l)
        for t in range(T):
            js = [j for j in range(k) if 0 <= idx[t, j] < E]
            if mask[t] and js:
                gate = p[t, idx[t, js]] if mode == "softmax_all" else R.softmax(l[t, idx[t, js]][None])[0]
                total += float(gate @ d_gate[t, js])
        return total

    d, _ = R.backward(logits, idx, mask, group, E, k, d_loss, d_gate, mode)
    step = 1e-6
    for t in range(T):
        for e in range(E):
            up, down = logits.copy(), logits.copy()
            up[t, e] += step
            down[t, e] -= step
            assert abs((value(up) - value(down)) / (2 * step) - d[t, e]) < 1e-7


def _desc(E=8, k=2):
    return P.make_desc(64, 64, E, k)


def test_refusals_before_any_launch():
    lib = P.load_library()
    d = _desc()
    n = ctypes.c_size_t(0)
    assert lib.prism_balance_workspace_bytes(ctypes.byref(d), None) == 1
    assert lib.prism_balance_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == 0 and n.value % 256 == 0
    p = ctypes.c_void_p(0x10000)                # never dereferenced
    bad = ctypes.c_void_p(0x10010)

    def loss(desc=d, logits=p, idx=p, mask=None, group=0, T=4, loss=p, counts=p, probs=p, tokens=p, ws=p, size=n.value):
        return lib.prism_balance_loss(ctypes.byref(desc), logits, idx, mask, group, T, loss, counts, probs, tokens, ws, size, None)

    assert loss(T=-1) == 1 and loss(group=-1) == 1
    for name in ("logits", "idx", "loss", "counts", "probs", "tokens", "ws"):
        assert loss(**{name: None}) == 1, name
    assert loss(ws=bad) == 1
    assert loss(size=n.value - 1) == 3
    assert loss(desc=_desc(257, 2)) == 2
    assert loss(T=(1 << 23) + 1, group=1) == 2  # more groups than workgroups are started for

    def backward(desc=d, logits=p, idx=p, mask=None, group=0, T=4, counts=p, tokens=p, d_loss=p, d_gate=p, out=p):
        return lib.prism_route_backward(ctypes.byref(desc), logits, idx, mask, group, T, counts, tokens, d_loss, d_gate, out, None)

    assert backward(T=-1) == 1 and backward(group=-1) == 1
    for name in ("logits", "idx", "counts", "tokens", "d_loss", "out"):
        assert backward(**{name: None}) == 1, name
    assert backward(counts=None, tokens=None, d_loss=None, d_gate=None) == 1
    assert backward(T=(1 << 23) + 1, group=1) == 2
    assert backward(T=0) == 0                   # nothing to do, nothing launched
    assert loss(T=0, group=4) == 0


def test_workspace_depends_on_the_experts_alone():
    lib = P.load_library()
    sizes = []
    for E in (1, 8, 64, 256):
        n = ctypes.c_size_t(0)
        d = _desc(E, 1)
        assert lib.prism_balance_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == 0
        sizes.append(n.value)
    assert sizes == sorted(sizes) and sizes[0] > 0
