"""Balance loss of very many groups and of very long ones."""
import pytest
import torch

import paper_2508_12851_amd as P
import balance_reference as R

pytestmark = pytest.mark.gpu


def _picks(T, E, k, gen):
    """k different experts of each token."""
    first, step = (torch.randint(0, E, (T, 1), generator=gen, device="cuda") for _ in range(2))
    return ((first + torch.arange(k, device="cuda") * (1 + step % max(1, E // k))) % E).int().contiguous()


@pytest.mark.parametrize("T,group", [((1 << 22) - 1, 1), ((1 << 22) + 3, 1), (2 * ((1 << 22) + 1) + 1, 2), (1 << 23, 1)])
def test_more_groups_than_one_grid_has_workgroups(T, group):
    """A group has a workgroup of 1024 threads, and a grid fewer than 2^32 of them."""
    E, k, G = 3, 2, -(-T // group)
    gen = torch.Generator(device="cuda").manual_seed(T)
    logits = torch.randn((T, E), generator=gen, device="cuda").clamp(-3, 3)
    idx = _picks(T, E, k, gen)
    desc = P.make_desc(64, 64, E, k)
    b = P.prism_balance_loss(desc, logits, idx, P.alloc_balance_workspace(desc), group_tokens=group)

    def of_groups(rows):
        return torch.cat([rows, rows.new_zeros((G * group - T, E))]).view(G, group, E).sum(1)
    n = torch.full((G,), group, device="cuda")
    n[-1] = T - (G - 1) * group
    counts = of_groups(torch.zeros((T, E), dtype=torch.int64, device="cuda").scatter_add_(1, idx.long(), torch.ones_like(idx).long()))
    assert torch.equal(b.n_tokens.long(), n) and torch.equal(b.counts.long(), counts)
    probs = of_groups(torch.softmax(logits.double(), 1)) / n[:, None]
    # the derived error of a p, the addition of two of them, their mean rounded
    tol = R.relative_error_of_p(6.0) + 2 * R.EPS
    assert bool(((b.probs.double() - probs).abs() <= tol * probs).all())
    loss = E / (k * n) * (counts * probs).sum(1)
    assert bool(((b.loss.double() - loss).abs() <= (tol + R.EPS) * loss).all())
    # the gradient of the loss of every group
    d_loss = torch.randn(G, generator=gen, device="cuda")
    d = P.prism_route_backward(desc, logits, idx, b, d_loss, group_tokens=group)
    at = torch.arange(T, device="cuda") // group
    u = (d_loss.double() * E / (k * n.double() ** 2))[at, None] * (counts - counts.double().mean(1, keepdim=True))[at]
    p = torch.softmax(logits.double(), 1)
    want, size = p * (u - (u * p).sum(1, keepdim=True)), p * (u.abs() + (u.abs() * p).sum(1, keepdim=True))
    assert bool(((d.double() - want).abs() <= (2 * R.relative_error_of_p(6.0) + 12 * R.EPS) * size + 1e-38).all())


@pytest.mark.parametrize("E,group", [(3, 1 << 20), (40, 1 << 16), (256, 1 << 14), (256, (1 << 14) - 77)])
def test_the_error_of_a_long_group_does_not_grow_with_it(E, group):
    """Equal rows, whose probabilities a sum of fp32 rounds the same way a thousand times; so many groups that each is one workgroup's."""
    G, k = 129, 1
    T = G * group
    row = torch.randn(E, generator=torch.Generator().manual_seed(E), dtype=torch.float32).clamp(-3, 3).cuda()
    logits = row.expand(T, E).contiguous()
    idx = (torch.arange(T, device="cuda", dtype=torch.int32) % E)[:, None].contiguous()
    desc = P.make_desc(64, 64, E, k)
    b = P.prism_balance_loss(desc, logits, idx, P.alloc_balance_workspace(desc), group_tokens=group)
    p = torch.softmax(row.double(), 0)
    # the derived error of a p; 15 additions of a lane's rows, their sum, at most 6 lanes' and 15 wavefronts' additions, the mean
    tol = R.relative_error_of_p(6.0) + (15 + 1 + 6 + 15 + 1) * R.EPS
    assert bool(((b.probs.double() - p).abs() <= tol * p).all()), float(((b.probs.double() - p).abs() / p).max() / R.EPS)
    loss = E / (k * group) * (b.counts.double() * p).sum(1)
    assert torch.equal(b.counts.sum(1), b.n_tokens)
    assert bool(((b.loss.double() - loss).abs() <= (tol + R.EPS) * loss).all())
