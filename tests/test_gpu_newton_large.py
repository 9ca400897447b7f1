"""Updates of matrices that do not fit LDS (many launches), beside small ones: the direction and
all that an update does with it."""
import numpy as np
import pytest
import torch

import routed_reference as rr
from test_gpu_newton import blocks, check, pm, randn  # noqa: F401

pytestmark = pytest.mark.gpu

# (F, widths): matrices of more than 128 rows and columns or more than 1,280 columns, turned
# and not, beside ones that fit LDS
LARGE = [(200, [9, 140, 300]), (131, [129, 3, 133]), (1300, [1, 40, 2]), (5, [1500, 9, 1281]),
         (257, [255, 256, 258]), (1, [1281, 1, 5000])]
shapes = pytest.mark.parametrize("F,hs", LARGE, ids=lambda v: str(v) if isinstance(v, int) else "M%d" % len(v))


def through_launches(net):
    return net.kernel_variants()["hidden2"][0] == "k_ns_product"


@shapes
@pytest.mark.parametrize("n", [1, 2, 3, 10])
def test_steps(pm, F, hs, n):
    net = pm.PackedMLP(F, 2, hs, [0] * len(hs))
    G = randn(F + n, sum(hs), F)
    got = net.orthogonalize(G.cuda(), steps=n)
    assert through_launches(net)
    check(got, G, blocks(F, hs), n)
    again = G.cuda()
    net.orthogonalize(again, steps=n, out=again)
    assert torch.equal(got, again)


@pytest.mark.parametrize("O", [2, 16])
def test_output_weights(pm, O):
    hs = [1281, 3, 20000, 4096]
    net = pm.PackedMLP(5, O, hs, [0] * len(hs))
    G = randn(O, O, sum(hs))
    got = net.orthogonalize(G.cuda(), "W2")
    assert through_launches(net)
    check(got.t(), G.t(), blocks(O, hs))


@pytest.mark.parametrize("scale", [1e-38, 1e-12, 1e30, 1e37])
def test_any_scale(pm, scale):
    hs = [9, 140, 300]
    net = pm.PackedMLP(200, 2, hs, [0] * 3)
    G = (randn(7, sum(hs), 200).double() * scale).float()
    check(net.orthogonalize(G.cuda()), G, blocks(200, hs))
    assert through_launches(net)


def test_zero_and_low_rank_and_diverged_matrices(pm):
    hs = [140, 9, 200, 300, 160, 150]
    net = pm.PackedMLP(201, 2, hs, [0] * len(hs))
    parts = blocks(201, hs)
    G = randn(8, sum(hs), 201)
    G[parts[0]] = 0
    G[parts[2]] = torch.outer(randn(9, 200), randn(10, 201))
    G[parts[3], 10:] = 0
    clean = net.orthogonalize(G.cuda())
    check(clean, G, parts)
    assert through_launches(net)
    assert not bool(clean[parts[0]].any()) and not bool(clean[parts[3], 10:].any())
    for bad in (float("nan"), float("inf"), -float("inf")):
        H = G.clone()
        for k in (1, 4):
            H[parts[k].start + 1, 3] = bad
        got = net.orthogonalize(H.cuda())
        for k, r in enumerate(parts):
            if k in (1, 4):
                assert bool(got[r].isnan().all())
            else:
                assert torch.equal(got[r], clean[r])


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_momentum(pm, nesterov, in_place):
    hs = [9, 140, 300]
    net = pm.PackedMLP(200, 2, hs, [0] * 3)
    G, mom = randn(1, sum(hs), 200), randn(2, sum(hs), 200)
    g, m = G.cuda(), mom.cuda()
    new = m if in_place else torch.empty_like(m)
    out = g if in_place else None
    got = net.orthogonalize(g, momentum=m, mu=0.9, nesterov=nesterov,
                            momentum_out=None if in_place else new, out=out)
    mu = float(np.float32(0.9))
    want = mu * mom.double() + G.double()
    assert bool(((new.cpu().double() - want).abs() <= rr.U * 2 * (mom.abs() + want.abs())).all())
    held = new.cpu().double()
    check(got, G.double() + mu * held if nesterov else held, blocks(200, hs))
    if not in_place:
        assert torch.equal(m.cpu(), mom) and torch.equal(g.cpu(), G)


@pytest.mark.parametrize("per_model", [False, True])
@pytest.mark.parametrize("kind", ["W1", "V1", "W2", "W12", "masked"])
def test_muon_step(pm, kind, per_model):
    """Weights from the direction, rates, decay, the gain of tall matrices and masks."""
    F, hs, k = 200, [9, 140, 300, 150], 0
    M, N = 4, sum(hs)
    mask = None
    if kind == "V1":
        net, k = pm.BlockPackedMLP(F, 2, hs, [7] * M, gated=True), 1
        shapes = [(h, F) for h in hs]
    elif kind == "W2":
        hs = [1281, 3, 2000, 1500]
        net, k = pm.PackedMLP(5, 3, hs, [0] * M), 1
        shapes = [(3, h) for h in hs]
    elif kind == "W12":
        h2 = [9, 300, 140, 400]
        net, k = pm.DeepPackedMLP(7, 3, hs, h2, [2] * M), 1
        shapes = [(b, a) for a, b in zip(hs, h2)]
    else:
        net = pm.PackedMLP(F, 2, hs, [0] * M)
        shapes = [(h, F) for h in hs]
        if kind == "masked":
            mask = np.random.default_rng(1).random((M, F)) < 0.7
            net.set_feature_mask(mask)
    name = "W1" if kind == "masked" else kind

    def parts(t):  # each model's matrix
        t = torch.as_tensor(t).double()
        if kind == "W2":
            return [t[:, r] for r in blocks(3, hs)]
        return [v.reshape(s) for v, s in zip(t.reshape(-1).split([a * b for a, b in shapes]), shapes)]

    size = sum(a * b for a, b in shapes)
    shape = {"W2": (3, size // 3), "W12": (size,)}.get(kind, (N, F))
    G, mom = randn(3, *shape), randn(4, *shape)
    rates = torch.tensor([0.1, 0.0, 0.5, 0.25])
    before = net.get_params()
    m = mom.cuda()
    net.muon_step(G.cuda(), rates.cuda() if per_model else 0.3, name, momentum=m, mu=0.8, decay=0.05)
    assert through_launches(net)
    after = net.get_params()
    assert all(np.array_equal(a, b) for i, (a, b) in enumerate(zip(before, after)) if i != k)
    mu, decay = float(np.float32(0.8)), float(np.float32(0.05))
    U = G.double() + mu * m.cpu().double()
    for i, (w, got, u) in enumerate(zip(parts(before[k]), parts(after[k]), parts(U))):
        lr = float(rates[i]) if per_model else float(np.float32(0.3))
        d, bound = rr.orthogonalized(u, 5)
        gain = max(1.0, u.shape[0] / u.shape[1]) ** 0.5
        d, bound = gain * d, gain * bound
        want = w - lr * (decay * w + d)
        if mask is not None:
            want = want * torch.from_numpy(mask[i]).double()
        off = (got - want).abs()
        assert bool((off <= lr * bound + 4 * rr.U * (w.abs() + lr * d.abs())).all()), (kind, i)


def test_bad_rate_of_a_large_matrix_is_reported(pm):
    net = pm.PackedMLP(200, 2, [300, 9], [2, 2])
    X, y = randn(6, 40, 200).cuda(), torch.zeros(40, dtype=torch.int32).cuda()
    net.train_step(X, y, 0.1)
    net.losses()
    G = randn(5, 309, 200).cuda()
    for rates in ([float("nan"), 0.1], [0.1, float("inf")]):
        net.muon_step(G, torch.tensor(rates).cuda())
        assert through_launches(net)
        with pytest.raises(pm.PmlpError, match="learning rate"):
            net.losses()
        net.losses()


def test_more_matrices_than_a_workspace_holds(pm):
    """150 of 1,000 x 1,000: their halves in both orders are more than the 2 GiB that a run of
    matrices takes, so that they go in two; three of each run are compared.  In place, as the
    second run starts when the first has written its results."""
    M = 150
    hs = [1000] * M
    net = pm.PackedMLP(1000, 2, hs, [0] * M)
    g = torch.Generator(device="cuda").manual_seed(3)
    G = torch.randn(1000 * M, 1000, generator=g, device="cuda")
    some = [0, 60, 94, 120, 149]
    U = [G[1000 * k:1000 * (k + 1)].cpu() for k in some]
    got = net.orthogonalize(G)
    net.orthogonalize(G, out=G)
    assert through_launches(net) and torch.equal(G, got)
    for k, u in zip(some, U):
        check(got[1000 * k:1000 * (k + 1)], u, [slice(0, 1000)])
