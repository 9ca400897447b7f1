"""Orthogonalised updates against the 64-bit steps, matrix by matrix."""
import numpy as np
import pytest
import torch

import routed_reference as rr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pm():
    import paper_2206_08369_amd as pm
    assert torch.cuda.is_available()
    return pm


def blocks(F, hs):
    off = np.concatenate([[0], np.cumsum(hs)])
    return [slice(int(a), int(b)) for a, b in zip(off, off[1:])]


def check(got, U, parts, n=5):
    """Every model's matrix of `got` against the steps on that of U (both [N, F])."""
    got, U = got.cpu().double(), U.cpu().double()
    for m, r in enumerate(parts):
        want, bound = rr.orthogonalized(U[r], n)
        off = float((got[r] - want).abs().max())
        assert off <= float(bound), "model %d %s off by %.3g, %.3g allowed" % (
            m, tuple(want.shape), off, float(bound))


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


SHAPES = [(1, [1]), (1, [1, 2, 70, 300]), (2, [1, 3]), (10, list(range(1, 11))), (33, [31, 32, 33, 100]),
          (64, [64, 65, 1, 7]), (100, [1, 50, 99, 100, 101, 140, 250]), (127, [128, 129, 127, 400]),
          (130, [130, 260, 3]), (300, [16, 17, 200, 350]), (1000, [5, 100, 130])]


@pytest.mark.parametrize("strong", [False, True])
@pytest.mark.parametrize("F,hs", SHAPES, ids=lambda v: str(v) if isinstance(v, int) else "M%d" % len(v))
def test_input_weights(pm, F, hs, strong):
    net = pm.PackedMLP(F, 2, hs, [0] * len(hs))
    N = sum(hs)
    G = randn(F, N, F)
    if strong:
        G = 0.01 * G + randn(F + 1, N, 2) @ randn(F + 2, 2, F)
    G = 1e-4 * G
    got = net.orthogonalize(G.cuda())
    check(got, G, blocks(F, hs))
    assert torch.equal(got, net.orthogonalize(G.cuda()))


@pytest.mark.parametrize("F,top", [(100, 100), (128, 128), (9, 128), (140, 70)])
def test_many_matrices(pm, F, top):
    """More than 2,048 small ones go in launches by size; every ninth is compared."""
    hs = [1 + (37 * m) % top for m in range(2100)] + [150]
    net = pm.PackedMLP(F, 2, hs, [0] * len(hs))
    G = randn(F + top, sum(hs), F)
    got = net.orthogonalize(G.cuda())
    check(got, G, blocks(F, hs)[::9] + blocks(F, hs)[-1:])
    assert torch.equal(got, net.orthogonalize(G.cuda()))


def test_many_large_matrices(pm):
    """Enough of them for the larger tiles; three are compared."""
    hs = [1000] * 17 + [129, 900]
    net = pm.PackedMLP(1000, 2, hs, [0] * len(hs))
    G = randn(3, sum(hs), 1000)
    got = net.orthogonalize(G.cuda())
    check(got, G, [blocks(1000, hs)[k] for k in (0, 17, 18)])
    assert torch.equal(got, net.orthogonalize(G.cuda()))


@pytest.mark.parametrize("n", [1, 2, 3, 8, 10])
def test_steps(pm, n):
    hs = [3, 40, 150]
    net = pm.PackedMLP(60, 2, hs, [0] * 3)
    G = randn(n, 193, 60)
    check(net.orthogonalize(G.cuda(), steps=n), G, blocks(60, hs), n)


@pytest.mark.parametrize("O", [2, 3, 16])
def test_output_weights(pm, O):
    hs = [1, 2, 3, 16, 17, 200, 1500]
    net = pm.PackedMLP(5, O, hs, [0] * len(hs))
    G = randn(O, O, sum(hs))
    got = net.orthogonalize(G.cuda(), "W2")
    check(got.t(), G.t(), blocks(O, hs))


def test_gate_weights(pm):
    hs = [5, 70]
    net = pm.BlockPackedMLP(40, 2, hs, [7, 2], gated=True)
    G = randn(1, 75, 40)
    check(net.orthogonalize(G.cuda(), "V1"), G, blocks(40, hs))


def test_two_layer_packs(pm):
    h1, h2 = [1, 5, 40, 130, 64], [3, 5, 150, 33, 200]
    net = pm.DeepPackedMLP(7, 3, h1, h2, [2] * 5)
    sizes = [a * b for a, b in zip(h1, h2)]
    G = randn(2, sum(sizes))
    got = net.orthogonalize(G.cuda(), "W12")
    for a, b, g, u in zip(h1, h2, got.cpu().split(sizes), G.split(sizes)):
        check(g.reshape(b, a), u.reshape(b, a), [slice(0, b)])
    G2 = randn(3, 3, sum(h2))
    check(net.orthogonalize(G2.cuda(), "W2").t(), G2.t(), blocks(0, h2))
    G1 = randn(4, sum(h1), 7)
    check(net.orthogonalize(G1.cuda(), "W1"), G1, blocks(7, h1))
    before = net.get_params()
    net.muon_step(G.cuda(), 0.25, "W12")
    net.muon_step(G2.cuda(), 0.25, "W2")
    after = net.get_params()
    scale = np.concatenate([np.full(n, max(1, b / a) ** 0.5) for n, a, b in zip(sizes, h1, h2)])
    assert np.allclose(before[1] - after[1], 0.25 * scale * got.cpu().numpy(), rtol=0, atol=1e-6)
    assert np.array_equal(before[0], after[0]) and not np.array_equal(before[2], after[2])


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-12, 1e12, 1e30, 1e37])
def test_any_scale(pm, scale):
    hs = [4, 70, 130]
    net = pm.PackedMLP(50, 2, hs, [0] * 3)
    G = (randn(7, 204, 50).double() * scale).float()
    check(net.orthogonalize(G.cuda()), G, blocks(50, hs))


def test_zero_and_low_rank_and_diverged_matrices(pm):
    hs = [4, 4, 70, 70, 70, 200, 200, 9]
    net = pm.PackedMLP(50, 2, hs, [0] * len(hs))
    parts = blocks(50, hs)
    G = randn(8, sum(hs), 50)
    G[parts[0]] = 0
    G[parts[2]] = 0
    G[parts[3]] = torch.outer(randn(9, 70), randn(10, 50))
    G[parts[5], 10:] = 0
    clean = net.orthogonalize(G.cuda())
    check(clean, G, parts)
    assert not bool(clean[parts[0]].any()) and not bool(clean[parts[5], 10:].any())
    for bad in (float("nan"), float("inf"), -float("inf")):
        H = G.clone()
        for k in (1, 4, 6):
            H[parts[k].start + 1, 3] = bad
        got = net.orthogonalize(H.cuda())
        for k, r in enumerate(parts):
            if k in (1, 4, 6):
                assert bool(got[r].isnan().all())
            else:
                assert torch.equal(got[r], clean[r])


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_momentum(pm, nesterov, in_place):
    hs = [3, 40, 150]
    net = pm.PackedMLP(60, 2, hs, [0] * 3)
    G, mom = randn(1, 193, 60), randn(2, 193, 60)
    g, m = G.cuda(), mom.cuda()
    new = m if in_place else torch.empty_like(m)
    out = g if in_place else None
    got = net.orthogonalize(g, momentum=m, mu=0.9, nesterov=nesterov,
                            momentum_out=None if in_place else new, out=out)
    mu = float(np.float32(0.9))
    want = mu * mom.double() + G.double()
    # a product and a sum
    assert bool(((new.cpu().double() - want).abs()
                 <= rr.U * 2 * (mom.abs() + want.abs())).all())
    held = new.cpu().double()
    check(got, G.double() + mu * held if nesterov else held, blocks(60, hs))
    if not in_place:
        assert torch.equal(m.cpu(), mom) and torch.equal(g.cpu(), G)


@pytest.mark.parametrize("matrix", ["W1", "W2"])
@pytest.mark.parametrize("steps", [0, 5])
@pytest.mark.parametrize("per_model", [False, True])
def test_muon_step(pm, matrix, steps, per_model):
    hs = [3, 40, 150, 2]
    F, O, N = 33, 4, 195
    net = pm.PackedMLP(F, O, hs, [0] * 4)
    G = randn(3, *((N, F) if matrix == "W1" else (O, N)))
    mom = randn(4, *G.shape)
    rates = torch.tensor([0.1, 0.0, 0.5, 0.25])
    before = [torch.from_numpy(v).double() for v in net.get_params()]
    m = mom.cuda()
    net.muon_step(G.cuda(), rates.cuda() if per_model else 0.3, matrix, momentum=m, mu=0.8,
                  steps=steps, decay=0.05)
    after = [torch.from_numpy(v).double() for v in net.get_params()]
    mu, decay = float(np.float32(0.8)), float(np.float32(0.05))
    held = m.cpu().double()
    U = G.double() + mu * held
    k = 0 if matrix == "W1" else 1
    assert torch.equal(before[1 - k], after[1 - k])
    for i, r in enumerate(blocks(F, hs)):
        view = (r, slice(None)) if matrix == "W1" else (slice(None), r)
        lr = float(rates[i]) if per_model else float(np.float32(0.3))
        u, w = U[view], before[k][view]
        if steps:
            d, bound = rr.orthogonalized(u, steps)
            gain = max(1.0, u.shape[0] / u.shape[1]) ** 0.5
            d, bound = gain * d, gain * bound
        else:
            d, bound = u, 2 * rr.U * u.abs().max()
        want = w - lr * (decay * w + d)
        off = (after[k][view] - want).abs()
        assert bool((off <= lr * bound + 4 * rr.U * (w.abs() + lr * d.abs())).all())


def test_no_momentum_equals_orthogonalize(pm):
    hs = [30, 9]
    net = pm.PackedMLP(20, 2, hs, [0, 0])
    G = randn(5, 39, 20).cuda()
    before = net.get_params()[0]
    net.muon_step(G, 1.0)
    gain = np.repeat(np.float32([np.sqrt(1.5), 1.0]), hs)[:, None]
    want = before - gain * net.orthogonalize(G).cpu().numpy()
    assert np.allclose(net.get_params()[0], want, rtol=0, atol=1e-6)


def test_update_reaches_the_bf16_copy(pm):
    net = pm.PackedMLP(20, 2, [30, 9], [2, 2], precision=pm.PMLP_BF16_GEMM)
    X = randn(6, 40, 20).cuda()
    old = net.forward(X)
    net.muon_step(randn(5, 39, 20).cuda(), 1.0)
    new = net.forward(X)
    other = pm.PackedMLP(20, 2, [30, 9], [2, 2], precision=pm.PMLP_BF16_GEMM)
    other.set_params(*net.get_params())
    assert torch.equal(new, other.forward(X)) and not torch.equal(old, new)


def test_bad_rate_is_reported(pm):
    net = pm.PackedMLP(20, 2, [30, 9], [2, 2])
    X, y = randn(6, 40, 20).cuda(), torch.zeros(40, dtype=torch.int32).cuda()
    net.train_step(X, y, 0.1)
    net.losses()
    for steps in (0, 5):
        net.muon_step(randn(5, 39, 20).cuda(), torch.tensor([0.1, float("nan")]).cuda(), steps=steps)
        with pytest.raises(pm.PmlpError, match="learning rate"):
            net.losses()
        net.losses()


def test_biases_keep_out_of_it(pm):
    hs = [30, 9]
    net = pm.PackedMLP(22, 2, hs, [2, 2], biases=True)
    b = net.get_biases()
    G = randn(5, 39, 22)
    check(net.orthogonalize(G.cuda()), G, blocks(22, hs))
    net.muon_step(G.cuda(), 0.5)
    assert all(np.array_equal(x, y) for x, y in zip(b, net.get_biases()))


@pytest.mark.parametrize("big", [False, True])
def test_captured_and_replayed(pm, big):
    hs = [300, 140] if big else [30, 9]
    N = sum(hs)
    net = pm.PackedMLP(200 if big else 20, 2, hs, [0, 0])
    G, mom = randn(1, N, net.F).cuda(), torch.zeros(N, net.F).cuda()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        net.orthogonalize(G, momentum=mom)
    s.synchronize()
    mom.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        U = net.orthogonalize(G, momentum=mom)
    want_mom = torch.zeros_like(mom)
    for turn in range(4):
        G.copy_(randn(turn, N, net.F))
        want = net.orthogonalize(G, momentum=want_mom)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(U, want) and torch.equal(mom, want_mom), turn


def test_nothing_else_is_written(pm):
    hs = [31, 9]
    net = pm.PackedMLP(21, 3, hs, [0, 0])
    for matrix, n in (("W1", 40 * 21), ("W2", 120)):
        buf = torch.full((3, n + 128), 7.5).cuda()
        buf[0, 64:64 + n] = randn(1, n).cuda()
        buf[1, 64:64 + n] = randn(2, n).cuda()
        at = [v[64:].data_ptr() for v in buf]
        pm.pmlp_set_stream(net.handle, torch.cuda.current_stream().cuda_stream)
        pm.pmlp_orthogonalize(net.handle, pm.MATRIX_IDS[matrix], at[0], at[1], at[1], 0.9, True, 5, at[2])
        torch.cuda.synchronize()
        assert bool((buf[:, :64] == 7.5).all()) and bool((buf[:, 64 + n:] == 7.5).all())


def test_refusals(pm):
    net = pm.PackedMLP(20, 2, [30, 9], [2, 2])
    G = randn(5, 39, 20).cuda()
    for call in (lambda: net.orthogonalize(G.cpu()), lambda: net.orthogonalize(G.double()),
                 lambda: net.orthogonalize(G.t()), lambda: net.orthogonalize(G, "W2"),
                 lambda: net.orthogonalize(G, "W9"), lambda: net.orthogonalize(G, momentum_out=G),
                 lambda: net.orthogonalize(G, momentum=G[:3]), lambda: net.orthogonalize(G, out=G.t()),
                 lambda: net.muon_step(G, torch.ones(3).cuda()), lambda: net.muon_step(G, torch.ones(2))):
        with pytest.raises(ValueError):
            call()
    for matrix in ("V1", "W12"):
        with pytest.raises((pm.PmlpError, ValueError)):
            net.orthogonalize(G, matrix)
    h = net.handle
    out = torch.empty_like(G)
    for args, msg in (((9, G, None, None, 0.9, True, 5, out), "unknown matrix"),
                      ((-1, G, None, None, 0.9, True, 5, out), "unknown matrix"),
                      ((0, None, None, None, 0.9, True, 5, out), "null gradient"),
                      ((0, G, None, None, 0.9, True, 5, None), "null output"),
                      ((0, G, G, None, 0.9, True, 5, out), "both"),
                      ((0, G, None, out, 0.9, True, 5, out), "both"),
                      ((0, G, None, None, 0.9, True, 0, out), "steps"),
                      ((0, G, None, None, 0.9, True, 11, out), "steps"),
                      ((0, G, None, None, float("nan"), True, 5, out), "finite"),
                      ((0, G, out, G, 0.9, True, 5, out), "overlap"),
                      ((0, G, out, out, 0.9, True, 5, out), "overlap"),
                      ((0, G, None, None, 0.9, True, 5, G[1:]), "overlap")):
        with pytest.raises(pm.PmlpError, match=msg):
            pm.pmlp_orthogonalize(h, *args)
    for args, msg in (((0, G, G, 0.9, True, 5, 0.1), "overlap"), ((0, G, None, 0.9, True, -1, 0.1), "steps"),
                      ((0, G, None, 0.9, True, 5, float("inf")), "finite"),
                      ((1, G, None, 0.9, True, 5, 0.1), "no gate"),
                      ((3, G, None, 0.9, True, 5, 0.1), "second hidden layer")):
        with pytest.raises(pm.PmlpError, match=msg):
            pm.pmlp_muon_step(h, *args)


# plans of small matrices: (F, O, widths, matrix) with few rows only, with both kinds in one
# launch, in two, and by class
PLANS = [(10, 2, [1 + 7 * i % 16 for i in range(300)], "W1"),
         (300, 3, [512, 257, 129, 128, 16, 1] * 9, "W2"), (200, 2, [32, 31, 17, 16] * 5, "W1"),
         (40, 2, [3, 33, 40, 16] * 250, "W1"), (40, 2, [3, 33, 40, 16] * 300, "W1"),
         (140, 2, [3, 33, 16, 100] * 520, "W1"), (256, 16, [600, 513, 250, 8] * 4, "W2")]


@pytest.mark.parametrize("F,O,hs,matrix", PLANS, ids=lambda v: "M%d" % len(v) if isinstance(v, list) else str(v))
def test_plans_of_small_matrices(pm, F, O, hs, matrix):
    net = pm.PackedMLP(F, O, hs, [7] * len(hs))
    G = randn(F + len(hs), *((O, net.N) if matrix == "W2" else (net.N, F)))
    got = net.orthogonalize(G.cuda(), matrix)
    assert torch.equal(got, net.orthogonalize(G.cuda(), matrix))
    if matrix == "W2":
        got, G = got.t(), G.t()
    check(got, G, blocks(F, hs)[::len(hs) // 60 | 1])  # (an odd step: widths of all kinds)
