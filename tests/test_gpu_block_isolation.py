"""Block packs: a diverged model changes nothing for the models that share its
tiles, in the gradients and in the parameters after training steps."""
import numpy as np
import pytest

import block_reference as ref

pytestmark = pytest.mark.gpu

KINDS = {"gated": (True, False), "norm": (False, True), "both": (True, True)}


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    torch.cuda.set_device(0)
    return torch


@pytest.fixture(scope="module")
def pm(torch):
    import paper_2206_08369_amd as pm
    pm.load_library()
    return pm


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def units_of_others(hs, bad):
    off = np.concatenate([[0], np.cumsum(hs)])
    keep = np.ones(off[-1], bool)
    for m in bad:
        keep[off[m]:off[m + 1]] = False
    return off, keep


# One activation, so that tiles of the backward hold several models: batches that run
# in three launches (past 256 samples, or a pool past what one launch takes) and in one,
# and inputs whose pre-activations are stored.
@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("where", ["W1", "V1", "W2"])
@pytest.mark.parametrize("M, O, F, B", [(70, 5, 9, 290), (70, 10, 36, 300), (70, 16, 8, 257),
                                        (70, 4, 9, 290), (70, 2, 9, 290), (70, 16, 9, 40),
                                        (5000, 10, 6, 40), (70, 10, 140, 290)])
def test_a_diverged_model_stays_alone(pm, torch, kind, where, M, O, F, B):
    gated, norm = KINDS[kind]
    if where == "V1" and not gated:
        where = "W1"
    rng = np.random.default_rng(M + 10 * O + F + B)
    hs = rng.integers(1, 10, M).astype(np.int32)
    acts = np.full(M, 7, np.int32)
    good = ref.random_params(rng, hs, F, O, gated, norm)
    bad = [1, M // 2, M - 1]
    off, keep = units_of_others(hs, bad)
    broken = {k: v.copy() for k, v in good.items()}
    for m, v in zip(bad, (np.nan, np.inf, np.nan)):
        n = off[m] + (hs[m] - 1) // 2
        if where == "W2":
            broken["W2"][1, n] = v
        else:
            broken[where][n, 0] = v
    X = dev(torch, rng.standard_normal((B, F)).astype(np.float32))
    y = dev(torch, rng.integers(0, O, B).astype(np.int32))
    nets = []
    for p in (good, broken):
        net = pm.BlockPackedMLP(F, O, hs, acts, seed=3, gated=gated, norm=norm)
        net.set_params(**p)
        nets.append(net)
    others = dev(torch, keep)
    for k, a, b in zip(nets[0].param_names, nets[0].gradients(X, y), nets[1].gradients(X, y)):
        a, b = (a[:, others], b[:, others]) if k == "W2" else (a[others], b[others])
        assert torch.isfinite(a).all()
        assert torch.equal(a, b), "d" + k
    assert nets[1].nonfinite_count() == len(bad)
    for _ in range(3):
        for net in nets:
            net.train_step(X, y, 0.05)
    for k, a, b in zip(nets[0].param_names, nets[0].get_params(), nets[1].get_params()):
        a, b = (a[:, keep], b[:, keep]) if k == "W2" else (a[keep], b[keep])
        assert np.isfinite(a).all() and np.array_equal(a, b), k
    assert nets[0].nonfinite_count() == 0
    assert nets[1].nonfinite_count() == 3 * len(bad)
    for net in nets:
        net.close()


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_a_diverged_regression_stays_alone(pm, torch, kind):
    """Squared errors that overflow: the gradients of the outputs are infinite."""
    gated, norm = KINDS[kind]
    M, O, F, B = 50, 7, 5, 300
    rng = np.random.default_rng(2)
    hs = rng.integers(1, 6, M).astype(np.int32)
    p = ref.random_params(rng, hs, F, O, gated, norm)
    off, keep = units_of_others(hs, [20])
    X = dev(torch, rng.standard_normal((B, F)).astype(np.float32))
    Y = dev(torch, rng.standard_normal((B, O)).astype(np.float32))
    net = pm.BlockPackedMLP(F, O, hs, np.full(M, 2), gated=gated, norm=norm, head="mse")
    net.set_params(**p)
    want = net.gradients(X, Y)
    p["W2"][:, off[20]] = np.inf
    net.set_params(W2=p["W2"])
    others = dev(torch, keep)
    for k, a, b in zip(net.param_names, want, net.gradients(X, Y)):
        a, b = (a[:, others], b[:, others]) if k == "W2" else (a[others], b[others])
        assert torch.isfinite(a).all() and torch.equal(a, b), "d" + k
    net.close()
