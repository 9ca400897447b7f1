"""Block packs with a norm whose hidden values lie far from zero: the outputs keep
the precision of the deviations (H - mu), however large the mean beside them."""
import numpy as np
import pytest

import block_reference as ref

pytestmark = pytest.mark.gpu

U = ref.U


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


def problem(rng, hs, F, O, B, mean, gated, paired):
    """Identity units whose values are mean + k / 64, |k| <= 32 and thus exact in
    float32 (mean a power of two up to 2^17), as are the sums of the output weights
    (multiples of 1/64).  paired: the second half of a model's units has the values of
    the first half and the opposite weights, so that without the shifts its logits
    are zero."""
    N = int(hs.sum())
    W1 = np.zeros((N, F))
    W1[:, 0] = mean
    W1[:, F - 1] = rng.integers(-16, 17, N) / 64
    X = rng.integers(-3, 4, (B, F)).astype(np.float64)
    X[:, 0] = 1
    X[:, F - 1] = rng.choice([-2, -1, 1, 2], B)
    p = {"W1": W1, "gain": np.ones(N), "shift": rng.integers(-8, 9, N) / 64,
         "W2": rng.integers(1, 64, (O, N)) / 64}
    if gated:
        p["V1"] = np.zeros((N, F))
        p["V1"][:, 0] = 1
    at = 0
    for h in hs:
        if paired:
            half = int(h) // 2
            W1[at + half:at + 2 * half] = W1[at:at + half]
            p["W2"][:, at + half:at + 2 * half] = -p["W2"][:, at:at + half]
            p["W2"][:, at + 2 * half:at + int(h)] = 0
        else:
            p["W2"][:, at:at + int(h)] *= rng.choice([-1, 1], (O, int(h)))
        at += int(h)
    return {k: v.astype(np.float32) for k, v in p.items()}, X.astype(np.float32)


def logit_bounds(hs, p, X, gated):
    """The values H are exact in float32.  With d the largest deviation of a model's
    units from their mean mu, every sum that the outputs are made of has terms of at most
    4 d g W2 (a unit's value from another's 2 d, its piece's mean from another piece's
    2 d) and each of its h + 16 roundings counts U of their magnitudes.

    The mean of a piece is rounded to float32, up to six times where pieces are merged
    before they are stored, and is 40 U d off by its sum's own roundings: `off`.  That
    is what the whole mean may be off by, which counts as often as the sum of g W2, and
    it changes the variance v by up to 4 off sqrt(v) + 4 off^2 (the pieces' means enter
    as sum n_k (m_k - mu)^2), a share x of it."""
    H = X.astype(np.float64) @ p["W1"].astype(np.float64).T
    if gated:
        H = H * (X.astype(np.float64) @ p["V1"].astype(np.float64).T)
    out, at = [], 0
    for h in hs:
        s = slice(at, at + int(h))
        at += int(h)
        hm = H[:, s]
        mu = hm.mean(1, keepdims=True)
        d = np.abs(hm - mu).max(1, keepdims=True)
        var = ((hm - mu) ** 2).mean(1, keepdims=True)
        r = (var + ref.EPS) ** -0.5
        gw = (p["gain"][s] * p["W2"][:, s]).astype(np.float64)
        P = r * ((hm - mu) @ gw.T)
        D = p["W2"][:, s].astype(np.float64) @ p["shift"][s]
        off = 6 * U * (np.abs(mu) + d) + 40 * U * d
        x = 4 * off * r + 4 * (off * r) ** 2
        assert x.max() < 0.9
        most = (1 - x) ** -0.5
        bound = most * r * ((h + 16) * U * 4 * d * np.abs(gw).sum(1)
                            + off * (np.abs(gw.sum(1)) + (h + 8) * U * np.abs(gw).sum(1)))
        bound = bound + np.abs(P) * ((h + 32) * U + most - 1)
        bound = bound + (h + 8) * U * (np.abs(p["W2"][:, s]) @ np.abs(p["shift"][s])) \
            + 2 * U * np.abs(P + D)
        out.append((P + D, bound))
    return np.stack([v[0] for v in out], 1), np.stack([v[1] for v in out], 1)


# small packs (their gradients in one launch), packs whose waves take several tiles,
# wide models, pre-activations that are stored; batches of one, of some and past 256
SHAPES = [(30, 30, 70, 9, 2, 40), (30, 30, 70, 36, 10, 1), (12, 30, 90, 64, 3, 300),
          (700, 30, 100, 8, 2, 100), (300, 30, 360, 12, 10, 33), (3, 900, 1500, 20, 16, 50),
          (20, 30, 70, 140, 2, 40), (20, 30, 70, 140, 10, 300), (4, 300, 700, 133, 4, 17)]


@pytest.mark.parametrize("paired", [True, False])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M, lo, hi, F, O, B", SHAPES)
def test_outputs_of_hidden_values_far_from_zero(pm, torch, M, lo, hi, F, O, B, gated, paired):
    rng = np.random.default_rng(M + F + O + B)
    hs = rng.integers(lo, hi + 1, M).astype(np.int32)
    for mean in (2.0 ** 14, -1024.0):
        p, X = problem(rng, hs, F, O, B, mean, gated, paired)
        val, bound = logit_bounds(hs, p, X, gated)
        net = pm.BlockPackedMLP(F, O, hs, np.zeros(M), gated=gated, norm=True)
        net.set_params(**p)
        err = np.abs(net.forward(dev(torch, X)).cpu().numpy() - val)
        assert (err <= bound).all(), "mean %g: %.3g times its bound" % (mean, (err / bound).max())
        # the loss of the training path: a mean of log-sum-exps, none of which moves by
        # more than twice the largest of its logits' errors
        y = rng.integers(0, O, B).astype(np.int32)
        net.gradients(dev(torch, X), dev(torch, y))
        top = val.max(2)
        lse = top + np.log(np.exp(val - top[:, :, None]).sum(2))
        lp = lse - val[np.arange(B), :, y]
        tol = 2 * bound.max(2).mean(0) + 16 * U * (np.abs(lse) + np.abs(top) + 1).mean(0) \
            + (B + 8) * U * np.abs(lp).mean(0)
        err = np.abs(net.losses() - lp.mean(0))
        assert (err <= tol).all(), "mean %g: loss, %.3g times its bound" % (mean, (err / tol).max())
        net.close()


def test_hidden_values_whose_squares_overflow(pm, torch):
    """Values of 2^66 in every unit of a model: they deviate by nothing, and the norm
    is its shift."""
    hs = np.int32([40, 3, 17])
    N, F, O, B = int(hs.sum()), 4, 3, 9
    p = {"W1": np.zeros((N, F), np.float32), "gain": np.ones(N, np.float32),
         "shift": np.full(N, 0.25, np.float32), "W2": np.full((O, N), 0.5, np.float32)}
    p["W1"][:, 0] = 2.0 ** 66
    net = pm.BlockPackedMLP(F, O, hs, [0, 0, 0], gated=False, norm=True)
    net.set_params(**p)
    L = net.forward(dev(torch, np.ones((B, F), np.float32))).cpu().numpy()
    assert np.array_equal(L, np.broadcast_to((hs / 8).astype(np.float32)[None, :, None], L.shape))
    net.close()
