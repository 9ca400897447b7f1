"""The float64 reference of the block packs against definitions that share
nothing with it: central differences of its losses, PyTorch's float64 layer norm
and autograd, and known special cases."""
import numpy as np
import pytest

import block_reference as ref

KINDS = [(True, False), (False, True), (True, True)]
SMOOTH = (0, 2, 3, 4, 6, 7, 8, 9, 12)


def problem(gated, norm, head, hs, acts, F=5, O=3, B=7, seed=0):
    rng = np.random.default_rng(seed)
    p = ref.random_params(rng, hs, F, O, gated, norm)
    X = rng.standard_normal((B, F)).astype(np.float32)
    y = rng.standard_normal((B, O)) if head == "mse" else rng.integers(0, O, B)
    return p, X, y


@pytest.mark.parametrize("head", ["ce", "mse"])
@pytest.mark.parametrize("gated,norm", KINDS)
def test_gradients_against_differences(gated, norm, head):
    hs, acts = np.arange(1, 10), np.array(SMOOTH)
    p, X, y = problem(gated, norm, head, hs, acts)
    p = {k: v.astype(np.float64) for k, v in p.items()}
    got = ref.pack(hs, acts, p, X, y, head)
    rng = np.random.default_rng(1)
    step = 1e-6
    for name, v in p.items():
        for _ in range(12):
            at = tuple(rng.integers(0, n) for n in v.shape)
            d = []
            for s in (step, -step):
                q = {k: w.copy() for k, w in p.items()}
                q[name][at] += s
                d.append(ref.pack(hs, acts, q, X, y, head)["loss"][0].sum())
            # truncation step^2 f''' / 6 (f''' up to 1e4 through the norm of two
            # units), rounding 1e-15 / step
            assert abs((d[0] - d[1]) / (2 * step) - got[name][0][at]) < 2e-8, (name, at)


@pytest.mark.parametrize("gated,norm", KINDS)
def test_against_autograd(gated, norm):
    torch = pytest.importorskip("torch")
    t = torch.nn.functional
    F, O, B, h = 6, 4, 9, 11
    p, X, y = problem(gated, norm, "ce", np.array([h]), [7], F=F, O=O, B=B)
    w = {k: torch.tensor(v, dtype=torch.float64, requires_grad=True) for k, v in p.items()}
    x = torch.tensor(X, dtype=torch.float64)
    H = t.silu(x @ w["W1"].T)
    if gated:
        H = H * (x @ w["V1"].T)
    if norm:
        H = t.layer_norm(H, (h,), w["gain"], w["shift"], eps=ref.EPS)
    L = H @ w["W2"].T
    t.cross_entropy(L, torch.tensor(y)).backward()
    got = ref.pack([h], [7], p, X, y)
    assert np.abs(got["logits"][0][:, 0] - L.detach().numpy()).max() < 1e-13
    for k, v in w.items():
        assert np.abs(got[k][0] - v.grad.numpy()).max() < 1e-13, k


def test_bounds_hold_for_float32():
    """A float32 evaluation of the same formulas stays inside the bounds, and the
    bounds are of float32's order."""
    hs, acts = np.array([8, 40]), np.array([7, 6])
    p, X, y = problem(True, True, "ce", hs, acts, F=30, B=20)
    val, bound = ref.pack(hs, acts, p, X, y)["logits"]
    L = []
    for m in range(2):
        q = ref.model_params(p, hs, m)
        z = X @ q["W1"].T
        H = ref.act(int(acts[m]), z)[0].astype(np.float32) * (X @ q["V1"].T)
        D = H - H.mean(1, keepdims=True, dtype=np.float32)
        n = D / np.sqrt((D * D).mean(1, keepdims=True, dtype=np.float32) + np.float32(1e-5))
        L.append((n * q["gain"] + q["shift"]) @ q["W2"].T)
    assert np.all(np.abs(np.stack(L, 1) - val) <= bound)
    assert np.median(bound / np.abs(val)) < 1e-3


def test_norm_of_one_unit_is_its_shift():
    p, X, y = problem(True, True, "ce", np.array([1]), [7])
    got = ref.pack([1], [7], p, X, y)
    assert np.allclose(got["logits"][0], (p["W2"].astype(float) @ p["shift"])[None, None])
    assert not got["W1"][0].any() and not got["V1"][0].any() and not got["gain"][0].any()
