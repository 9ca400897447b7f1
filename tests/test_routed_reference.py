"""The 64-bit reference of routed packs against differences, and of the orthogonalised
update against its singular values."""
import numpy as np
import pytest
import torch

import routed_reference as rr


@pytest.mark.parametrize("gated", [False, True])
def test_gradients_against_differences(gated):
    rng = np.random.default_rng(3)
    hs, acts = [3, 1, 4, 2], [2, 7, 6, 9]
    F, O, B, K = 5, 3, 6, 2
    t = lambda *s: torch.from_numpy(rng.standard_normal(s))
    X, W1, V1, W2, dY = t(B, F), t(10, F), t(10, F) if gated else None, t(O, 10), t(B, O)
    w = t(B, K)
    idx = torch.from_numpy(rng.integers(-1, 4, (B, K)))
    idx[0], idx[1] = torch.tensor([2, 2]), torch.tensor([-1, -1])
    grads = rr.mixture(hs, acts, X, idx, w, W1, V1, W2, dY)
    loss = lambda: float((rr.mixture(hs, acts, X, idx, w, W1, V1, W2)["Y"][0] * dY).sum())
    for name, p in (("W1", W1), ("V1", V1), ("W2", W2), ("weight", w)):
        if p is None:
            continue
        flat = p.reshape(-1)
        for i in range(flat.numel()):
            old, e = float(flat[i]), 1e-5
            flat[i] = old + e
            up = loss()
            flat[i] = old - e
            down = loss()
            flat[i] = old
            # (central differences: e^2 f''' / 6, and 2^-53 / e of the loss)
            assert abs((up - down) / (2 * e) - float(grads[name][0].reshape(-1)[i])) < 1e-7


def test_route_gradient_against_differences():
    rng = np.random.default_rng(4)
    s = rng.standard_normal((1, 6))
    idx, w = rr.route(s, 3)
    dw = rng.standard_normal(3)
    ds = w[0] * (dw - (w[0] * dw).sum())
    for k, m in enumerate(idx[0]):
        e = 1e-6
        up, down = s.copy(), s.copy()
        up[0, m] += e
        down[0, m] -= e
        diff = ((rr.route(up, 3)[1] - rr.route(down, 3)[1])[0] * dw).sum() / (2 * e)
        assert abs(diff - ds[k]) < 1e-8


@pytest.mark.parametrize("shape", [(1, 1), (1, 9), (9, 1), (6, 17), (17, 6)])
def test_steps_are_the_scalar_polynomial_of_the_singular_values(shape):
    g = torch.Generator().manual_seed(5)
    M = torch.randn(*shape, generator=g).double()
    want, _ = rr.orthogonalized(M, 5)
    u, s, vh = torch.linalg.svd(M / M.norm(), full_matrices=False)
    a, b, c = rr.COEF
    for _ in range(5):
        s = s * (a + b * s ** 2 + c * s ** 4)
    assert float((want - u @ torch.diag(s) @ vh).abs().max()) < 1e-12
