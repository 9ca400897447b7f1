"""The bounds for rows and columns of unlike size hold for plain fp32 steps, and not for
values that are held to a fraction of the largest one."""
import pytest
import torch

import newton_bounds as nb


def float32_steps(M, n):
    X = (M / M.norm()).float()
    turned = X.shape[0] > X.shape[1]
    X = X.T if turned else X
    for _ in range(n):
        A = X @ X.T
        X = 3.4445 * X + (-4.7750 * A + 2.0315 * (A @ A)) @ X
    return (X.T if turned else X).double()


def excess(got, want_bound):
    want, bound = want_bound
    return float(((got - want).abs() / bound).max())


@pytest.mark.parametrize("n", [1, 5, 10])
@pytest.mark.parametrize("kind", nb.KINDS)
@pytest.mark.parametrize("r,c", [(2, 9), (8, 100), (70, 40), (64, 64)])
def test_fp32_keeps_small_rows_and_columns(r, c, kind, n):
    M, rows, cols = nb.unlike(r, c, kind)
    assert excess(float32_steps(M, n), nb.orthogonalized(M, n, rows, cols)) <= 1


@pytest.mark.parametrize("kind", nb.KINDS)
def test_values_held_beside_the_largest_do_not(kind):
    M, rows, cols = nb.unlike(8, 100, kind)
    X = M / M.norm()

    def held(t):  # steps of 2^-38 whatever the value
        return (t * 2.0 ** 38).round() * 2.0 ** -38

    import routed_reference as rr
    assert excess(rr.steps(X, 5, held), nb.orthogonalized(M, 5, rows, cols)) > 10
