"""Bounds of the Newton-Schulz steps for matrices whose rows and columns are of unlike size.

A matrix is D M0 E with D and E diagonal and M0 of even size.  The steps commute with E
(X <- (a + P) X) and treat a row of X as a whole, so what fp32 keeps is measured beside a row's
and a column's own size, not beside the largest entry."""
import torch

import routed_reference as rr


def orthogonalized(M, n, rows, cols):
    """The direction of M (float64, of r <= c or not) after n steps and a bound of the error of
    every entry; rows and cols: the sizes of its rows and columns (D and E).

    As routed_reference.orthogonalized: the arithmetic holds values to 23 bits and leaves out
    2^-22 of a product, modelled by the steps with every operand and result moved by up to
    2^-22 of itself at random (four times), and a sum of k products in fp32 adds up to
    sqrt(k / 2) of that.  Here the effect is measured row by row, each entry beside its
    column's size: 8 (1 + sqrt(k / 2)) times its mean size.  (A scale of powers of two that a
    row or column is held with and that is up to 2^15 above its entries adds 2^-39 + 15, a
    quarter of 2^-22, to what a value is held to.)"""
    want = rr.steps(M / M.norm(), n)
    moved = torch.zeros_like(want)
    for seed in range(4):
        gen = torch.Generator().manual_seed(M.numel() + seed)
        move = lambda t: t * (1 + 2 ** -22 * (2 * torch.rand(t.shape, generator=gen).double() - 1))
        moved += (rr.steps(M / M.norm(), n, move) - want).pow(2) / 4
    size = lambda t: (t / cols.pow(2)).mean(1, keepdim=True).sqrt()
    typical = size(moved) + 2 ** -22 * size(want.pow(2))
    return want, 8 * (1 + (max(M.shape) / 2) ** 0.5) * typical * cols


def unlike(r, c, kind, seed=0, least=-12):
    """(M, rows, cols): an r x c matrix of float32 values whose rows, columns or both are up to
    10^least times as large as others; "aligned": its small rows are nearly multiples of the
    first one, so that they do not grow in the steps as small singular values do."""
    g = torch.Generator().manual_seed(100 * r + c + seed)
    M = torch.randn(r, c, generator=g).double()
    sizes = lambda n: 10.0 ** torch.randint(least, 1, (n,), generator=g).double()
    rows, cols = torch.ones(r, 1).double(), torch.ones(1, c).double()
    if kind != "columns":
        rows = sizes(r)[:, None]
        rows[0] = 1
    if kind in ("columns", "both"):
        cols = sizes(c)[None]
        cols[0, 0] = 1
    if kind == "aligned":
        M[1:] = M[0] * torch.randn(r - 1, 1, generator=g).double() + 0.01 * M[1:]
    return (M * rows * cols).float().double(), rows, cols


KINDS = ("rows", "columns", "both", "aligned")
