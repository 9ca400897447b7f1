"""Routed packs and orthogonalised updates in 64 bits, with bounds of what float32
kernels may be off by.

U is half a step of float32 (2^-24).  A sum of n float32 products is off by at most
(n + 2) U times the sum of the absolute products, whatever its order; the products of
three-piece operands leave out at most 2 U of each (the bounds below take 2 (n + 8) U)."""
import numpy as np
import torch

U = 2.0 ** -24
SMOOTH = (0, 2, 3, 4, 6, 7, 8, 9, 12)  # activations with a continuous slope
L1, L2 = 1.2, 2.6   # no slope of an activation is above L1, no change of one above L2
ACT_ABS, ACT_REL = 4e-7, 16 * U  # what the activations themselves are off by


def act(a, z):
    """Value and slope of activation a, float64."""
    s = torch.sigmoid(z)
    if a == 0:
        return z, torch.ones_like(z)
    if a == 1:
        return torch.relu(z), (z > 0).double()
    if a == 2:
        t = torch.tanh(z)
        return t, 1 - t * t
    if a == 3:
        return s, s * (1 - s)
    if a == 4:
        return torch.where(z > 0, z, torch.expm1(z)), torch.where(z > 0, 1.0, torch.exp(z))
    if a == 5:
        return torch.where(z > 0, z, 0.01 * z), torch.where(z > 0, 1.0, 0.01).double()
    if a == 6:
        c = 0.5 * torch.special.erfc(-z / 2 ** 0.5)
        return z * c, c + z * torch.exp(-0.5 * z * z) / (2 * np.pi) ** 0.5
    if a == 7:
        return z * s, s + z * s * (1 - s)
    if a == 8:
        return torch.nn.functional.softplus(z), s
    if a == 9:
        t = torch.sigmoid(2 * z)
        return z * t, t + 2 * z * t * (1 - t)
    if a == 10:
        k, l = 1.6732632423543772, 1.0507009873554805
        return (torch.where(z > 0, l * z, l * k * torch.expm1(z)),
                torch.where(z > 0, l, l * k * torch.exp(z)))
    if a == 11:
        on = z.abs() > 0.5
        return torch.where(on, z, 0.0), on.double()
    t = torch.tanh(torch.nn.functional.softplus(z))
    return z * t, t + z * (1 - t * t) * s


def route(scores, K):
    """idx [B, K] and weights of the K best scores (float64 numpy arrays)."""
    B, M = scores.shape
    idx = np.full((B, K), -1, np.int32)
    w = np.zeros((B, K))
    for b in range(B):
        live = [m for m in range(M) if scores[b, m] > -np.inf]
        live.sort(key=lambda m: (-scores[b, m], m))
        live = live[:K]
        if live:
            s = scores[b, live].astype(np.float64)
            e = np.exp(s - s[0])
            idx[b, :len(live)] = live
            w[b, :len(live)] = e / e.sum()
    return idx, w


def mixture(hs, acts, X, idx, w, W1, V1, W2, dY=None):
    """Y, or with dY the gradients, each with the bound of its error:
    {"Y": (value, bound)} or {"W1", "V1", "W2", "weight"}.  All float64 tensors."""
    hs = [int(h) for h in hs]
    B, K = idx.shape
    O, F = W2.shape[0], X.shape[1]
    off = np.concatenate([[0], np.cumsum(hs)])
    gated = V1 is not None
    zeros = lambda t: torch.zeros_like(t)
    Y, eY = torch.zeros(B, O).double(), torch.zeros(B, O).double()
    out = {}
    if dY is not None:
        out = {k: (zeros(v), zeros(v)) for k, v in (("W1", W1), ("V1", V1), ("W2", W2))
               if v is not None}
        out["weight"] = (torch.zeros(B, K).double(), torch.zeros(B, K).double())
    flat = idx.reshape(-1)
    for m, h in enumerate(hs):
        s = torch.nonzero(flat == m).reshape(-1)
        if len(s) == 0:
            continue
        b, k = s // K, s % K
        n = slice(off[m], off[m + 1])
        x, ws = X[b], w[b, k][:, None]
        prod = 2 * (F + 8) * U
        z, ez = x @ W1[n].T, prod * (x.abs() @ W1[n].abs().T)
        v, d = act(int(acts[m]), z)
        ev = L1 * ez + ACT_ABS + ACT_REL * v.abs()
        ed = L2 * ez + 2 * ACT_ABS + ACT_REL * d.abs()
        if gated:
            u, eu = x @ V1[n].T, prod * (x.abs() @ V1[n].abs().T)
            H, eH = v * u, ev * u.abs() + v.abs() * eu + ev * eu + U * (v * u).abs()
        else:
            H, eH = v, ev
        logits = H @ W2[:, n].T
        el = eH @ W2[:, n].abs().T + 2 * (h + 8) * U * (H.abs() @ W2[:, n].abs().T)
        Y.index_add_(0, b, ws * logits)
        eY.index_add_(0, b, ws.abs() * (el + (K + 2) * U * logits.abs()))
        if dY is None:
            continue
        g, G = dY[b] @ W2[:, n], dY[b].abs() @ W2[:, n].abs()
        eg = (O + 2) * U * G
        out["weight"][0][b, k] = (H * g).sum(1)
        out["weight"][1][b, k] = (eH * g.abs() + H.abs() * eg + eH * eg
                                  + 2 * (h + 8) * U * (H * g).abs()).sum(1)
        r = 2 * (len(s) + 8) * U
        wy = ws * dY[b]
        out["W2"][0][:, n] = wy.T @ H
        out["W2"][1][:, n] = wy.abs().T @ eH + r * (wy.abs().T @ H.abs())
        dh, edh = ws * g, ws.abs() * (eg + U * g.abs())
        t, et = (u, eu) if gated else (torch.ones_like(g), torch.zeros_like(g))
        for name, f, ef in (("W1", d * t, ed * t.abs() + d.abs() * et + ed * et), ("V1", v, ev)):
            if name not in out:
                continue
            dz = dh * f
            edz = edh * f.abs() + dh.abs() * ef + edh * ef + 3 * U * dz.abs()
            out[name][0][n] = dz.T @ x
            out[name][1][n] = edz.T @ x.abs() + r * (dz.abs().T @ x.abs())
    return out if dY is not None else {"Y": (Y, eY)}


COEF = (3.4445, -4.7750, 2.0315)


def steps(X, n, held=lambda t: t):
    """n Newton-Schulz steps on X (the side of the smaller A); `held` is applied to every
    operand and result, as an arithmetic would hold it."""
    turned = X.shape[0] > X.shape[1]
    X = held(X.T if turned else X)
    a, b, c = COEF
    for _ in range(n):
        A = held(X @ X.T)
        P = held(b * A + c * (A @ A))
        X = held(a * X + P @ X)
    return X.T if turned else X


def orthogonalized(M, n):
    """The direction of matrix M (float64) and the bound of its error.

    The arithmetic holds values to 23 bits and leaves out 2^-22 of a product; its effect on
    the result (singular values grow up to 3.4 times in a step, errors with them) is modelled
    by the same steps in 64 bits with every operand and result moved by up to 2^-22 of itself
    at random.  A sum of k products accumulated in float32 adds up to k / 2 roundings of the
    same size with random signs, sqrt(k / 2) of one of them; the bound takes 8 (largest of
    a few thousand normal values against their typical one) times both together."""
    norm = M.norm()
    if norm == 0:
        return torch.zeros_like(M), torch.tensor(0.0).double()
    X = M / norm
    want = steps(X, n)
    gen = torch.Generator().manual_seed(M.numel())
    move = lambda t: t * (1 + 2 ** -22 * (2 * torch.rand(t.shape, generator=gen).double() - 1))
    d = (steps(X, n, move) - want).abs()
    typical = d.pow(2).mean().sqrt() + 2 ** -22 * want.pow(2).mean().sqrt()
    return want, 8 * (1 + (max(M.shape) / 2) ** 0.5) * typical
