"""Block packs (a gated hidden layer, a layer norm over each model's hidden
units) in float64, model by model, with first-order bounds on what float32
arithmetic may change.

Every quantity is computed as a value and an error bound: a sum of k terms in
any order is off by at most (k + 8) u times the sum of their magnitudes (u =
2^-24; the 8 covers the products' own roundings and the three-piece products'
2^-23), an activation by its slope times the error of its argument, 8 u of its
value and 4e-7 (the rational approximation of the normal distribution function is
off by 1.5e-7 |z| and the hardware's exponential and reciprocal by a few u), and
errors propagate by the derivative of each step.  A result whose float32
evaluation is right lies within its bound whatever the order of its sums.
"""
import math

import numpy as np

U = 2.0 ** -24
EPS = float(np.float32(1e-5))


def act(a, z):
    """Value and derivative of activation id a (float64)."""
    one = np.ones_like(z)
    with np.errstate(over="ignore"):
        sig = 1 / (1 + np.exp(-z))
        ez = np.exp(np.minimum(z, 0))
        sp = np.logaddexp(z, 0)
    pos = z > 0
    if a == 0:
        return z, one
    if a == 1:
        return np.where(pos, z, 0), pos * one
    if a == 2:
        return np.tanh(z), 1 - np.tanh(z) ** 2
    if a == 3:
        return sig, sig * (1 - sig)
    if a == 4:
        return np.where(pos, z, ez - 1), np.where(pos, 1, ez)
    if a == 5:
        return np.where(pos, z, 0.01 * z), np.where(pos, 1, 0.01)
    if a == 6:
        cdf = np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in z.ravel()]).reshape(z.shape)
        return z * cdf, cdf + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if a == 7:
        return z * sig, sig + z * sig * (1 - sig)
    if a == 8:
        return sp, sig
    if a == 9:
        s2 = 1 / (1 + np.exp(-2 * z))
        return z * s2, s2 + 2 * z * s2 * (1 - s2)
    if a == 10:
        al, la = 1.6732632423543772, 1.0507009873554805
        return np.where(pos, la * z, la * al * (ez - 1)), np.where(pos, la, la * al * ez)
    if a == 11:
        on = np.abs(z) > 0.5
        return np.where(on, z, 0), on * one
    t = np.tanh(sp)
    return z * t, t + z * (1 - t * t) * sig


def dot(a, ea, b, eb):
    """a @ b with bounds, in any order of summation."""
    k = a.shape[-1]
    mag = np.abs(a) @ np.abs(b)
    return a @ b, ea @ np.abs(b) + np.abs(a) @ eb + ea @ eb + (k + 8) * U * mag


def one_model(a, p, X, y, head, B_total=None):
    """Logits, loss and gradients of one model, each as (value, bound).  p: its
    W1 [h, F], W2 [O, h] and, if it has them, V1, gain, shift."""
    X = X.astype(np.float64)
    W1, W2 = p["W1"].astype(np.float64), p["W2"].astype(np.float64)
    h, O, B = W1.shape[0], W2.shape[0], X.shape[0]
    zX, z1, z2 = np.zeros_like(X), np.zeros_like(W1), np.zeros_like(W2)
    Z, eZ = dot(X, zX, W1.T, z1.T)
    A, S = act(a, Z)
    eA = (np.abs(S) + eZ) * eZ + 8 * U * np.abs(A) + 4e-7
    eS = 2 * eZ + 1e-6
    gated, norm = "V1" in p, "gain" in p
    if gated:
        V1 = p["V1"].astype(np.float64)
        Q, eQ = dot(X, zX, V1.T, np.zeros_like(V1).T)
        H = A * Q
        eH = np.abs(A) * eQ + np.abs(Q) * eA + eA * eQ + U * np.abs(H)
    else:
        Q, eQ, H, eH = np.ones_like(A), np.zeros_like(A), A, eA
    if norm:
        g, s = p["gain"].astype(np.float64), p["shift"].astype(np.float64)
        mu = H.mean(1, keepdims=True)
        emu = eH.mean(1, keepdims=True) + (h + 8) * U * np.abs(H).mean(1, keepdims=True)
        D = H - mu
        eD = eH + emu + U * np.abs(D)
        var = (D * D).mean(1, keepdims=True)
        ev = (2 * np.abs(D) * eD + eD * eD).mean(1, keepdims=True) + (h + 8) * U * var
        r = (var + EPS) ** -0.5
        er = 0.5 * r ** 3 * ev + 4 * U * r
        N = D * r
        eN = r * eD + np.abs(D) * er + 2 * U * np.abs(N)
        T = g * N + s
        eT = np.abs(g) * eN + 3 * U * (np.abs(g * N) + np.abs(s))
        C = W2 @ g
        eC = (h + 8) * U * (np.abs(W2) @ np.abs(g))
        # the outputs come as r (sum H g W2 - mu C) + sum s W2
        gw = np.abs(g * W2).T
        eP = eN @ gw + (h + 8) * U * r * ((np.abs(H) + np.abs(mu)) @ gw)
        P = N @ (g * W2).T
        L = P + W2 @ s
        eL = eP + (h + 8) * U * (np.abs(W2) @ np.abs(s)) + 2 * U * np.abs(L)
    else:
        T, eT = H, eH
        L, eL = dot(T, eT, W2.T, z2.T)
    out = {"logits": (L, eL)}
    if y is None:
        return out
    if head == "mse":
        R = L - y
        loss = (R * R).mean()
        G = 2 * R / (B * O)
        eG = 2 * eL / (B * O) + 4 * U * np.abs(G) + 2 * U * np.abs(y) / (B * O)
        eloss = (2 * np.abs(R) * eL + eL ** 2).mean() + (B * O + 8) * U * loss
    else:
        m = L.max(1, keepdims=True)
        lse = m + np.log(np.exp(L - m).sum(1, keepdims=True))
        pr = np.exp(L - lse)
        hot = np.eye(O)[y]
        lp = (lse - L)[np.arange(B), y]
        loss = lp.mean()
        # the fp32 log-sum-exp carries a few u of its magnitude into the probabilities
        top = eL.max(1, keepdims=True) + 8 * U * (np.abs(lse) + np.abs(m) + 1)
        G = (pr - hot) / B
        eG = (2 * pr * top + 16 * U) / B
        eloss = 2 * top.mean() + (B + 8) * U * np.abs(lp).mean()
    out["loss"] = (loss, eloss)
    dT, edT = dot(G, eG, W2, z2)
    if norm:
        # T_o = sum_b G_o N, then dW2 = g T_o + s sum_b G_o, dgain = sum_o W2 T_o
        To, eTo = dot(G.T, eG.T, N, eN)
        Gs, eGs = G.sum(0), eG.sum(0) + (B + 8) * U * np.abs(G).sum(0)
        out["W2"] = (g * To + np.outer(Gs, s),
                     np.abs(g) * eTo + np.outer(eGs, np.abs(s))
                     + 4 * U * (np.abs(g * To) + np.abs(np.outer(Gs, s))))
        out["gain"] = ((W2 * To).sum(0), (np.abs(W2) * eTo + (O + 8) * U * np.abs(W2 * To)).sum(0))
        out["shift"] = (Gs @ W2, eGs @ np.abs(W2) + (O + 8) * U * (np.abs(Gs) @ np.abs(W2)))
        a1, a2 = (G * C).sum(1, keepdims=True) / h, (G * P).sum(1, keepdims=True) / h
        k = (O + 8) * U
        ea1 = (eG * np.abs(C) + np.abs(G) * eC + k * np.abs(G * C)).sum(1, keepdims=True) / h
        ea2 = (eG * np.abs(P) + np.abs(G) * eP + eG * eP + k * np.abs(G * P)).sum(1, keepdims=True) / h
        inner = g * dT - a1 - N * a2
        ein = (np.abs(g) * edT + ea1 + eN * np.abs(a2) + np.abs(N) * ea2
               + 4 * U * (np.abs(g * dT) + np.abs(a1) + np.abs(N * a2)))
        dH = r * inner
        edH = r * ein + er * (np.abs(inner) + ein) + 2 * U * np.abs(dH)
        if h == 1:  # the norm of one value is constant
            dH, edH = 0 * dH, 0 * edH
    else:
        out["W2"] = dot(G.T, eG.T, T, eT)
        dH, edH = dT, edT
    dZ = dH * Q * S
    edZ = (edH * np.abs(Q * S) + np.abs(dH) * (eQ * np.abs(S) + np.abs(Q) * eS)
           + edH * (eQ + np.abs(Q)) * eS + 4 * U * np.abs(dZ))
    out["W1"] = dot(dZ.T, edZ.T, X, zX)
    if gated:
        dQ = dH * A
        edQ = edH * (np.abs(A) + eA) + np.abs(dH) * eA + 4 * U * np.abs(dQ)
        out["V1"] = dot(dQ.T, edQ.T, X, zX)
    return out


def model_params(params, hs, m):
    off = np.concatenate([[0], np.cumsum(np.asarray(hs, np.int64))])
    s = slice(off[m], off[m + 1])
    return {k: v[:, s] if k == "W2" else v[s] for k, v in params.items()}


def pack(hs, acts, params, X, y=None, head="ce"):
    """The whole pack: {"logits": [B, M, O], "loss": [M], parameter gradients in
    the packed layout}, each (value, bound)."""
    got = [one_model(int(acts[m]), model_params(params, hs, m), X, y, head)
           for m in range(len(hs))]
    join = {"logits": lambda v: np.stack(v, 1), "loss": np.array,
            "W2": lambda v: np.concatenate(v, 1)}
    return {k: tuple(join.get(k, np.concatenate)([g[k][i] for g in got]) for i in (0, 1))
            for k in got[0]}


def random_params(rng, hs, F, O, gated, norm):
    """Parameters of the ranges that packs start from; gains and shifts of a net
    under training."""
    N = int(np.sum(hs))
    f = lambda *s: rng.uniform(-1, 1, s)  # noqa: E731
    p = {"W1": f(N, F) / math.sqrt(F), "W2": f(O, N) / np.sqrt(np.repeat(hs, hs))}
    if gated:
        p["V1"] = f(N, F) / math.sqrt(F)
    if norm:
        p["gain"] = 1 + 0.2 * f(N)
        p["shift"] = 0.2 * f(N)
    return {k: v.astype(np.float32) for k, v in p.items()}
