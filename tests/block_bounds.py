"""First-order bounds on the float32 evaluation of block packs, relative where the
values are: what block_reference.py grants an activation absolutely (4e-7), a norm
multiplies by up to 316, and hidden values that are small beside 1 need it relative.

An activation may be off by its slope times the error of its argument and by
(8 + 2 |z|) u of its value (u = 2^-24; the exponential of z carries |z| u), GELU by
1.5e-7 |z| more (the rational approximation of the normal distribution function).
Normalised outputs are sums of deviations from the mean, with the roundings of the
mean and of the sums beside the error of the hidden values themselves."""
import numpy as np

import block_reference as ref

U = ref.U


def one_model(a, p, X, y=None):
    """Logits, and with labels y the gradients, of one model of the softmax
    cross-entropy head, each as (value, bound); parameters as in
    block_reference.one_model."""
    p = {k: v.astype(np.float64) for k, v in p.items()}
    X = X.astype(np.float64)
    W1, W2 = p["W1"], p["W2"]
    h, O, B = W1.shape[0], W2.shape[0], X.shape[0]
    zero = lambda v: np.zeros_like(v)  # noqa: E731
    Z, eZ = ref.dot(X, zero(X), W1.T, zero(W1).T)
    A, S = ref.act(a, Z)
    # (slopes grow by at most 1.3 |dz|; SELU's jumps by 0.7 at 0)
    eA = (np.abs(S) + 0.8 + 2 * eZ) * eZ + (8 + 2 * np.abs(Z)) * U * np.abs(A)
    if a in (2, 3, 8):
        eA = (np.abs(S) + eZ) * eZ + (8 + 2 * np.abs(Z)) * U * np.abs(A)
    if a == 6:
        eA = eA + 1.5e-7 * np.abs(Z)
    eS = 2 * eZ + 1e-6
    if a == 2:  # 1 / cosh^2 z: relative, twice the error of z (and of its exponential)
        eS = np.abs(S) * (2 * eZ + 4 * eZ * eZ + (12 + 4 * np.abs(Z)) * U)
    if "V1" in p:
        Q, eQ = ref.dot(X, zero(X), p["V1"].T, zero(p["V1"]).T)
        H = A * Q
        eH = np.abs(A) * eQ + np.abs(Q) * eA + eA * eQ + U * np.abs(H)
    else:
        Q, eQ, H, eH = np.ones_like(A), zero(A), A, eA
    norm = "gain" in p
    if norm:
        g, s = p["gain"], p["shift"]
        mu = H.mean(1, keepdims=True)
        D = H - mu
        d = np.abs(D).max(1, keepdims=True)
        eD = eH + eH.mean(1, keepdims=True) + 6 * U * (np.abs(mu) + d) + 40 * U * d
        var = (D * D).mean(1, keepdims=True)
        ev = (2 * np.abs(D) * eD + eD * eD).mean(1, keepdims=True) + (h + 8) * U * var
        r = (var + ref.EPS) ** -0.5
        er = 0.5 * r ** 3 * ev + 4 * U * r
        N = D * r
        eN = r * eD + np.abs(D) * er + er * eD + 2 * U * np.abs(N)
        gw = np.abs(g * W2).T
        P = N @ (g * W2).T
        eP = eN @ gw + (h + 16) * U * 4 * d * r * gw.sum(0)
        L = P + W2 @ s
        eL = eP + (h + 8) * U * (np.abs(W2) @ np.abs(s)) + 2 * U * np.abs(L)
    else:
        L, eL = ref.dot(H, eH, W2.T, zero(W2).T)
    out = {"logits": (L, eL)}
    if y is None:
        return out
    m = L.max(1, keepdims=True)
    lse = m + np.log(np.exp(L - m).sum(1, keepdims=True))
    pr = np.exp(L - lse)
    G = (pr - np.eye(O)[y]) / B
    # probabilities move by their logits' differences
    eG = pr * (eL + eL.max(1, keepdims=True)) / B + 16 * U * (pr + np.eye(O)[y]) / B
    dT, edT = ref.dot(G, eG, W2, zero(W2))
    if norm:
        To, eTo = ref.dot(G.T, eG.T, N, eN)
        Gs, eGs = G.sum(0), eG.sum(0) + (B + 8) * U * np.abs(G).sum(0)
        out["W2"] = (g * To + np.outer(Gs, s), np.abs(g) * eTo + np.outer(eGs, np.abs(s))
                     + 4 * U * (np.abs(g * To) + np.abs(np.outer(Gs, s))))
        out["gain"] = ((W2 * To).sum(0), (np.abs(W2) * eTo + (O + 8) * U * np.abs(W2 * To)).sum(0))
        out["shift"] = (Gs @ W2, eGs @ np.abs(W2) + (O + 8) * U * (np.abs(Gs) @ np.abs(W2)))
        C, k = W2 @ g, (O + 8) * U
        eC = (h + 8) * U * gw.sum(0)
        a1, a2 = (G * C).sum(1, keepdims=True) / h, (G * P).sum(1, keepdims=True) / h
        ea1 = (eG * np.abs(C) + np.abs(G) * eC + k * np.abs(G * C)).sum(1, keepdims=True) / h
        ea2 = (eG * np.abs(P) + np.abs(G) * eP + eG * eP
               + k * np.abs(G * P)).sum(1, keepdims=True) / h
        inner = g * dT - a1 - N * a2
        ein = (np.abs(g) * edT + ea1 + eN * np.abs(a2) + np.abs(N) * ea2
               + 4 * U * (np.abs(g * dT) + np.abs(a1) + np.abs(N * a2)))
        dH, edH = r * inner, r * ein + er * (np.abs(inner) + ein) + 2 * U * np.abs(r * inner)
        if h == 1:  # the norm of one value is constant
            dH, edH = 0 * dH, 0 * edH
    else:
        out["W2"] = ref.dot(G.T, eG.T, H, eH)
        dH, edH = dT, edT
    dZ = dH * Q * S
    edZ = (edH * np.abs(Q * S) + np.abs(dH) * (eQ * np.abs(S) + np.abs(Q) * eS)
           + edH * (eQ + np.abs(Q)) * eS + 4 * U * np.abs(dZ))
    out["W1"] = ref.dot(dZ.T, edZ.T, X, zero(X))
    if "V1" in p:
        out["V1"] = ref.dot((dH * A).T, (edH * (np.abs(A) + eA) + np.abs(dH) * eA
                                         + 4 * U * np.abs(dH * A)).T, X, zero(X))
    return out


def pack(hs, acts, params, X, y=None):
    """The whole pack, as block_reference.pack."""
    got = [one_model(int(acts[m]), ref.model_params(params, hs, m), X, y) for m in range(len(hs))]
    join = {"logits": lambda v: np.stack(v, 1), "W2": lambda v: np.concatenate(v, 1)}
    return {k: tuple(join.get(k, np.concatenate)([g[k][i] for g in got]) for i in (0, 1))
            for k in got[0]}
