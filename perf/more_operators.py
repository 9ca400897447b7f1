"""Routed packs and the orthogonalised update of packed MLPs, measured.

A pool of M independent MLPs owns the N = sum h_m hidden units of its models;
model m maps x to W2_m act_m(W1_m x), or, gated, to W2_m (act_m(W1_m x) * V1_m x).

* "forward" and "gradients": the pool as a mixture.  A router takes the K best of
  the scores [B, M] of each sample (ties: the lowest index; a score of -inf is a
  model that is switched off, and a slot that finds none left has index -1 and
  weight 0) and weighs them by the softmax over the chosen.  Only the chosen models
  compute: y_b = sum_k w_bk logits_{m(b, k)}(x_b).  The gradients are those of the
  parameters and of the scores, from dY = dLoss/dy.
* "orthogonalize": a matrix of every model (W1 [N, F], W2 [O, N] or the
  hidden-to-hidden blocks W12) as the optimiser updates it: mom' = mu mom + G,
  U = G + mu mom', X = U / |U|_F per model, then five Newton-Schulz steps
  A = X X^T, X <- a X + (b A + c A A) X on the side where A is smaller.
"""
import math

import numpy as np
import torch

own = False

MU, STEPS = 0.95, 5
COEF = (3.4445, -4.7750, 2.0315)

# identity, tanh, sigmoid, GELU, SiLU, Swish with beta 2: activations without a kink.
# (At a kink two correct float32 results may take different slopes.)
SMOOTH = (0, 2, 3, 6, 7, 9)

BASE = dict(op="forward", gated=False, grid="paper", models=0, wmin=1, wmax=10, acts=6, repeats=1,
            F=10, O=2, B=32, K=2, skew=0.0, off=0.0, matrix="W1")


def _case(**kw):
    c = dict(BASE)
    c.update(kw)
    return c


def listed():
    return [
        # one sample, two of 60 small models: the latency of a single answer
        _case(name="answer_one", B=1, K=2),
        # 32 requests at once, each to four of 6,000 models of 1..100 units
        _case(name="serve_pool", gated=True, wmax=100, repeats=10, F=100, B=32, K=4),
        # a random pool, odd sizes, a fifth of the models switched off
        _case(name="ragged_forward", grid="random", models=130, wmax=250, F=37, O=3, B=777, K=3,
              skew=1.0, off=0.2),
        # validation of a mixture of few wide models in one call
        _case(name="wide_forward", gated=True, grid="random", models=48, wmin=500, wmax=1000, F=1000,
              O=10, B=16384, K=4, skew=0.5),
        # the smallest pool on its ordinary batch
        _case(name="small_gradients", op="gradients", B=32, K=2),
        # 600 models of 1..100 units, 100 features, batches of 4,096: many ragged groups
        _case(name="pool_gradients", op="gradients", gated=True, wmax=100, F=100, B=4096, K=8,
              skew=0.5),
        # few models, one of which most samples prefer, and a long batch
        _case(name="skewed_gradients", op="gradients", grid="random", models=9, wmin=40, wmax=300, F=61,
              O=7, B=9999, K=2, skew=3.0),
        # 1,000 features, models of 500..1,000 units: the products count
        _case(name="wide_gradients", op="gradients", grid="random", models=32, wmin=500, wmax=1000,
              F=1000, O=10, B=8192, K=2, skew=0.5),
        # the update of 60 models of 1..10 units on ten features: the latency of a step
        _case(name="small_update", op="orthogonalize"),
        # the paper's grid of widths, ten repeats: 6,000 matrices of 1..100 rows, 100 columns
        _case(name="paper_update", op="orthogonalize", wmax=100, repeats=10, F=100),
        # hidden-to-hidden blocks of two-layer models
        _case(name="hidden_update", op="orthogonalize", grid="random", models=300, wmin=32, wmax=200,
              F=50, matrix="W12"),
        # 1,000 features, models of 500..1,000 units
        _case(name="wide_update", op="orthogonalize", grid="random", models=40, wmin=500, wmax=1000,
              F=1000),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    c = _case(op=rng.choice(["forward", "gradients", "orthogonalize"]), grid="random",
              models=_log(rng, 2, 6000), F=_log(rng, 4, 1000), O=rng.choice([2, 2, 3, 4, 7, 10, 16]),
              acts=rng.choice([1, 2, 6]))
    c["wmin"] = _log(rng, 1, 500)
    c["wmax"] = _log(rng, c["wmin"], 1000)
    if c["op"] == "orthogonalize":
        c["matrix"] = rng.choice(["W1", "W1", "W1", "W2", "W12"])
        while _newton_work(c) > 0.9e12 or _entries(c) > 6e7:
            c["models"] = max(1, c["models"] * 2 // 3)
        return c
    c["gated"] = rng.random() < 0.5
    c["B"] = _log(rng, 1, 16384 if c["op"] == "forward" else 9999)
    c["K"] = min(c["models"], rng.choice([1, 2, 2, 3, 4, 8]))
    c["skew"] = rng.choice([0.0, 0.5, 1.0, 3.0])
    c["off"] = rng.choice([0.0, 0.0, 0.2])
    # no dearer than the listed cases: products, weights, scores
    while True:
        h = (c["wmin"] + c["wmax"]) / 2
        k = 2 if c["gated"] else 1
        products = c["B"] * c["K"] * h * c["F"] * k * (2 if c["op"] == "gradients" else 1)
        if products <= 6e10 and c["models"] * h * c["F"] * k <= 6e7 and c["B"] * c["models"] <= 2e7:
            return c
        if c["models"] * h * c["F"] * k > 6e7 or c["B"] * c["models"] > 2e7:
            c["models"] = max(1, c["models"] * 2 // 3)
            c["K"] = min(c["K"], c["models"])
        else:
            c["B"] = max(1, c["B"] * 2 // 3)


# --- inputs -----------------------------------------------------------------

def _pool(c):
    """Hidden widths and activation ids of the models."""
    acts = np.array(SMOOTH[:c["acts"]], np.int32)
    if c["grid"] == "paper":  # activation-major, width-ascending
        w = np.arange(c["wmin"], c["wmax"] + 1)
        hs = np.tile(np.repeat(w, c["repeats"]), len(acts))
        ac = np.repeat(acts, len(w) * c["repeats"])
    else:
        r = np.random.default_rng([c["models"], c["wmin"], c["wmax"], c["acts"]])
        hs = r.integers(c["wmin"], c["wmax"] + 1, c["models"])
        ac = np.sort(acts[r.integers(0, len(acts), c["models"])])
    return hs.astype(np.int32), ac.astype(np.int32)


def _second(c, hs):
    """Second-layer widths of a two-layer pool."""
    r = np.random.default_rng([len(hs), c["wmin"], c["wmax"], 2])
    return r.integers(c["wmin"], c["wmax"] + 1, len(hs)).astype(np.int32)


def _blocks(c):
    """(rows, columns) of every model's matrix."""
    hs, _ = _pool(c)
    if c["matrix"] == "W1":
        return [(int(h), c["F"]) for h in hs]
    if c["matrix"] == "W2":
        return [(c["O"], int(h)) for h in hs]
    return [(int(h2), int(h)) for h, h2 in zip(hs, _second(c, hs))]


def _entries(c):
    return sum(float(a * b) for a, b in _blocks(c))


def _newton_work(c):
    """Multiplications and additions of the steps, symmetric products counted once."""
    total = 0.0
    for a, b in _blocks(c):
        r, w = float(min(a, b)), float(max(a, b))
        total += STEPS * (r * r * w + r * r * r + 2 * r * r * w)
    return total


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(6151 * seed + 17)


def _mixture_tensors(c, seed):
    """Samples, scores, output gradients and parameters (float32), from the seed
    alone.  The parameters have the ranges that the packs start from; the scores are
    a gate's outputs, with models that are liked by more samples than others."""
    hs, _ = _pool(c)
    g = _generator(seed)
    N, M, F, O, B = int(hs.sum()), len(hs), c["F"], c["O"], c["B"]

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda") * 2 - 1

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    p = {"X": normal(B, F), "scores": normal(B, M) + c["skew"] * normal(M)}
    if c["off"]:
        p["scores"][:, torch.rand(M, generator=g, device="cuda") < c["off"]] = -math.inf
        p["scores"][B - B // 32:] = -math.inf  # the padding of a batch: no model at all
    p["dY"] = normal(B, O) / B
    p["W1"] = uniform(N, F) / math.sqrt(F)
    if c["gated"]:
        p["V1"] = uniform(N, F) / math.sqrt(F)
    h = torch.from_numpy(hs).cuda()
    p["W2"] = uniform(O, N) / torch.repeat_interleave(h.float(), h.long()).sqrt()
    return p


def _update_tensors(c, seed):
    """Gradient and momentum of one matrix of every model: noise and a few strong
    directions, at scales that differ from model to model."""
    hs, _ = _pool(c)
    g = _generator(seed)
    N = int(hs.sum())

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if c["matrix"] == "W12":
        blocks = _blocks(c)
        size = torch.tensor([a * b for a, b in blocks], device="cuda")
        scale = torch.repeat_interleave(torch.exp(2 * normal(len(blocks))), size)
        out = {k: normal(int(size.sum())) * scale for k in ("G", "mom")}
    else:
        scale = torch.exp(2 * normal(len(hs))).repeat_interleave(torch.from_numpy(hs).cuda().long())
        shape = (N, c["F"]) if c["matrix"] == "W1" else (N, c["O"])
        out = {}
        for k in ("G", "mom"):
            strong = normal(N, 3) @ normal(3, shape[1])
            out[k] = (normal(*shape) + strong) * scale[:, None]
        if c["matrix"] == "W2":
            out = {k: v.t().contiguous() for k, v in out.items()}
    return {"G": 1e-3 * out["G"], "mom": 1e-2 * out["mom"]}


def prepare(case, seed):
    """What a program holds before the call: the batch or the gradient on the GPU,
    and the pool.  The framework's pool owns its parameters: they are set once."""
    c = dict(BASE, **case)
    hs, ac = _pool(c)
    state = {"c": c}
    if c["op"] == "orthogonalize":
        state.update(_update_tensors(c, seed), blocks=_blocks(c))
        if own:
            import paper_2206_08369_amd as pm
            if c["matrix"] == "W12":
                state["net"] = pm.DeepPackedMLP(c["F"], c["O"], hs, _second(c, hs), ac)
            else:
                state["net"] = pm.PackedMLP(c["F"], c["O"], hs, ac)
            state["new"] = torch.empty_like(state["mom"])
            return state
        state["groups"] = _equal_blocks(c)
        return state
    p = _mixture_tensors(c, seed)
    state.update(X=p["X"], scores=p["scores"], dY=p["dY"])
    if own:
        import paper_2206_08369_amd as pm
        net = (pm.BlockPackedMLP(c["F"], c["O"], hs, ac, gated=True) if c["gated"]
               else pm.PackedMLP(c["F"], c["O"], hs, ac))
        net.set_params(**{k: p[k].cpu().numpy() for k in ("W1", "V1", "W2") if k in p})
        state["net"] = net
        return state
    edges = np.concatenate([[0], np.cumsum(hs.astype(np.int64))])
    state.update(p, edges=[int(e) for e in edges], acts=[int(a) for a in ac])
    return state


# --- one pass, in plain operations ----------------------------------------------

def _gate(a, z):
    if a == 0:
        return z
    if a == 2:
        return torch.tanh(z)
    if a == 3:
        return 1 / (1 + torch.exp(-z))
    if a == 6:
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z / (1 + torch.exp(-(z if a == 7 else 2 * z)))


def _slope(a, z):
    if a == 0:
        return torch.ones_like(z)
    if a == 2:
        return 1 - torch.tanh(z) ** 2
    if a == 3:
        s = 1 / (1 + torch.exp(-z))
        return s * (1 - s)
    if a == 6:
        return (0.5 * (1 + torch.erf(z / math.sqrt(2)))
                + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi))
    b = 1 if a == 7 else 2
    s = 1 / (1 + torch.exp(-b * z))
    return s + b * z * s * (1 - s)


def _plain_route(scores, K):
    best, idx = torch.sort(scores, dim=1, descending=True, stable=True)
    best, idx = best[:, :K], idx[:, :K]
    live = best > -math.inf
    e = torch.where(live, torch.exp(best - best[:, :1]), torch.zeros_like(best))
    w = torch.where(live, e / e.sum(1, keepdim=True), torch.zeros_like(best))
    return torch.where(live, idx, torch.full_like(idx, -1)).to(torch.int32), w


def _plain_mixture(s):
    c, X, W1, V1, W2 = s["c"], s["X"], s["W1"], s.get("V1"), s["W2"]
    B, K, O, M = c["B"], c["K"], c["O"], len(s["acts"])
    idx, w = _plain_route(s["scores"], K)
    flat, wflat = idx.reshape(-1).long(), w.reshape(-1)
    order = torch.sort(flat, stable=True).indices  # slots by model, the unused ones first
    counts = torch.bincount(flat + 1, minlength=M + 1).tolist()
    P = torch.zeros(B * K, O, device=X.device)
    train = c["op"] == "gradients"
    if train:
        dW1, dW2 = torch.zeros_like(W1), torch.zeros_like(W2)
        dV1 = None if V1 is None else torch.zeros_like(V1)
    at = counts[0]
    for m in range(M):
        n = counts[m + 1]
        if n == 0:
            continue
        slots, at = order[at:at + n], at + n
        i, j, a = s["edges"][m], s["edges"][m + 1], s["acts"][m]
        rows = slots // K
        x = X[rows]
        z = x @ W1[i:j].t()
        h = act = _gate(a, z)
        if V1 is not None:
            u = x @ V1[i:j].t()
            h = act * u
        P[slots] = h @ W2[:, i:j].t()
        if train:
            d = wflat[slots, None] * s["dY"][rows]
            dh = d @ W2[:, i:j]
            dW2[:, i:j] = d.t() @ h
            if V1 is not None:
                dV1[i:j] = (dh * act).t() @ x
                dh = dh * u
            dW1[i:j] = (dh * _slope(a, z)).t() @ x
    P = P.reshape(B, K, O)
    if not train:
        return idx, w, (w[:, :, None] * P).sum(1)
    dw = (P * s["dY"][:, None, :]).sum(2)
    ds = w * (dw - (w * dw).sum(1, keepdim=True))
    dscores = torch.zeros(B, M + 1, device=X.device).scatter_add_(1, idx.long() + 1, ds)[:, 1:]
    out = {"W1": dW1, "W2": dW2, "scores": dscores.contiguous()}
    if V1 is not None:
        out["V1"] = dV1
    return out


def _equal_blocks(c):
    """Models by the shape of their matrix: (shape, positions of their entries)."""
    hs, _ = _pool(c)
    blocks = _blocks(c)
    edges = np.concatenate([[0], np.cumsum(hs.astype(np.int64))])
    start = np.concatenate([[0], np.cumsum([a * b for a, b in blocks])])
    by_shape = {}
    for m, shape in enumerate(blocks):
        by_shape.setdefault(shape, []).append(m)
    out = []
    for (a, b), members in by_shape.items():
        i = torch.arange(a, device="cuda")[None, :, None]
        j = torch.arange(b, device="cuda")[None, None, :]
        if c["matrix"] == "W2":
            at = torch.tensor(edges[members], device="cuda")[:, None, None] + i * int(edges[-1]) + j
        elif c["matrix"] == "W1":
            at = (torch.tensor(edges[members], device="cuda")[:, None, None] + i) * b + j
        else:
            at = torch.tensor(start[members], device="cuda")[:, None, None] + i * b + j
        out.append(((a, b), at))
    return out


def _plain_update(s):
    a, b, c = COEF
    mom = MU * s["mom"] + s["G"]
    U = (s["G"] + MU * mom).reshape(-1)
    out = torch.empty_like(U)
    for (rows, cols), at in s["groups"]:
        X = U[at]
        if rows > cols:
            X = X.transpose(1, 2).contiguous()
        X = X / torch.sqrt((X * X).sum((1, 2), keepdim=True))
        for _ in range(STEPS):
            A = X @ X.transpose(1, 2).contiguous()
            X = a * X + (b * A + c * (A @ A)) @ X
        out[at] = X.transpose(1, 2) if rows > cols else X
    return mom, out.reshape(s["G"].shape)


def run(state):
    c = state["c"]
    if not own:
        return _plain_update(state) if c["op"] == "orthogonalize" else _plain_mixture(state)
    net = state["net"]
    if c["op"] == "orthogonalize":
        U = net.orthogonalize(state["G"], matrix=c["matrix"], steps=STEPS, momentum=state["mom"],
                              mu=MU, nesterov=True, momentum_out=state["new"])
        return state["new"], U
    idx, w = net.route(state["scores"], c["K"])
    if c["op"] == "forward":
        return idx, w, net.forward_routed(state["X"], idx, w)
    *grads, dw = net.gradients_routed(state["X"], idx, w, state["dY"])
    names = ("W1", "V1", "W2") if c["gated"] else ("W1", "W2")
    out = dict(zip(names, grads))
    out["scores"] = net.route_backward(idx, w, dw)
    return out


def work(case):
    """Inputs read once, outputs written once, of the weights those of models that a
    sample chose; products of the chosen (sample, model) pairs, and for gradients
    those of the weights' gradients and of the hidden gradient.  The steps of the
    update as _newton_work."""
    c = dict(BASE, **case)
    if c["op"] == "orthogonalize":
        return {"bytes": 16.0 * _entries(c), "flops": _newton_work(c)}
    hs, _ = _pool(c)
    N, M, F, O, B, K = int(hs.sum()), len(hs), c["F"], c["O"], c["B"], c["K"]
    k = 2 if c["gated"] else 1
    share = 1 - (1 - 1 / M) ** (B * K)  # of the models, that some sample chose
    params = float(N) * (k * F + O)
    io = float(B) * (M + F + O)
    pairs = float(B) * K * N / M
    if c["op"] == "forward":
        return {"bytes": 4.0 * (share * params + io + 2 * B * K), "flops": 2.0 * pairs * (k * F + O)}
    return {"bytes": 4.0 * (share * params + params + io + B * M),
            "flops": 2.0 * pairs * (2 * k * F + 3 * O)}


# --- the definition, in 64 bits -------------------------------------------------

def _value_and_slope(a, z):
    if a == 0:
        return z, torch.ones_like(z)
    if a == 2:
        t = torch.tanh(z)
        return t, 1 - t * t
    if a == 3:
        t = torch.sigmoid(z)
        return t, t * (1 - t)
    if a == 6:
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    beta = 1.0 if a == 7 else 2.0
    t = torch.sigmoid(beta * z)
    return z * t, t + beta * z * t * (1 - t)


def _exact_mixture(c, seed):
    hs, ac = _pool(c)
    p = {k: v.double() for k, v in _mixture_tensors(c, seed).items()}
    B, K, O, M = c["B"], c["K"], c["O"], len(hs)
    left = p["scores"].clone()
    row = torch.arange(B, device="cuda")
    idx = torch.empty(B, K, dtype=torch.int32, device="cuda")
    best = torch.empty(B, K, dtype=torch.double, device="cuda")
    column = torch.arange(M, device="cuda")
    for k in range(K):  # the best of what is left, the lowest index of equals
        top = left.max(1).values
        first = torch.where(left == top[:, None], column[None], M).min(1).values
        best[:, k], idx[:, k] = top, first.int()
        left[row, first] = -math.inf
    none = best == -math.inf
    idx[none] = -1
    w = torch.softmax(torch.where(none, -1e300, best), 1)
    w[none] = 0
    train = c["op"] == "gradients"
    logits = torch.zeros(B, K, O, dtype=torch.double, device="cuda")
    grads = {k: torch.zeros_like(p[k]) for k in ("W1", "V1", "W2") if k in p}
    at, model = torch.sort(idx.reshape(-1).long()), 0
    ends = torch.searchsorted(at.values, torch.arange(M + 1, device="cuda")).tolist()
    n1 = 0
    for model in range(M):
        n0, n1 = n1, n1 + int(hs[model])
        pick = at.indices[ends[model]:ends[model + 1]]
        if len(pick) == 0:
            continue
        b, k = torch.div(pick, K, rounding_mode="floor"), pick % K
        x = p["X"][b]
        act, dact = _value_and_slope(int(ac[model]), x @ p["W1"][n0:n1].T)
        lin = x @ p["V1"][n0:n1].T if c["gated"] else torch.ones_like(act)
        logits[b, k] = (act * lin) @ p["W2"][:, n0:n1].T
        if train:
            dy = p["dY"][b] * w[b, k][:, None]
            dhid = dy @ p["W2"][:, n0:n1]
            grads["W2"][:, n0:n1] = dy.T @ (act * lin)
            grads["W1"][n0:n1] = (dhid * lin * dact).T @ x
            if c["gated"]:
                grads["V1"][n0:n1] = (dhid * act).T @ x
    if not train:
        return idx, w, torch.einsum("bk,bko->bo", w, logits)
    dw = torch.einsum("bko,bo->bk", logits, p["dY"])
    ds = w * (dw - (w * dw).sum(1, keepdim=True))
    grads["scores"] = torch.zeros(B, M, dtype=torch.double, device="cuda")
    grads["scores"].scatter_add_(1, idx.clamp(min=0).long(), ds)
    return {k: grads[k] for k in ("W1", "W2", "scores", "V1") if k in grads}


def _exact_update(c, seed):
    hs, _ = _pool(c)
    t = _update_tensors(c, seed)
    G, old = t["G"].double(), t["mom"].double()
    mom = MU * old + G
    U = G + MU * mom
    out = torch.empty_like(U)
    a, b, coef = COEF
    n = e = 0
    for (rows, cols), h in zip(_blocks(c), hs):
        if c["matrix"] == "W1":
            view = (slice(n, n + rows),)
        elif c["matrix"] == "W2":
            view = (slice(None), slice(n, n + cols))
        else:
            view = (slice(e, e + rows * cols),)
        X = U[view].reshape(rows, cols)
        X = X / X.norm()
        for _ in range(STEPS):
            if rows <= cols:
                A = X @ X.T
                X = a * X + (b * A + coef * A @ A) @ X
            else:
                A = X.T @ X
                X = a * X + X @ (b * A + coef * A @ A)
        out[view] = X.reshape(out[view].shape)
        n, e = n + int(h), e + rows * cols
    return mom, out


def exact(case, seed):
    c = dict(BASE, **case)
    return _exact_update(c, seed) if c["op"] == "orthogonalize" else _exact_mixture(c, seed)
