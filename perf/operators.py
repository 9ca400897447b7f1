"""The gated hidden layer and the layer norm of packed MLPs, measured.

A pool of M independent MLPs shares its inputs X [B, F]; model m owns h_m
consecutive hidden units of the N = sum h_m of the pool.  Two operators, each
with and without the other:

* gated: H = act_m(X W1^T) * (X V1^T), the feed-forward block of two
  projections, one of them through the model's activation (without the gate
  H = act_m(X W1^T));
* norm: each model's hidden vector is normalised over its own h_m units, per
  sample, with a gain and a shift per unit: N = gain * (H - mu) / sqrt(var +
  1e-5) + shift.  The normalised models here have four units and more: the norm
  of two values is their difference's sign wherever that is above sqrt(1e-5), and
  next to that border float32 says little about its gradient.

The logits [B, M, O] are every model's sums over its own units of N (or H) times
W2 [O, N].  kind "forward" returns them; kind "gradients" returns the gradients
of the sum over models of the mean loss (softmax cross-entropy, or squared error
for head "mse") with regard to every parameter.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5

# identity, tanh, sigmoid, GELU, SiLU, Swish with beta 2: the activations of gated
# feed-forward blocks without a kink.  (At a kink two correct float32 results may
# take different slopes.)
SMOOTH = (0, 2, 3, 6, 7, 9)

BASE = dict(kind="gradients", gated=True, norm=False, grid="paper", models=0, wmin=1, wmax=10,
            acts=6, repeats=1, F=10, O=2, B=32, head="ce")


def _case(**kw):
    c = dict(BASE)
    c.update(kw)
    return c


def listed():
    return [
        # one sample through a pool of 42 small models, 4..10 units wide: the latency
        # of a single prediction
        _case(name="predict_one", kind="forward", norm=True, wmin=4, B=1),
        # one sample through 6,000 models of 1..100 units, 100 features: serving a
        # large pool request by request, which reads every weight for one sample
        _case(name="serve_pool", kind="forward", wmax=100, repeats=10, F=100, B=1),
        # the gradients of the smallest pool on its ordinary batch
        _case(name="small_gated", B=32),
        _case(name="small_norm", gated=False, norm=True, wmin=4, B=32),
        # 582 models of 4..100 units, 50 features, batches of 128
        _case(name="hundreds_both", norm=True, wmin=4, wmax=100, F=50, B=128),
        # validation: the same pool on all its 10,000 samples in one call
        _case(name="validate_both", kind="forward", norm=True, wmin=4, wmax=100, F=50, B=10000),
        # the paper's grid of widths, ten repeats: 303,000 units, 100 features, batches of 256
        _case(name="paper_gated", wmax=100, repeats=10, F=100, B=256),
        _case(name="paper_norm", gated=False, norm=True, wmin=4, wmax=100, repeats=10, F=100, B=256),
        # models up to 1,000 units wide, ten classes, batches of 32 on 32 features:
        # weight traffic and the output layer count
        _case(name="ten_class_both", norm=True, acts=2, wmin=4, wmax=1000, F=32, O=10, B=32),
        # 1,000 features and batches of 1,024: the input-layer products count
        _case(name="wide_input_gated", wmax=200, F=1000, B=1024),
        # a random pool: widths of 4..250, odd feature count, three targets, a ragged
        # batch, regression
        _case(name="ragged_both", norm=True, grid="random", models=700, wmin=4, wmax=250, F=37, O=3,
              B=201, head="mse"),
        # few wide models on a batch of 1,000: validation of a short list
        _case(name="wide_norm_forward", kind="forward", gated=False, norm=True, grid="random",
              models=40, wmin=500, wmax=1000, F=100, O=16, B=1000),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    c = _case(kind=rng.choice(["gradients", "gradients", "forward"]), grid="random",
              models=_log(rng, 2, 10000), F=_log(rng, 4, 1000),
              O=rng.choice([2, 2, 3, 4, 7, 10, 16]), acts=rng.choice([1, 2, 6]))
    c["gated"], c["norm"] = rng.choice([(True, False), (False, True), (True, True)])
    c["wmin"] = 4 if c["norm"] else 1
    c["wmax"] = _log(rng, c["wmin"], 1000)
    c["B"] = _log(rng, 1, 1024 if c["kind"] == "gradients" else 10000)
    c["head"] = "mse" if c["kind"] == "gradients" and rng.random() < 0.2 else "ce"
    # no dearer than the listed cases: products, activations, logits, weights
    while True:
        n = c["models"] * (c["wmin"] + c["wmax"]) / 2
        if (n * c["F"] * c["B"] <= 4e10 and n * c["B"] * c["O"] <= 3e8 and n * c["F"] <= 1e8
                and c["models"] * c["B"] * c["O"] <= 6e7):
            return c
        c["models"] = max(1, c["models"] * 2 // 3)


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


def _tensors(c, seed):
    """Samples, targets and parameters (float32), from the seed alone.  The
    parameters have the ranges that the packs start from, the gains and shifts
    those of a net under training."""
    hs, _ = _pool(c)
    g = torch.Generator(device="cuda").manual_seed(7919 * seed + 101)
    N, F, O, B = int(hs.sum()), c["F"], c["O"], c["B"]

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda") * 2 - 1

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    p = {"X": normal(B, F)}
    score = p["X"] @ normal(F, O) / math.sqrt(F) + 0.1 * normal(B, O)
    p["y"] = score.contiguous() if c["head"] == "mse" else score.argmax(1).to(torch.int32)
    p["W1"] = uniform(N, F) / math.sqrt(F)
    if c["gated"]:
        p["V1"] = uniform(N, F) / math.sqrt(F)
    h = torch.from_numpy(hs).cuda()
    p["W2"] = uniform(O, N) / torch.repeat_interleave(h.float(), h.long()).sqrt()
    if c["norm"]:
        p["gain"] = 1 + 0.1 * normal(N)
        p["shift"] = 0.1 * normal(N)
    return p


def prepare(case, seed):
    """The batch on the GPU and the pool.  The framework's pool owns its
    parameters: they are set once, as a program does before it trains or serves.
    The plain form keeps the tensors and each unit's model."""
    c = dict(BASE, **case)
    hs, ac = _pool(c)
    p = _tensors(c, seed)
    state = {"kind": c["kind"], "X": p["X"], "y": p["y"]}
    if own:
        import paper_2206_08369_amd as pm
        net = pm.BlockPackedMLP(c["F"], c["O"], hs, ac, gated=c["gated"], norm=c["norm"],
                                head=c["head"])
        net.set_params(**{k: v.cpu().numpy() for k, v in p.items() if k not in ("X", "y")})
        state["net"] = net
        return state
    h = torch.from_numpy(hs).cuda().long()
    edges = np.concatenate([[0], np.cumsum(hs.astype(np.int64))])
    first = np.flatnonzero(np.diff(ac, prepend=-1))
    runs = [(int(ac[m]), int(edges[m]), int(edges[k]))
            for m, k in zip(first, list(first[1:]) + [len(ac)])]
    state.update(p, M=len(hs), head=c["head"], runs=runs, h=h.float(),
                 mid=torch.repeat_interleave(torch.arange(len(hs), device="cuda"), h))
    return state


# --- one pass -----------------------------------------------------------------

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


def _by_run(f, s, Z):
    return torch.cat([f(a, Z[i:j]) for a, i, j in s["runs"]])


def _per_model(s, v):
    """Sums of v [N, ...] over each model's units."""
    return torch.zeros(s["M"], *v.shape[1:], device=v.device).index_add_(0, s["mid"], v)


def _plain(s):
    X, W2, mid = s["X"], s["W2"], s["mid"]
    B, O = X.shape[0], W2.shape[0]
    Z = s["W1"] @ X.t()
    A = _by_run(_gate, s, Z)
    U = s["V1"] @ X.t() if "V1" in s else None
    H = A if U is None else A * U
    if "gain" in s:
        mu = _per_model(s, H) / s["h"][:, None]
        D = H - mu[mid]
        r = 1 / torch.sqrt(_per_model(s, D * D) / s["h"][:, None] + EPS)
        Hn = D * r[mid]
        T = s["gain"][:, None] * Hn + s["shift"][:, None]
    else:
        T = H
    L = _per_model(s, (T[:, :, None] * W2.t()[:, None, :]).reshape(len(mid), B * O))
    L = L.reshape(s["M"], B, O)
    if s["kind"] == "forward":
        return L.transpose(0, 1).contiguous()
    if s["head"] == "mse":
        G = 2 * (L - s["y"][None]) / (B * O)
    else:
        e = torch.exp(L - L.max(2, keepdim=True).values)
        hot = (s["y"][:, None] == torch.arange(O, device=X.device)[None]).float()
        G = (e / e.sum(2, keepdim=True) - hot[None]) / B
    Gu = G[mid]
    out = {"W2": (Gu * T[:, :, None]).sum(1).t().contiguous()}
    dT = (Gu * W2.t()[:, None, :]).sum(2)
    if "gain" in s:
        out["gain"], out["shift"] = (dT * Hn).sum(1), dT.sum(1)
        dN = dT * s["gain"][:, None]
        m1 = _per_model(s, dN) / s["h"][:, None]
        m2 = _per_model(s, dN * Hn) / s["h"][:, None]
        dT = r[mid] * (dN - m1[mid] - Hn * m2[mid])
    S = _by_run(_slope, s, Z)
    if U is not None:
        out["V1"] = (dT * A) @ X
        dT = dT * U
    out["W1"] = (dT * S) @ X
    return out


def run(state):
    if not own:
        return _plain(state)
    net = state["net"]
    if state["kind"] == "forward":
        return net.forward(state["X"])
    return dict(zip(net.param_names, net.gradients(state["X"], state["y"])))


def work(case):
    """Parameters and the batch read once, logits or gradients written once; the
    products of the input layer and of the output layer, forward and, for
    gradients, those of the weights' gradients and of the hidden gradient."""
    c = dict(BASE, **case)
    hs, _ = _pool(c)
    N, M, F, O, B = int(hs.sum()), len(hs), c["F"], c["O"], c["B"]
    k = 2 if c["gated"] else 1
    params = N * (k * F + O + (2 if c["norm"] else 0))
    if c["kind"] == "forward":
        return {"bytes": 4.0 * (params + B * F + B * M * O), "flops": 2.0 * N * B * (k * F + O)}
    return {"bytes": 4.0 * (2 * params + B * (F + (O if c["head"] == "mse" else 1))),
            "flops": 2.0 * N * B * (2 * k * F + 3 * O)}


# --- the definition, in 64 bits -------------------------------------------------

def _value_and_slope(ids, z):
    """Activation ids [n, 1] of z [n, B] and its derivative."""
    beta = torch.where(ids == 9, 2.0, 1.0).double()
    sig = torch.sigmoid(beta * z)
    tanh = torch.tanh(z)
    cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    pdf = torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    v = torch.where((ids == 7) | (ids == 9), z * sig, z)
    d = torch.where((ids == 7) | (ids == 9), sig + beta * z * sig * (1 - sig), torch.ones_like(z))
    v, d = torch.where(ids == 2, tanh, v), torch.where(ids == 2, 1 - tanh * tanh, d)
    v, d = torch.where(ids == 3, sig, v), torch.where(ids == 3, sig * (1 - sig), d)
    return torch.where(ids == 6, z * cdf, v), torch.where(ids == 6, cdf + z * pdf, d)


def exact(case, seed):
    c = dict(BASE, **case)
    hs, ac = _pool(c)
    B, O = c["B"], c["O"]
    p = {k: v.double() if v.is_floating_point() else v for k, v in _tensors(c, seed).items()}
    X, y = p["X"], p["y"]
    got = {k: [] for k in p if k not in ("X", "y")}
    logits = []
    m0 = n0 = 0
    while m0 < len(hs):  # whole models at a time, about 4e7 products with W2
        m1, n = m0 + 1, int(hs[m0])
        while m1 < len(hs) and (n + int(hs[m1])) * B * O <= 4e7:
            n += int(hs[m1])
            m1 += 1
        rows = slice(n0, n0 + n)
        cnt = torch.from_numpy(hs[m0:m1].astype(np.int64)).cuda()
        owner = torch.repeat_interleave(torch.arange(m1 - m0, device="cuda"), cnt)
        ids = torch.from_numpy(np.repeat(ac[m0:m1], hs[m0:m1])).cuda()[:, None]

        def total(v):
            return torch.zeros(m1 - m0, v.shape[1], dtype=torch.double,
                               device="cuda").index_add_(0, owner, v)

        def mean(v):
            return (total(v) / cnt[:, None])[owner]

        act, dact = _value_and_slope(ids, p["W1"][rows] @ X.t())
        lin = p["V1"][rows] @ X.t() if c["gated"] else torch.ones_like(act)
        hid = act * lin
        if c["norm"]:
            dev = hid - mean(hid)
            inv = (mean(dev * dev) + EPS) ** -0.5
            unit = dev * inv
            top = unit * p["gain"][rows, None] + p["shift"][rows, None]
        else:
            top = hid
        w2 = p["W2"][:, rows]
        L = torch.stack([total(top * w2[o][:, None]) for o in range(O)], 2)
        if c["kind"] == "forward":
            logits.append(L.transpose(0, 1))
            m0, n0 = m1, n0 + n
            continue
        if c["head"] == "mse":
            G = (L - y[None]) * (2.0 / (B * O))
        else:
            G = torch.softmax(L, 2)
            G[:, torch.arange(B, device="cuda"), y.long()] -= 1
            G = G / B
        dtop = torch.zeros_like(top)
        dw2 = torch.empty_like(w2)
        for o in range(O):
            go = G[:, :, o][owner]
            dtop += go * w2[o][:, None]
            dw2[o] = (go * top).sum(1)
        got["W2"].append(dw2)
        dhid = dtop
        if c["norm"]:
            got["gain"].append((dtop * unit).sum(1))
            got["shift"].append(dtop.sum(1))
            dunit = dtop * p["gain"][rows, None]
            dhid = inv * (dunit - mean(dunit) - unit * mean(dunit * unit))
        got["W1"].append((dhid * lin * dact) @ X)
        if c["gated"]:
            got["V1"].append((dhid * act) @ X)
        m0, n0 = m1, n0 + n
    if c["kind"] == "forward":
        return torch.cat(logits, 1)
    return {k: torch.cat(v, 1 if k == "W2" else 0) for k, v in got.items()}
