"""Routed packs against the 64-bit reference, model by model and slot by slot."""
import numpy as np
import pytest
import torch

import routed_reference as rr

pytestmark = pytest.mark.gpu

ALL = tuple(range(13))


@pytest.fixture(scope="module")
def pm():
    import paper_2206_08369_amd as pm
    assert torch.cuda.is_available()
    return pm


class Pool:
    """A pack and its parameters as the reference takes them."""

    def __init__(self, pm, F, O, hs, acts, gated, seed=0):
        self.hs, self.acts, self.gated = list(hs), list(acts), gated
        self.F, self.O, self.N = F, O, int(sum(hs))
        self.g = torch.Generator().manual_seed(1000 + seed)
        self.net = (pm.BlockPackedMLP(F, O, hs, acts, gated=True) if gated
                    else pm.PackedMLP(F, O, hs, acts))
        self.W1 = self.rand(self.N, F) / F ** 0.5
        self.V1 = self.rand(self.N, F) / F ** 0.5 if gated else None
        self.W2 = self.rand(O, self.N) / max(hs) ** 0.5
        self.put()

    def rand(self, *shape):
        return torch.randn(*shape, generator=self.g)

    def put(self):
        kw = {"V1": self.V1.numpy()} if self.gated else {}
        self.net.set_params(W1=self.W1.numpy(), W2=self.W2.numpy(), **kw)

    def choices(self, B, K, unused=0.1, negative=True):
        M = len(self.hs)
        idx = torch.randint(0, M, (B, K), generator=self.g, dtype=torch.int32)
        idx[torch.rand(B, K, generator=self.g) < unused] = -1
        w = self.rand(B, K) if negative else torch.rand(B, K, generator=self.g)
        return idx, w

    def want(self, X, idx, w, dY=None):
        d = lambda t: None if t is None else t.double()
        return rr.mixture(self.hs, self.acts, d(X), idx.long(), d(w), d(self.W1), d(self.V1),
                          d(self.W2), d(dY))

    def forward(self, X, idx, w):
        return self.net.forward_routed(X.cuda(), idx.cuda(), w.cuda())

    def gradients(self, X, idx, w, dY):
        got = self.net.gradients_routed(X.cuda(), idx.cuda(), w.cuda(), dY.cuda())
        return dict(zip(("W1", "V1", "W2", "weight") if self.gated else ("W1", "W2", "weight"), got))


def close(got, want, what=""):
    value, bound = want
    off = (got.cpu().double() - value).abs()
    assert bool((off <= bound + 1e-30).all()), "%s off by %.3g where %.3g is allowed" % (
        what, float(off.max()), float(bound.reshape(-1)[(off - bound).argmax()]))


# --- the router ---------------------------------------------------------------------

def check_route(pm, net, scores, K):
    idx, w = net.route(torch.from_numpy(scores).cuda(), K)
    ri, rw = rr.route(scores.astype(np.float64), K)
    assert np.array_equal(idx.cpu().numpy(), ri)
    # a difference, an exponential, a sum of K and a quotient: each within 2 U; the
    # difference's rounding moves the exponential by U times its size, at most 90
    assert np.all(np.abs(w.cpu().numpy() - rw) <= (2 * K + 200) * rr.U * rw + 1e-44)
    return idx, w


@pytest.mark.parametrize("M", [1, 2, 63, 64, 65, 256, 257, 1024, 1025, 5000, 8193])
@pytest.mark.parametrize("K", [1, 2, 5, 16])
def test_route(pm, M, K):
    rng = np.random.default_rng(M * 17 + K)
    net = pm.PackedMLP(3, 2, [1] * M, [0] * M)
    s = rng.standard_normal((7, M)).astype(np.float32)
    s[1] = rng.integers(-1, 2, M)               # many ties
    s[2] = -np.inf                              # nothing left
    s[3, rng.random(M) < 0.7] = -np.inf
    s[4, rng.random(M) < 0.5] = np.nan
    s[5] = -0.0
    s[5, ::2] = 0.0                             # equal, whatever the sign
    s[6] = np.finfo(np.float32).min
    check_route(pm, net, s, K)


@pytest.mark.parametrize("B", [1, 3, 4, 5, 1000])
def test_route_batches_and_extremes(pm, B):
    rng = np.random.default_rng(B)
    net = pm.PackedMLP(3, 2, [1] * 40, [0] * 40)
    s = (rng.standard_normal((B, 40)) * 10.0 ** rng.integers(-3, 3, (B, 1))).astype(np.float32)
    s[0, 3] = np.finfo(np.float32).max
    check_route(pm, net, s, 3)


def test_route_infinite_score(pm):
    net = pm.PackedMLP(3, 2, [1] * 4, [0] * 4)
    s = torch.tensor([[0.0, float("inf"), 1.0, 2.0], [0.0, 1.0, 2.0, 3.0]]).cuda()
    idx, w = net.route(s, 2)
    assert idx.tolist() == [[1, 3], [3, 2]]
    assert bool(w[0].isnan().all()) and bool(w[1].isfinite().all())


@pytest.mark.parametrize("M,K", [(1, 1), (5, 3), (64, 2), (65, 16), (2000, 8)])
def test_route_backward(pm, M, K):
    rng = np.random.default_rng(M + K)
    net = pm.PackedMLP(3, 2, [1] * M, [0] * M)
    s = rng.standard_normal((9, M)).astype(np.float32)
    s[2] = -np.inf
    s[3, 1:] = -np.inf
    idx, w = check_route(pm, net, s, K)
    dw = torch.from_numpy(rng.standard_normal((9, K)).astype(np.float32)).cuda()
    got = net.route_backward(idx, w, dw).cpu().double()
    wd, dd = w.cpu().double(), dw.cpu().double()
    mean = (wd * dd).sum(1, keepdim=True)
    ds = wd * (dd - mean)
    want = torch.zeros(9, M + 1).double().scatter_add_(1, idx.cpu().long() + 1, ds)[:, 1:]
    bound = (K + 4) * rr.U * wd * (dd.abs() + (wd * dd.abs()).sum(1, keepdim=True))
    bound = torch.zeros(9, M + 1).double().scatter_add_(1, idx.cpu().long() + 1, bound)[:, 1:]
    assert bool(((got - want).abs() <= bound).all())


def test_route_backward_same_model_twice(pm):
    net = pm.PackedMLP(3, 2, [1] * 3, [0] * 3)
    idx = torch.tensor([[1, 1]], dtype=torch.int32).cuda()
    w, dw = torch.tensor([[0.5, 0.25]]).cuda(), torch.tensor([[4.0, 8.0]]).cuda()
    # mean 4: 0.5 (4 - 4) + 0.25 (8 - 4)
    assert net.route_backward(idx, w, dw).tolist() == [[0.0, 1.0, 0.0]]


# --- the mixture ----------------------------------------------------------------------

SHAPES = [
    # F, O, widths, B, K: few slots
    (1, 2, [1], 1, 1),
    (10, 2, list(range(1, 11)), 1, 2),
    (37, 3, [5, 64, 65, 130, 1], 3, 2),
    (130, 16, [200, 3, 17], 4, 4),
    # tiles
    (1, 2, [1], 40, 1),
    (3, 2, [1, 2, 3], 33, 2),
    (31, 3, [7, 64, 63, 65], 64, 2),
    (32, 4, [128, 129], 100, 3),
    (37, 5, [250, 1, 40], 201, 2),
    (100, 16, [33, 100, 7, 64, 128, 300], 257, 4),
    (129, 10, [96], 300, 1),
    (500, 7, [70, 200], 150, 2),
    # wide waves of models and rows
    (40, 2, [150, 90, 260], 500, 1),
    (66, 9, [150, 190], 1000, 2),
    (20, 3, [10, 30], 400, 2),
    # more slots than one workgroup groups
    (9, 2, [5, 33, 8], 5000, 2),
]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "F%d-O%d-M%d-B%d-K%d" % (s[0], s[1], len(s[2]), s[3], s[4]))
def test_forward_and_gradients(pm, shape, gated):
    F, O, hs, B, K = shape
    acts = [rr.SMOOTH[(3 * m + len(hs)) % len(rr.SMOOTH)] for m in range(len(hs))]
    p = Pool(pm, F, O, hs, acts, gated, seed=F)
    X, dY = p.rand(B, F), p.rand(B, O)
    idx, w = p.choices(B, K)
    if B > 2:
        idx[1] = -1
        idx[2] = 0
    close(p.forward(X, idx, w), p.want(X, idx, w)["Y"], "Y")
    got = p.gradients(X, idx, w, dY)
    want = p.want(X, idx, w, dY)
    for k in got:
        close(got[k], want[k], k)
    again = p.gradients(X, idx, w, dY)
    assert all(torch.equal(got[k], again[k]) for k in got)
    p.net.check_routed()


# forward passes that group the rows: their slots read more than 128 MB
GROUPED = [(1000, 3, [70, 200], 300, 1), (531, 5, [250, 1, 40], 700, 1), (131, 16, [64, 128], 3000, 1),
           (29, 4, [1200], 1300, 1), (999, 2, [33, 520, 64, 700], 90, 3), (40, 10, [600, 260], 23000, 2)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", GROUPED, ids=lambda s: "F%d-O%d-M%d-B%d-K%d" % (s[0], s[1], len(s[2]), s[3], s[4]))
def test_grouped_forward(pm, shape, gated):
    F, O, hs, B, K = shape
    p = Pool(pm, F, O, hs, [rr.SMOOTH[(2 * m + F) % len(rr.SMOOTH)] for m in range(len(hs))], gated, seed=B)
    X = p.rand(B, F)
    idx, w = p.choices(B, K)
    idx[1], idx[2] = -1, 0
    X[1] = float("nan")
    got = p.forward(X, idx, w)
    X[1] = 0
    close(got, p.want(X, idx, w)["Y"], "Y")
    assert "k_rt_tile" == p.net.kernel_variants()["gemm_fwd"][0]
    X[1] = float("inf")
    assert torch.equal(got, p.forward(X, idx, w))
    p.net.check_routed()


# .. and that do not: a wave to 64 units of a slot (up to 64 columns), or a workgroup
SLOTS = [(37, 3, [250, 1, 66, 130], 500, 2, "k_rt_few_waves"), (64, 16, [300, 64, 65], 400, 1, "k_rt_few_waves"),
         (3, 2, [1030], 80, 1, "k_rt_few_waves"), (4, 5, [17, 16, 700, 2], 111, 16, "k_rt_few_waves"),
         (65, 4, [250, 1, 66, 130], 500, 2, "k_rt_few"), (37, 9, [300, 64, 65], 40, 2, "k_rt_few")]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", SLOTS, ids=lambda s: "F%d-O%d-M%d-B%d-K%d" % (s[0], s[1], len(s[2]), s[3], s[4]))
def test_slot_by_slot_forward(pm, shape, gated):
    F, O, hs, B, K, kernel = shape
    p = Pool(pm, F, O, hs, [rr.SMOOTH[(2 * m + F) % len(rr.SMOOTH)] for m in range(len(hs))], gated, seed=B)
    X = p.rand(B, F)
    idx, w = p.choices(B, K)
    idx[1], idx[2] = -1, 0
    X[1] = float("nan")
    got = p.forward(X, idx, w)
    X[1] = 0
    close(got, p.want(X, idx, w)["Y"], "Y")
    assert kernel == p.net.kernel_variants()["gemm_fwd"][0]
    # units of an infinite output weight behind a model's last one add nothing to it
    if len(hs) > 1:
        first = p.choices(B, K, unused=0)[0] * 0
        p.W2[:, hs[0]] = float("inf")
        p.put()
        assert bool(torch.isfinite(p.forward(X, first, w)).all())
    p.net.check_routed()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("B", [2, 200])
def test_every_activation(pm, gated, B):
    p = Pool(pm, 20, 2, [5 + m for m in range(13)], ALL, gated, seed=B)
    X = 2 * p.rand(B, 20)
    idx, w = p.choices(B, 3)
    value, bound = p.want(X, idx, w)["Y"]
    if 11 in ALL:  # hardshrink jumps by 0.5 at its border: the samples near it are left out
        z = X.double() @ p.W1.double().T
        n0 = sum(p.hs[:11])
        near = ((z[:, n0:n0 + p.hs[11]].abs() - 0.5).abs() < 1e-4).any(1)
        value[near], bound[near] = 0, float("inf")
    close(p.forward(X, idx, w), (value, bound), "Y")


def test_agrees_with_forward(pm):
    """All models chosen with weight 1 / M: the mean of pmlp_forward's logits."""
    p = Pool(pm, 19, 3, [4, 9, 30], [2, 7, 3], True)
    X = p.rand(50, 19)
    idx = torch.arange(3, dtype=torch.int32).expand(50, 3).contiguous()
    w = torch.full((50, 3), 1 / 3)
    value, bound = p.want(X, idx, w)["Y"]
    dense = p.net.forward(X.cuda()).mean(1)
    close(dense, (value, 2 * bound), "dense")
    close(p.forward(X, idx, w), (value, bound), "routed")


def test_one_model_takes_every_row(pm):
    """Parts of the rows are summed beside each other, and models without rows get zeros."""
    p = Pool(pm, 21, 4, [30, 50, 7], [7, 2, 6], True, seed=5)
    B, K = 1500, 2
    X, dY = p.rand(B, 21), p.rand(B, 4)
    idx, w = torch.ones(B, K, dtype=torch.int32), p.rand(B, K)
    got, want = p.gradients(X, idx, w, dY), p.want(X, idx, w, dY)
    for k in got:
        close(got[k], want[k], k)
    assert not bool(got["W1"][:30].any()) and not bool(got["W2"][:, 80:].any())


def test_no_slot_used(pm):
    p = Pool(pm, 6, 2, [3, 4], [2, 3], False)
    X, dY = p.rand(70, 6), p.rand(70, 2)
    idx, w = torch.full((70, 3), -1, dtype=torch.int32), p.rand(70, 3)
    assert not bool(p.forward(X, idx, w).any())
    assert not any(bool(v.any()) for v in p.gradients(X, idx, w, dY).values())


@pytest.mark.parametrize("M", [3000, 20000])  # (above 16,384 the counters leave LDS)
def test_many_models(pm, M):
    rng = np.random.default_rng(M)
    hs = rng.integers(1, 4, M)
    p = Pool(pm, 5, 2, hs, rng.choice(rr.SMOOTH, M), False, seed=M)
    B, K = 3500 if M == 3000 else 21000, 2
    X, dY = p.rand(B, 5), p.rand(B, 2)
    idx, w = p.choices(B, K)
    few = slice(0, 300)
    close(p.forward(X[few], idx[few].contiguous(), w[few].contiguous()),
          p.want(X[few], idx[few], w[few])["Y"], "few")
    close(p.forward(X, idx, w), p.want(X, idx, w)["Y"], "Y")
    got, want = p.gradients(X, idx, w, dY), p.want(X, idx, w, dY)
    for k in got:
        close(got[k], want[k], k)


def test_more_slots_than_a_launch_has_workgroups(pm):
    # 3,600,000 slots of models of one unit, and one of 300: slot by slot they were 18 million
    # workgroups of 256 threads, more than a launch may have
    M, K, B, F, wide = 1_200_000, 4, 900_000, 4, 300
    pack = Pool(pm, F, 2, [1] * (M - 1) + [wide], [0] * M, False, seed=5)
    X = pack.rand(B, F)
    idx, w = pack.choices(B, K)
    idx[::1000, 1] = M - 1
    got = pack.forward(X, idx, w).cpu().double()
    Y, bound = torch.zeros(B, 2).double(), torch.zeros(B, 2).double()
    W1, W2, Xd = pack.W1.double(), pack.W2.double(), X.double()

    def add(b, units, weight):  # samples b, their slots' units [len(b), n]: the identity's sums
        z, r = ((Xd[b][:, None] * W1[units]).sum(2), (Xd[b][:, None] * W1[units]).abs().sum(2))
        e = 2 * (F + 8) * rr.U * r + rr.ACT_ABS + rr.ACT_REL * z.abs()
        for o in range(2):
            v = W2[o][units]
            Y[b, o] += weight * (z * v).sum(1)
            bound[b, o] += weight.abs() * ((e * v.abs()).sum(1) + (2 * (units.shape[1] + 8) + K + 2)
                                           * rr.U * (z * v).abs().sum(1))
    for k in range(K):
        i, wk = idx[:, k].long(), w[:, k].double()
        b = torch.nonzero((i >= 0) & (i < M - 1)).reshape(-1)
        add(b, i[b][:, None], wk[b])
        b = torch.nonzero(i == M - 1).reshape(-1)
        add(b, torch.arange(M - 1, M - 1 + wide).repeat(len(b), 1), wk[b])
    close(got, (Y, bound))


@pytest.mark.parametrize("models", [9, 700])  # grouped by one workgroup, or by several
def test_a_few_models_take_most_rows(pm, models):
    hs = [1 + 5 * m % 20 for m in range(models)]
    p = Pool(pm, 20, 3, hs, [rr.SMOOTH[m % len(rr.SMOOTH)] for m in range(models)], True, seed=models)
    B = 1900 if models == 9 else 3000
    X, dY = p.rand(B, 20), p.rand(B, 3)
    idx, w = p.choices(B, 2)
    idx[:B // 3, 0], idx[B // 2:, 1], idx[B // 2:B // 2 + 300, 0] = 5, models - 1, 0
    got, want = p.gradients(X, idx, w, dY), p.want(X, idx, w, dY)
    for k in got:
        close(got[k], want[k], k)


@pytest.mark.parametrize("gated,lo,hi", [(False, 1, 9), (True, 1, 9), (False, 60, 90)])
def test_many_tiles(pm, gated, lo, hi):
    """Enough tiles of the weight gradients for the wider ones."""
    M, F = 1100, 70
    rng = np.random.default_rng(hi)
    p = Pool(pm, F, 3, rng.integers(lo, hi, M), rng.choice(rr.SMOOTH, M), gated, seed=hi)
    X, dY = p.rand(2000, F), p.rand(2000, 3)
    idx, w = p.choices(2000, 2)
    close(p.forward(X, idx, w), p.want(X, idx, w)["Y"], "Y")
    got, want = p.gradients(X, idx, w, dY), p.want(X, idx, w, dY)
    for k in got:
        close(got[k], want[k], k)


def test_regression_packs(pm):
    """The head of a pack is its own loss's; the mixture takes a gradient from outside."""
    p = Pool(pm, 6, 2, [3, 40], [2, 7], False)
    p.net.close()
    p.net = pm.PackedMLP(6, 2, [3, 40], [2, 7], head="mse")
    p.put()
    X, dY = p.rand(90, 6), p.rand(90, 2)
    idx, w = p.choices(90, 2)
    close(p.forward(X, idx, w), p.want(X, idx, w)["Y"], "Y")
    got, want = p.gradients(X, idx, w, dY), p.want(X, idx, w, dY)
    for k in got:
        close(got[k], want[k], k)
    with pytest.raises(pm.PmlpError) as e:
        p.net.losses()  # (no call of its own loss has run)
    assert e.value.code == pm.PMLP_ESTATE


def test_calls_under_way_keep_their_workspace(pm):
    """A larger batch on another stream while calls that use the smaller workspace run."""
    p = Pool(pm, 90, 2, [70, 200, 33], [7, 2, 3], True, seed=4)
    small = [t.cuda() for t in (p.rand(800, 90), *p.choices(800, 2), p.rand(800, 2))]
    large = [t.cuda() for t in (p.rand(9000, 90), *p.choices(9000, 2), p.rand(9000, 2))]
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(a):
        first = [p.net.gradients_routed(*small) for _ in range(4)][-1]
    with torch.cuda.stream(b):
        second = p.net.gradients_routed(*large)
    torch.cuda.synchronize()
    for got, data in ((first, small), (second, large)):
        want = p.want(*[t.cpu() for t in data[:3]], data[3].cpu())
        for g, k in zip(got, ("W1", "V1", "W2", "weight")):
            close(g, want[k], k)


def test_memory_is_given_back(pm):
    def in_use():
        torch.cuda.synchronize()
        free, total = torch.cuda.mem_get_info()
        return total - free

    p = Pool(pm, 40, 2, [300, 200], [7, 2], False)
    before = in_use()
    for B in range(20000, 60001, 10000):
        X = torch.zeros(B, 40).cuda()
        idx, w = torch.zeros(B, 1, dtype=torch.int32).cuda(), torch.zeros(B, 1).cuda()
        p.net.gradients_routed(X, idx, w, torch.zeros(B, 2).cuda())
        del X, idx, w
    torch.cuda.empty_cache()
    # hidden values of 60,000 rows of the widest model twice, and the rest: not one
    # workspace a size
    assert in_use() - before < 2 * 300 * 60100 * 4 + (128 << 20)
    p.net.close()
    torch.cuda.empty_cache()
    assert in_use() - before < (64 << 20)


@pytest.mark.parametrize("B", [1, 300])
def test_bad_indices_are_reported(pm, B):
    p = Pool(pm, 4, 2, [3, 5], [2, 2], False)
    X, dY = p.rand(B, 4), p.rand(B, 2)
    for bad in (2, -2, 2 ** 31 - 1, -2 ** 31):
        idx, w = p.choices(B, 2, unused=0)
        as_unused = idx.clone()
        idx[B - 1, 1], as_unused[B - 1, 1] = bad, -1
        close(p.forward(X, idx, w), p.want(X, as_unused, w)["Y"], "Y")
        with pytest.raises(pm.PmlpError, match="outside"):
            p.net.check_routed()
        p.net.check_routed()
        got, want = p.gradients(X, idx, w, dY), p.want(X, as_unused, w, dY)
        for k in got:
            close(got[k], want[k], k)
        with pytest.raises(pm.PmlpError, match="outside"):
            p.net.check_routed()


def test_diverged_model_stays_alone(pm):
    p = Pool(pm, 40, 2, [20, 70, 33], [2, 7, 6], False)
    X, dY = p.rand(300, 40), p.rand(300, 2)
    idx, w = p.choices(300, 2, unused=0)
    want, grads = p.want(X, idx, w)["Y"], p.want(X, idx, w, dY)
    p.W1[20:90] = float("nan")
    p.put()
    hit = (idx == 1).any(1)
    got = p.forward(X, idx, w).cpu()
    assert bool(got[hit].isnan().all())
    close(got[~hit], (want[0][~hit], want[1][~hit]))
    g = p.gradients(X, idx, w, dY)
    for rows in (slice(0, 20), slice(90, 123)):
        close(g["W1"][rows], tuple(t[rows] for t in grads["W1"]))
        close(g["W2"][:, rows], tuple(t[:, rows] for t in grads["W2"]))


@pytest.mark.parametrize("B", [2, 200])
def test_samples_nobody_answers_may_hold_anything(pm, B):
    p = Pool(pm, 13, 2, [9, 70], [7, 3], True)
    X, dY = p.rand(B, 13), p.rand(B, 2)
    idx, w = p.choices(B, 2, unused=0)
    idx[B // 2:] = -1
    clean = X.clone()
    clean[B // 2:] = 0
    X[B // 2:], w[B // 2:], dY[B // 2:] = float("nan"), float("inf"), float("nan")
    cw, cdY = w.clone(), dY.clone()
    cw[B // 2:], cdY[B // 2:] = 0, 0
    close(p.forward(X, idx, w), p.want(clean, idx, cw)["Y"], "Y")
    got, want = p.gradients(X, idx, w, dY), p.want(clean, idx, cw, cdY)
    for k in got:
        close(got[k], want[k], k)


def test_feature_masks(pm):
    p = Pool(pm, 35, 2, [20, 70], [2, 7], False)
    mask = torch.rand(2, 35, generator=p.g) < 0.5
    p.net.set_feature_mask(mask.numpy())
    rows = torch.cat([mask[0].expand(20, 35), mask[1].expand(70, 35)])
    p.W1 = p.W1 * rows
    X, dY = p.rand(90, 35), p.rand(90, 2)
    idx, w = p.choices(90, 2)
    close(p.forward(X, idx, w), p.want(X, idx, w)["Y"], "Y")
    got, want = p.gradients(X, idx, w, dY), p.want(X, idx, w, dY)
    want["W1"] = tuple(t * rows for t in want["W1"])
    for k in got:
        close(got[k], want[k], k)
    G = torch.randn(90, 35, generator=p.g).cuda()
    p.net.muon_step(G, 0.1)
    W1 = torch.from_numpy(p.net.get_params()[0])
    assert not bool(W1[~rows].any()) and bool((W1 != p.W1).any())


@pytest.mark.parametrize("B", [4, 400])
def test_other_stream_and_growing_batches(pm, B):
    p = Pool(pm, 23, 3, [40, 8, 90], [7, 2, 3], True, seed=B)
    s = torch.cuda.Stream()
    for n in (1, B, 3 * B, B):
        X, dY = p.rand(n, 23), p.rand(n, 3)
        idx, w = p.choices(n, 2)
        args = [t.cuda() for t in (X, idx, w, dY)]
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            Y = p.net.forward_routed(*args[:3])
            got = p.net.gradients_routed(*args)
        s.synchronize()
        close(Y, p.want(X, idx, w)["Y"], "Y")
        want = p.want(X, idx, w, dY)
        for g, k in zip(got, ("W1", "V1", "W2", "weight")):
            close(g, want[k], k)


@pytest.mark.parametrize("B", [4, 300])
def test_captured_and_replayed(pm, B):
    p = Pool(pm, 23, 3, [40, 8, 90], [7, 2, 3], False, seed=B)
    X, idx, w, dY = p.rand(B, 23).cuda(), *[t.cuda() for t in p.choices(B, 2)], p.rand(B, 3).cuda()
    scores = p.rand(B, 3).cuda()
    mom = torch.zeros(138, 23).cuda()

    def calls():
        i, v = p.net.route(scores, 2)
        Y = p.net.forward_routed(X, i, v)
        dW1, dW2, dw = p.net.gradients_routed(X, i, v, dY)
        ds = p.net.route_backward(i, v, dw)
        U = p.net.orthogonalize(dW1, momentum=mom, momentum_out=out)
        return i, v, Y, dW1, dW2, dw, ds, U

    out = torch.empty_like(mom)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        calls()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        kept = calls()
    for turn in range(4):
        X.copy_(p.rand(B, 23))
        scores.copy_(p.rand(B, 3))
        eager = [t.clone() for t in calls()]
        torch.cuda.synchronize()
        for t in kept:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, eager)), turn


def test_capture_refuses_to_grow(pm):
    p = Pool(pm, 23, 3, [40, 8, 90], [7, 2, 3], False)
    X, dY = p.rand(2000, 23).cuda(), p.rand(2000, 3).cuda()
    idx, w = [t.cuda() for t in p.choices(2000, 2)]
    G = p.rand(138, 23).cuda()
    out = torch.empty(2000, 3).cuda()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(pm.PmlpError, match="graph capture") as e:
            p.net.gradients_routed(X, idx, w, dY)
        assert e.value.code == pm.PMLP_ESTATE
        with pytest.raises(pm.PmlpError, match="graph capture"):
            p.net.orthogonalize(G)
        out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    close(p.net.forward_routed(X, idx, w, out=out).cpu(), p.want(X.cpu(), idx.cpu(), w.cpu())["Y"])


def test_two_packs_at_once(pm):
    a = Pool(pm, 23, 3, [40, 8, 90], [7, 2, 3], False, seed=1)
    b = Pool(pm, 11, 2, [60, 9], [6, 3], True, seed=2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    data = []
    for p in (a, b):
        X, dY = p.rand(700, p.F), p.rand(700, p.O)
        data.append((X, *p.choices(700, 2), dY))
    dev = [[t.cuda() for t in d] for d in data]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, p in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i] = p.net.gradients_routed(*dev[i])
    torch.cuda.synchronize()
    for i, (p, names) in enumerate(((a, ("W1", "W2", "weight")), (b, ("W1", "V1", "W2", "weight")))):
        want = p.want(data[i][0], data[i][1], data[i][2], data[i][3])
        for g, k in zip(got[i], names):
            close(g, want[k], k)


def test_neighbours_are_left_alone(pm):
    """Nothing is written outside the outputs."""
    p = Pool(pm, 37, 3, [5, 64, 65], [7, 2, 3], False)
    B, K = 70, 2
    X, dY = p.rand(B, 37).cuda(), p.rand(B, 3).cuda()
    idx, w = [t.cuda() for t in p.choices(B, K)]
    sizes = {"Y": B * 3, "W1": 134 * 37, "W2": 3 * 134, "weight": B * K}
    bufs = {k: torch.full((n + 128,), 7.5).cuda() for k, n in sizes.items()}
    at = {k: v[64:].data_ptr() for k, v in bufs.items()}
    h = p.net.handle
    pm.pmlp_set_stream(h, torch.cuda.current_stream().cuda_stream)
    pm.pmlp_forward_routed(h, X, B, idx, w, K, at["Y"])
    pm.pmlp_gradients_routed(h, X, B, idx, w, K, dY, at["W1"], None, at["W2"], at["weight"])
    torch.cuda.synchronize()
    want = p.want(X.cpu(), idx.cpu(), w.cpu(), dY.cpu())
    want["Y"] = p.want(X.cpu(), idx.cpu(), w.cpu())["Y"]
    for k, v in bufs.items():
        assert bool((v[:64] == 7.5).all()) and bool((v[64 + sizes[k]:] == 7.5).all()), k
        close(v[64:64 + sizes[k]].reshape(want[k][0].shape), want[k], k)


def test_training_as_a_mixture(pm):
    """Routing, the mixture, its gradients and the updates together, three steps."""
    p = Pool(pm, 12, 3, [6, 30, 70], [7, 2, 3], True, seed=9)
    M, B, K, lr, mu = 3, 120, 2, 0.05, 0.9
    X, target = p.rand(B, 12), p.rand(B, 3)
    gate = p.rand(12, M)
    moms = {k: torch.zeros(84 + 22, 12).cuda() for k in ("W1", "V1")}
    rmoms = {k: torch.zeros(106, 12).double() for k in ("W1", "V1")}
    edges = [0, 6, 36, 106]
    P = {k: getattr(p, k).double() for k in ("W1", "V1", "W2")}
    dgate = gate.cuda()
    rgate = gate.double()
    for step in range(3):
        scores = X.cuda() @ dgate
        idx, w = p.net.route(scores, K)
        Y = p.net.forward_routed(X.cuda(), idx, w)
        dY = 2 * (Y - target.cuda()) / B
        dW1, dV1, dW2, dw = p.net.gradients_routed(X.cuda(), idx, w, dY)
        ds = p.net.route_backward(idx, w, dw)
        p.net.muon_step(dW1, lr, "W1", momentum=moms["W1"], mu=mu)
        p.net.muon_step(dV1, lr, "V1", momentum=moms["V1"], mu=mu)
        p.net.muon_step(dW2, lr, "W2", steps=0)
        dgate -= lr * (X.cuda().t() @ ds)
        # the same in 64 bits
        s = X.double() @ rgate
        ri, rw = (torch.from_numpy(t) for t in rr.route(s.numpy(), K))
        assert torch.equal(ri, idx.cpu())
        ref = lambda d=None: rr.mixture(p.hs, p.acts, X.double(), ri.long(), rw, P["W1"], P["V1"],
                                        P["W2"], d)
        rdY = 2 * (ref()["Y"][0] - target.double()) / B
        g = ref(rdY)
        for k in ("W1", "V1"):
            rmoms[k] = mu * rmoms[k] + g[k][0]
            for m in range(M):
                r = slice(edges[m], edges[m + 1])
                d, _ = rr.orthogonalized((g[k][0] + mu * rmoms[k])[r], 5)
                P[k][r] -= lr * max(1.0, d.shape[0] / d.shape[1]) ** 0.5 * d
        P["W2"] -= lr * g["W2"][0]
        rdw = g["weight"][0]
        rds = rw * (rdw - (rw * rdw).sum(1, keepdim=True))
        full = torch.zeros(B, M).double().scatter_add_(1, ri.long(), rds)
        rgate = rgate - lr * (X.double().t() @ full)
    got = dict(zip(p.net.param_names, p.net.get_params()))
    for k in ("W1", "V1", "W2"):
        # gradients agree to about 1e-5 of their size; an orthogonalised direction multiplies
        # what is off in weak directions by up to 3.4445^5 = 485: 5e-3 of its entries (at most
        # 1.2 sqrt(rows / cols) = 2.9), times three rates
        assert float((torch.from_numpy(got[k]).double() - P[k]).abs().max()) < 3 * lr * 5e-3 * 2.9
    assert float((dgate.cpu().double() - rgate).abs().max()) < 1e-3


# --- refusals ---------------------------------------------------------------------------

def test_refusals(pm):
    p = Pool(pm, 4, 2, [3, 5], [2, 2], False)
    X, dY = p.rand(6, 4).cuda(), p.rand(6, 2).cuda()
    idx, w = [t.cuda() for t in p.choices(6, 2)]
    net = p.net
    for call in (lambda: net.forward_routed(X.cpu(), idx, w), lambda: net.forward_routed(X, idx.long(), w),
                 lambda: net.forward_routed(X, idx[:5].contiguous(), w[:5].contiguous()),
                 lambda: net.forward_routed(X, idx, w[:, :1].contiguous()),
                 lambda: net.forward_routed(X, idx, w.double()), lambda: net.forward_routed(X, idx[0], w[0]),
                 lambda: net.forward_routed(X, idx, w, out=dY.t()),
                 lambda: net.gradients_routed(X, idx, w, dY[:3]), lambda: net.route(X, 2),
                 lambda: net.route(dY.double(), 1), lambda: net.route_backward(idx, w, dY[:5]),
                 lambda: net.forward_routed(X, idx.t(), w.t())):
        with pytest.raises(ValueError):
            call()
    for K in (0, -1, 17):
        with pytest.raises(pm.PmlpError, match="K must be") as e:
            net.route(dY, K)
        assert e.value.code == pm.PMLP_EINVAL
    h = net.handle
    with pytest.raises(pm.PmlpError, match="batch size"):
        pm.pmlp_forward_routed(h, X, 0, idx, w, 2, dY)
    with pytest.raises(pm.PmlpError, match="null"):
        pm.pmlp_forward_routed(h, X, 6, None, w, 2, dY)
    with pytest.raises(pm.PmlpError, match="null"):
        pm.pmlp_gradients_routed(h, X, 6, idx, w, 2, dY, None, None, None, None)
    for out in (X, idx, w):
        with pytest.raises(pm.PmlpError, match="overlaps"):
            pm.pmlp_forward_routed(h, X, 6, idx, w, 2, out)
    a = torch.empty(8 * 4 + 16).cuda()
    with pytest.raises(pm.PmlpError, match="overlap"):
        pm.pmlp_gradients_routed(h, X, 6, idx, w, 2, dY, a, None, a[16:], torch.empty(12).cuda())
    with pytest.raises(pm.PmlpError, match="overlap"):
        pm.pmlp_route(h, dY, 6, 2, idx, idx)
    for other in (pm.PackedMLP(4, 2, [3, 5], [2, 2], biases=True),
                  pm.DeepPackedMLP(4, 2, [3, 5], [2, 2], [2, 2]),
                  pm.BlockPackedMLP(4, 2, [3, 5], [2, 2], gated=True, norm=True)):
        with pytest.raises(pm.PmlpError) as e:
            other.forward_routed(X, idx, w)
        assert e.value.code == pm.PMLP_ESTATE
        other.route(dY, 1)   # (the router is for every pack)
    net.set_precision(pm.PMLP_BF16_GEMM)
    with pytest.raises(pm.PmlpError) as e:
        net.gradients_routed(X, idx, w, dY)
    assert e.value.code == pm.PMLP_ESTATE
