"""Orthogonalised updates of matrices whose rows and columns are of unlike size: what fp32
keeps of the small ones (nearly dead units, rare features) is kept."""
import pytest
import torch

import newton_bounds as nb
from test_gpu_newton import pm  # noqa: F401

pytestmark = pytest.mark.gpu

# widths of models of 100, 130 and 1,300 inputs: matrices in LDS (of every number of 16 rows),
# and ones that are not
SHAPES = [(100, [1, 2, 8, 20, 33, 50, 70, 90, 100, 112, 128, 250]), (9, [3, 9, 40, 1000]),
          (700, [1, 5, 16, 20, 40]), (130, [3, 140, 129, 260]), (1300, [1, 7, 40]),
          (64, [64] * 3)]


def parts(F, hs, kind, seed=0):
    return [nb.unlike(h, F, kind, seed + m) for m, h in enumerate(hs)]


def check(got, mats, n, what):
    at = 0
    for m, (M, rows, cols) in enumerate(mats):
        mine = got[at:at + M.shape[0]].cpu().double()
        at += M.shape[0]
        want, bound = nb.orthogonalized(M, n, rows, cols)
        over = float(((mine - want).abs() / bound).max())
        assert over <= 1, "%s model %d %s: %.3g times what is allowed" % (what, m, tuple(M.shape), over)


@pytest.mark.parametrize("kind", nb.KINDS)
@pytest.mark.parametrize("n", [1, 5, 10])
@pytest.mark.parametrize("F,hs", SHAPES, ids=lambda v: str(v) if isinstance(v, int) else "M%d" % len(v))
def test_input_weights(pm, F, hs, n, kind):
    if kind == "aligned":
        hs = [h for h in hs if h > 1]
    net = pm.PackedMLP(F, 2, hs, [0] * len(hs))
    mats = parts(F, hs, kind)
    G = torch.cat([M for M, _, _ in mats]).float().cuda()
    got = net.orthogonalize(G, steps=n)
    check(got, mats, n, kind)
    assert torch.equal(got, net.orthogonalize(G, steps=n))


@pytest.mark.parametrize("O", [2, 3, 16])
@pytest.mark.parametrize("n", [5, 10])
def test_output_weights(pm, O, n):
    """Units that hardly count are columns of W2."""
    hs = [1, 7, 300, 500, 1500, 3000]
    net = pm.PackedMLP(4, O, hs, [0] * len(hs))
    mats = [nb.unlike(O, h, "columns", m) for m, h in enumerate(hs)]
    G = torch.cat([M for M, _, _ in mats], 1).float().cuda()
    got = net.orthogonalize(G, "W2", steps=n)
    at = 0
    for m, (M, rows, cols) in enumerate(mats):
        want, bound = nb.orthogonalized(M, n, rows, cols)
        over = float(((got[:, at:at + M.shape[1]].cpu().double() - want).abs() / bound).max())
        at += M.shape[1]
        assert over <= 1, (m, M.shape, over)


@pytest.mark.parametrize("F", [100, 140])
def test_many_models(pm, F):
    """More than 2,048 matrices go in launches by size."""
    hs = [1 + (37 * m) % 128 for m in range(2100)] + [150]
    net = pm.PackedMLP(F, 2, hs, [0] * len(hs))
    mats = [nb.unlike(h, F, nb.KINDS[m % 3], m) for m, h in enumerate(hs)]
    got = net.orthogonalize(torch.cat([M for M, _, _ in mats]).float().cuda())
    at = [0]
    for h in hs:
        at.append(at[-1] + h)
    for m in list(range(0, 2100, 19)) + [2100]:
        check(got[at[m]:at[m + 1]], mats[m:m + 1], 5, "model %d" % m)


@pytest.mark.parametrize("F,h,M", [(380, 250, 90), (250, 380, 90), (200, 256, 130)])
def test_large_tiles(pm, F, h, M):
    """512 tiles of 128 x 128 and more, with partly empty ones at their ends; turned and not."""
    net = pm.PackedMLP(F, 2, [h] * M, [0] * M)
    mats = [nb.unlike(h, F, nb.KINDS[m % 4], m) for m in range(M)]
    G = torch.cat([A for A, _, _ in mats]).float().cuda()
    got = net.orthogonalize(G)
    assert net.kernel_variants()["hidden2"][0] == "k_ns_product"
    for m in (0, 1, 2, 3, M - 4, M - 3, M - 2, M - 1):
        check(got[h * m:h * (m + 1)], mats[m:m + 1], 5, "model %d" % m)
    assert torch.equal(got, net.orthogonalize(G))


@pytest.mark.parametrize("F,hs", [(50, [8, 40]), (200, [150, 9])])
def test_tiny_rows_do_not_vanish(pm, F, hs):
    """Rows of 1e-20 of the others grow by 3.4445 in each of five steps, as they do in fp32."""
    net = pm.PackedMLP(F, 2, hs, [0] * 2)
    G = torch.randn(sum(hs), F, generator=torch.Generator().manual_seed(1)).double()
    small = [1, hs[0] + 2]
    G[small] *= 1e-20
    got = net.orthogonalize(G.float().cuda()).cpu().double()
    for s, r in zip(small, (slice(0, hs[0]), slice(hs[0], sum(hs)))):
        want, bound = nb.orthogonalized(G[r].float().double(), 5, torch.ones(r.stop - r.start, 1).double(),
                                        torch.ones(1, F).double())
        assert bool(((got[r] - want).abs() <= bound).all())
        assert bool(want[s - r.start].abs().max() > 1e-20)


def test_a_lone_entry_of_each_row(pm):
    """A diagonal of sizes down to 1e-24."""
    F, hs = 70, [40, 70, 300]
    net = pm.PackedMLP(F, 2, hs, [0] * 3)
    mats = []
    for h in hs:
        M = torch.zeros(h, F).double()
        k = min(h, F)
        rows = torch.ones(h, 1).double()
        rows[:k, 0] = 10.0 ** -(torch.arange(k).double() % 25)
        M[torch.arange(k), torch.arange(k)] = 1.0
        M = (M * rows).float().double()
        mats.append(M)
    got = net.orthogonalize(torch.cat(mats).float().cuda()).cpu().double()
    at = 0
    for M in mats:
        x = M / M.norm()
        want = x.clone()
        for _ in range(5):
            want = want * (3.4445 - 4.7750 * want ** 2 + 2.0315 * want ** 4)
        mine = got[at:at + M.shape[0]]
        at += M.shape[0]
        # each value by itself: five steps, each within 2^-20 of the value it had
        assert bool(((mine - want).abs() <= 5 * 3.5 * 2.0 ** -20 * want.abs()).all())
