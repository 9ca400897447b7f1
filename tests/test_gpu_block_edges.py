"""Block packs: calls that the header allows at the ends of their ranges and next to
each other."""
import numpy as np
import pytest

import block_bounds
import block_reference as ref

pytestmark = pytest.mark.gpu

SMOOTH = (0, 2, 3, 4, 6, 7, 8, 9, 12)
KINDS = {"gated": (True, False), "norm": (False, True), "both": (True, True)}


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    torch.cuda.set_device(0)
    return torch


@pytest.fixture(scope="module")
def pm(torch):
    import paper_2206_08369_amd as pm
    pm.load_library()
    return pm


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make(pm, hs, acts, p, F, O, kind):
    net = pm.BlockPackedMLP(F, O, hs, acts, gated=KINDS[kind][0], norm=KINDS[kind][1])
    net.set_params(**p)
    return net


def compare(torch, net, hs, acts, p, X, y):
    want = block_bounds.pack(hs, acts, p, X, y)
    got = {"logits": net.forward(dev(torch, X))}
    got.update(zip(net.param_names, net.gradients(dev(torch, X), dev(torch, y))))
    for k, v in got.items():
        val, bound = want[k]
        err = np.abs(v.cpu().numpy().astype(np.float64) - val) / (bound + 1e-30)
        assert err.max() <= 1, "%s: %.3g times its bound" % (k, err.max())


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("O, B", [(16, 100), (10, 64), (16, 300), (4, 128), (2, 1100)])
def test_few_wide_models(pm, torch, kind, O, B):
    """Models of hundreds of pieces, which groups of threads merge: every number of
    groups and threads that the output and loss kernels run with."""
    rng = np.random.default_rng(O + B)
    hs, acts, F = np.int32([6000, 5, 900]), np.int32([2, 7, 8]), 7
    p = ref.random_params(rng, hs, F, O, *KINDS[kind])
    X = rng.standard_normal((B, F)).astype(np.float32)
    y = rng.integers(0, O, B).astype(np.int32)
    net = make(pm, hs, acts, p, F, O, kind)
    compare(torch, net, hs, acts, p, X, y)
    net.close()


def test_batch_sizes_in_any_order(pm, torch):
    """Plans and workspaces of a handle that sees many batch sizes, back and forth."""
    rng = np.random.default_rng(4)
    hs = rng.integers(1, 70, 25).astype(np.int32)
    acts, F, O = rng.choice(SMOOTH, 25).astype(np.int32), 20, 3
    p = ref.random_params(rng, hs, F, O, True, True)
    X = rng.standard_normal((700, F)).astype(np.float32)
    y = rng.integers(0, O, 700).astype(np.int32)
    net = make(pm, hs, acts, p, F, O, "both")
    whole = net.forward(dev(torch, X))
    seen = {}
    for B in (1, 700, 33, 256, 5, 257, 32, 700, 64, 1, 31, 512, 33, 256):
        L = net.forward(dev(torch, X[:B]))
        g = net.gradients(dev(torch, X[:B]), dev(torch, y[:B]))
        # (another batch size may sum a model's pieces in another order)
        assert (L - whole[:B]).abs().max() < 1e-4
        if B in seen:
            assert torch.equal(L, seen[B][0])
            assert all(torch.equal(a, b) for a, b in zip(g, seen[B][1]))
        seen[B] = (L, g)
    for B in (5, 33, 257):
        compare(torch, net, hs, acts, p, X[:B], y[:B])
    net.close()


def test_two_handles_at_once(pm, torch):
    """Handles on two streams, whose calls overlap, next to the same calls one by one."""
    rng = np.random.default_rng(5)
    F, O, B = 16, 10, 300
    pools = []
    for seed in (1, 2):
        hs = rng.integers(4, 90, 400).astype(np.int32)
        acts = rng.choice(SMOOTH, 400).astype(np.int32)
        pools.append((hs, acts, ref.random_params(rng, hs, F, O, True, True)))
    X = dev(torch, rng.standard_normal((B, F)).astype(np.float32))
    y = dev(torch, rng.integers(0, O, B).astype(np.int32))
    alone = []
    for hs, acts, p in pools:
        net = make(pm, hs, acts, p, F, O, "both")
        for _ in range(4):
            net.train_step(X, y, 0.1)
        alone.append((net.forward(X), net.get_params()))
        net.close()
    nets = [make(pm, hs, acts, p, F, O, "both") for hs, acts, p in pools]
    streams = [torch.cuda.Stream() for _ in nets]
    torch.cuda.synchronize()
    out = [None, None]
    for i in range(5):
        for k, (net, s) in enumerate(zip(nets, streams)):
            with torch.cuda.stream(s):
                if i < 4:
                    net.train_step(X, y, 0.1)
                else:
                    out[k] = net.forward(X)
    torch.cuda.synchronize()
    for net, o, (L, params) in zip(nets, out, alone):
        assert torch.equal(o, L)
        assert all(np.array_equal(a, b) for a, b in zip(net.get_params(), params))
        net._stream()
        net.close()


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("F, B", [(12, 40), (12, 400), (150, 70)])
def test_a_captured_epoch_equals_an_eager_one(pm, torch, kind, F, B):
    """Steps of a whole and of a ragged batch and a validation pass in one graph,
    replayed, with the handle's own eager calls in between."""
    rng = np.random.default_rng(F + B)
    hs = rng.integers(4, 50, 40).astype(np.int32)
    acts, O, rest = rng.choice(SMOOTH, 40).astype(np.int32), 6, B // 3
    p = ref.random_params(rng, hs, F, O, *KINDS[kind])
    nets = [make(pm, hs, acts, p, F, O, kind) for _ in range(2)]
    X = dev(torch, rng.standard_normal((B + rest, F)).astype(np.float32))
    y = dev(torch, rng.integers(0, O, B + rest).astype(np.int32))
    out = torch.zeros(B + rest, 40, O, device="cuda")

    def epoch(net, out):
        net.train_step(X[:B], y[:B], 0.05)
        net.train_step(X[B:], y[B:], 0.05)
        net.forward(X, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        epoch(nets[0], out)      # sizes the workspace
    side.synchronize()
    nets[0]._stream()
    nets[0].set_params(**p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        epoch(nets[0], out)
    want = torch.zeros_like(out)
    for rep in range(4):
        graph.replay()
        torch.cuda.synchronize()
        epoch(nets[1], want)
        assert torch.equal(out, want)
        assert np.array_equal(nets[0].losses(), nets[1].losses())
        one = X[rep:rep + 1].contiguous()
        assert torch.equal(nets[0].forward(one), nets[1].forward(one))
    for net in nets:
        net._stream()
        net.close()
