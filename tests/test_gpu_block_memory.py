"""Device memory of block packs: what a larger batch replaces is given back, what a
captured graph holds is kept."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

MIB = 1 << 20


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


def in_use(torch):
    torch.cuda.synchronize()
    free, total = torch.cuda.mem_get_info()
    return total - free


def pool(pm, torch, F, B, units=20000, O=2):
    """A pool (two of a kind start with the same weights) and a batch."""
    hs = np.full(units // 100, 100, np.int32)
    net = pm.BlockPackedMLP(F, O, hs, np.full(hs.size, 7), gated=True, norm=True)
    X = torch.randn(B, F, device="cuda")
    y = torch.randint(0, O, (B,), device="cuda", dtype=torch.int32)
    return net, X, y


def test_batches_that_grow_keep_one_workspace(pm, torch):
    """Twelve batch sizes of 160 to 340 MB of pre-activations each: one workspace at the
    end, not one a size."""
    net, X, y = pool(pm, torch, 140, 2100)
    before = in_use(torch)
    for B in range(1000, 2101, 100):
        net.train_step(X[:B], y[:B], 0.0)
    largest = 2 * 20000 * 2304 * 4 + 64 * MIB  # Z and U of a padded batch, and the rest
    assert in_use(torch) - before <= largest + 64 * MIB
    assert net.nonfinite_count() == 0
    net.close()


def test_calls_under_way_keep_their_workspace(pm, torch):
    """A larger batch on another stream, while calls that use the smaller workspace are
    still to run."""
    net, X, y = pool(pm, torch, 140, 600)
    twin, _, _ = pool(pm, torch, 140, 600)
    want = twin.forward(X[:300].contiguous())
    other = twin.forward(X)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    small = X[:300].contiguous()
    with torch.cuda.stream(a):
        late = torch.zeros_like(small)
        for _ in range(200):
            late.add_(small, alpha=0.005)
        late.copy_(small)
        got = net.forward(late)
    with torch.cuda.stream(b):
        rest = net.forward(X)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(rest, other)
    net._stream()
    net.close()
    twin.close()


def test_a_captured_workspace_outlives_larger_batches(pm, torch):
    """Two graphs of two batch sizes, both replayed after a third, larger batch: each
    still writes into the workspace that it was captured with."""
    net, X, y = pool(pm, torch, 12, 5000, units=3000)
    twin, _, _ = pool(pm, torch, 12, 5000, units=3000)
    side = torch.cuda.Stream()
    graphs = []
    for B in (40, 900):
        Xs, out = X[:B].contiguous(), torch.zeros(B, net.M, 2, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            net.forward(Xs, out=out)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            net.forward(Xs, out=out)
        graphs.append((g, Xs, out))
    for rep in range(3):
        assert torch.equal(net.forward(X[rep:].contiguous()), twin.forward(X[rep:].contiguous()))
        for g, Xs, out in graphs:
            Xs.copy_(torch.randn_like(Xs))
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, twin.forward(Xs))
    net._stream()
    net.close()
    twin.close()


def test_a_pool_that_fits_is_created(pm, torch):
    """A gated pool of two weight matrices of 4 GiB, where the device has 11 GiB left: it
    needs no third one on the way."""
    F, hs = 1024, np.full(10486, 100, np.int32)
    torch.cuda.empty_cache()
    free, _ = torch.cuda.mem_get_info()
    held = torch.empty(free - (11 << 30), dtype=torch.uint8, device="cuda")
    try:
        net = pm.BlockPackedMLP(F, 2, hs, np.zeros(hs.size), seed=1, gated=True)
        with pytest.raises(pm.PmlpError) as e:
            pm.BlockPackedMLP(F, 2, hs, np.zeros(hs.size), seed=1, gated=True)
        assert e.value.code == pm.PMLP_ENOMEM
        L = net.forward(torch.ones(1, F, device="cuda"))
        assert torch.isfinite(L).all()
        net.close()
    finally:
        del held
        torch.cuda.empty_cache()
