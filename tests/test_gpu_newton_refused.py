"""An update that is refused leaves the momentum, the weights and the output as they were."""
import numpy as np
import pytest
import torch

from test_gpu_newton import pm, randn  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_refused_update_changes_nothing(pm):
    """Under capture, where the plan is there and the workspace of the large matrix is not."""
    net = pm.PackedMLP(200, 2, [9, 300], [0, 0])
    N = 309
    G, mom = randn(1, N, 200).cuda(), randn(2, N, 200).cuda()
    net.muon_step(G, 0.1, momentum=mom, steps=0)
    torch.cuda.synchronize()
    weights, held, out = net.get_params(), mom.clone(), torch.full((N, 200), 7.5).cuda()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    mark = torch.ones(3).cuda()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(pm.PmlpError, match="graph capture") as e:
            net.muon_step(G, 0.1, momentum=mom)
        assert e.value.code == pm.PMLP_ESTATE
        with pytest.raises(pm.PmlpError, match="graph capture"):
            net.orthogonalize(G, momentum=mom, out=out)
        mark.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert not bool(mark.any())
    assert torch.equal(mom, held) and bool((out == 7.5).all())
    assert all(np.array_equal(a, b) for a, b in zip(net.get_params(), weights))
    net.muon_step(G, 0.1, momentum=mom)  # the pack as it was: one update, of every model
    assert torch.allclose(mom, 0.95 * held + G, rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("steps", [0, 5])
def test_rates_inside_the_momentum_are_refused(pm, steps):
    """The momentum is written while models still read their rates."""
    net = pm.PackedMLP(20, 2, [30, 9], [2, 2])
    G, mom = randn(1, 39, 20).cuda(), randn(2, 39, 20).cuda()
    weights, held = net.get_params(), mom.clone()
    for rates in (mom.reshape(-1)[:2], mom.reshape(-1)[-2:]):
        with pytest.raises(pm.PmlpError, match="overlap"):
            net.muon_step(G, rates, momentum=mom, steps=steps)
    torch.cuda.synchronize()
    assert torch.equal(mom, held)
    assert all(np.array_equal(a, b) for a, b in zip(net.get_params(), weights))
