"""Device memory of routed gradients where one model is much wider than the others."""
import numpy as np
import pytest
import torch

from test_gpu_routed import Pool, close, pm  # noqa: F401

pytestmark = pytest.mark.gpu


def test_hidden_values_take_their_own_models_width(pm):
    """Hidden values of 32,768 slots and of up to 31 places more for each model, as wide as
    that model: not all of them as wide as the widest."""
    def in_use():
        torch.cuda.synchronize()
        free, total = torch.cuda.mem_get_info()
        return total - free

    hs = [1 + m % 9 for m in range(5999)] + [1000]
    p = Pool(pm, 8, 2, hs, [2] * 6000, False)
    B = 32768
    X, dY = torch.randn(B, 8).cuda(), torch.randn(B, 2).cuda()
    idx = torch.randint(0, 6000, (B, 1), dtype=torch.int32).cuda()
    w = torch.ones(B, 1).cuda()
    out = p.net.gradients_routed(X[:1], idx[:1], w[:1], dY[:1])
    del out
    torch.cuda.empty_cache()
    before = in_use()
    out = p.net.gradients_routed(X, idx, w, dY)
    grads = sum(t.numel() for t in out) * 4
    need = 2 * 4 * (1000 * B + 31 * sum(hs))  # two buffers of hidden values
    assert in_use() - before <= need + grads + (96 << 20)


@pytest.mark.parametrize("gated", [False, True])
def test_models_of_unlike_width(pm, gated):
    """The last places of the last model lie at the end of the hidden values."""
    hs = [1, 2, 3, 700]
    for picks in ([3] * 64, [3] * 65 + [0], list(range(4)) * 17):
        p = Pool(pm, 11, 3, hs, [7, 2, 3, 0], gated, seed=len(picks))
        B = len(picks)
        idx = torch.tensor(picks, dtype=torch.int32).reshape(B, 1)
        X, w, dY = p.rand(B, 11), p.rand(B, 1), p.rand(B, 3)
        want, got = p.want(X, idx, w, dY), p.gradients(X, idx, w, dY)
        for k in got:
            close(got[k], want[k], k)
