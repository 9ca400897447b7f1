"""Routed packs with one model much wider than the others: few slots each on its own, many grouped,
and a launch of few slots over all dies."""
import pytest
import torch

from test_gpu_routed import Pool, close, pm  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("picks", ["any", "wide", "half"])
@pytest.mark.parametrize("F,B,K,kernel", [(20, 64, 1, "k_rt_few_waves"), (20, 300, 1, "k_rt_few_waves"),
                                          (100, 131, 2, "k_rt_few"), (20, 16384, 1, "k_rt_tile"),
                                          (100, 700, 3, "k_rt_tile")])
@pytest.mark.parametrize("gated", [False, True])
def test_one_wide_model(pm, gated, F, B, K, kernel, picks):
    hs = [1 + m % 9 for m in range(99)] + [3000]
    p = Pool(pm, F, 2, hs, [2] * 100, gated, seed=B)
    idx, w = p.choices(B, K)
    if picks != "any":
        idx[::1 if picks == "wide" else 2] = 99
    X = p.rand(B, F)
    got = p.forward(X, idx, w)
    assert p.net.kernel_variants()["gemm_fwd"][0] == kernel
    some = torch.arange(0, B, 1 + B // 500)  # (a sample's answer is its own)
    close(got[some.cuda()], p.want(X[some], idx[some], w[some])["Y"], "Y")
    assert torch.equal(got, p.forward(X, idx, w))
    p.net.check_routed()
