"""Block packs whose pre-activations are small, or so far below zero that the
activation is: the hidden values are accurate relative to themselves, which a norm
of such values needs (it divides by a deviation as small as they are)."""
import numpy as np
import pytest

import block_bounds
import block_reference as ref

pytestmark = pytest.mark.gpu

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


def check(pm, torch, acts_of, kind, F, O, B, scale, offset, seed, M=24, grads=True):
    gated, norm = KINDS[kind]
    rng = np.random.default_rng(seed)
    hs = rng.integers(5, 60, M).astype(np.int32)
    acts = np.resize(np.int32(acts_of), M)
    p = ref.random_params(rng, hs, F, O, gated, norm)
    X = rng.standard_normal((B, F)).astype(np.float32)
    X[:, 0] = 1
    p["W1"] = (p["W1"] * np.float32(scale)).astype(np.float32)
    p["W1"][:, 0] += np.float32(offset)
    if gated:
        p["V1"][:, 0] += 1
    y = rng.integers(0, O, B).astype(np.int32)
    want = block_bounds.pack(hs, acts, p, X, y)
    net = pm.BlockPackedMLP(F, O, hs, acts, gated=gated, norm=norm)
    net.set_params(**p)
    got = {"logits": net.forward(dev(torch, X))}
    if grads:
        got.update(zip(net.param_names, net.gradients(dev(torch, X), dev(torch, y))))
    net.close()
    for k, v in got.items():
        val, bound = want[k]
        err = np.abs(v.cpu().numpy().astype(np.float64) - val) / (bound + 1e-30)
        assert err.max() <= 1, "%s: %.3g times its bound at %s" % (
            k, err.max(), np.unravel_index(err.argmax(), err.shape))


# batches that run in one launch and in three, pre-activations that are stored
SIZES = [(9, 2, 40), (36, 10, 300), (100, 3, 20), (140, 4, 50), (140, 10, 40)]


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("F, O, B", SIZES)
@pytest.mark.parametrize("scale", [1.0, 0.3, 1e-2, 1e-3, 1e-5])
def test_small_pre_activations(pm, torch, kind, F, O, B, scale):
    """Identity, tanh, ELU, GELU, SiLU, Swish and Mish, all near z or z / 2 at 0."""
    check(pm, torch, (0, 2, 4, 6, 7, 9, 12), kind, F, O, B, scale, 0, F + O + B)


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("F, O, B", SIZES)
@pytest.mark.parametrize("scale", [1.0, 1e-3])
def test_small_pre_activations_of_selu(pm, torch, kind, F, O, B, scale):
    check(pm, torch, (10,), kind, F, O, B, scale, 0, F + O + B, grads=False)


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("F, O, B", SIZES)
@pytest.mark.parametrize("offset", [0, -3, -9, 12])
def test_softplus_and_sigmoid_off_zero(pm, torch, kind, F, O, B, offset):
    check(pm, torch, (8, 3), kind, F, O, B, 1.0, offset, F + O + B)


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("F, O, B", SIZES)
@pytest.mark.parametrize("offset", [-6, -4, 4, 6])
def test_slopes_of_saturated_tanh(pm, torch, kind, F, O, B, offset):
    """Slopes of 1e-3 to 1e-6, accurate relative to themselves: one minus the square of a
    value next to one is not."""
    check(pm, torch, (2,), kind, F, O, B, 1.0, offset, F + O + B)
