"""Host-side checks of the routed calls and the orthogonalised update that need no GPU:
arguments are refused before any device work."""
import pytest

from test_block_host import pm  # noqa: F401  (the loaded library)


def test_null_handles_and_buffers(pm):
    lib = pm.load_library()
    assert lib.pmlp_route(None, None, 1, 1, None, None) == pm.PMLP_EINVAL
    assert lib.pmlp_route_backward(None, None, None, None, 1, 1, None) == pm.PMLP_EINVAL
    assert lib.pmlp_forward_routed(None, None, 1, None, None, 1, None) == pm.PMLP_EINVAL
    assert lib.pmlp_gradients_routed(None, None, 1, None, None, 1, *[None] * 5) == pm.PMLP_EINVAL
    assert lib.pmlp_routed_status(None) == pm.PMLP_EINVAL
    assert lib.pmlp_orthogonalize(None, 0, None, None, None, 0.9, 1, 5, None) == pm.PMLP_EINVAL
    assert lib.pmlp_muon_step(None, 0, None, None, 0.9, 1, 5, 0.1, None, 0.0) == pm.PMLP_EINVAL
    assert "null handle" in pm.pmlp_last_error()


def test_matrix_names(pm):
    assert pm.MATRIX_IDS == {"W1": 0, "V1": 1, "W2": 2, "W12": 3}
    net = pm.PackedMLP.__new__(pm.PackedMLP)
    with pytest.raises(ValueError, match="matrix must be"):
        net._matrix("W3")
