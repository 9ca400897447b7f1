"""Host-side checks of pmlp_create_block and its calls that need no GPU:
arguments are refused before any device work."""
import ctypes as C

import numpy as np
import pytest


@pytest.fixture(scope="module")
def pm():
    import os
    import paper_2206_08369_amd as pm
    if not os.path.exists(pm.library_path()):
        from paper_2206_08369_amd import build
        build.build()
    pm.load_library()
    return pm


@pytest.mark.parametrize("F,O,hs,acts,flags,msg", [
    (3, 2, [1], [0], 0, "gate, a norm or both"),
    (3, 2, [1], [0], 2, "gate, a norm or both"),
    (3, 2, [1], [0], 4 | 1, "unknown flags"),
    (3, 2, [1], [0], 16, "unknown flags"),
    (3, 2, [1], [0], -1, "unknown flags"),
    (0, 2, [1], [0], 4, "F must be"),
    (3, 1, [1], [0], 8, "O must be"),
    (3, 17, [1], [0], 12, "O must be"),
    (3, 2, [0], [0], 4, "hidden size"),
    (3, 2, [2, -1], [0, 0], 4, "hidden size"),
    (3, 2, [1], [13], 4, "activation id"),
])
def test_create_rejects_bad_arguments(pm, F, O, hs, acts, flags, msg):
    with pytest.raises(pm.PmlpError) as e:
        pm.pmlp_create_block(F, O, hs, acts, 0, flags)
    assert e.value.code == pm.PMLP_EINVAL
    assert msg in str(e.value)


def test_null_arguments_rejected(pm):
    lib = pm.load_library()
    h, one = C.c_void_p(), np.ones(2, np.int32)
    assert lib.pmlp_create_block(None, 3, 2, 2, one.ctypes.data, one.ctypes.data, 0, 4) == pm.PMLP_EINVAL
    assert lib.pmlp_create_block(C.byref(h), 3, 2, 2, None, one.ctypes.data, 0, 4) == pm.PMLP_EINVAL
    assert lib.pmlp_create_block(C.byref(h), 3, 2, 0, one.ctypes.data, one.ctypes.data, 0, 4) == pm.PMLP_EINVAL
    assert h.value is None
    assert lib.pmlp_gradients_block(None, None, None, 1, *[None] * 5) == pm.PMLP_EINVAL
    assert lib.pmlp_gradients_block_mse(None, None, None, 1, *[None] * 5) == pm.PMLP_EINVAL
    assert lib.pmlp_get_params_block(None, *[None] * 5) == pm.PMLP_EINVAL
    assert lib.pmlp_set_params_block(None, *[None] * 5) == pm.PMLP_EINVAL


def test_wrapper_rejects_bad_arguments(pm):
    with pytest.raises(ValueError):
        pm.pmlp_create_block(3, 2, [1, 2], [0], 0, 4)
    with pytest.raises(ValueError):
        pm.BlockPackedMLP(3, 2, [1], [0], head="other")
