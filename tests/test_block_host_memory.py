"""Host memory that runs out while a pack is made is an error code at the C entry: no
C++ exception leaves it, which would end the process."""
import os
import subprocess
import sys

import pytest

CODE = """
import os, resource, sys
import numpy as np
import paper_2206_08369_amd as pm
pm.load_library()
size = int(open("/proc/self/statm").read().split()[0]) * os.sysconf("SC_PAGE_SIZE")
wide, act = np.int32([2 ** 31 - 2]), np.int32([0])
# (8 GiB for the model of each unit, where there is room for one more)
resource.setrlimit(resource.RLIMIT_AS, (size + (1 << 30), resource.RLIM_INFINITY))
for call in ({calls}):
    try:
        call()
        print("made")
    except pm.PmlpError as e:
        print(e.code == pm.PMLP_ENOMEM, "host allocation" in str(e))
"""
CALLS = {
    "block": "lambda: pm.pmlp_create_block(1, 2, wide, act, 0, 4 | 8),",
    "one_layer": "lambda: pm.pmlp_create(1, 2, wide, act, 0, 1),",
    "deep": "lambda: pm.pmlp_create_deep(1, 2, np.int32([1]), wide, act, 0), "
            "lambda: pm.pmlp_create_deep(1, 2, wide, np.int32([1]), act, 0),",
}


@pytest.mark.parametrize("kind", sorted(CALLS))
def test_no_memory_for_the_units(kind):
    import paper_2206_08369_amd as pm
    if not os.path.exists(pm.library_path()):
        from paper_2206_08369_amd import build
        build.build()
    run = subprocess.run([sys.executable, "-c", CODE.format(calls=CALLS[kind])],
                         capture_output=True, text=True, timeout=120,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(pm.__file__))))
    assert run.returncode == 0, run.stderr[-500:]
    lines = run.stdout.split("\n")[:-1]
    # (without a device the second layer's units are never reached)
    assert lines and all(v in ("True True", "False False") for v in lines)
    assert lines[-1] == "True True"
