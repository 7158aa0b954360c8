"""The loss head without logits and the rows kept in 8 bits on their host side, on a CPU: sizes at their limits over host_launches.c, which refuses the
launches that the runtime refuses, and the training loop's checks of its head."""
import ctypes as C
import json
import os
import subprocess
import sys

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "libhostlaunches.so")
    subprocess.run(["cc", "-O1", "-shared", "-fPIC", os.path.join(HERE, "host_launches.c"), "-o", so], check=True)
    return so


def _child(runtime, what, *args):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), runtime, what, json.dumps(args)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout.splitlines()[-1])


# ---- in the child -----------------------------------------------------------------------------------------------
def _trainer(rt, d_top, n_classes, bf16, fused):
    """Workspace size, message, what gnntrain_create returns and its message, for a stage whose last level is d_top wide."""
    from test_host_launches import _Stage

    from paper_2308_10087_amd.binding import gnntrain_desc, lib
    st = _Stage("gcn", [8, d_top], 2, n=60, bf16=bf16)
    some = np.zeros(4096, np.uint8)
    at = (some.ctypes.data + 255) // 256 * 256
    d = gnntrain_desc()
    hs = (C.c_void_p * 1)(st.h)
    d.n_stages, d.stages, d.n_classes = 1, C.cast(hs, C.c_void_p), n_classes
    d.head_W = d.head_b = d.head_dW = d.head_db = d.labels = at
    d.optimizer, d.alpha_hist, d.head_fused = 0, 1, fused
    size = lib.gnntrain_workspace_size(C.byref(d))
    why = lib.gnntrain_last_error(None).decode()
    d.workspace, d.workspace_bytes = at, 1 << 60
    h = C.c_void_p(None)
    rc = lib.gnntrain_create(C.byref(d), C.byref(h))
    return [size, why, rc, lib.gnntrain_last_error(None).decode(), h.value is not None]


if __name__ == "__main__":
    _rt = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
    from test_host_launches import _Launch
    _rt.host_launch.restype, _rt.host_launch.argtypes = C.POINTER(_Launch), [C.c_size_t]
    _rt.host_launches.restype = C.c_size_t
    _rt.host_clear.argtypes = [C.c_int64]
    sys.path.insert(0, os.path.dirname(HERE))
    print(json.dumps(globals()[sys.argv[2]](_rt, *json.loads(sys.argv[3]))))
    sys.stdout.flush()
    os._exit(0)


# ---- tests ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bf16", [False, True])
def test_the_loop_refuses_what_its_head_refuses(runtime, bf16):
    """Before anything is launched, and with the head's own reason."""
    size, why, rc, again, made = _child(runtime, "_trainer", 1024, 1 << 24, bf16, 1)
    assert size == 0 and rc == -1 and not made
    assert "2^33" in why and "2^33" in again
    size, why, rc, again, made = _child(runtime, "_trainer", 65536, 3, bf16, 1)
    assert size == 0 and rc == -1 and not made
    assert "65534" in why and "65534" in again


def test_the_loop_takes_what_its_head_takes(runtime):
    for args in ((1024, 1 << 23, True, 1), (64, 70001, False, 1), (64, 41, False, 0), (256, 5, True, 1)):
        size, _, rc, again, made = _child(runtime, "_trainer", *args)
        assert size > 0 and rc == 0 and made, again
    size, why, rc, _, made = _child(runtime, "_trainer", 64, 65537, False, 0)
    assert size == 0 and rc == -1 and not made and "65536" in why
