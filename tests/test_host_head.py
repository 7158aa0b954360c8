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
def _trainer(rt, d_top, n_classes, bf16, fused, n=60):
    """Workspace size, message, what gnntrain_create returns and its message, for a stage whose last level is d_top wide."""
    from test_host_launches import _Stage

    from paper_2308_10087_amd.binding import gnntrain_desc, lib
    st = _Stage("gcn", [8, d_top], 2, n=n, bf16=bf16)
    some = np.zeros(4096, np.uint8)
    at = (some.ctypes.data + 255) // 256 * 256
    d = gnntrain_desc()
    hs = (C.c_void_p * 1)(st.h)
    d.n_stages, d.stages, d.n_classes = 1, C.cast(hs, C.c_void_p), n_classes
    labels = np.zeros(n, np.int32)
    d.head_W = d.head_b = d.head_dW = d.head_db = at
    d.labels = labels.ctypes.data
    d.optimizer, d.alpha_hist, d.head_fused = 0, 1, fused
    size = lib.gnntrain_workspace_size(C.byref(d))
    why = lib.gnntrain_last_error(None).decode()
    d.workspace, d.workspace_bytes = at, 1 << 60
    h = C.c_void_p(None)
    rc = lib.gnntrain_create(C.byref(d), C.byref(h))
    return [size, why, rc, lib.gnntrain_last_error(None).decode(), h.value is not None]


def _buffer():
    """A 256-byte aligned address that is never read: launches are listed, not run."""
    some = np.zeros(4096, np.uint8)
    return some, (some.ctypes.data + 255) // 256 * 256


def _each(rt, what, cases):
    return [globals()[what](rt, *c) for c in cases]


def _weight_grad(rt, rows, d, d_out, bf16):
    """Size, return code, message, launches."""
    from paper_2308_10087_amd.binding import lib
    keep, at = _buffer()
    size = lib.gnnstage_rows8_weight_grad_workspace_size(rows, d, d_out, bf16)
    rt.host_clear(-1)
    rc = lib.gnnstage_rows8_weight_grad(at, (d + 31) // 32 * 32, at, (d + 31) // 32, at, bf16, d_out, rows, d, d_out, at, at, at, size or 1 << 60, None)
    return [size, rc, lib.gnnstage_last_error(None).decode() if rc else "", rt.host_launches()]


def _head(rt, rows, d, n_classes, bf16, grads):
    from paper_2308_10087_amd.binding import lib
    keep, at = _buffer()
    size = lib.gnntrain_head_xent_workspace_size(rows, d, n_classes, bf16, grads)
    rt.host_clear(-1)
    g = at + 256 if grads else None
    rc = lib.gnntrain_head_xent(at, d, at, bf16, at, at, None, rows, d, n_classes, 1.0, at, g, d, g, g, at, size, None)
    return [size, rc, lib.gnntrain_last_error(None).decode() if rc else "", rt.host_launches()]


def _save8_sizes(rt, variant, dims, bf16, need_input_grad, n):
    """Workspace of a stage without save_8bit and with."""
    from test_host_launches import _Stage

    from paper_2308_10087_amd import binding
    real, seen = binding.lib, []

    class Listening:
        def __getattr__(self, name):
            if name == "gnnstage_workspace_size":
                return lambda d: (seen.append(d._obj), real.gnnstage_workspace_size(d))[1]
            return getattr(real, name)

    binding.lib = Listening()
    stage = _Stage(variant, dims, 4, n=n, bf16=bool(bf16))
    binding.lib = real
    d = seen[0]
    d.need_input_grad = need_input_grad
    sizes = []
    for d.save_8bit in (0, 1):
        sizes.append(real.gnnstage_workspace_size(C.byref(d)))
    return sizes


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


def test_the_largest_weight_gradients_can_be_launched(runtime):
    cases = [(rows, d, d_out, bf16) for rows, d, d_out in [(100, 65536, 16382), (100, 16382, 65536), (5, 32767, 32764), (1 << 31, 65536, 1), (3, 1, 65536)] for bf16 in (0, 1)]
    for c, (size, rc, why, launches) in zip(cases, _child(runtime, "_each", "_weight_grad", cases)):
        assert size > 0 and rc == 0 and launches > 0, (c, why)


def test_larger_weight_gradients_are_refused_before_anything_runs(runtime):
    cases = [(rows, d, d_out, bf16) for rows, d, d_out in [(100, 65536, 16385), (100, 65536, 16383), (100, 16385, 65536), (1, 65536, 65536)] for bf16 in (0, 1)]
    for c, (size, rc, why, launches) in zip(cases, _child(runtime, "_each", "_weight_grad", cases)):
        assert size == 0 and rc == -1 and "2^30" in why and launches == 0, (c, size, rc, why)


def test_heads_at_their_limits_can_be_launched(runtime):
    """Every launch is one that the runtime takes: the widest rows, the most classes, the most weights, several slabs, few rows."""
    cases = [c + (bf16, grads) for c in [(1, 1, 1), (1, 65534, 131072), (1, 512, 1 << 24), (300, 512, 1 << 24), (5000, 8, 1 << 24), (2200001, 256, 47), (2200001, 300, 47),
                                         (140000, 65534, 2), (140000, 1, 200000), (4096, 65534, 8192), (4097, 40000, 8192), (1 << 21, 1, 1)]
             for bf16 in (0, 1) for grads in (0, 1)]
    for c, (size, rc, why, launches) in zip(cases, _child(runtime, "_each", "_head", cases)):
        assert size > 0 and rc == 0 and launches > 0, (c, why)


@pytest.mark.parametrize("n,d_top,n_classes", [(232965, 256, 41), (169343, 128, 40), (700001, 128, 47), (46657, 256, 10007), (46657, 64, 16)])
def test_a_loop_without_logits_needs_no_more_memory(runtime, n, d_top, n_classes):
    """bf16 levels of a width that is read in place: the head without logits in the place of the one that keeps them, from 16 classes on."""
    fused = _child(runtime, "_trainer", d_top, n_classes, True, 1, n)
    kept = _child(runtime, "_trainer", d_top, n_classes, True, 0, n)
    assert fused[2] == kept[2] == 0 and 0 < fused[0] <= kept[0], (fused[0], kept[0])


def test_saved_rows_in_8_bits_never_take_more_room(runtime):
    """Layers that aggregate first are as wide as their input at most where they write, so the backward pass has rows for an aggregation to borrow, also without a
    gradient of the input."""
    cases = [(v, dims, bf16, grad, 4000) for v, dims in [("gcn", [128, 128]), ("gcn", [256, 256]), ("gcn", [100, 256, 46]), ("gcn", [34, 64, 64]), ("sage", [128, 128]),
                                                         ("sage", [64, 100, 100]), ("resgcn", [64, 64, 64])] for bf16 in (0, 1) for grad in (0, 1)]
    for c, (plain, small) in zip(cases, _child(runtime, "_each", "_save8_sizes", cases)):
        assert 0 < small < plain, (c, plain, small)
