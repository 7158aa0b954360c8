"""What the AdamW step launches, on a CPU: over host_adamw_launches.c, which lists kernel launches with their arguments instead of running them (no buffer is
touched, so tensors of any size take no memory)."""
import ctypes as C
import json
import os
import subprocess
import sys

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = (1 << 24) - 1  # workgroups of 256 that a launch may have
GAMMA, MASK = 0x9E3779B97F4A7C15, (1 << 64) - 1


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "libhostadamw.so")
    subprocess.run(["cc", "-O1", "-shared", "-fPIC", os.path.join(HERE, "host_adamw_launches.c"), "-o", so], check=True)
    return so


# what a launch's arguments hold (csrc/adamw.hip: Tensor, Args)
TENSOR = np.dtype([("p", "u8"), ("g", "u8"), ("m", "u8"), ("v", "u8"), ("m_scale", "u8"), ("v_scale", "u8"), ("compute", "u8"), ("n", "i8"), ("key", "u8"), ("keep", "f4"),
                   ("g_bf16", "i1"), ("compute_bf16", "i1"), ("unused", "i1", 2)])
ARGS = np.dtype([("t", TENSOR, 40), ("first", "i4", 40)])


def _child(rt, counts, bits):
    """Return code, and per launch its workgroups and (p, n, key, first workgroup) of the tensors that some of them work on."""
    from paper_2308_10087_amd.binding import gnntrain_adamw_tensor, lib
    a, at = (gnntrain_adamw_tensor * len(counts))(), 1 << 40
    places = []
    for i, n in enumerate(counts):
        places.append(at)
        for name, size in (("p", 4), ("g", 2), ("m", bits // 8), ("v", bits // 8), ("m_scale", 1), ("v_scale", 1)):
            setattr(a[i], name, at)
            at += (size * n + 256) // 256 * 256
        a[i].g_dtype, a[i].count = 1, n
    rc = lib.gnntrain_adamw_step(a, len(counts), bits, 1e-3, 0.9, 0.999, 1e-8, None, 3, 7, None)
    launches = []
    for i in range(rt.adamw_launches()):
        raw = C.string_at(rt.adamw_args(i), 4096)
        x = np.frombuffer(raw, ARGS, 1)[0]
        blocks, threads = np.frombuffer(raw, "u4", 2, 4080).tolist()
        launches.append([blocks, threads, [[int(t["p"]), int(t["n"]), int(t["key"]), int(f)] for t, f in zip(x["t"], x["first"]) if f < blocks]])
    return [rc, places, launches]


if __name__ == "__main__":
    _rt = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)  # before the library, whose calls it takes
    _rt.adamw_launches.restype = C.c_size_t
    _rt.adamw_args.restype, _rt.adamw_args.argtypes = C.c_void_p, [C.c_size_t]
    sys.path.insert(0, os.path.dirname(HERE))
    print(json.dumps(_child(_rt, *json.loads(sys.argv[2]))))
    sys.stdout.flush()
    os._exit(0)


def _output(z):
    z &= MASK
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & MASK
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & MASK
    return z ^ (z >> 31)


LIMIT = MOST * 1024  # elements that a launch's workgroups take of 8-bit states


@pytest.mark.parametrize("bits,counts", [(8, [LIMIT - 1024]), (8, [LIMIT]), (8, [LIMIT + 1]), (8, [1 << 35]), (8, [100, LIMIT + 5, 70]), (8, [1 << 35, 1000, (1 << 34) + 7]),
                                         (32, [1 << 35]), (32, [5, 1 << 35, 1 << 35, 9]), (8, [0, 33, 0] * 50), (32, [1 << 20] * 45)],
                         ids=lambda x: str(x) if isinstance(x, int) else f"{len(x)} of {max(x)}")
def test_every_element_is_stepped_once_by_launches_that_the_runtime_takes(runtime, bits, counts):
    """Counts go up to 2^35; a launch has fewer than 2^32 threads.  A tensor that needs more goes on in the next one, with its own key and its elements' own numbers."""
    r = subprocess.run([sys.executable, os.path.abspath(__file__), runtime, json.dumps([counts, bits])], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    rc, places, launches = json.loads(r.stdout.splitlines()[-1])
    assert rc == 0
    per = 4096 if bits == 32 and sum(counts) >= 1 << 21 else 1024
    base = _output(7 + 3 * GAMMA)
    reached = {}  # by the place of p: workgroups so far
    for blocks, threads, tensors in launches:
        assert threads == 256 and 0 < blocks <= MOST
        firsts = [t[3] for t in tensors]
        assert firsts == sorted(firsts) and firsts[0] <= 0
        for (p, n, key, first), end in zip(tensors, firsts[1:] + [blocks]):
            i = places.index(p) if p not in reached else reached[p][0]
            assert n == counts[i] and key == _output(base + (i + 1) * GAMMA)
            begin = max(first, 0) - first  # the tensor's workgroup that this launch begins with
            assert begin == (reached[p][1] if p in reached else 0)
            reached[p] = (i, end - first)
    assert sorted((i, b) for i, b in reached.values()) == [(i, (n + per - 1) // per) for i, n in enumerate(counts) if n]
