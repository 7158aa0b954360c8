"""What the AdamW step refuses (every refusal comes before the first launch), and what states in 8 bits keep, by their formula alone.  No GPU."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest
import torch

import adamw_formula as formula
import paper_2308_10087_amd as g
from paper_2308_10087_amd.binding import gnntrain_adamw_tensor, lib

BUF = (C.c_char * (1 << 16))()
AT = (C.addressof(BUF) + 255) // 256 * 256  # never read


def _tensor(k=0, **more):
    t = gnntrain_adamw_tensor()
    values = dict(p=AT + 8192 * k, g=AT + 8192 * k + 1000, m=AT + 8192 * k + 2000, v=AT + 8192 * k + 3000, m_scale=AT + 8192 * k + 4096,
                  v_scale=AT + 8192 * k + 4200, compute=None, count=100, g_dtype=0, compute_dtype=0, weight_decay=0.1)
    values.update(more)
    for name, x in values.items():
        setattr(t, name, x)
    return t


def _step(*tensors, bits=8, b1=0.9, b2=0.999, t=1, n=None):
    a = (gnntrain_adamw_tensor * max(len(tensors), 1))(*tensors)
    return lib.gnntrain_adamw_step(a, len(tensors) if n is None else n, bits, 1e-3, b1, b2, 1e-8, None, t, 0, None)


ONE = [dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(count=-1), dict(count=(1 << 35) + 1), dict(g_dtype=2), dict(compute=AT + 5000, compute_dtype=3),
       dict(m_scale=None), dict(v_scale=None), dict(p=AT + 2), dict(g=AT + 1001), dict(m=AT + 2001), dict(compute=AT + 5001, compute_dtype=1),
       dict(p=AT + 1000), dict(p=AT + 996), dict(m=AT + 396), dict(v=AT + 2100 - 4), dict(compute=AT, compute_dtype=1), dict(compute=AT + 4, compute_dtype=0),
       dict(m_scale=AT + 4200), dict(m_scale=AT + 4197), dict(v=AT + 2000)]


@pytest.mark.parametrize("bad", ONE)
def test_step_refuses_a_tensor(bad):
    for list_ in ((_tensor(**bad),), (_tensor(1), _tensor(**bad))):
        assert _step(*list_) == -1
        assert "gnntrain_adamw_step: " in lib.gnntrain_last_error(None).decode()


def test_step_refuses_other_arguments():
    for bad in (dict(bits=16), dict(bits=0), dict(b1=1.0), dict(b2=1.0), dict(b1=-0.1), dict(b2=float("nan")), dict(t=0), dict(t=-3), dict(n=-1)):
        assert _step(_tensor(), **bad) == -1, bad
    assert lib.gnntrain_adamw_step(None, 1, 8, 1e-3, 0.9, 0.999, 1e-8, None, 1, 0, None) == -1
    assert _step(_tensor(), _tensor()) == -1  # the same tensor twice
    assert "overlaps" in lib.gnntrain_last_error(None).decode()
    assert _step(_tensor(), _tensor(1, g=AT + 8)) == -1  # another one's gradients are what a step writes
    assert _step(_tensor(1, compute=AT + 20000, compute_dtype=1), _tensor(m=AT + 20000 + 196)) == -1


def test_nothing_to_do():
    assert _step(n=0) == 0
    assert _step(_tensor(count=0, p=None, g=None, m=None)) == 0
    assert g.gnntrain_adamw_step(g.gnntrain_adamw_tensors([]), 1e-3, 0.9, 0.999, 1e-8, 1) is None


def test_tensors_are_checked_before_anything_else():
    f = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)
    u8 = torch.uint8
    good = dict(p=f(40), g=f(40), m=f(40), v=f(40))
    eight = dict(p=f(40), g=f(40), m=f(40, t=u8), v=f(40, t=u8), m_scale=f(2, t=u8), v_scale=f(2, t=u8))
    g.gnntrain_adamw_tensors([good, {**good, "g": f(40, t=torch.bfloat16), "compute": f(40, t=torch.bfloat16), "weight_decay": 0.1}])
    g.gnntrain_adamw_tensors([eight])
    bad = [{**good, "g": f(39)}, {**good, "p": f(40).double()}, {**good, "g": f(40).half()}, {**good, "m": f(40).bfloat16()}, {**good, "v": f(40, t=u8)},
           {**good, "compute": f(40).half()}, {**good, "p": f(80)[::2]}, {**good, "decay": 0.1}, {"p": f(40), "g": f(40), "m": f(40)},
           {**eight, "m_scale": f(1, t=u8)}, {**eight, "v_scale": None}, {**eight, "v_scale": f(2)}]
    for i, x in enumerate(bad):
        with pytest.raises(g.GnnStageError):
            g.gnntrain_adamw_tensors([x])
    with pytest.raises(g.GnnStageError):
        g.gnntrain_adamw_tensors([good, eight])
    with pytest.raises(g.GnnStageError):  # on the CPU
        g.gnntrain_adamw_step(g.gnntrain_adamw_tensors([good]), 1e-3, 0.9, 0.999, 1e-8, 1)


def test_codes_are_mxfp8():
    """decode() agrees with torch's e4m3 for every code that is stored."""
    code = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(code).view(torch.float8_e4m3fn).double().numpy()
    got = formula.decode(code, np.full(8, 127, np.uint8))
    assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(want[~np.isnan(want)], got[~np.isnan(want)])


def test_a_stored_value_is_a_neighbour_and_its_mean_is_kept():
    """Over 512 draws of a value between neighbours a distance s apart the mean is off by at most s / 2 / sqrt(512) as a standard deviation, plus
    2^-16 s of the draws' steps; six of them."""
    rng = np.random.default_rng(7)
    for positive in (False, True):
        x = (rng.normal(size=4000) * np.exp(3 * rng.normal(size=4000))).astype(np.float32)
        x = np.abs(x) if positive else x
        codes = [formula.encode(x, rng.integers(0, 65536, 4000), positive) for _ in range(512)]
        values = np.stack([formula.decode(*c) for c in codes])
        scale = codes[0][1].astype(np.float64)
        factor = np.repeat(2.0 ** (scale - 127), 32)[:4000]
        y = np.abs(x.astype(np.float64)) / factor
        spacing = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-30))), -6) - 3) * factor
        assert np.all(np.abs(values - x) <= spacing * (1 + 2.0 ** -15))
        assert not positive or np.all(values[:, x > 0] > 0)
        small = positive & (y < 2.0 ** -9)  # kept above zero: not the mean
        off = np.abs(values.mean(0) - x)[~small]
        assert np.all(off <= spacing[~small] * (6 * 0.5 / np.sqrt(512) + 2.0 ** -15))


def test_a_mean_of_a_thousand_steps_follows():
    """v under a constant gradient from a hundredth of its square: nearest rounding would never move it (a step is 2^-10 of the distance), the
    draws let it arrive.  After 8,000 steps 1 - e^-8 of the way is made; the draws' noise in a root is below a quarter (a step adds
    at most (1/8)^2 2^-10 / 2 of relative variance, which decays at 2^-10 a step: 0.09 of deviation), 32 of them average it."""
    g0, n = 0.01, 32
    rng = np.random.default_rng(3)
    code, scale = formula.encode(np.full(n, 0.1 * g0, np.float32), np.full(n, 0), True)
    for _ in range(8000):
        r = formula.decode(code, scale).astype(np.float32)
        root = formula.means_32(np.full(n, g0, np.float32), np.zeros(n), r * r, 0.9, 0.999)[1]
        code, scale = formula.encode(root, rng.integers(0, 65536, n), True)
    assert abs(np.sqrt((formula.decode(code, scale) ** 2).mean()) / g0 - 1) < 0.15
