"""What rows in 4 bits refuse (before the first launch), and their formula.  No GPU."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest
import torch

import paper_2308_10087_amd as g
import rows4_formula as formula
from paper_2308_10087_amd.binding import lib

BUF = (C.c_char * 8192)()
AT = (C.addressof(BUF) + 255) // 256 * 256  # never read


def _store(x=AT, dtype=1, ld_x=100, rows=10, d=100, q=AT, ld_q=64, scale=AT, ld_s=4):
    return lib.gnnstage_rows4_store(x, dtype, ld_x, rows, d, q, ld_q, scale, ld_s, None)


def _columns(x=AT, dtype=1, ld_x=100, rows=10, d=100, q=AT, ld_q=64, scale=AT, ld_s=4):
    return lib.gnnstage_rows4_store_columns(x, dtype, 9 if ld_x < 100 else ld_x, rows, d, q, ld_q, scale, ld_s, None)


def _load(q=AT, ld_q=64, scale=AT, ld_s=4, rows=10, d=100, x=AT, dtype=1, ld_x=100):
    return lib.gnnstage_rows4_load(q, ld_q, scale, ld_s, rows, d, x, dtype, ld_x, None)


def _product(q=AT, ld_q=64, scale=AT, ld_s=4, rows=10, other_q=AT, ld_oq=64, other_scale=AT, ld_os=4, others=7, d=100, bias=None, x=AT, dtype=1, ld_out=7):
    return lib.gnnstage_rows4_product(q, ld_q, scale, ld_s, rows, other_q, ld_oq, other_scale, ld_os, others, d, bias, x, dtype, ld_out, None)


SHARED = [dict(dtype=2), dict(rows=-1), dict(rows=1 << 41), dict(d=0), dict(d=65537), dict(q=None), dict(q=AT + 8), dict(ld_q=56), dict(ld_q=48), dict(scale=None), dict(ld_s=3),
          dict(x=None), dict(x=AT + 1)]


@pytest.mark.parametrize("bad", SHARED + [dict(ld_x=99)])
def test_store_and_load_refuse(bad):
    for call in (_store, _columns, _load):
        assert call(**bad) == -1
        assert "gnnstage_rows4_" in lib.gnnstage_last_error(None).decode()


@pytest.mark.parametrize("bad", SHARED + [dict(other_q=None), dict(other_q=AT + 4), dict(other_scale=None), dict(ld_oq=48), dict(ld_os=3), dict(others=-1), dict(others=(1 << 29) + 1, ld_out=1 << 30),
                                          dict(ld_out=6), dict(x=AT + 2, dtype=0)])
def test_product_refuses(bad):
    assert _product(**bad) == -1
    assert "gnnstage_rows4_product: " in lib.gnnstage_last_error(None).decode()


def test_nothing_to_do():
    assert _store(rows=0, x=None, q=None, scale=None) == 0 and _load(rows=0, x=None, q=None, scale=None) == 0 and _columns(rows=0, x=None, q=None, scale=None) == 0
    assert _product(rows=0, q=None, x=None) == 0 and _product(others=0, other_q=None, x=None) == 0


def test_tensors_are_checked_before_anything_else():
    f = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)
    u8 = torch.uint8
    x, q, s = f(6, 40), f(6, 32, t=u8), f(6, 2, t=u8)
    calls = [
        lambda: g.gnnstage_rows4_store(x, q, s), lambda: g.gnnstage_rows4_load(q, s, x), lambda: g.gnnstage_rows4_store_columns(f(40, 6), q, s),  # on the CPU
        lambda: g.gnnstage_rows4_product(q, s, q, s, 40, f(6, 6)),
        lambda: g.gnnstage_rows4_store(x.half(), q, s), lambda: g.gnnstage_rows4_store(x, f(6, 16, t=u8), s), lambda: g.gnnstage_rows4_store(x, q, f(6, 1, t=u8)),
        lambda: g.gnnstage_rows4_store(x, f(6, 32, t=torch.int8), s), lambda: g.gnnstage_rows4_store(f(40, 6).t(), q, s), lambda: g.gnnstage_rows4_store_columns(x, q, s),
        lambda: g.gnnstage_rows4_load(q[:5], s, x), lambda: g.gnnstage_rows4_product(q, s, q, s, 65, f(6, 6)), lambda: g.gnnstage_rows4_product(q, s, q, s, 40, f(6, 5)),
        lambda: g.gnnstage_rows4_product(q, s, q, s, 40, f(6, 6), bias=f(5)), lambda: g.gnnstage_rows4_product(q, s, q, s, 40, f(6, 6), bias=f(6).bfloat16()),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(g.GnnStageError) as e:
            call()
        assert e.value.code == -1, i


def test_the_formula_keeps_the_nearest():
    """A block's factor is at least a seventh of its largest value and below two sevenths of it; a value is off by at most half the distance of its neighbours, a factor at most,
    a quarter of it below twice the factor; what is kept stays as it is."""
    rng = np.random.default_rng(1)
    x = rng.normal(size=(200, 100)) * np.exp(3 * rng.normal(size=(200, 1)))
    q, s = formula.encode(x)
    back, factor = formula.decode(q, s, 100), np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, axis=1)[:, :100]
    for b in range(4):
        part = slice(32 * b, min(100, 32 * b + 32))
        a, f = np.abs(x[:, part]).max(1), factor[:, 32 * b]
        assert np.all(a <= 7 * f) and np.all(a > 3.5 * f)
    assert np.all(np.abs(back - x) <= factor) and np.all(np.abs(back - x)[np.abs(x) <= 2 * factor] <= 0.25 * factor[np.abs(x) <= 2 * factor])
    again = formula.encode(back)
    assert np.array_equal(formula.decode(*again, 100), back)
