"""What gnntrain_logprobs and its gradient refuse (before the first launch), their workspaces, and the formula's gradient against differences.  No GPU."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest
import torch

import logprobs_formula as formula
import paper_2308_10087_amd as g
from paper_2308_10087_amd.binding import lib

BUF = (C.c_char * 8192)()
AT = (C.addressof(BUF) + 255) // 256 * 256  # never read


def _answer(logits=AT, dtype=0, ld=10, bias=None, ids=AT, mask=None, rows=5, n_classes=10, n_top=3, logp=AT, entropy=AT, norm=AT, top_ids=AT, top_logp=AT, ws=AT, size=1 << 40):
    return lib.gnntrain_logprobs(logits, dtype, ld, bias, ids, mask, rows, n_classes, n_top, logp, entropy, norm, top_ids, top_logp, ws, size, None)


def _grad(logits=AT, dtype=0, ld=10, bias=None, ids=AT, mask=None, rows=5, n_classes=10, logp=AT, entropy=AT, norm=AT, g_logp=AT, g_entropy=AT, dlogits=AT + 4096,
          dl_dtype=0, ld_dl=10, dbias=None, ws=AT, size=1 << 40):
    return lib.gnntrain_logprobs_grad(logits, dtype, ld, bias, ids, mask, rows, n_classes, logp, entropy, norm, g_logp, g_entropy, dlogits, dl_dtype, ld_dl, dbias, ws, size, None)


SHARED = [(dict(rows=-1), -1), (dict(rows=1 << 41), -1), (dict(n_classes=0), -1), (dict(n_classes=(1 << 24) + 1, ld=1 << 25), -1), (dict(dtype=2), -1), (dict(ld=9), -1),
          (dict(logits=None), -1), (dict(logits=AT + 2), -1), (dict(logits=AT + 1, dtype=1), -1), (dict(ws=None), -1), (dict(ws=AT + 16), -1), (dict(size=255), -4)]


@pytest.mark.parametrize("bad,code", SHARED + [(dict(n_top=-1), -1), (dict(n_top=11), -1), (dict(n_top=65, n_classes=100, ld=100), -1), (dict(top_ids=None), -1),
                                               (dict(top_logp=None), -1), (dict(ids=None), -1)])
def test_answer_refuses(bad, code):
    assert _answer(**bad) == code
    assert "gnntrain_logprobs: " in lib.gnntrain_last_error(None).decode()


@pytest.mark.parametrize("bad,code", SHARED + [(dict(dl_dtype=5), -1), (dict(ld_dl=9), -1), (dict(dlogits=None), -1), (dict(norm=None), -1), (dict(ids=None), -1), (dict(logp=None), -1),
                                               (dict(entropy=None), -1), (dict(dlogits=AT + 4098), -1), (dict(dlogits=AT, dl_dtype=1), -1), (dict(dlogits=AT, ld_dl=11), -1)])
def test_gradient_refuses(bad, code):
    assert _grad(**bad) == code
    assert "gnntrain_logprobs_grad: " in lib.gnntrain_last_error(None).decode()


def test_no_rows_are_nothing_to_do():
    assert _answer(rows=0, logits=None, ws=None, size=0) == 0
    assert _grad(rows=0, logits=None, dlogits=None, ws=None, size=0) == 0


def test_workspace_sizes():
    for bad in ((-1, 5, 0), (5, 0, 0), (5, 3, 4), (5, 100, 65)):
        assert lib.gnntrain_logprobs_workspace_size(*bad) == 0
        with pytest.raises(g.GnnStageError):
            g.gnntrain_logprobs_workspace_size(*bad)
    for bad in ((-1, 5), (5, 0), (5, (1 << 24) + 1)):
        assert lib.gnntrain_logprobs_grad_workspace_size(*bad) == 0
    for rows in (0, 1, 7, 300, 511, 512, 100000, 1 << 40):
        for n_classes in (1, 41, 4096, 100003, 1 << 24):
            assert 0 < g.gnntrain_logprobs_workspace_size(rows, n_classes, min(64, n_classes)) < 1 << 20
            assert 0 < g.gnntrain_logprobs_grad_workspace_size(rows, n_classes) <= (1 << 27) + 256


def test_tensors_are_checked_before_anything_else():
    f = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)
    i32, u8 = torch.int32, torch.uint8
    z, b, y, k, r, norm, ws = f(6, 8), f(8), f(6, t=i32), f(6, t=u8), f(6), f(6, 2), f(256, t=u8)
    A = lambda *a, **m: g.gnntrain_logprobs(*a, **m)
    G = lambda *a, **m: g.gnntrain_logprobs_grad(*a, **m)
    calls = [
        lambda: A(z, b, y, k, r, r, norm, ws),  # on the CPU
        lambda: A(z.double(), b, y, k, r, r, norm, ws), lambda: A(f(8, 6).t(), b, y, k, r, r, norm, ws), lambda: A(f(1, 8).expand(6, 8), b, y, k, r, r, norm, ws),
        lambda: A(z, f(7), y, k, r, r, norm, ws), lambda: A(z, b, y.long(), k, r, r, norm, ws), lambda: A(z, b, y, k.bool(), r, r, norm, ws),
        lambda: A(z, b, y, k, f(5), r, norm, ws), lambda: A(z, b, y, k, r, r.bfloat16(), norm, ws), lambda: A(z, b, y, k, r, r, f(2, 6), ws),
        lambda: A(z, b, y, k, r, r, norm, ws.float()), lambda: A(z, b, y, k, r, r, norm, ws, top_ids=f(6, 2, t=i32)), lambda: A(z, b, y, k, r, r, norm, ws, top_logp=f(6, 2)),
        lambda: A(z, b, y, k, r, r, norm, ws, top_ids=f(6, 2, t=torch.int64), top_logp=f(6, 2)), lambda: A(z, b, y, k, r, r, norm, ws, top_ids=f(6, 2, t=i32), top_logp=f(6, 3)),
        lambda: G(z, b, y, k, r, r, norm, r, r, f(6, 8), ws),  # on the CPU
        lambda: G(z, b, y, k, r, r, norm, r, r, f(6, 9), ws), lambda: G(z, b, y, k, r, r, norm, r, r, f(6, 8).half(), ws), lambda: G(z, b, y, k, r, r, norm, f(5), r, f(6, 8), ws),
        lambda: G(z, b, y, k, r, r, f(6), r, r, f(6, 8), ws), lambda: G(z, b, y, k, r, r, norm, r, r, f(6, 8), ws, dbias=f(8).bfloat16()),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(g.GnnStageError) as e:
            call()
        assert e.value.code == -1, i


@pytest.mark.parametrize("C", [2, 5, 41])
def test_the_formulas_gradient_is_the_differences(C):
    """Central differences with a step of 1e-5: off by a third derivative times 1e-10 / 6 (at most 10 here) and 1e-16 / 1e-5 of rounding."""
    rng = np.random.default_rng(C)
    z, ids = 3 * rng.normal(size=(6, C)), rng.integers(0, C, 6)
    z[4] = 0
    z[5, 0] += 12
    gl, gh = rng.normal(size=6), rng.normal(size=6)
    ids[3] = -1
    w = formula.answer(z, ids)
    got = formula.gradient(z, ids, w["M"], w["log_s"], w["logp"], w["entropy"], gl, gh)[0]
    for c in range(C):
        f = []
        for step in (1e-5, -1e-5):
            moved = z.copy()
            moved[:, c] += step
            v = formula.answer(moved, ids)
            f.append(v["logp"] * gl + v["entropy"] * gh)
        assert np.all(np.abs((f[0] - f[1]) / 2e-5 - got[:, c]) < 1e-8)
