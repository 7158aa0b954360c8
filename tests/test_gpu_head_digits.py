"""How many digits the gradients of the loss head without logits (gnntrain_head_xent) have, where its other tests' bounds leave room for fewer.

u = 2^-24 is half a step of fp32 relative to the value, v = 2^-8 of bf16, so v^2 what the sum of two bf16 numbers leaves out."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_head_rows8 import DT, U, V, check_head, counts, head_formula, head_inputs, run_head

pytestmark = pytest.mark.gpu

COARSE = 2.0 ** -5  # a probability up to this share of its row's sum may enter dh as one bf16 number


def leaning(rows, d, C, dtype, seed, common, lean=2.0):
    """Rows that lean towards their class.  Of the columns in which they are zero, which logits do not see, the classes' weights share one ``common`` times as
    large as what tells them apart."""
    rng = np.random.default_rng(seed)
    seen = (d + 1) // 2
    W = rng.normal(size=(d, C)) / np.sqrt(seen)
    y = rng.integers(0, C, size=rows).astype(np.int32)
    h = np.zeros((rows, d))
    h[:, :seen] = np.maximum(rng.normal(size=(rows, seen)) + lean * rng.random((rows, 1)) * W[:seen, y].T * np.sqrt(seen), 0.0)
    W[seen:] += common * rng.normal(size=(d - seen, 1)) / np.sqrt(seen)
    to = lambda x: torch.from_numpy(x.astype(np.float32)).to(DT[dtype])
    return to(h), to(W), (0.1 * rng.normal(size=C)).astype(np.float32), y


def dh_and_bound(h, W, b, y, inv_n, coarse):
    """float64: dh and a bound for it as bf16.  With p the other classes' probabilities, q = p / sum p and t = sum p: dh = inv_n t (sum q W - W_y).
      * the rounding of the result: v |dh|
      * factors p (1 + e) weighted against their own sum: what classes' weights have in common cancels, sum e q |W_c - sum q W| is left.  e is v for q up to
        ``coarse`` and 2 v^2 for the others; and 4 dz for all, dz being how far a logit is off, (d + 3) u of its terms
      * t as a whole: 8 dz and the rounding of a sum of C terms, of dh
      * fp32 sums of C terms, and the difference of t sum q W and t W_y: (C + 64) u of their magnitudes"""
    h, W, b = h.double().numpy(), W.double().numpy(), b.astype(np.float64)
    n, d = h.shape
    C = W.shape[1]
    z = h @ W + b
    z -= z.max(1, keepdims=True)
    p = np.exp(z)
    own = p[np.arange(n), y].copy()
    p[np.arange(n), y] = 0.0
    o = p.sum(1)
    t, q = inv_n * o / (o + own), p / o[:, None]
    mean = q @ W.T
    dh = t[:, None] * (mean - W[:, y].T)
    dz = (d + 3) * U * (np.abs(h) @ np.abs(W) + np.abs(b)).max(1)[:, None]
    e = np.where(q <= coarse, V / (1 - V), 2 * V * V) + 4 * dz
    away = np.empty((n, d))
    for k in range(d):
        away[:, k] = (e * q * np.abs(W[k][None, :] - mean[:, k:k + 1])).sum(1)
    mag = q @ np.abs(W).T + np.abs(W[:, y].T)
    return dh, V * np.abs(dh) + ((8 * dz + (C + 64) * U) * np.abs(dh) + t[:, None] * (away + (C + 64) * U * mag)) * (1 + V)


@pytest.mark.parametrize("rows,d,C,common", [(2000, 256, 41, 0), (2000, 256, 41, 16), (900, 128, 172, 4), (700, 100, 300, 16), (900, 64, 60, 64), (40, 200, 3000, 64),
                                             (300, 256, 2100, 16), (517, 33, 5000, 16), (9001, 250, 41, 16), (1, 64, 2, 16)])
def test_input_gradients_to_the_rounding_of_their_type(rows, d, C, common):
    """bf16 rows of up to 256 columns: dh is as good as its type, also where all classes' weights have most in common and cancel."""
    h, W, b, y = leaning(rows, d, C, "bf16", rows + d + C, common)
    want, bound = dh_and_bound(h, W, b, y, 1.0 / 64, COARSE)
    got = run_head(h, W, b, y, None, 1.0 / 64, "bf16")["dh"]
    off = np.abs(got - want)
    assert np.all(off <= bound), (float((off / bound).max()), float(np.linalg.norm(off) / np.linalg.norm(want)))


def test_probabilities_that_all_round_the_same_way():
    """All other classes have the same logit and the label's a larger one: every factor is the same number, and rounds by the same part of itself.  Weighted against
    their own sum nothing of that is left, however coarse the factors."""
    rows, d, C = 200, 64, 2000
    rng = np.random.default_rng(3)
    W = torch.from_numpy((8.0 + 0.5 * rng.integers(-2, 3, size=(d, C))).astype(np.float32)).bfloat16()
    W[0] = 0.0
    W[0, 0] = 1.3
    h = torch.zeros(rows, d, dtype=torch.bfloat16)
    h[:, 0] = torch.from_numpy((1.0 + rng.random(rows)).astype(np.float32))
    b, y = np.zeros(C, np.float32), np.zeros(rows, np.int32)
    want, bound = dh_and_bound(h, W, b, y, 1.0, 0.0)
    got = run_head(h, W, b, y, None, 1.0, "bf16")["dh"]
    off = np.abs(got - want)
    assert np.all(off <= bound), float((off / bound).max())


@pytest.mark.parametrize("rows,d,C,common", [(2000, 500, 41, 0), (2000, 500, 41, 16), (700, 300, 1000, 4), (300, 500, 9001, 0), (37, 264, 9001, 64), (4200, 264, 9001, 4),
                                             (1, 1000, 2, 16)])
def test_input_gradients_of_wide_rows(rows, d, C, common):
    """bf16 rows of more than 256 columns: every g, the label's too, enters dh as the sum of two bf16 numbers, v^2 of it off at most; where classes are many, rows few or
    many, or both in pieces.  Beside that dh_and_bound's errors, of terms as they are: nothing cancels on its own here."""
    h, W, b, y = leaning(rows, d, C, "bf16", rows + d + C, common)
    # logits are made of multiples of 2^-9 below 2^14: every sum of theirs is exact, and what comes after is off by a few roundings of theirs
    h, W[:(d + 1) // 2], b = (h * 8).round() / 8, (W[:(d + 1) // 2] * 64).round() / 64, np.round(b * 64) / 64
    z = h.double().numpy() @ W.double().numpy() + b
    assert np.abs(h.double().numpy()).max() < 32 and float(W[:(d + 1) // 2].abs().max()) < 4 and np.abs(z).max() < 2 ** 12
    inv_n = 1.0 / 64
    want, mag = head_formula(h.double().numpy(), W.double().numpy(), b.astype(np.float64), y, np.ones(rows, bool), inv_n)
    dz = 4 * U * (1 + z.max(1) - z.min(1))[:, None]
    got = run_head(h, W, b, y, None, inv_n, "bf16")["dh"]
    bound = V * np.abs(want["dh"]) + (V * V + 12 * dz + (2 * C + 64) * U) * mag["dh"] * (1 + V)
    off = np.abs(got - want["dh"])
    assert np.all(off <= bound), (float((off / bound).max()), float(np.linalg.norm(off) / np.linalg.norm(want["dh"])))


@pytest.mark.parametrize("rows,d,C", [(500, 64, 8000), (70, 300, 8000), (9001, 256, 6000), (8400, 33, 8300), (300, 64, 20001), (700, 390, 12000), (5, 1000, 4000)])
def test_long_sums_of_fp32_input_gradients(rows, d, C):
    """All logits are equal, so dh is a sum of C - 1 equal terms and the label's: in one chain the additions' roundings go the same way for thousands of terms.  In
    chains of at most 256 that are added up, or in tiles of them, a sum is off by (256 + C / 64 + 64) u; g by a few roundings, its own sum being one of ones."""
    rng = np.random.default_rng(rows)
    w, v = (1.0 + rng.random(d)).astype(np.float32), (-1.0 - rng.random(d)).astype(np.float32)
    W = torch.from_numpy(np.repeat(w[:, None], C, 1))
    W[:, 0] = torch.from_numpy(v)
    y = np.zeros(rows, np.int32)
    got = run_head(torch.zeros(rows, d), W, None, y, None, 1.0 / 64, "f32")
    own = (C - 1) / C / 64
    want = own * (w.astype(np.float64) - v)
    mag = own * (w.astype(np.float64) + np.abs(v))
    off = np.abs(got["dh"] - want).max(0)
    bound = (256 + C / 64 + 64) * U * mag
    assert np.all(off <= bound), float((off / bound).max())
    assert np.abs(got["loss"] - np.log(C)).max() <= 8 * U * np.log(C)


def one_hot(rows, d, C, seed, active=8):
    """Rows of one number each in a column of its own, then rows of zeros: an element of dW is one term and zeros.  All classes but ``active`` are left out.  Logits are
    multiples of 2^-13 within -3 and 3: exact."""
    rng = np.random.default_rng(seed)
    at = np.sort(rng.choice(C, active, replace=False))
    h = np.zeros((rows, d), np.float32)
    k = min(rows, d)
    h[np.arange(k), np.arange(k)] = 1.0 + rng.integers(0, 128, size=k) / 128
    W = rng.integers(-64, 65, size=(d, C)) / 64
    b = np.full(C, -np.inf, np.float32)
    b[at] = rng.integers(-16, 17, size=active) / 16
    y = at[rng.integers(0, active, size=rows)].astype(np.int32)
    return torch.from_numpy(h).bfloat16(), torch.from_numpy(W.astype(np.float32)).bfloat16(), b, y, at


@pytest.mark.parametrize("rows,d,C", [(1, 64, 8), (300, 256, 8), (300, 100, 40), (129, 128, 70), (16384, 200, 64), (17000, 256, 200), (20000, 128, 300), (20000, 40, 1000),
                                      (60000, 100, 1000), (300, 300, 40), (17000, 300, 200)])
def test_weight_gradients_have_all_bits_where_a_class_has_few_rows(rows, d, C):
    """Every element of dW is h_ik g_ic inv_n with h and inv_n short numbers, so it is as good as g, and g's of a row's own class are large: all bits.  g is off by its
    exponent, 12 at most, whose last digit is 16 u: 2 * 16 u ln 2 for it and its part log2 of the sum; by its sum of 8 terms, 8 u; by two functions, 8 u: 40 u."""
    h, W, b, y, at = one_hot(rows, d, C, rows + d + C)
    want, _ = head_formula(h.double().numpy(), W.double().numpy(), b.astype(np.float64), y, np.ones(rows, bool), 1.0 / 64)
    got = run_head(h, W, b, y, None, 1.0 / 64, "bf16", grads=("dW", "db"))["dW"]
    k = np.arange(min(rows, d))
    own = (k, y[k])
    off = np.abs(got / np.where(want["dW"] == 0, 1.0, want["dW"]) - (want["dW"] != 0))
    assert off[own].max() <= 40 * U, float(off[own].max() / U)
    assert off[k].max() <= 40 * U + V * V
    assert np.all(got[want["dW"] == 0] == 0)


@pytest.mark.parametrize("rows,d,C", [(33, 128, 8200), (257, 64, 20011), (1, 256, 50021), (700, 250, 9001), (90, 300, 9001), (17500, 100, 8300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norms_over_many_classes(rows, d, C, dtype):
    """A sum of C roundings of random signs is 4 sqrt(C) u off at most (four of its standard deviations); g to 16 bits 2^-16; logits of d terms 4 sqrt(d) u of
    their magnitudes, which is what g is off by.  As norms: what only the worst case of every rounding allows does not pass here."""
    h, W, b, y, mask = head_inputs(rows, d, C, dtype, rows + C, "some" if rows > 1 else "all")
    on = counts(y, mask, C)
    inv_n = 1.0 / max(1, int(on.sum()))
    want, mag = head_formula(h.double().numpy(), W.double().numpy(), b.astype(np.float64), y, on, inv_n)
    got = run_head(h, W, b, y, mask, inv_n, dtype)
    sums = 4 * np.sqrt(C) * U + 4 * np.sqrt(d) * U * float(mag["z"].max()) + 64 * U
    for key, more in (("loss", 0.0), ("dW", V * V), ("db", V * V), ("dh", V if dtype == "bf16" else 0.0)):
        rel = np.linalg.norm(got[key] - want[key]) / np.linalg.norm(want[key])
        assert rel <= sums + 4 * np.sqrt(max(rows, C)) * U + more, (key, rel)


@pytest.mark.parametrize("d", [256, 200, 128, 64])
def test_weight_gradients_of_classes_with_many_rows(d):
    """More than 16,384 labelled rows and more than 128 a class: two bf16 numbers of every g, of rows as they are and packed."""
    check_head(34000, d, 100, "bf16", "some")


@pytest.mark.parametrize("d,C,pad", [(8, 3, 0), (64, 5, 8)])
def test_more_rows_than_a_slab(d, C, pad):
    """2^20 rows go at a time: weights and biases of the first slab serve the next, whose labels, mask, losses and gradient rows begin further on, and whose sums are
    added to the first one's.  Labelled rows on both sides of the border."""
    rows = (1 << 20) + 129

    def edit(h, W, b, y, mask):
        mask[(1 << 20) - 3:(1 << 20) + 5] = 1
        y[(1 << 20) - 3:(1 << 20) + 5] = np.arange(8) % C
        mask[-1], y[-1] = 1, C - 1

    got = check_head(rows, d, C, "bf16", "some", pad=pad, edit=edit)
    border = slice((1 << 20) - 3, (1 << 20) + 5)
    assert np.all(got["loss"][border] > 0) and np.all(np.abs(got["dh"][border]).max(1) > 0) and got["loss"][-1] > 0
