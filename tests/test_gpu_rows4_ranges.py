"""Products of rows in 4 bits whose blocks differ by many powers of two, to the ends of the factors' range.

u = 2^-24, v = 2^-8.  What is multiplied are the stored values (products of two codes and a power of two, exact however small or large); an fp32 sum of d products and a bias, in
any order, is off by at most (d + 2) u times the sum of their magnitudes, and where a sum comes below 2^-126 each of its d + 1 additions may lose that much more (whether fp32
numbers below 2^-126 are kept or are zero).  Sums that stay below 2^128 whatever their order, magnitudes together below 2^127, are finite."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import rows4_formula as formula

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, V, TINY = 2.0 ** -24, 2.0 ** -8, 2.0 ** -126


def _g():
    import paper_2308_10087_amd as g
    return g


def _store(x):
    """fp32 numpy rows, stored; and what is stored"""
    g = _g()
    rows, d = x.shape
    wide = -(-d // 32)
    q, s = torch.empty(rows, 16 * wide, dtype=torch.uint8, device=DEV), torch.empty(rows, wide, dtype=torch.uint8, device=DEV)
    g.gnnstage_rows4_store(torch.from_numpy(x).to(DEV), q, s)
    want_q, want_s = formula.encode(x.astype(np.float64))
    assert np.array_equal(s.cpu().numpy(), want_s) and np.array_equal(q.cpu().numpy(), want_q)
    return q, s, formula.decode(want_q, want_s, d)


def _blocks(rng, rows, d, lo, hi):
    """Normal numbers times a power of two of lo .. hi per block of 32 columns"""
    wide = -(-d // 32)
    power = np.repeat(rng.integers(lo, hi + 1, size=(rows, wide)), 32, axis=1)[:, :d]
    with np.errstate(over="ignore"):
        x = np.ldexp(np.clip(rng.normal(size=(rows, d)), -3, 3), power)
    return np.clip(x, -3.4e38, 3.4e38).astype(np.float32)


def _product(a, b, bias, out_dtype=torch.float32):
    g = _g()
    (qa, sa, A), (qb, sb, B) = a, b
    out = torch.empty(A.shape[0], B.shape[0], dtype=out_dtype, device=DEV)
    g.gnnstage_rows4_product(qa, sa, qb, sb, A.shape[1], out, bias=None if bias is None else torch.from_numpy(bias).to(DEV))
    return out.double().cpu().numpy()


def _check(a, b, bias=None, out_dtype=torch.float32):
    A, B = a[2], b[2]
    d = A.shape[1]
    got = _product(a, b, bias, out_dtype)
    beta = 0.0 if bias is None else bias.astype(np.float64)
    want, size = A @ B.T + beta, np.abs(A) @ np.abs(B).T + np.abs(beta)
    fine = size < 2.0 ** 127
    half = V if out_dtype == torch.bfloat16 else U
    bound = (d + 2) * U * size + (d + 1) * TINY
    off = np.abs(got - want)
    assert np.all(np.isfinite(got[fine]))
    assert np.all((off <= bound * (1 + half) + half * np.abs(want) + TINY)[fine]), (float((off / np.maximum(bound, 1e-300))[fine].max()), np.argwhere(fine & (off > bound))[:4])
    return got, want, size


SHAPES = [(33, 129, 64), (65, 300, 256), (5, 1000, 100), (40, 90, 602)]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("M,N,d", SHAPES)
def test_blocks_far_apart(M, N, d, out_dtype):
    rng = np.random.default_rng(M + d)
    _check(_store(_blocks(rng, M, d, -20, 20)), _store(_blocks(rng, N, d, -20, 20)), rng.normal(size=N).astype(np.float32), out_dtype)


@pytest.mark.parametrize("M,N,d", [(33, 129, 96), (40, 90, 288)])
def test_large_parts_that_cancel(M, N, d):
    """Of three parts the first and the last are the same and 2^18 times the one between, against others that differ in sign: it alone is left."""
    rng = np.random.default_rng(d)
    third = d // 3
    a, b = _blocks(rng, M, d, 0, 0), _blocks(rng, N, d, 0, 0)
    a[:, :third] *= 2.0 ** 18
    a[:, 2 * third:] = a[:, :third]
    b[:, 2 * third:] = -b[:, :third]
    _, want, size = _check(_store(a), _store(b))
    assert np.median(np.abs(want) / size) < 2.0 ** -14


@pytest.mark.parametrize("M,N,d", SHAPES)
def test_factors_at_both_ends(M, N, d):
    """2^-120 .. 2^-100 against 2^100 .. 2^120: products of ordinary size."""
    rng = np.random.default_rng(M + d + 1)
    a, b = _store(_blocks(rng, M, d, -117, -100)), _store(_blocks(rng, N, d, 100, 120))
    assert int(a[1].min()) <= 127 - 110 and int(b[1].max()) >= 127 + 110
    _check(a, b)
    _check(b, a)


@pytest.mark.parametrize("low", [-118, -75, -64])
def test_products_below_the_least_number(low):
    rng = np.random.default_rng(-low)
    a, b = _store(_blocks(rng, 40, 160, low, -60)), _store(_blocks(rng, 130, 160, low, -60))
    got, want, _ = _check(a, b)
    assert (np.abs(want) < TINY).any() and np.all(np.abs(got) <= np.abs(want).max() * 2 + 200 * TINY)
    # the bias is there whatever the products are
    bias = rng.normal(size=130).astype(np.float32)
    got, _, _ = _check(a, b, bias)
    assert np.array_equal(got, np.broadcast_to(bias.astype(np.float64), got.shape))


def test_products_beyond_the_largest_number():
    """Sums of one sign beyond it are infinite, below it they are what they are; of both signs they are not finite or within the bound of the others (not told apart)."""
    rng = np.random.default_rng(9)
    a, b = np.abs(_blocks(rng, 40, 96, 50, 68)), np.abs(_blocks(rng, 70, 96, 50, 68))
    got, want, size = _check(_store(a), _store(b))
    beyond = want >= 2.0 ** 128 * (1 + 100 * U)
    assert beyond.any() and (size < 2.0 ** 127).any()
    assert np.all(got[beyond] == np.inf)
    _check(_store(_blocks(rng, 40, 96, 50, 68)), _store(_blocks(rng, 70, 96, 50, 68)))
    _check(_store(_blocks(rng, 40, 96, 100, 126)), _store(_blocks(rng, 70, 96, 100, 126)))


def test_large_finite_rows():
    """To the type's largest number: a block's largest value is 7 factors at most, or the factor is 2^125 and 6 of them is the largest that is kept."""
    g = _g()
    rng = np.random.default_rng(4)
    x = (rng.uniform(-1, 1, size=(6, 96)) * 3.4028234663852886e38).astype(np.float32)
    x[0, 5] = np.finfo(np.float32).max
    x[1, 40] = -np.finfo(np.float32).max
    x[2] *= np.float32(2.0 ** -7)
    assert np.all(np.isfinite(x))
    q, s, want = _store(x)
    assert int(s.max()) == 125 + 127
    back = torch.empty(6, 96, device=DEV)
    g.gnnstage_rows4_load(q, s, back)
    assert np.array_equal(back.double().cpu().numpy(), want)
    _check((q, s, want), _store(_blocks(rng, 30, 96, -40, -20)))
