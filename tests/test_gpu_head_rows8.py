"""The loss head without logits (gnntrain_head_xent) and rows kept in 8 bits (gnnstage_rows8_*) against their formulas in 64 bits.

u = 2^-24 is half a step of fp32 relative to the value, v = 2^-8 of bf16.  Bounds are per element and follow the sums: a sum of n products in
fp32, in any order, is off by at most (n + 1) u times the sum of the products' magnitudes."""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, V = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _g():
    import paper_2308_10087_amd as g
    return g


def _code(g, dtype):
    return g.GNNSTAGE_BF16 if dtype == "bf16" else g.GNNSTAGE_F32


# ---- the head ------------------------------------------------------------------------------------------------------
def head_formula(h, W, b, labels, on, inv_n):
    """float64 arrays; on: which rows count.  Loss, dh, dW, db and the sums of magnitudes that bound their errors."""
    n, d = h.shape
    C = W.shape[1]
    loss, dh, dW, db = np.zeros(n), np.zeros((n, d)), np.zeros((d, C)), np.zeros(C)
    at = np.flatnonzero(on)
    h, y = h[at], labels[at]
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        z = h @ W + b
        z = z - z.max(1, keepdims=True)
        e = np.exp(z)
        own = e[np.arange(len(at)), y]
        e[np.arange(len(at)), y] = 0.0
        others = e.sum(1)
        total = others + own
        loss[at] = np.where(own > 0.5 * total, np.log1p(others / own), np.log(total) - z[np.arange(len(at)), y])
        g = e * (inv_n / total)[:, None]
        g[np.arange(len(at)), y] = -inv_n * others / total
        dh[at] = g @ W.T
        dW[:], db[:] = h.T @ g, g.sum(0)
        fine = np.where(np.isfinite(b), b, 0.0)
        mag_z = np.zeros(n)
        mag_z[at] = (np.abs(h) @ np.abs(W) + np.abs(fine)).max(1, initial=0.0)
        mag_dh = np.zeros((n, d))
        mag_dh[at] = np.abs(g) @ np.abs(W).T
    return dict(loss=loss, dh=dh, dW=dW, db=db), dict(z=mag_z, dh=mag_dh, dW=np.abs(h).T @ np.abs(g), db=np.abs(g).sum(0))


def head_bounds(want, mag, d, C, n_on, dtype):
    """logits: d + 1 additions; a loss is the difference of a logarithm of C terms and a logit; a softmax's relative error is the absolute
    one of its exponent (twice: numerator and maximum cancel, the sum has the same) plus C + 16 roundings of sums and functions."""
    dz = (d + 2) * U * mag["z"]
    loss = 2 * dz + (C + 16) * U * (1 + np.abs(want["loss"])) + 16 * U * mag["z"]
    rho = float((2 * (dz + 8 * U * mag["z"])).max(initial=0.0)) + (C + 32) * U
    bf = dtype == "bf16"
    dh = (rho + (C + 2) * U + (V if bf else 0)) * mag["dh"] * (1 + V) + ((V if bf else U) * np.abs(want["dh"]))
    two = V * V if bf else 0.0  # the second of two bf16 numbers is rounded
    dW = (rho + two + (n_on + 4) * U) * mag["dW"]
    db = (rho + two + (n_on + 4) * U) * mag["db"]
    return dict(loss=loss, dh=dh, dW=dW, db=db)


def head_inputs(rows, d, C, dtype, seed, masked, lean=2.0):
    rng = np.random.default_rng(seed)
    W = torch.from_numpy((rng.normal(size=(d, C)) / np.sqrt(d)).astype(np.float32)).to(DT[dtype])
    y = rng.integers(0, C, size=rows).astype(np.int32)
    h = rng.normal(size=(rows, d)) + lean * rng.random((rows, 1)) * W.float().numpy()[:, y].T * np.sqrt(d)
    h = torch.from_numpy(h.astype(np.float32)).to(DT[dtype])
    b = (0.3 * rng.normal(size=C)).astype(np.float32)
    mask = None
    if masked == "none left":
        mask = np.zeros(rows, np.uint8)
    elif masked == "some":
        mask = (rng.random(rows) < 0.5).astype(np.uint8) * rng.integers(1, 256, size=rows).astype(np.uint8)
        y[rng.random(rows) < 0.1] = -1          # labels outside the classes count as none
        y[rng.random(rows) < 0.1] = C
        y[rng.random(rows) < 0.02] = -2147483648
    return h, W, b, y, mask


def run_head(h, W, b, y, mask, inv_n, dtype, grads=("dh", "dW", "db"), pad=0, start=None, workspace=None):
    """Returns numpy float64 outputs; checks what must not be written."""
    g = _g()
    rows, d = h.shape
    C = W.shape[1]
    wide = torch.full((rows + 1, d + pad), 7.0, dtype=DT[dtype], device=DEV)
    wide[:rows, :d] = h.to(DEV)
    dh_wide = torch.full((rows + 2, d + pad), 5.0, dtype=DT[dtype], device=DEV)
    loss = torch.full((rows + 1,), -3.0, device=DEV)
    dW = None if "dW" not in grads else torch.zeros(d, C, device=DEV) if start is None else torch.from_numpy(start[0]).to(DEV)
    db = None if "db" not in grads else torch.zeros(C, device=DEV) if start is None else torch.from_numpy(start[1]).to(DEV)
    if workspace is None:
        size = g.gnntrain_head_xent_workspace_size(rows, d, C, _code(g, dtype), bool(grads))
        workspace = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device=DEV)  # NaNs: nothing in it may be counted on
    size = workspace.numel() - 256
    g.gnntrain_head_xent(wide[:rows, :d], W.to(DEV), None if b is None else torch.from_numpy(b).to(DEV), torch.from_numpy(y).to(DEV),
                         None if mask is None else torch.from_numpy(mask).to(DEV), inv_n, loss[:rows], workspace[:size],
                         dh=dh_wide[:rows, :d] if "dh" in grads else None, dW=dW, db=db)
    torch.cuda.synchronize()
    assert loss[rows].item() == -3.0
    assert bool((workspace[size:] == 0xFF).all())
    assert bool((dh_wide[rows:] == 5.0).all()) and bool((dh_wide[:, d:] == 5.0).all())
    out = {"loss": loss[:rows], "dh": dh_wide[:rows, :d], "dW": dW, "db": db}
    return {k: x.double().cpu().numpy() for k, x in out.items() if x is not None and (k == "loss" or k in grads)}


def counts(y, mask, C):
    return (y >= 0) & (y < C) & (np.ones(len(y), bool) if mask is None else mask != 0)


def check_head(rows, d, C, dtype, masked, pad=0, bias=True, seed=0, edit=None, lean=2.0):
    h, W, b, y, mask = head_inputs(rows, d, C, dtype, 1000 * rows + 10 * d + C + seed, masked, lean)
    if not bias:
        b = None
    if edit:
        edit(h, W, b, y, mask)
    on = counts(y, mask, C)
    inv_n = float(np.float32(1.0 / max(1, on.sum())))
    want, mag = head_formula(h.double().numpy(), W.double().numpy(), np.zeros(C) if b is None else b.astype(np.float64), y, on, inv_n)
    bound = head_bounds(want, mag, d, C, int(on.sum()), dtype)
    got = run_head(h, W, b, y, mask, inv_n, dtype, pad=pad)
    for k in ("loss", "dh", "dW", "db"):
        finite = np.isfinite(want[k])
        assert np.array_equal(np.isnan(want[k]), np.isnan(got[k])), (k, "NaN elsewhere")
        assert np.array_equal(want[k][~finite & ~np.isnan(want[k])], got[k][~finite & ~np.isnan(want[k])]), k
        off = np.abs(got[k][finite] - want[k][finite])
        assert np.all(off <= bound[k][finite] + 1e-30), (k, float(off.max()), float((off - bound[k][finite]).max()))
    assert np.all(got["loss"][~on] == 0) and np.all(got["dh"][~on] == 0)
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", ["all", "some", "none left"])
@pytest.mark.parametrize("rows,d,C", [(1, 1, 1), (1, 8, 2), (2, 3, 3), (7, 33, 5), (33, 16, 31), (64, 64, 33), (130, 100, 100), (65, 17, 257),
                                      (255, 128, 41), (257, 65, 64), (300, 256, 1000), (31, 250, 513), (513, 129, 130), (96, 600, 77)])
def test_head_against_the_formula(rows, d, C, dtype, masked):
    check_head(rows, d, C, dtype, masked, pad=(rows % 3) * (8 if d % 8 == 0 else 1), bias=rows % 2 == 1 or d == 256)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,C", [(33, 128, 8200), (257, 64, 20011), (1, 256, 50021), (20, 520, 9001)])
def test_head_over_many_classes(rows, d, C, dtype):
    check_head(rows, d, C, dtype, "some" if rows > 1 else "all")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,C", [(140001, 16, 3), (70001, 128, 41), (9001, 256, 300)])
def test_head_over_many_rows(rows, d, C, dtype):
    check_head(rows, d, C, dtype, "some", pad=8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_most_classes(dtype):
    """2^24 of them (the formula on the GPU, in 64 bits).  The softmax's sum over 2^24 terms is one of partial sums of 2^17 at most."""
    g = _g()
    rows, d, C = 3, 4, 1 << 24
    gen = torch.Generator(device=DEV).manual_seed(3)
    W = torch.randn(d, C, device=DEV, generator=gen).to(DT[dtype])
    h = torch.randn(rows, d, device=DEV, generator=gen).to(DT[dtype])
    y = torch.tensor([0, C - 1, 12345678], dtype=torch.int32, device=DEV)
    loss, dh = torch.empty(rows, device=DEV), torch.empty_like(h)
    dW, db = torch.zeros(d, C, device=DEV), torch.zeros(C, device=DEV)
    ws = torch.empty(g.gnntrain_head_xent_workspace_size(rows, d, C, _code(g, dtype)), dtype=torch.uint8, device=DEV)
    g.gnntrain_head_xent(h, W, None, y, None, 1.0, loss, ws, dh=dh, dW=dW, db=db)
    z = h.double() @ W.double()
    lse = torch.logsumexp(z, 1, keepdim=True)
    want = (lse - z.gather(1, y.long().unsqueeze(1))).squeeze(1)
    p = torch.exp(z - lse)
    p[torch.arange(rows, device=DEV), y.long()] -= 1.0
    rel = 2 * 2 ** 17 * U  # of the softmax: its sum's, and what the logits' own roundings come to beside that
    assert float((loss.double() - want).abs().max()) <= rel + 1e-5
    assert float((db.double() - p.sum(0)).abs().max()) <= rel + 1e-6
    big = p.abs().sum(0)
    assert bool(((db.double() - p.sum(0)).abs() <= (rel + 8 * U + V * V) * big + 1e-30).all())
    for k in range(d):
        terms = h[:, k].double().unsqueeze(1) * p
        assert bool(((dW[k].double() - terms.sum(0)).abs() <= (rel + 8 * U + V * V) * terms.abs().sum(0) + 1e-30).all())
    dh_mag = p.abs() @ W.double().abs().t().contiguous()
    dh_want = p @ W.double().t().contiguous()
    assert bool(((dh.double() - dh_want).abs() <= (rel + (2 * V if dtype == "bf16" else 0)) * dh_mag + V * dh_want.abs()).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,C", [(3011, 520, 2003), (2900, 397, 2741), (1500, 300, 9001), (1299, 390, 8999), (8400, 392, 8300)])
def test_head_of_wide_rows_over_many_classes(rows, d, C, dtype):
    """Wide products; classes in more than one piece, for the last one of rows in more than one as well."""
    check_head(rows, d, C, dtype, "some", pad=1 if rows == 2900 else 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,C", [(70, 64, 300), (40, 128, 9000)])
def test_masked_rows_may_hold_anything(rows, d, C, dtype):
    def edit(h, W, b, y, mask):
        off = torch.from_numpy(~counts(y, mask, C))
        h[off] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38])[torch.arange(int(off.sum())) % 4].to(h.dtype)[:, None]

    check_head(rows, d, C, dtype, "some", edit=edit)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,C,pad", [(300, 64, 41, 0), (300, 64, 41, 8), (300, 64, 41, 1), (260, 512, 70, 0), (260, 512, 70, 8), (140001, 392, 30, 0), (90, 33, 8200, 7)])
def test_losses_alone_beside_masked_rows_of_anything(rows, d, C, pad, dtype):
    h, W, b, y, mask = head_inputs(rows, d, C, dtype, 17, "some")
    on = counts(y, mask, C)
    h[~torch.from_numpy(on)] = float("nan")
    want, mag = head_formula(h.double().numpy(), W.double().numpy(), b.astype(np.float64), y, on, 1.0)
    got = run_head(h, W, b, y, mask, 1.0, dtype, grads=(), pad=pad)["loss"]
    assert np.all(np.abs(got - want["loss"]) <= head_bounds(want, mag, d, C, int(on.sum()), dtype)["loss"])
    assert np.all(got[~on] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lowest", [-float("inf"), -3.4028234663852886e38])
def test_classes_left_out_by_their_bias(dtype, lowest):
    """Left out first, last, in whole runs longer than any tile; none of the rows' own."""
    def edit(h, W, b, y, mask):
        b[:] = lowest
        b[700:720] = 0.5
        y[:] = 700 + np.arange(len(y)) % 20

    got = check_head(90, 64, 1500, dtype, "all", edit=edit)
    assert np.all(got["dW"][:, :700] == 0) and np.all(got["db"][720:] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [-3.4028234663852886e38, 1e30, -1e9, 3e8])
def test_all_classes_at_a_bias_beyond_every_logit(dtype, bias):
    """All logits are the bias then, a step of fp32 above what products add: the softmax is flat, and a large logit is its own maximum."""
    h, W, b, y, mask = head_inputs(50, 48, 300, dtype, 12, "all")
    got = run_head(h * 2.0 ** -10, W, np.full_like(b, bias), y, mask, 1.0, dtype)
    assert np.abs(got["loss"] - np.log(300.0)).max() <= 1e-5
    assert np.abs(got["db"].sum()) <= 1e-3 and np.isfinite(got["dW"]).all() and np.isfinite(got["dh"]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e3, 1e7, 1e18])
def test_large_logits_stay_numbers(dtype, scale):
    """Logits so large that every row is sure of some class: the loss is the difference of two of them, and the gradient one-hot."""
    h, W, b, y, mask = head_inputs(70, 64, 200, dtype, 13, "all", lean=0.0)
    h, W = (h.float() * scale).to(DT[dtype]), (W.float() * scale).to(DT[dtype])
    got = run_head(h, W, np.zeros_like(b), y, mask, 1.0, dtype)
    z = h.double().numpy() @ W.double().numpy()
    top = z.max(1)
    second = np.sort(z, 1)[:, -2]
    mag = (np.abs(h.double().numpy()) @ np.abs(W.double().numpy())).max(1)
    own = z[np.arange(70), y]
    off = np.abs(got["loss"] - (top - own))
    clear = (top - second) > 40 + 8 * 66 * U * mag  # rows whose largest logit leads in any order of additions
    assert clear.sum() >= 40
    assert np.all(off[clear] <= (2 * 66 * U * mag + U * np.abs(top - own) + 1e-6)[clear])
    assert np.isfinite(got["dh"]).all() and np.isfinite(got["dW"]).all() and np.isfinite(got["db"]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_row_whose_label_is_left_out(dtype):
    def edit(h, W, b, y, mask):
        b[5] = -np.inf
        y[:] = 9
        y[3] = 5

    got = check_head(40, 32, 64, dtype, "all", edit=edit)
    assert np.isposinf(got["loss"][3]) and np.isfinite(np.delete(got["loss"], 3)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", ["all classes out", "nan row", "inf logit"])
def test_rows_without_a_softmax_are_nan(dtype, bad):
    h, W, b, y, mask = head_inputs(40, 32, 70, dtype, 4, "all")
    if bad == "all classes out":
        b[:] = -np.inf
    elif bad == "nan row":
        h[7, 3] = float("nan")
    else:
        b[11] = np.inf
    got = run_head(h, W, b, y, mask, 0.1, dtype)
    hit = [7] if bad == "nan row" else list(range(40))
    assert np.isnan(got["loss"][hit]).all() and np.isnan(got["dh"][hit]).all()
    rest = np.setdiff1d(np.arange(40), hit)
    assert np.isfinite(got["loss"][rest]).all() and np.isfinite(got["dh"][rest]).all()
    assert np.isnan(got["db"]).all() and np.isnan(got["dW"]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_sure_keep_their_digits(dtype):
    """Losses of 1e-9 and gradients to match: what a difference of two numbers near one would lose."""
    n, d, C = 64, 64, 200
    W = torch.zeros(d, C)
    W[torch.arange(d), torch.arange(d)] = 4.0
    h = torch.zeros(n, d)
    h[torch.arange(n), torch.arange(n)] = torch.linspace(2.0, 6.0, n)
    h, W = h.to(DT[dtype]), W.to(DT[dtype])
    y = np.arange(n, dtype=np.int32)
    want, _ = head_formula(h.double().numpy(), W.double().numpy(), np.zeros(C), y, np.ones(n, bool), 1.0)
    got = run_head(h, W, None, y, None, 1.0, dtype)
    assert want["loss"].min() < 1e-8
    # the logits are exact here but for their scaling by log2 e: 24 * 2 u in the exponent, and a few functions
    assert np.abs(got["loss"] / want["loss"] - 1).max() <= (C + 200) * U
    tol = (V * 2 + 1e-4) if dtype == "bf16" else (2 * C + 200) * U
    big = np.abs(want["dh"]) > 0
    assert np.abs(got["dh"][big] / want["dh"][big] - 1).max() <= tol


def test_head_outputs_one_by_one_and_added_to():
    for dtype in ("f32", "bf16"):
        h, W, b, y, mask = head_inputs(150, 96, 333, dtype, 8, "some")
        whole = run_head(h, W, b, y, mask, 0.01, dtype)
        for grads in ((), ("dh",), ("dW",), ("db",), ("dh", "db"), ("dW", "db")):
            part = run_head(h, W, b, y, mask, 0.01, dtype, grads=grads)
            for k in part:
                assert np.abs(part[k] - whole[k]).max() <= 1e-4 * np.abs(whole[k]).max(), (k, grads)
        start = (np.random.default_rng(1).normal(size=(96, 333)).astype(np.float32), np.arange(333, dtype=np.float32))
        more = run_head(h, W, b, y, mask, 0.01, dtype, start=start)
        # one more rounding, of the sum
        assert np.all(np.abs(more["dW"] - (whole["dW"] + start[0])) <= 2 * U * np.abs(start[0]) + 4 * U * np.abs(whole["dW"]) + 1e-12)
        assert np.all(np.abs(more["db"] - (whole["db"] + start[1])) <= 2 * U * np.abs(start[1]) + 4 * U * np.abs(whole["db"]) + 1e-12)


def test_the_same_call_gives_the_same_bits_and_workspaces_can_be_shared_in_turn():
    g = _g()
    sizes = [(3000, 256, 5000), (40, 64, 41), (1, 256, 50021), (700, 100, 300)]
    room = max(g.gnntrain_head_xent_workspace_size(*s, _code(g, dt)) for s in sizes for dt in DT)
    ws = torch.zeros(room + 256, dtype=torch.uint8, device=DEV)
    ws[room:] = 0xFF
    first = {}
    for turn in range(2):
        for s in sizes:
            for dtype in DT:
                got = run_head(*head_inputs(*s, dtype, 5, "some"), 0.01, dtype, workspace=ws)
                for k, x in got.items():
                    if turn:
                        assert np.array_equal(x, first[s, dtype][k]), (s, dtype, k)
                first.setdefault((s, dtype), got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_head_gradients_against_differences(dtype):
    """Along a random direction: (f(x + t v) - f(x - t v)) / 2t of the summed loss.  The third derivative of a row's loss is at most the cubed
    range of its logits' change; the losses' own errors go in over t."""
    n, d, C, t = 60, 24, 50, 2.0 ** -5
    rng = np.random.default_rng(3)
    h, W, b, y, _ = head_inputs(n, d, C, dtype, 6, "all")
    got = run_head(h, W, b, y, None, 1.0, dtype)
    # directions whose steps are exact in the operands' type: a multiple of the operand's own last digit
    def total(hh, WW, bb):
        return run_head(hh, WW, bb, y, None, 1.0, dtype, grads=())["loss"].sum()

    for what in ("h", "W", "b"):
        x = {"h": h.float(), "W": W.float(), "b": torch.from_numpy(b)}[what]
        v = torch.from_numpy(rng.normal(size=tuple(x.shape)).astype(np.float32))
        hi, lo = ((x + t * v).to(DT[dtype] if what != "b" else torch.float32), (x - t * v).to(DT[dtype] if what != "b" else torch.float32))
        step = (hi.double() - lo.double()).numpy() / 2          # what was really gone
        mid = (hi.double() + lo.double()).numpy() / 2 - x.double().numpy()
        args = {"h": ((hi, W, b), (lo, W, b)), "W": ((h, hi, b), (h, lo, b)), "b": ((h, W, hi.float().numpy()), (h, W, lo.float().numpy()))}[what]
        diff = (total(*args[0]) - total(*args[1])) / 2
        grad = {"h": got["dh"], "W": got["dW"], "b": got["db"]}[what]
        slope = float((grad * step).sum())

        def of_logits(change):
            change = np.abs(change)
            if what == "h":
                return change @ np.abs(W.double().numpy())
            return np.abs(h.double().numpy()) @ change if what == "W" else change[None].repeat(n, 0)

        reach, shift = 2 * of_logits(step).max(1), of_logits(mid)
        z = float((np.abs(h.double().numpy()) @ np.abs(W.double().numpy())).max()) + 2
        # third order; the midpoint off x by a rounding (second order: range times range); the losses' errors; the gradient's own
        bound = (reach ** 3 / 6).sum() + (reach * 2 * shift.max(1)).sum() + n * (2 * (d + 2) * U * z + (C + 16) * U * 6 + 16 * U * z)
        bound += (V * 2 if dtype == "bf16" else 1e-4) * float(np.abs(grad * step).sum())
        assert abs(diff - slope) <= bound, (what, diff, slope, bound)


def test_head_on_another_stream_and_in_a_graph():
    """Captured once, replayed with other inputs in the same buffers, eager work between the replays."""
    g = _g()
    for dtype, (rows, d, C) in (("bf16", (700, 128, 3000)), ("f32", (300, 64, 500)), ("bf16", (90, 300, 200)), ("bf16", (5000, 64, 41))):
        ws = torch.empty(g.gnntrain_head_xent_workspace_size(rows, d, C, _code(g, dtype)), dtype=torch.uint8, device=DEV)
        h, W, b, y, mask = head_inputs(rows, d, C, dtype, 1, "some")
        t = [x.to(DEV) for x in (h, W, torch.from_numpy(b), torch.from_numpy(y), torch.from_numpy(mask))]
        loss, dh = torch.zeros(rows, device=DEV), torch.zeros(rows, d, dtype=DT[dtype], device=DEV)
        dW, db = torch.zeros(d, C, device=DEV), torch.zeros(C, device=DEV)
        call = lambda: g.gnntrain_head_xent(*t, 0.01, loss, ws, dh=dh, dW=dW, db=db)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for turn in range(3):
            new = head_inputs(rows, d, C, dtype, 20 + turn, "some")
            for dst, src in zip(t, (new[0], new[1], torch.from_numpy(new[2]), torch.from_numpy(new[3]), torch.from_numpy(new[4]))):
                dst.copy_(src)
            dW.zero_()
            db.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = [x.clone() for x in (loss, dh, dW, db)]
            dW.zero_()
            db.zero_()
            call()
            torch.cuda.synchronize()
            for a, e in zip(got, (loss, dh, dW, db)):
                assert torch.equal(a, e), (dtype, rows, turn)


@pytest.mark.parametrize("dtype,rows,d,C", [("f32", 1299, 390, 8999), ("bf16", 200, 300, 9000), ("f32", 3011, 520, 2003), ("bf16", 20000, 128, 172), ("bf16", 20000, 40, 300),
                                            ("bf16", 1, 256, 20011)])
def test_replays_and_calls_at_once(dtype, rows, d, C):
    """A graph whose replays find few labelled rows, all, none; two streams at work at the same time, each with a workspace of its own."""
    g = _g()
    size = g.gnntrain_head_xent_workspace_size(rows, d, C, _code(g, dtype))
    h, W, b, y, _ = head_inputs(rows, d, C, dtype, 31, "all")
    inputs = [x.to(DEV) for x in (h, W, torch.from_numpy(b), torch.from_numpy(y))] + [torch.ones(rows, dtype=torch.uint8, device=DEV)]

    def outputs():
        return (torch.empty(rows, device=DEV), torch.empty(rows, d, dtype=DT[dtype], device=DEV), torch.zeros(d, C, device=DEV), torch.zeros(C, device=DEV),
                torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV))

    def call(out):
        out[2].zero_()
        out[3].zero_()
        g.gnntrain_head_xent(*inputs, 0.01, out[0], out[4], dh=out[1], dW=out[2], db=out[3])

    first, second, want = outputs(), outputs(), outputs()
    call(first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(first)
    side = torch.cuda.Stream()
    for share in (1.0, 0.1, 0.0, 0.95, 1.0):
        inputs[4].copy_((torch.rand(rows, generator=torch.Generator().manual_seed(7)) < share).to(torch.uint8))
        call(want)
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(second)
        graph.replay()
        torch.cuda.synchronize()
        for out in (first, second):
            assert all(torch.equal(x, e) for x, e in zip(out[:4], want[:4])), share


# ---- rows in 8 bits ------------------------------------------------------------------------------------------------
def stored(x):
    """q, scale and the values they stand for, of float64 rows, from the definition."""
    n, d = x.shape
    wide = (d + 31) // 32
    full = np.zeros((n, wide * 32))
    full[:, :d] = x
    blocks = full.reshape(n, wide, 32)
    bad = ~np.isfinite(blocks).all(2)
    a = np.where(bad, 0.0, np.abs(np.where(np.isfinite(blocks), blocks, 0.0)).max(2))
    e = np.full(a.shape, -120)
    for power in range(-120, 121):       # the least e with a <= 127 * 2^e
        e[a > 127.0 * 2.0 ** power] = power + 1
    q = np.clip(np.rint(np.where(bad[..., None], 0.0, blocks) * np.exp2(-e.astype(np.float64))[..., None]), -127, 127)
    value = q * np.exp2(e.astype(np.float64))[..., None]
    value[bad] = np.nan
    return q.reshape(n, -1).astype(np.int8), np.where(bad, 255, e + 127).astype(np.uint8), value.reshape(n, -1)[:, :d]


def rows_input(n, d, dtype, seed, extremes=True):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(n, d)) * np.exp2(rng.integers(-6, 7, size=(n, 1)))
    x[rng.random((n, d)) < 0.4] = 0.0
    if extremes and n >= 8:
        x[0] = 0.0
        x[1] = np.exp2(rng.integers(-149, 127, size=d))
        x[2] = 127.0 * 2.0 ** -3 * rng.choice([-1, 1, 0.5, 1 / 127], size=d)
        x[3, 0], x[4, -1], x[5, d // 2] = np.nan, np.inf, -np.inf
        x[6] = 3.3e38 * rng.choice([-1, 1, 0.3], size=d)
        x[7] = 2.0 ** -121 * rng.choice([0.9, 1.1, 3.0], size=d)
    with np.errstate(over="ignore"):
        return torch.from_numpy(x.astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 1), (1, 32), (3, 31), (9, 33), (64, 100), (257, 64), (40, 250), (17, 602), (1000, 128), (70001, 8)])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_store_and_load_are_exact(n, d, dtype, pad):
    g = _g()
    x = rows_input(n, d, dtype, 100 * n + d)
    q_want, s_want, value = stored(x.double().numpy())
    wide = torch.full((n + 1, d + pad), 9.0, dtype=DT[dtype], device=DEV)
    wide[:n, :d] = x.to(DEV)
    cols = (d + 31) // 32
    q = torch.full((n + 1, cols * 32 + 16 * (pad > 0)), 77, dtype=torch.int8, device=DEV)
    s = torch.full((n + 1, cols + pad), 77, dtype=torch.uint8, device=DEV)
    g.gnnstage_rows8_store(wide[:n, :d], q[:n, :cols * 32], s[:n, :cols])
    torch.cuda.synchronize()
    assert np.array_equal(q[:n, :cols * 32].cpu().numpy(), q_want) and np.array_equal(s[:n, :cols].cpu().numpy(), s_want)
    assert bool((q[n] == 77).all()) and bool((s[n] == 77).all()) and bool((q[:, cols * 32:] == 77).all()) and bool((s[:, cols:] == 77).all())
    for out_type in DT.values():
        back = torch.full((n + 1, d + pad), 9.0, dtype=out_type, device=DEV)
        g.gnnstage_rows8_load(q[:n, :cols * 32], s[:n, :cols], back[:n, :d])
        torch.cuda.synchronize()
        assert np.array_equal(back[:n, :d].double().cpu().numpy(), value, equal_nan=True)
        assert bool((back[n] == 9.0).all()) and bool((back[:, d:] == 9.0).all())
    # half a step of the block's largest value, 2^e / 2 <= a / 127 (the blocks beyond the factors' range: a whole step)
    want = x.double().numpy()
    with np.errstate(invalid="ignore"):
        step = np.exp2(s_want.astype(np.float64) - 127).repeat(32, 1)[:, :d] * np.where(np.abs(want) > 127.0 * 2.0 ** 121, 1.0, 0.5)
        fine = np.isfinite(value)
        assert np.all(np.abs(value - want)[fine] <= step[fine])


def check_weight_grad(n, d, out, dtype, pad=0, bias=True, nan=False):
    g = _g()
    rng = np.random.default_rng(n + d * 7 + out)
    x = rows_input(n, d, "f32", n + d, extremes=False)
    if nan:
        x[n // 2, d // 2] = float("nan")
    q, s, value = stored(x.double().numpy())
    dy = torch.from_numpy(rng.normal(size=(n, out)).astype(np.float32)).to(DT[dtype])
    # nothing behind the last row's columns: the tensor ends there
    flat = torch.zeros((n - 1) * (out + pad) + out, dtype=DT[dtype], device=DEV)
    view = flat.as_strided((n, out), (out + pad, 1))
    view.copy_(dy)
    start = rng.normal(size=(d, out)).astype(np.float32)
    dW = torch.from_numpy(start).to(DEV)
    db = torch.ones(out, device=DEV) if bias else None
    size = g.gnnstage_rows8_weight_grad_workspace_size(n, d, out, _code(g, dtype))
    ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    g.gnnstage_rows8_weight_grad(torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV), view, dW, ws[:size], dbias=db)
    torch.cuda.synchronize()
    assert bool((ws[size:] == 0xFF).all())
    dy = dy.double().numpy()
    got = dW.double().cpu().numpy()
    if nan:
        block = slice(d // 2 // 32 * 32, min(d, d // 2 // 32 * 32 + 32))
        assert np.isnan(got[block]).all() and np.isfinite(np.delete(got, np.arange(block.start, block.stop), 0)).all()
        value = np.nan_to_num(value)
        got[block] = (value.T @ dy + start)[block]
    want = value.T @ dy
    bound = (n + 2) * U * (np.abs(value).T @ np.abs(dy)) + 2 * U * (np.abs(start) + np.abs(want))
    assert np.all(np.abs(got - (want + start)) <= bound), np.abs(got - want - start).max()
    if bias:
        assert np.all(np.abs(db.double().cpu().numpy() - 1 - dy.sum(0)) <= (n + 2) * U * np.abs(dy).sum(0) + 2 * U * (1 + np.abs(dy.sum(0))))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,out", [(1, 1, 1), (1, 33, 8), (5, 3, 2), (63, 32, 3), (64, 64, 64), (65, 100, 100), (130, 250, 41), (257, 256, 256),
                                     (333, 602, 128), (1000, 128, 257), (3000, 31, 500), (4100, 129, 255)])
def test_weight_gradient_from_stored_rows(n, d, out, dtype):
    check_weight_grad(n, d, out, dtype, pad=(n % 3) * (8 if out % 8 == 0 else 1), bias=n % 2 == 0)


@pytest.mark.parametrize("dtype,n,d,out,pad", [("bf16", 70001, 256, 256, 0), ("bf16", 66000, 256, 200, 8), ("bf16", 90001, 130, 256, 0), ("f32", 66000, 100, 100, 0),
                                               ("bf16", 300001, 64, 41, 0), ("bf16", 131072, 256, 128, 0)])
def test_weight_gradient_over_many_rows(dtype, n, d, out, pad):
    check_weight_grad(n, d, out, dtype, pad=pad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [200, 70001])
def test_a_nan_block_reaches_the_weight_gradient(dtype, n):
    check_weight_grad(n, 100, 64, dtype, nan=True)


def test_stored_rows_on_another_stream_and_in_a_graph():
    g = _g()
    for dtype, n, d, out in (("bf16", 3000, 256, 256), ("f32", 2000, 100, 41), ("bf16", 70001, 256, 100)):
        x = torch.empty(n, d, dtype=DT[dtype], device=DEV)
        dy = torch.empty(n, out, dtype=DT[dtype], device=DEV)
        q = torch.empty(n, (d + 31) // 32 * 32, dtype=torch.int8, device=DEV)
        s = torch.empty(n, (d + 31) // 32, dtype=torch.uint8, device=DEV)
        back = torch.empty(n, d, dtype=DT[dtype], device=DEV)
        dW, db = torch.zeros(d, out, device=DEV), torch.zeros(out, device=DEV)
        ws = torch.empty(g.gnnstage_rows8_weight_grad_workspace_size(n, d, out, _code(g, dtype)), dtype=torch.uint8, device=DEV)

        def call():
            g.gnnstage_rows8_store(x, q, s)
            g.gnnstage_rows8_load(q, s, back)
            g.gnnstage_rows8_weight_grad(q, s, dy, dW, ws, dbias=db)

        x.normal_()
        dy.normal_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(3):
            x.normal_()
            dy.normal_()
            dW.zero_()
            db.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (q, s, back, dW, db)]
            dW.zero_()
            db.zero_()
            call()
            torch.cuda.synchronize()
            for a, e in zip(got, (q, s, back, dW, db)):
                assert torch.equal(a, e), dtype


def test_a_step_with_stored_rows_and_a_head_without_logits():
    """The operators as a training step uses them: a layer's rows are stored, the head gives losses and the layer's output gradient,
    the layer's weight gradient reads the stored rows.  Against the same step in 64 bits on the values that were stored."""
    g = _g()
    n, d, hid, C = 3000, 100, 128, 10007
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.normal(size=(n, d)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    W1 = torch.from_numpy((rng.normal(size=(d, hid)) / 10).astype(np.float32)).to(torch.bfloat16).to(DEV)
    W2 = torch.from_numpy((rng.normal(size=(hid, C)) / 11).astype(np.float32)).to(torch.bfloat16).to(DEV)
    y = torch.from_numpy(rng.integers(0, C, size=n).astype(np.int32)).to(DEV)
    mask = torch.from_numpy((rng.random(n) < 0.7).astype(np.uint8)).to(DEV)
    inv_n = float(np.float32(1.0 / int(mask.sum())))
    q, s = torch.empty(n, 128, dtype=torch.int8, device=DEV), torch.empty(n, 4, dtype=torch.uint8, device=DEV)
    g.gnnstage_rows8_store(x, q, s)
    pre = x.float() @ W1.float()
    h = torch.relu(pre).to(torch.bfloat16)
    loss, dh = torch.empty(n, device=DEV), torch.empty_like(h)
    dW2, db2 = torch.zeros(hid, C, device=DEV), torch.zeros(C, device=DEV)
    ws = torch.empty(g.gnntrain_head_xent_workspace_size(n, hid, C, g.GNNSTAGE_BF16), dtype=torch.uint8, device=DEV)
    g.gnntrain_head_xent(h, W2, None, y, mask, inv_n, loss, ws, dh=dh, dW=dW2, db=db2)
    dy = dh * (h > 0)
    dW1, db1 = torch.zeros(d, hid, device=DEV), torch.zeros(hid, device=DEV)
    ws2 = torch.empty(g.gnnstage_rows8_weight_grad_workspace_size(n, d, hid, g.GNNSTAGE_BF16), dtype=torch.uint8, device=DEV)
    g.gnnstage_rows8_weight_grad(q, s, dy, dW1, ws2, dbias=db1)
    torch.cuda.synchronize()
    on = counts(y.cpu().numpy(), mask.cpu().numpy(), C)
    want, mag = head_formula(h.double().cpu().numpy(), W2.double().cpu().numpy(), np.zeros(C), y.cpu().numpy(), on, inv_n)
    bound = head_bounds(want, mag, hid, C, int(on.sum()), "bf16")
    for k, got in (("loss", loss), ("dh", dh), ("dW", dW2), ("db", db2)):
        assert np.all(np.abs(got.double().cpu().numpy() - want[k]) <= bound[k]), k
    value = stored(x.double().cpu().numpy())[2]
    keep = (h > 0).double().cpu().numpy()
    # the layer's gradient from the formula's dh: off by dh's bound carried through the stored rows
    want1 = value.T @ (want["dh"] * keep)
    bound1 = np.abs(value).T @ (bound["dh"] * keep) + (n + 2) * U * (np.abs(value).T @ np.abs(want["dh"]))
    assert np.all(np.abs(dW1.double().cpu().numpy() - want1) <= bound1)
