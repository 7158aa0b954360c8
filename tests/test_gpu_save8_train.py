"""Stages that keep their saved aggregations in 8 bits (save_8bit) and the epoch loop with a head that keeps no logits (head_fused)."""
from __future__ import annotations

import functools

import numpy as np
import pytest
import torch

import gpu_harness
from gpu_harness import GpuRun, GpuTrainRun
from helpers import make_problem, make_train_problem, max_rel, new_oracle_trainer
from synth.configs import Workload

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture
def save8(monkeypatch):
    """Stages of the harness are created with save_8bit from here on."""
    g = gpu_harness.g

    def on():
        monkeypatch.setattr(gpu_harness, "g", _With(g, save_8bit=True))

    yield on


class _With:
    """The package, whose stages take one more option."""

    def __init__(self, g, **options):
        self._g, self._options = g, options

    def __getattr__(self, name):
        x = getattr(self._g, name)
        return functools.partial(x, **self._options) if name == "GnnStage" else x


def _outputs(run):
    out = {f"cur{j}": t for j, t in enumerate(run.cur)}
    for name in ("dbias", "d_ln_gamma", "d_ln_beta"):
        if getattr(run, name) is not None:
            out.update({f"{name}{j}": t for j, t in enumerate(getattr(run, name))})
    if run.grad_in is not None:
        out["grad_in"] = run.grad_in
    if run.grad_h0 is not None:
        out["grad_h0"] = run.grad_h0
    return out


CASES = [Workload("s8_gcn", "er", 700, 21, [48, 64, 40], 4, avg_degree=8.0),
         Workload("s8_gcn_narrow", "er", 700, 22, [64, 24, 33], 3, avg_degree=8.0),
         Workload("s8_sage", "er", 700, 23, [33, 48, 32], 4, variant="sage", avg_degree=8.0),
         Workload("s8_res", "er", 700, 24, [36, 36, 36], 4, variant="resgcn", avg_degree=8.0),
         Workload("s8_gcnii", "er", 700, 25, [64, 64, 64], 4, variant="gcnii", avg_degree=8.0, gcnii_first_layer=3),
         Workload("s8_gcn_bf16", "er", 700, 26, [48, 64, 40], 4, dtype="bf16", avg_degree=8.0),
         Workload("s8_sage_bf16", "er", 700, 27, [34, 48, 64], 4, variant="sage", dtype="bf16", avg_degree=8.0),
         Workload("s8_res_bf16", "er", 700, 28, [128, 128, 128], 4, variant="resgcn", dtype="bf16", avg_degree=8.0),
         Workload("s8_gcnii_bf16", "er", 700, 29, [64, 64, 64], 4, variant="gcnii", dtype="bf16", avg_degree=8.0, gcnii_first_layer=3)]


@pytest.mark.parametrize("w", CASES, ids=lambda w: w.name)
@pytest.mark.parametrize("need_input_grad", [True, False])
def test_nothing_but_weight_gradients_changes(w, need_input_grad, save8):
    """Levels, gradients of rows and LayerNorm parameters are the same bits.  Bias gradients are the same sums, of bf16 rows in another order: two
    sums of n terms are apart by at most 2 n u times their magnitudes' sum, which for terms of random signs is at most the root
    of n times the largest of the sums.  A weight gradient is off by what its rows are off: a stored
    value by at most 1 / 127 of its block's largest, evenly over that range, so by about 0.6 / 127 / sqrt(3) of twice to four times the
    rows' root mean square; with gradient rows of random signs that is 1 to 2 % of the sum's size.  5 % at most."""
    p = make_problem(w)
    plain = GpuRun(p, need_input_grad=need_input_grad).run()
    save8()
    small = GpuRun(p, need_input_grad=need_input_grad).run()
    want, got = _outputs(plain), _outputs(small)
    for k in want:
        if k.startswith("dbias") and w.dtype == "bf16":
            assert float((want[k] - got[k]).abs().max()) <= 2 * p.n * U * np.sqrt(p.n) * float(want[k].abs().max()), k
        else:
            assert torch.equal(want[k], got[k]), k
    for j in range(p.L):
        a, b = plain.dW[j].double(), small.dW[j].double()
        assert float((a - b).norm() / a.norm()) <= 0.05, j
        if not torch.equal(a, b):
            assert plain.stage.gnnstage_layer_order(j) == 0
    # another pass over the same handle, chunk by chunk this time
    for t in small.dW + (small.dbias or []) + (small.d_ln_gamma or []) + (small.d_ln_beta or []):
        t.zero_()
    if small.grad_h0 is not None:
        small.grad_h0.zero_()
    for pos, k in enumerate(p.order):
        small.stage.stage_forward_chunk(int(k), pos)
    for k in reversed(list(p.order)):
        small.stage.stage_backward_chunk(int(k), small.grad_out[small.stage.rows(int(k))])
    torch.cuda.synchronize()
    for j in range(p.L):
        a, b = plain.dW[j].double(), small.dW[j].double()
        assert float((a - b).norm() / a.norm()) <= 0.05, j
    for k in want:
        if k.startswith("cur") or k.startswith("grad"):
            assert torch.equal(want[k], _outputs(small)[k]), k


@pytest.mark.parametrize("variant", ["gcn", "sage"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("whole", [True, False])
def test_what_8_bits_hold_exactly_changes_nothing(variant, dtype, whole):
    """Small whole numbers everywhere: every aggregation is one of at most 127, which 8 bits keep, so the weight gradients are those of a stage
    that keeps everything, up to the order of a sum."""
    g = gpu_harness.g
    n, K, dims = 900, 4, [40, 33 if dtype == "f32" else 34, 48]
    rng = np.random.default_rng(5)
    rows = [np.unique(np.concatenate([[v], rng.integers(0, n, size=4)])) for v in range(n)]
    row_ptr = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int64)
    col = np.concatenate(rows).astype(np.int32)
    chunk_ptr = np.array([0, 200, 200, 611, n], dtype=np.int64)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    two = 2 if variant == "sage" else 1

    def stage(save):
        r = np.random.default_rng(6)
        W = []
        for j in range(2):  # every output copies one input
            w = np.zeros((two * dims[j], dims[j + 1]), np.float32)
            w[r.integers(0, dims[j], size=dims[j + 1]) + (two - 1) * dims[j], np.arange(dims[j + 1])] = 1.0
            W.append(torch.from_numpy(w).to(t).to(DEV))
        x = torch.from_numpy(r.integers(-2, 3, size=(n, dims[0])).astype(np.float32)).to(t).to(DEV)
        cur = [x] + [torch.zeros(n, d, dtype=t, device=DEV) for d in dims[1:]]
        hist = [torch.from_numpy(r.integers(-2, 3, size=(n, dims[j])).astype(np.float32)).to(t).to(DEV) for j in range(2)]
        dW = [torch.zeros(two * dims[j], dims[j + 1], device=DEV) for j in range(2)]
        db = [torch.zeros(dims[j + 1], device=DEV) for j in range(2)]
        st = g.GnnStage(row_ptr, col, chunk_ptr, dims, W=W, cur=cur, hist=hist, dW=dW, bias=[torch.zeros_like(b) for b in db], dbias=db,
                        edge_val=np.ones(len(col), np.float32), variant=g.GNNSTAGE_SAGE if variant == "sage" else g.GNNSTAGE_GCN,
                        dtype=g.GNNSTAGE_BF16 if dtype == "bf16" else g.GNNSTAGE_F32, grad_in=torch.zeros_like(x), save_8bit=save)
        grad = torch.from_numpy(r.integers(-3, 4, size=(n, dims[2])).astype(np.float32)).to(t).to(DEV)
        order = [2, 0, 3, 1]
        if whole:
            st.forward_pass(order)
            st.backward_pass(order, grad)
        else:
            for pos, k in enumerate(order):
                st.stage_forward_chunk(k, pos)
            for k in reversed(order):
                st.stage_backward_chunk(k, grad[st.rows(k)])
        torch.cuda.synchronize()
        return st, dW, db, cur

    a, b = stage(False), stage(True)
    assert b[0].workspace_bytes < a[0].workspace_bytes
    for x, y in zip(a[1] + a[2] + a[3], b[1] + b[2] + b[3]):
        assert torch.equal(x, y)  # whole numbers below 2^24: no order of additions changes them


def test_the_workspace_shrinks_by_the_saved_rows():
    """Ten layers of width 128: 10 n 256 bytes less, 10 n 132 more."""
    w = Workload("s8_deep", "er", 4000, 30, [128] * 11, 4, variant="gcnii", dtype="bf16", avg_degree=6.0, gcnii_first_layer=3)
    p = make_problem(w)
    plain = GpuRun(p)
    gpu_harness_g = gpu_harness.g
    try:
        gpu_harness.g = _With(gpu_harness_g, save_8bit=True)
        small = GpuRun(p)
    finally:
        gpu_harness.g = gpu_harness_g
    saved = plain.stage.workspace_bytes - small.stage.workspace_bytes
    assert saved >= 10 * 4000 * (256 - 132) - 20 * 512


@pytest.mark.parametrize("variants,stage_dims,C", [(None, ((24, 16), (16, 16, 12)), 5), (("sage", "resgcn", "gcn"), ((24, 16), (16, 16, 16), (16, 8)), 41),
                                                   (None, ((20, 24, 100),), 300), (None, ((24, 300),), 9000)])
def test_epochs_without_logits_fp32(variants, stage_dims, C):
    """The loop against the oracle's, as with the head that keeps its logits."""
    kw = {} if variants is None else {"variants": variants}
    tp = make_train_problem(n=1500, n_classes=C, stage_dims=stage_dims, K=4, ragged=True, **kw)
    opt = dict(optimizer="sgd", lr=float(np.float32(0.05)), shuffle=True, seed=7, alpha_hist=1)
    ref = new_oracle_trainer(tp, **opt)
    run = GpuTrainRun(tp, head_fused=True, **opt)
    for e in range(3):
        want, got = ref.epoch(e), run.epoch(e)
        assert abs(got - want) <= 1e-4 * want
        for a, b in zip(run.grads(), ref.grads()):
            assert max_rel(a.reshape(b.shape), b) <= 1e-4, e
    for a, b in zip(run.master_values(), ref.master):
        assert max_rel(a.reshape(b.shape), b) <= 1e-4


@pytest.mark.parametrize("C", [5, 1000])
def test_an_epoch_without_logits_bf16(C):
    """Against the loop with the other head on the same inputs: both round the logits' gradients for the rows' to bf16 (the other one for the weights'
    too), 2^-8 of each factor at most, and ReLU decisions are the same (one forward pass): 1e-2 of a tensor's largest."""
    tp = make_train_problem(n=1500, n_classes=C, stage_dims=((24, 16), (16, 16, 64)), K=4, dtype="bf16")
    opt = dict(optimizer="sgd", lr=float(np.float32(0.05)), shuffle=True, seed=7, alpha_hist=1)
    a, b = GpuTrainRun(tp, **opt), GpuTrainRun(tp, head_fused=True, **opt)
    la, lb = a.epoch(0), b.epoch(0)
    assert abs(la - lb) <= 1e-5 * la
    for x, y in zip(a.grads(), b.grads()):
        assert max_rel(x, y) <= 1e-2


def test_more_classes_than_the_other_head_takes():
    tp = make_train_problem(n=300, n_classes=70001, stage_dims=((8, 16),), K=3)
    with pytest.raises(gpu_harness.g.GnnStageError):
        GpuTrainRun(tp)
    run = GpuTrainRun(tp, head_fused=True, optimizer="adam", lr=0.01)
    head_W, head_b = run.head_master.double().cpu().numpy(), run.head_b.double().cpu().numpy()
    loss = run.epoch(0)
    z = run.cur[0][-1].double().cpu().numpy() @ head_W + head_b
    top = z.max(1, keepdims=True)
    rows = np.log(np.exp(z - top).sum(1)) + top[:, 0] - z[np.arange(300), tp.labels]
    on = np.ones(300, bool) if tp.mask is None else tp.mask != 0
    assert abs(loss - rows[on].mean()) <= 1e-5 * abs(rows[on].mean())
    assert run.epoch(1) < loss


def test_both_options_in_one_model(save8):
    """bf16, three layer types, dropout: the options' loop against the plain one.  The losses of the first epoch are the same forward pass; the
    weight gradients differ by the stored rows' 5 % (above)."""
    tp = make_train_problem(n=1500, n_classes=41, stage_dims=((24, 16), (16, 16, 16), (16, 32)), K=4, ragged=True, dtype="bf16",
                            variants=("sage", "resgcn", "gcn"))
    tp.dropout_p = 0.5
    opt = dict(optimizer="sgd", lr=float(np.float32(0.05)), shuffle=True, seed=11, alpha_hist=2)
    a = GpuTrainRun(tp, **opt)
    save8()
    b = GpuTrainRun(tp, head_fused=True, **opt)
    la, lb = a.epoch(0), b.epoch(0)
    assert abs(la - lb) <= 1e-5 * la
    for x, y in zip(a.grads(), b.grads()):
        assert np.linalg.norm(x - y) <= 0.06 * np.linalg.norm(x)
    for e in range(1, 4):
        la, lb = a.epoch(e), b.epoch(e)
        assert np.isfinite(lb)
