"""A classifier's step and its answers, as a program runs them: logits, log probabilities and entropies, their gradients, the AdamW step, the new weights in 4 bits, answers from
those.  Every stage is checked from what the stage before it gave; bounds as in the operators' own tests."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import adamw_formula
import logprobs_formula
import rows4_formula

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


def _program(rows, d, classes, top, bits, seed):
    import paper_2308_10087_amd as g
    gen = torch.Generator(device=DEV).manual_seed(seed)
    f = lambda *shape: torch.randn(*shape, device=DEV, generator=gen)
    empty = lambda *shape, t=torch.float32: torch.zeros(*shape, dtype=t, device=DEV)
    u8, wide = torch.uint8, (d + 31) // 32
    s = dict(h=torch.relu(f(rows, d)), W=f(d, classes) / d ** 0.5, b=0.1 * f(classes), ids=torch.randint(0, classes, (rows,), device=DEV, generator=gen, dtype=torch.int32),
             gl=-torch.ones(rows, device=DEV) / rows, gh=torch.full((rows,), -0.1 / rows, device=DEV), dW=empty(d, classes), db=empty(classes), dl=empty(rows, classes),
             logp=empty(rows), H=empty(rows), norm=empty(rows, 2), ws=empty(max(g.gnntrain_logprobs_workspace_size(rows, classes, top), 256), t=u8),
             ws2=empty(g.gnntrain_logprobs_grad_workspace_size(rows, classes), t=u8), hq=empty(rows, 16 * wide, t=u8), hs=empty(rows, wide, t=u8), Wq=empty(classes, 16 * wide, t=u8),
             Ws=empty(classes, wide, t=u8), z4=empty(rows, classes), top_ids=empty(rows, top, t=torch.int32), top_logp=empty(rows, top), copy=empty(d, classes, t=torch.bfloat16))
    state = torch.float32 if bits == 32 else u8
    model = []
    for name, grad, copy in (("W", "dW", s["copy"]), ("b", "db", None)):
        x = dict(p=s[name], g=s[grad], m=torch.zeros_like(s[name], dtype=state), v=torch.zeros_like(s[name], dtype=state), compute=copy, weight_decay=0.01 if name == "W" else 0.0)
        if bits == 8:
            x.update({k: empty((x["p"].numel() + 31) // 32, t=u8) for k in ("m_scale", "v_scale")})
        model.append(x)
    s["model"], tensors = model, g.gnntrain_adamw_tensors(model)

    def step(t):
        logits = s["h"] @ s["W"]
        g.gnntrain_logprobs(logits, s["b"], s["ids"], None, s["logp"], s["H"], s["norm"], s["ws"])
        s["db"].zero_()
        g.gnntrain_logprobs_grad(logits, s["b"], s["ids"], None, s["logp"], s["H"], s["norm"], s["gl"], s["gh"], s["dl"], s["ws2"], dbias=s["db"])
        s["dW"].copy_(s["h"].t() @ s["dl"])
        g.gnntrain_adamw_step(tensors, 1e-2, 0.9, 0.999, 1e-8, t, seed=5)
        return logits

    def answer():
        g.gnnstage_rows4_store(s["h"], s["hq"], s["hs"])
        g.gnnstage_rows4_store_columns(s["W"], s["Wq"], s["Ws"])
        g.gnnstage_rows4_product(s["hq"], s["hs"], s["Wq"], s["Ws"], d, s["z4"], bias=s["b"])
        g.gnntrain_logprobs(s["z4"], None, s["ids"], None, s["logp"], s["H"], s["norm"], s["ws"], top_ids=s["top_ids"], top_logp=s["top_logp"])
    return s, step, answer


def _np(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rows,d,classes,top", [(150, 40, 41, 3), (33, 96, 5003, 10), (1, 256, 20011, 5)])
def test_steps_and_answers(rows, d, classes, top, bits):
    s, step, answer = _program(rows, d, classes, top, bits, rows + bits)
    for t in (1, 2, 3):
        before = {k: _np(s[k]) for k in ("W", "b")}
        states = [{k: x[k].cpu().numpy() for k in ("m", "v", "m_scale", "v_scale") if k in x} for x in s["model"]]
        logits = step(t)
        torch.cuda.synchronize()
        ids = s["ids"].cpu().numpy()
        z = logprobs_formula.logits_32(logits.cpu().numpy(), before["b"].astype(np.float32))
        w = logprobs_formula.answer(z, ids)
        bound = logprobs_formula.bounds(w, classes)
        assert np.all(np.abs(_np(s["logp"]) - w["logp"]) <= bound["logp"]) and np.all(np.abs(_np(s["H"]) - w["entropy"]) <= bound["entropy"])
        norm = _np(s["norm"])
        dl, slack = logprobs_formula.gradient(z, ids, norm[:, 0], norm[:, 1], _np(s["logp"]), _np(s["H"]), _np(s["gl"]), _np(s["gh"]))
        assert np.all(np.abs(_np(s["dl"]) - dl) <= slack + U * np.abs(dl))
        assert np.all(np.abs(_np(s["db"]) - dl.sum(0)) <= slack.sum(0) + (rows + 8) * U * np.abs(dl).sum(0))
        for k, (name, grad, x, old) in enumerate(zip(("W", "b"), ("dW", "db"), s["model"], states)):
            G = s[grad].cpu().numpy().reshape(-1)
            m0, v0 = (old["m"].reshape(-1).astype(np.float64), old["v"].reshape(-1).astype(np.float64)) if bits == 32 else \
                (adamw_formula.decode(old["m"].reshape(-1), old["m_scale"]), adamw_formula.decode(old["v"].reshape(-1), old["v_scale"]) ** 2)
            p, m, v = adamw_formula.step_64(before[name].reshape(-1), G, m0, v0, 1e-2, 0.9, 0.999, 1e-8, 0.01 * (name == "W"), t)
            c1, c2 = 1 / (1 - float(np.float32(0.9)) ** t), 1 / (1 - float(np.float32(0.999)) ** t)
            dm = 4 * U * (0.9 * np.abs(m0) + 0.1001 * np.abs(G)) + 2.0 ** -140
            off = np.abs(_np(s[name]).reshape(-1) - p)
            assert np.all(off <= 7 * U * np.maximum(np.abs(p), np.abs(before[name].reshape(-1))) + 1e-2 * c1 * (dm + 12 * U * np.abs(m)) / (np.sqrt(v * c2) + 1e-8)), (t, name)
            if bits == 8:
                m32, root = adamw_formula.means_32(G, m0, adamw_formula.decode(old["v"].reshape(-1), old["v_scale"]).astype(np.float32) ** 2, 0.9, 0.999)
                um, uv = adamw_formula.draws(5, t, k, len(G))
                for key, value, u, positive in (("m", m32, um, False), ("v", root, uv, True)):
                    code, byte = adamw_formula.encode(value, u, positive)
                    assert np.array_equal(x[key].cpu().numpy().reshape(-1), code) and np.array_equal(x[key + "_scale"].cpu().numpy(), byte)
        assert torch.equal(s["copy"], s["W"].bfloat16())
    answer()
    torch.cuda.synchronize()
    A = rows4_formula.decode(*rows4_formula.encode(_np(s["h"])), d)
    B = rows4_formula.decode(*rows4_formula.encode(_np(s["W"]).T), d)
    b, z4 = _np(s["b"]), _np(s["z4"])
    assert np.all(np.abs(z4 - (A @ B.T + b)) <= (d + 3) * U * (np.abs(A) @ np.abs(B).T + np.abs(b)))
    z = logprobs_formula.logits_32(z4, None)
    w = logprobs_formula.answer(z, s["ids"].cpu().numpy())
    assert np.all(np.abs(_np(s["logp"]) - w["logp"]) <= logprobs_formula.bounds(w, classes)["logp"])
    assert np.array_equal(s["top_ids"].cpu().numpy(), logprobs_formula.best(z, top))


def test_a_captured_step_and_answer_replayed():
    """The graph of one step (its number is the host's: every replay is step 1 again) and the answers behind it, next to the same calls made eagerly on tensors of
    their own, with eager work between."""
    (one, step_one, answer_one), (two, step_two, answer_two) = _program(64, 64, 1000, 5, 8, 3), _program(64, 64, 1000, 5, 8, 3)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # the library's products set themselves up outside of the capture
        _ = one["h"] @ one["W"], one["h"].t() @ one["dl"]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step_one(1)
        answer_one()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        step_two(1)
        answer_two()
        torch.cuda.synchronize()
        for k in ("W", "b", "copy", "dW", "db", "logp", "H", "top_ids", "top_logp", "z4", "Wq"):
            assert torch.equal(one[k], two[k]), k
