"""Operators around what a training step keeps between its forward and its backward pass, as cases to be timed: the loss head over many
classes without logits (``gnntrain_head_xent``) and activation checkpoints in 8 bits with the weight gradient that reads them
(``gnnstage_rows8_*``), each next to its plain form in elementary torch operations.

Fields of a case
  call      head: row losses and all gradients of a linear softmax cross-entropy head
            loss: the row losses alone (an evaluation pass)
            keep: rows stored in 8 bits and restored
            use:  weight and bias gradient of a layer from its rows in 8 bits and its gradient rows
  dtype     f32 or bf16: of rows, weights and gradient rows (row losses, weight and bias gradients are fp32)
  rows, d   rows of the operand and its width
  out       classes (head, loss) or output width of the layer (use)
  share     share of labelled rows (head, loss)
  pad       columns behind the row's d in memory (leading dimension d + pad)
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
BLOCK = 32  # columns that share a scale


def _case(name, call, dtype, rows, d, out=0, share=1.0, pad=0):
    c = {} if name is None else {"name": name}
    c.update(call=call, dtype=dtype, rows=rows, d=d, out=out, share=share, pad=pad)
    return c


def listed():
    return [
        # The head of the smallest benchmark configuration's size, in fp32, the usual handful of classes.  Launches and latency.
        _case("head_tiny_f32", "head", "f32", 4096, 64, 41),
        # One full-graph pass over the labelled two thirds of a graph with a few ten classes.
        _case("head_few_classes_bf16", "head", "bf16", 232965, 256, 41, share=0.66),
        # A citation graph where one vertex in a hundred has a label.
        _case("head_rare_labels_bf16", "head", "bf16", 700001, 128, 172, share=0.011),
        # A sampled batch of vertices against a catalogue of entities: few rows, many classes.
        _case("head_batch_bf16", "head", "bf16", 517, 256, 50021),
        # The catalogue as the classes of a whole graph; the largest case.
        _case("head_entities_bf16", "head", "bf16", 20011, 256, 100003, share=0.9),
        # Hidden width 100 (rows of 200 bytes), ten thousand classes.
        _case("head_h100_bf16", "head", "bf16", 46657, 100, 10007, share=0.5),
        # The paper's small wide model in its fp32, with a large label set.
        _case("head_wide_f32", "head", "f32", 5196, 1000, 2003),
        # Evaluation: the losses of held-out vertices.
        _case("loss_entities_bf16", "loss", "bf16", 16384, 128, 100003, share=0.5),
        # A saved aggregation of a small fp32 stage, and one of the benchmark's 2.45 M vertices.
        _case("keep_small_f32", "keep", "f32", 4096, 100),
        _case("keep_large_bf16", "keep", "bf16", 2450000, 128),
        # Weight gradients from saved rows: hidden 100 in fp32, and a whole pass over 700 k vertices at hidden 256.
        _case("use_h100_f32", "use", "f32", 34493, 100, 100),
        _case("use_large_bf16", "use", "bf16", 700001, 256, 256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = 20011 * 100003 * 256  # rows * classes * width of the largest listed head


def draw(rng):
    """One more case of the same ranges."""
    call = rng.choice(["head", "head", "head", "loss", "keep", "use"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 0, 3, 8])
    if call in ("head", "loss"):
        d = rng.choice([16, 64, 100, 128, 200, 256, 256, 500]) if dtype == "bf16" else rng.choice([16, 64, 100, 128, 256, 600, 1000])
        most = MOST if dtype == "bf16" else MOST // 16
        out = _log_int(rng, 2, 120000)
        rows = _log_int(rng, 1, max(2, min(700001, most // (out * d), 2000000000 // out)))
        share = rng.choice([1.0, 1.0, 0.66, 0.3, 0.02])
        return _case(None, call, dtype, rows, d, out, share, pad)
    d = rng.choice([8, 33, 64, 100, 128, 250, 256, 512, 602])
    rows = _log_int(rng, 1, 2450000 * 128 // max(d, 128))
    if call == "keep":
        return _case(None, "keep", dtype, rows, d, pad=pad)
    out = rng.choice([8, 41, 64, 100, 128, 256, 256])
    rows = min(rows, 700001 * 256 * 256 // (max(d, 128) * max(out, 128)) // (1 if dtype == "bf16" else 8))
    return _case(None, "use", dtype, max(rows, 1), d, out, pad=pad)


# ---- inputs ----------------------------------------------------------------------------------------------------
def _rows(gen, rows, d, pad, dtype, relu=False):
    x = torch.randn(rows, d + pad, device=DEV, generator=gen)
    return (torch.relu_(x) if relu else x).to(dtype)[:, :d]


def _power_of_two(e):
    """2^e in fp32 for whole e of -126 .. 127, from its bits (a power function may be off in the last one)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _in_8_bits(x):
    """Blocks of 32 columns of fp32 rows (zeros behind the last column): whole numbers of -127 .. 127, and the byte e + 127 of their
    common factor 2^e."""
    n, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % BLOCK)).view(n, -1, BLOCK)
    a = x.abs().amax(2)
    part, power = torch.frexp(a)
    e = torch.where(a > 0, (power - 7 + (part > 127 / 128)).clamp(-120, 121), torch.full_like(power, -120))
    q = torch.round(x * _power_of_two(-e).unsqueeze(2)).clamp(-127, 127)
    return q.to(torch.int8).view(n, -1), (e + 127).to(torch.uint8)


def _from_8_bits(q, scale, d):
    n = q.shape[0]
    return (q.view(n, -1, BLOCK).float() * _power_of_two(scale.int() - 127).unsqueeze(2)).view(n, -1)[:, :d]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n, d, out, call = case["rows"], case["d"], case["out"], case["call"]
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = {"case": case}
    if call in ("head", "loss"):
        # rows as a trained model has them: an activated level that leans towards the row's class, some rows sure of it
        w = torch.randn(d, out, device=DEV, generator=gen) / math.sqrt(d)
        y = torch.randint(0, out, (n,), device=DEV, generator=gen, dtype=torch.int32)
        lean = 6 * torch.rand(n, 1, device=DEV, generator=gen)
        h = torch.zeros(n, d + case["pad"], device=DEV)
        h[:, :d] = torch.relu(torch.randn(n, d, device=DEV, generator=gen) + lean * w[:, y.long()].t())
        s.update(h=h.to(t)[:, :d], W=w.to(t), bias=0.1 * torch.randn(out, device=DEV, generator=gen), labels=y)
        s["mask"] = None if case["share"] == 1.0 else (torch.rand(n, device=DEV, generator=gen) < case["share"]).to(torch.uint8)
        if s["mask"] is not None:
            s["mask"][0] = 1
        s["inv_n"] = 1.0 / max(1, round(n * case["share"]))
        s["loss"] = torch.empty(n, device=DEV)
        if call == "head":
            s.update(dh=torch.empty(n, d, dtype=t, device=DEV), dW=torch.empty(d, out, device=DEV), db=torch.empty(out, device=DEV))
        return s
    x = _rows(gen, n, d, case["pad"], t, relu=call == "use")
    if call == "keep":
        wide = (d + BLOCK - 1) // BLOCK
        s.update(x=x, q=torch.empty(n, wide * BLOCK, dtype=torch.int8, device=DEV), scale=torch.empty(n, wide, dtype=torch.uint8, device=DEV),
                 back=torch.empty(n, d, dtype=t, device=DEV))
        return s
    s["q"], s["scale"] = _in_8_bits(x.float())
    s.update(dy=_rows(gen, n, out, case["pad"], t), dW=torch.empty(d, out, device=DEV), db=torch.empty(out, device=DEV))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------
def _workspace(s, size):
    """Made on the first pass and kept, as a program keeps it."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    return s["workspace"]


def _run_own(s):
    import paper_2308_10087_amd as g

    case, call = s["case"], s["case"]["call"]
    code = g.GNNSTAGE_BF16 if case["dtype"] == "bf16" else g.GNNSTAGE_F32
    if call in ("head", "loss"):
        grads = call == "head"
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, g.gnntrain_head_xent_workspace_size(case["rows"], case["d"], case["out"], code, grads))
        if not grads:
            g.gnntrain_head_xent(s["h"], s["W"], s["bias"], s["labels"], s["mask"], s["inv_n"], s["loss"], ws)
            return {"loss": s["loss"]}
        s["dW"].zero_()
        s["db"].zero_()
        g.gnntrain_head_xent(s["h"], s["W"], s["bias"], s["labels"], s["mask"], s["inv_n"], s["loss"], ws, dh=s["dh"], dW=s["dW"], db=s["db"])
        return {"loss": s["loss"], "dh": s["dh"], "dW": s["dW"], "db": s["db"]}
    if call == "keep":
        g.gnnstage_rows8_store(s["x"], s["q"], s["scale"])
        g.gnnstage_rows8_load(s["q"], s["scale"], s["back"])
        return {"rows": s["back"], "scale": s["scale"]}
    ws = s.get("workspace")
    if ws is None:
        ws = _workspace(s, g.gnnstage_rows8_weight_grad_workspace_size(case["rows"], case["d"], case["out"], code))
    s["dW"].zero_()
    s["db"].zero_()
    g.gnnstage_rows8_weight_grad(s["q"], s["scale"], s["dy"], s["dW"], ws, dbias=s["db"])
    return {"dW": s["dW"], "db": s["db"]}


def run(state):
    s, case = state, state["case"]
    if own:
        return _run_own(s)
    if case["call"] == "keep":
        q, scale = _in_8_bits(s["x"].float())
        return {"rows": _from_8_bits(q, scale, case["d"]).to(s["x"].dtype), "scale": scale}
    if case["call"] == "use":
        dy = s["dy"].float()
        return {"dW": _from_8_bits(s["q"], s["scale"], case["d"]).t() @ dy, "db": dy.sum(0)}
    labels = s["labels"].long()
    counts = (labels >= 0) & (labels < case["out"])
    if s["mask"] is not None:
        counts &= s["mask"] != 0
    at = torch.nonzero(counts).squeeze(1)
    h, w, y = s["h"][at].float(), s["W"].float(), labels[at].unsqueeze(1)
    z = h @ w + s["bias"]
    z -= z.amax(1, keepdim=True)
    zy = z.gather(1, y)
    e = z.exp_()
    ey = e.gather(1, y)
    others = e.scatter_(1, y, 0.0).sum(1, keepdim=True)  # the label's own term apart: a sure row's loss has no cancellation
    total = others + ey
    loss = torch.zeros(case["rows"], device=DEV)
    loss[at] = torch.where(ey > 0.5 * total, torch.log1p(others / ey), torch.log(total) - zy).squeeze(1)
    if case["call"] == "loss":
        return {"loss": loss}
    grad = e.mul_(s["inv_n"] / total).scatter_(1, y, -s["inv_n"] * others / total)
    dh = torch.zeros(case["rows"], case["d"], dtype=s["h"].dtype, device=DEV)
    dh[at] = (grad @ w.t()).to(dh.dtype)
    return {"loss": loss, "dh": dh, "dW": h.t() @ grad, "db": grad.sum(0)}


# ---- 64 bits ---------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    n, d, out = case["rows"], case["d"], case["out"]
    if case["call"] == "keep":
        # from the definition: the least power of two of which 127 times reaches the block's largest value
        wide = (d + BLOCK - 1) // BLOCK
        x = torch.zeros(n, wide * BLOCK, dtype=torch.float64, device=DEV)
        x[:, :d] = s["x"].double()
        x = x.view(n, wide, BLOCK)
        largest = x.abs().amax(2, keepdim=True)
        power = torch.ceil(torch.log2((largest / 127).clamp_min(2.0 ** -120)) - 1e-13).long()
        step = ((power + 1023) << 52).view(torch.float64)
        return {"rows": (torch.round(x / step) * step).view(n, -1)[:, :d], "scale": None}
    if case["call"] == "use":
        dW, db = torch.zeros(d, out, dtype=torch.float64, device=DEV), torch.zeros(out, dtype=torch.float64, device=DEV)
        for i in range(0, n, 100000):
            factor = ((s["scale"][i:i + 100000].long() + 896) << 52).view(torch.float64).repeat_interleave(BLOCK, dim=1)
            x, dy = (s["q"][i:i + 100000].double() * factor)[:, :d], s["dy"][i:i + 100000].double()
            dW += x.t().contiguous() @ dy
            db += dy.sum(0)
        return {"dW": dW, "db": db}
    w, b = s["W"].double(), s["bias"].double()
    loss, dh = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, d, dtype=torch.float64, device=DEV)
    dW, db = torch.zeros(d, out, dtype=torch.float64, device=DEV), torch.zeros(out, dtype=torch.float64, device=DEV)
    has = torch.ones(n, device=DEV) if s["mask"] is None else (s["mask"] != 0).double()
    step = max(1, 200000000 // out)
    for i in range(0, n, step):
        h, y, on = s["h"][i:i + step].double(), s["labels"][i:i + step].long(), has[i:i + step].double().unsqueeze(1)
        z = h @ w + b
        lse = torch.logsumexp(z, 1, keepdim=True)
        loss[i:i + step] = ((lse - z.gather(1, y.unsqueeze(1))) * on).squeeze(1)
        if case["call"] == "loss":
            continue
        p = (torch.exp(z - lse) - torch.zeros_like(z).scatter_(1, y.unsqueeze(1), 1.0)) * on * s["inv_n"]
        dh[i:i + step] = p @ w.t().contiguous()
        dW += h.t().contiguous() @ p
        db += p.sum(0)
    return {"loss": loss} if case["call"] == "loss" else {"loss": loss, "dh": dh, "dW": dW, "db": db}


def work(case):
    """Inputs read once, outputs written once (weight gradients are added to: read and written); the products without the logits'
    second computation."""
    n, d, out, e = case["rows"], case["d"], case["out"], 2 if case["dtype"] == "bf16" else 4
    stored = d + (d + BLOCK - 1) // BLOCK
    if case["call"] == "keep":
        return {"bytes": float(n * (2 * d * e + 2 * stored)), "flops": 4.0 * n * d}
    if case["call"] == "use":
        return {"bytes": float(n * (stored + out * e) + 8 * out * (d + 1)), "flops": 2.0 * n * d * out}
    m = n if case["share"] == 1.0 else max(1, round(n * case["share"]))
    nbytes = m * (d * e + 4) + d * out * e + 4 * out + 4 * n + (n if case["share"] < 1.0 else 0)
    if case["call"] == "loss":
        return {"bytes": float(nbytes), "flops": 2.0 * m * d * out}
    return {"bytes": float(nbytes + n * d * e + 8 * out * (d + 1)), "flops": 6.0 * m * d * out}
