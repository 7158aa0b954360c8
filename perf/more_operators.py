"""Operators of a classifier over many classes between its training and its answers, as cases to be timed: the weight update of many tensors
at once (``gnntrain_adamw_step``), log probabilities with entropy and best classes (``gnntrain_logprobs``) and their gradient
(``gnntrain_logprobs_grad``), rows in 4 bits and their product (``gnnstage_rows4_*``), each next to its plain form in elementary torch operations.

Fields of a case
  call      adamw:   one AdamW step over all tensors of a model, states in fp32 or in 8 bits
            answer:  log probability of one class per row, entropy, the best classes
            push:    gradient of the logits (and the classes' bias) from the gradients of log probabilities and entropies
            keep4:   rows stored in 4 bits and restored
            logits4: rows stored in 4 bits and multiplied with classes' weights in 4 bits
  dtype     f32 or bf16: of gradients (adamw), of logits (answer, push), of rows (keep4, logits4) and of what is returned of them
  rows, d   rows and their width; adamw: classes of the head (its weights are d x rows) and hidden width
  out       classes (answer, push, logits4); adamw: layers in front of the head
  top       best classes asked for (answer)
  share     share of the rows that take part (answer, push)
  bits      of the optimizer's states (adamw)
  pad       columns behind a row's in memory; adamw: 1 for tensors right behind one another instead of on multiples of 64 elements
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
BLOCK = 32  # elements that share a factor
LR, B1, B2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
GOLDEN = 0x9E3779B97F4A7C15


def _case(name, call, dtype, rows, d, out=0, top=0, share=1.0, bits=0, pad=0):
    c = {} if name is None else {"name": name}
    c.update(call=call, dtype=dtype, rows=rows, d=d, out=out, top=top, share=share, bits=bits, pad=pad)
    return c


def listed():
    return [
        # Four layers of hidden width 256 and a head of 41 classes: 18 small tensors.  Launches and latency.
        _case("adamw_model_32", "adamw", "f32", 41, 256, 4, bits=32),
        # A catalogue of entities as classes: one large tensor and some small ones, states in fp32.
        _case("adamw_entities_32", "adamw", "f32", 100003, 256, 8, bits=32),
        # Hidden width 100, tensors behind one another (odd places), bf16 gradients, states in 8 bits.
        _case("adamw_h100_8", "adamw", "bf16", 10007, 100, 4, bits=8, pad=1),
        # The largest: four times the entities, whose states are why they are kept in 8 bits.
        _case("adamw_entities_8", "adamw", "bf16", 400009, 256, 4, bits=8),
        # One vertex asked for its five best of 100,003 classes.
        _case("answer_one_f32", "answer", "f32", 1, 0, 100003, top=5),
        # All vertices of a graph, a few ten classes, held-out two thirds.
        _case("answer_graph_f32", "answer", "f32", 232965, 0, 41, top=3, share=0.66),
        # A batch against the catalogue; rows whose lists are long.
        _case("answer_entities_bf16", "answer", "bf16", 8191, 0, 100003, top=10),
        # Gradients of a citation graph's logits, fp32, rows of odd length apart from one another.
        _case("push_citation_f32", "push", "f32", 70001, 0, 172, share=0.66, pad=3),
        # Gradients of a batch's logits over the catalogue.
        _case("push_entities_bf16", "push", "bf16", 8191, 0, 100003),
        # Rows of 200 bytes of a 700 k vertex graph, kept in 4 bits.
        _case("keep4_h100_bf16", "keep4", "bf16", 700001, 100),
        # Three vertices against four times the entities: bound by the classes' weights.
        _case("logits4_few_f32", "logits4", "f32", 3, 256, 400009),
        # A batch against the catalogue.
        _case("logits4_entities_bf16", "logits4", "bf16", 8191, 256, 100003),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = 8191 * 100003  # logits of the largest listed batch


def draw(rng):
    """One more case of the same ranges."""
    call = rng.choice(["adamw", "adamw", "answer", "answer", "push", "keep4", "logits4"])
    dtype = rng.choice(["bf16", "f32"])
    pad = rng.choice([0, 0, 3, 8])
    if call == "adamw":
        d = rng.choice([16, 64, 100, 128, 200, 256, 500])
        return _case(None, call, dtype, _log_int(rng, 2, 400009 * 256 // max(d, 256)), d, rng.choice([1, 2, 4, 8]), bits=rng.choice([8, 32]), pad=rng.choice([0, 0, 1]))
    if call in ("answer", "push"):
        out = _log_int(rng, 2, 400009)
        rows = _log_int(rng, 1, max(2, min(2450000, MOST // (1 if dtype == "bf16" else 2) // out)))
        share = rng.choice([1.0, 1.0, 0.66, 0.3, 0.02])
        top = min(out, rng.choice([0, 1, 3, 5, 10, 20, 64])) if call == "answer" else 0
        return _case(None, call, dtype, rows, 0, out, top, share, pad=pad)
    d = rng.choice([8, 33, 64, 100, 128, 250, 256, 512, 602])
    if call == "keep4":
        return _case(None, call, dtype, _log_int(rng, 1, 700001 * 100 // max(d, 100)), d, pad=pad)
    out = _log_int(rng, 2, 400009)
    rows = _log_int(rng, 1, max(2, min(700001, MOST // (1 if dtype == "bf16" else 2) // out * 256 // max(d, 256))))
    return _case(None, call, dtype, rows, d, out, pad=pad)


# ---- numbers in few bits -----------------------------------------------------------------------------------------
def _power_of_two(e):
    """2^e in fp32 for whole e of -126 .. 127, from its bits (a power function may be off in the last one)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _blocks(x):
    """fp32 rows in blocks of 32, zeros behind the last column"""
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK)).view(*x.shape[:-1], -1, BLOCK)


def _in_4_bits(x):
    """Bytes of two columns each (the first one in the low half: 0 .. 7 for 0, 1/2, 1, 3/2, 2, 3, 4, 6, and 8 more for minus) and the byte
    e + 127 of a block's factor 2^e, the least whose seven times reaches the block's largest value."""
    x = _blocks(x)
    a = x.abs().amax(-1)
    part, power = torch.frexp(a)  # a = part * 2^power, part in [1/2, 1)
    e = torch.where(a > 0, (power - 3 + (part > 7 / 8)).clamp(-120, 121), torch.full_like(power, -120))
    y = x.abs() * _power_of_two(-e).unsqueeze(-1)
    binade = ((y >= 2).int() + (y >= 4)).clamp_max(2)
    code = (2 * binade + torch.round(y * _power_of_two(1 - binade)).int()).clamp_max(7) + 8 * torch.signbit(x)
    code = code.to(torch.uint8).view(x.shape[0], -1)
    return code[:, 0::2] | code[:, 1::2] << 4, (e + 127).to(torch.uint8)


def _from_4_bits(q, scale, d):
    code = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1, BLOCK).int()
    size = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=q.device)[code & 7]
    return (torch.where(code > 7, -size, size) * _power_of_two(scale.int() - 127).unsqueeze(-1)).view(q.shape[0], -1)[:, :d]


def _mix(z):
    """The output function of SplitMix64 on int64 (whose products and sums wrap around)."""
    z = (z ^ ((z >> 30) & 0x3FFFFFFFF)) * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = (z ^ ((z >> 27) & 0x1FFFFFFFFF)) * (0x94D049BB133111EB - (1 << 64))
    return z ^ ((z >> 31) & 0x1FFFFFFFF)


def _mix_host(z):
    z &= (1 << 64) - 1
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & ((1 << 64) - 1)
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & ((1 << 64) - 1)
    return z ^ (z >> 31)


def _draws(seed, t, tensor, n):
    """Two numbers of 0 .. 65535 for each of a tensor's n elements: for its mean, for its root."""
    key = _mix_host(_mix_host(seed + t * GOLDEN) + (tensor + 1) * GOLDEN)
    signed = lambda x: (x & ((1 << 64) - 1)) - ((x & (1 << 63)) << 1)
    pair = torch.arange((n + 1) // 2, dtype=torch.int64, device=DEV)
    word = _mix((pair + 1) * signed(GOLDEN) + signed(key))
    half = torch.stack([word & 0xFFFFFFFF, (word >> 32) & 0xFFFFFFFF], 1).view(-1)[:n]
    return half & 0xFFFF, half >> 16


def _in_8_bits(x, random, least):
    """Codes of 8-bit floats (4 bits of exponent, 3 of mantissa) and the factors' bytes; ``random`` of 0 .. 65535 decides between a value's two
    neighbours.  least: what is above zero stays so."""
    n = x.shape[0]
    x = _blocks(x)
    size = x.abs()
    a = size.amax(-1)
    part, power = torch.frexp(a)
    e = torch.where(a > 0, (power - 9 + (part > 7 / 8)).clamp(-117, 119), torch.full_like(power, -117))
    y = size * _power_of_two(-e).unsqueeze(-1)
    binade = (y.view(torch.int32) >> 23).clamp_min(121)  # of 2^-6 at least
    u = _blocks(random.float()) * 2.0 ** -16
    code = (binade - 121) * 8 + torch.floor(y * _power_of_two(130 - binade) + u).int()
    if least:
        code = torch.where(size > 0, code.clamp_min(1), code)
    code += 128 * torch.signbit(x)
    return code.to(torch.uint8).view(-1)[:n], (e + 127).to(torch.uint8)


def _from_8_bits(code, scale):
    n = code.shape[0]
    return (_blocks(code.view(torch.float8_e4m3fn).float()) * _power_of_two(scale.int() - 127).unsqueeze(-1)).view(-1)[:n]


# ---- inputs ----------------------------------------------------------------------------------------------------
def _tensors(case):
    """Sizes and weight decays of a model's tensors: weights, bias and the two vectors of a norm of each layer, the head's weights and bias."""
    d, classes = case["d"], case["rows"]
    return [x for _ in range(case["out"]) for x in ((d * d, DECAY), (d, 0.0), (d, 0.0), (d, 0.0))] + [(d * classes, DECAY), (classes, 0.0)]


def _places(case):
    """Where each tensor begins in the model's buffers, and where the last one's room ends."""
    at, places = 0, []
    step = 1 if case["pad"] else 64
    for n, _ in _tensors(case):
        places.append(at)
        at += -(-n // step) * step
    return places, at


def _prepare_adamw(case, gen):
    places, total = _places(case)
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    # gradients as a model has them: a tensor's columns (classes) differ by orders of magnitude, from one element to the next by a factor of ten
    rare = torch.exp(1.5 * torch.randn(1021, device=DEV, generator=gen)).repeat(total // 1021 + 1)[:total]
    g = 1e-3 * rare * torch.randn(total, device=DEV, generator=gen)
    m = 0.3 * (g + 1e-3 * rare * torch.randn(total, device=DEV, generator=gen))
    v = (1e-3 * rare).square_().mul_(0.5 + torch.rand(total, device=DEV, generator=gen))
    s = {"g": g.to(t), "p": 0.05 * torch.randn(total, device=DEV, generator=gen), "compute": torch.zeros(total, dtype=torch.bfloat16, device=DEV), "t": 999}
    if case["bits"] == 32:
        s.update(m=m, v=v)
        return s
    # codes of a tensor begin on a multiple of 32, whatever its values do
    sizes = [n for n, _ in _tensors(case)]
    where, room = [], 0
    for n in sizes:
        where.append(room)
        room += -(-n // BLOCK) * BLOCK
    s.update(where=where, m=torch.zeros(room, dtype=torch.uint8, device=DEV), v=torch.zeros(room, dtype=torch.uint8, device=DEV),
             m_scale=torch.zeros(room // BLOCK, dtype=torch.uint8, device=DEV), v_scale=torch.zeros(room // BLOCK, dtype=torch.uint8, device=DEV))
    half = torch.full((max(sizes),), 1 << 15, device=DEV)
    for n, a, w in zip(sizes, places, where):
        for name, x in (("m", m[a:a + n]), ("v", v[a:a + n].sqrt())):
            s[name][w:w + n], s[name + "_scale"][w // BLOCK:w // BLOCK + -(-n // BLOCK)] = _in_8_bits(x, half[:n], name == "v")
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n, d, out, call, pad = case["rows"], case["d"], case["out"], case["call"], case["pad"]
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = {"case": case, "seed": seed}
    if call == "adamw":
        s.update(_prepare_adamw(case, gen))
        return s
    if call in ("answer", "push"):
        # logits of a trained head: spread out, rows sure of their class to any degree; some classes left out by their bias
        y = torch.randint(0, out, (n,), device=DEV, generator=gen, dtype=torch.int32)
        z = torch.randn(n, out + pad, device=DEV, generator=gen).mul_(2.0)
        z.scatter_add_(1, y.long().unsqueeze(1), 20 * torch.rand(n, 1, device=DEV, generator=gen))
        s.update(logits=z.to(t)[:, :out], ids=y, bias=0.1 * torch.randn(out, device=DEV, generator=gen))
        s["bias"][1::97] = -math.inf
        s["ids"] = torch.where(y % 97 == 1, y - 1, y)
        s["mask"] = None if case["share"] == 1.0 else (torch.rand(n, device=DEV, generator=gen) < case["share"]).to(torch.uint8)
        if s["mask"] is not None:
            s["mask"][0] = 1
        if call == "answer":
            s.update(logp=torch.empty(n, device=DEV), entropy=torch.empty(n, device=DEV), norm=torch.empty(n, 2, device=DEV))
            if case["top"]:
                s.update(top_ids=torch.empty(n, case["top"], dtype=torch.int32, device=DEV), top_logp=torch.empty(n, case["top"], device=DEV))
            return s
        del z
        # what the forward pass has left
        kept = _answer(s, 0)
        s.update(logp=kept["logp"], entropy=kept["entropy"], norm=kept["norm"], g_logp=torch.randn(n, device=DEV, generator=gen) / n,
                 g_entropy=0.1 * torch.randn(n, device=DEV, generator=gen) / n, dlogits=torch.empty(n, out, dtype=t, device=DEV), dbias=torch.empty(out, device=DEV))
        return s
    x = torch.relu_(torch.randn(n, d + pad, device=DEV, generator=gen)) if call == "logits4" else torch.randn(n, d + pad, device=DEV, generator=gen)
    s["x"] = x.to(t)[:, :d]
    wide = (d + BLOCK - 1) // BLOCK
    s.update(q=torch.empty(n, 16 * wide, dtype=torch.uint8, device=DEV), scale=torch.empty(n, wide, dtype=torch.uint8, device=DEV))
    if call == "keep4":
        s["back"] = torch.empty(n, d, dtype=t, device=DEV)
        return s
    s["W_q"], s["W_scale"] = _in_4_bits(torch.randn(out, d, device=DEV, generator=gen) / math.sqrt(d))
    s.update(bias=0.1 * torch.randn(out, device=DEV, generator=gen), logits=torch.empty(n, out, dtype=t, device=DEV))
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
    if call == "adamw":
        if "tensors" not in s:  # the model's list, which a program makes once
            places, _ = _places(case)
            wheres = s.get("where", places)
            model = []
            for (n, decay), a, w in zip(_tensors(case), places, wheres):
                x = {"p": s["p"][a:a + n], "g": s["g"][a:a + n], "compute": s["compute"][a:a + n], "m": s["m"][w:w + n], "v": s["v"][w:w + n], "weight_decay": decay}
                if case["bits"] == 8:
                    b, c = w // BLOCK, -(-n // BLOCK)
                    x.update(m_scale=s["m_scale"][b:b + c], v_scale=s["v_scale"][b:b + c])
                model.append(x)
            s["tensors"] = g.gnntrain_adamw_tensors(model)
        s["t"] += 1
        g.gnntrain_adamw_step(s["tensors"], LR, B1, B2, EPS, s["t"], seed=s["seed"])
        if case["bits"] == 32:
            return {"p": s["p"], "compute": s["compute"], "m": s["m"], "v": s["v"]}
        return {"p": s["p"], "compute": s["compute"], "m": s["m"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn), "m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    if call == "answer":
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, g.gnntrain_logprobs_workspace_size(case["rows"], case["out"], case["top"]))
        top = {"top_ids": s["top_ids"], "top_logp": s["top_logp"]} if case["top"] else {}
        g.gnntrain_logprobs(s["logits"], s["bias"], s["ids"], s["mask"], s["logp"], s["entropy"], s["norm"], ws, **top)
        return {"logp": s["logp"], "entropy": s["entropy"], **top}
    if call == "push":
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, g.gnntrain_logprobs_grad_workspace_size(case["rows"], case["out"]))
        s["dbias"].zero_()
        g.gnntrain_logprobs_grad(s["logits"], s["bias"], s["ids"], s["mask"], s["logp"], s["entropy"], s["norm"], s["g_logp"], s["g_entropy"], s["dlogits"], ws, dbias=s["dbias"])
        return {"dlogits": s["dlogits"], "dbias": s["dbias"]}
    g.gnnstage_rows4_store(s["x"], s["q"], s["scale"])
    if call == "keep4":
        g.gnnstage_rows4_load(s["q"], s["scale"], s["back"])
        return {"rows": s["back"], "scale": s["scale"]}
    g.gnnstage_rows4_product(s["q"], s["scale"], s["W_q"], s["W_scale"], case["d"], s["logits"], bias=s["bias"])
    return {"logits": s["logits"]}


def _answer(s, top):
    """Rows that take no part: zeros, and no best classes."""
    rows, classes = s["logits"].shape
    at = slice(None) if s["mask"] is None else torch.nonzero(s["mask"]).squeeze(1)
    z = s["logits"][at].float() + s["bias"] + 0.0  # (minus zero becomes zero)
    y = s["ids"][at].long().unsqueeze(1)
    most = z.amax(1, keepdim=True)
    shifted = z - most
    e = torch.exp(shifted)
    total = e.sum(1, keepdim=True)
    log = torch.log(total)
    own_e = e.gather(1, y)
    others = e.scatter(1, y, 0.0).sum(1, keepdim=True)  # the class's own term apart: a sure row's result has no cancellation
    logp, entropy, norm = torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV), torch.zeros(rows, 2, device=DEV)
    logp[at] = torch.where(own_e > 0.5 * total, -torch.log1p(others / own_e), shifted.gather(1, y) - log).squeeze(1)
    entropy[at] = (log - torch.where(e > 0, e * shifted, torch.zeros_like(e)).sum(1, keepdim=True) / total).squeeze(1)
    norm[at] = torch.cat([most, log], 1)
    r = {"logp": logp, "entropy": entropy, "norm": norm}
    if top:
        # one whole number per class: larger for a larger logit, and of equals for the lower class
        bits = z.view(torch.int32).long()
        key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) - torch.arange(classes, device=DEV)
        best = key.topk(top, 1).indices
        r.update(top_ids=torch.full((rows, top), -1, dtype=torch.int32, device=DEV), top_logp=torch.full((rows, top), -math.inf, device=DEV))
        r["top_ids"][at] = best.int()
        r["top_logp"][at] = shifted.gather(1, best) - log
    return r


def run(state):
    s, case, call = state, state["case"], state["case"]["call"]
    if own:
        return _run_own(s)
    if call == "adamw":
        s["t"] += 1
        c1, c2 = 1 / (1 - B1 ** s["t"]), 1 / (1 - B2 ** s["t"])
        a1, a2 = (float(1 - torch.tensor(b, dtype=torch.float32)) for b in (B1, B2))
        places, _ = _places(case)
        for k, ((n, decay), a, w) in enumerate(zip(_tensors(case), places, s.get("where", places))):
            p, g, m, v = s["p"][a:a + n], s["g"][a:a + n].float(), s["m"][w:w + n], s["v"][w:w + n]
            if case["bits"] == 8:
                factors = [s[x][w // BLOCK:w // BLOCK + -(-n // BLOCK)] for x in ("m_scale", "v_scale")]
                m1 = B1 * _from_8_bits(m, factors[0]) + a1 * g
                # (a value next to a border is rounded like the definition's: each operation in fp32, the root to its nearest)
                root = (B2 * _from_8_bits(v, factors[1]).square() + a2 * g * g).double().sqrt().float()
                draws = _draws(s["seed"], s["t"], k, n)
                m[:], factors[0][:] = _in_8_bits(m1, draws[0], False)
                v[:], factors[1][:] = _in_8_bits(root, draws[1], True)
            else:
                m.mul_(B1).add_(a1 * g)
                v.mul_(B2).add_(a2 * g * g)
                m1, root = m, v.sqrt()
            p.mul_(1 - LR * decay).sub_(LR * c1 * m1 / (root * math.sqrt(c2) + EPS))
            s["compute"][a:a + n] = p
        if case["bits"] == 32:
            return {"p": s["p"], "compute": s["compute"], "m": s["m"], "v": s["v"]}
        return {"p": s["p"], "compute": s["compute"], "m": s["m"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn), "m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    if call == "answer":
        r = _answer(s, case["top"])
        del r["norm"]
        return r
    if call == "push":
        at = slice(None) if s["mask"] is None else torch.nonzero(s["mask"]).squeeze(1)
        column = lambda name: s[name][at].unsqueeze(1)
        y = s["ids"][at].long().unsqueeze(1)
        log = s["logits"][at].float() + s["bias"] - s["norm"][at, :1] - s["norm"][at, 1:]
        p = torch.exp(log)
        grad = -p * column("g_logp") - torch.where(p > 0, p * (log + column("entropy")), torch.zeros_like(p)) * column("g_entropy")
        # the class's own: 1 - p without the cancellation
        own_p, own_log = p.gather(1, y), column("logp")
        at_y = -torch.expm1(own_log) * column("g_logp") - torch.where(own_p > 0, own_p * (own_log + column("entropy")), torch.zeros_like(own_p)) * column("g_entropy")
        grad.scatter_(1, y, at_y)
        s["dlogits"].zero_()
        s["dlogits"][at] = grad.to(s["dlogits"].dtype)
        return {"dlogits": s["dlogits"], "dbias": grad.sum(0)}
    q, scale = _in_4_bits(s["x"].float())
    x = _from_4_bits(q, scale, case["d"])
    if call == "keep4":
        return {"rows": x.to(s["x"].dtype), "scale": scale}
    return {"logits": (x @ _from_4_bits(s["W_q"], s["W_scale"], case["d"]).t() + s["bias"]).to(s["logits"].dtype)}


# ---- 64 bits ---------------------------------------------------------------------------------------------------
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _factor_64(scale, block):
    return ((scale.long() + 896) << 52).view(torch.float64).repeat_interleave(block, dim=-1)


def _stored_64(x):
    """What 4 bits keep of fp64 rows, from the definition: the nearest of the block's sixteen numbers, of two as near the one with an even code."""
    n, d = x.shape
    wide = -(-d // BLOCK)
    full = torch.zeros(n, wide * BLOCK, dtype=torch.float64, device=DEV)
    full[:, :d] = x
    full = full.view(n, wide, BLOCK)
    largest = full.abs().amax(2, keepdim=True)
    power = torch.ceil(torch.log2((largest / 7).clamp_min(2.0 ** -120)) - 1e-13).long()
    step = ((power + 1023) << 52).view(torch.float64)
    size = full.abs() / step
    value = torch.zeros_like(size)
    for i in range(1, 8):
        border = (_E2M1[i - 1] + _E2M1[i]) / 2
        value = torch.where((size > border) | ((size == border) & (i % 2 == 0)), torch.full_like(size, _E2M1[i]), value)
    return (torch.copysign(value, full) * step).view(n, -1)[:, :d]


def _exact_adamw(s):
    case, t = s["case"], s["t"] + 1
    places, total = _places(case)
    r = {x: s[x].double().clone() for x in (("p", "m", "v") if case["bits"] == 32 else ("p",))}
    compute = torch.zeros(total, dtype=torch.float64, device=DEV)
    b1, b2, lr = (float(torch.tensor(x, dtype=torch.float32)) for x in (B1, B2, LR))
    for (n, decay), a, w in zip(_tensors(case), places, s.get("where", places)):
        g = s["g"][a:a + n].double()
        if case["bits"] == 32:
            m, v = r["m"][w:w + n], r["v"][w:w + n]
        else:
            of = lambda x: s[x][w:w + n].view(torch.float8_e4m3fn).double() * _factor_64(s[x + "_scale"][w // BLOCK:w // BLOCK + -(-n // BLOCK)], BLOCK)[:n]
            m, v = of("m"), of("v").square()
        m.copy_(b1 * m + (1 - b1) * g)
        v.copy_(b2 * v + (1 - b2) * g * g)
        r["p"][a:a + n] = r["p"][a:a + n] * (1 - lr * decay) - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + EPS)
        compute[a:a + n] = r["p"][a:a + n]
    r["compute"] = compute
    return r if case["bits"] == 32 else {**r, "m": None, "v": None, "m_scale": None, "v_scale": None}


def exact(case, seed):
    s = prepare(case, seed)
    n, d, out, call = case["rows"], case["d"], case["out"], case["call"]
    if call == "adamw":
        return _exact_adamw(s)
    if call == "keep4":
        return {"rows": _stored_64(s["x"].double()), "scale": None}
    step = max(1, 100000000 // out)
    if call == "logits4":
        code = torch.stack([s["W_q"] & 15, s["W_q"] >> 4], 2).view(out, -1).long()
        w = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=torch.float64, device=DEV)[code] * _factor_64(s["W_scale"], BLOCK)
        w = w[:, :d].t().contiguous()
        return {"logits": torch.cat([(_stored_64(s["x"][i:i + step].double()) @ w + s["bias"].double()).to(torch.float32 if n * out > 50000000 and case["dtype"] == "bf16" else torch.float64)
                                     for i in range(0, n, step)])}
    on = torch.ones(n, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] != 0
    dtype = torch.float32 if n * out > 200000000 else torch.float64  # of what is handed back: rounded once, the largest only
    logp, entropy = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    top_logp = torch.full((n, case["top"]), -math.inf, dtype=torch.float64, device=DEV)
    dlogits = torch.zeros(n, out, dtype=dtype, device=DEV) if call == "push" else None
    dbias = torch.zeros(out, dtype=torch.float64, device=DEV)
    for i in range(0, n, step):
        z = s["logits"][i:i + step].double() + s["bias"].double()
        y, take = s["ids"][i:i + step].long().unsqueeze(1), on[i:i + step].unsqueeze(1)
        log = z - torch.logsumexp(z, 1, keepdim=True)
        p = torch.exp(log)
        weighted = torch.where(p > 0, p * log, torch.zeros_like(p))
        H = -weighted.sum(1, keepdim=True)
        if call == "answer":
            logp[i:i + step] = (log.gather(1, y) * take).squeeze(1)
            entropy[i:i + step] = (H * take).squeeze(1)
            if case["top"]:
                top_logp[i:i + step] = torch.where(take, log.topk(case["top"], 1).values, torch.full_like(top_logp[i:i + step], -math.inf))
            continue
        gl, gh = s["g_logp"][i:i + step].double().unsqueeze(1), s["g_entropy"][i:i + step].double().unsqueeze(1)
        grad = (torch.zeros_like(p).scatter_(1, y, 1.0) - p) * gl - gh * (weighted + p * H)
        grad *= take
        dlogits[i:i + step] = grad
        dbias += grad.sum(0)
    if call == "push":
        return {"dlogits": dlogits, "dbias": dbias}
    return {"logp": logp, "entropy": entropy, **({"top_ids": None, "top_logp": top_logp} if case["top"] else {})}


def work(case):
    """Inputs read once, outputs written once (what an update changes is read and written)."""
    n, d, out, e = case["rows"], case["d"], case["out"], 2 if case["dtype"] == "bf16" else 4
    if case["call"] == "adamw":
        count = sum(x for x, _ in _tensors(case))
        return {"bytes": count * (8.0 + e + 2 + (16 if case["bits"] == 32 else 4 + 4 / BLOCK)), "flops": 15.0 * count}
    m = n if case["share"] == 1.0 else max(1, round(n * case["share"]))
    mask = n if case["share"] < 1.0 else 0
    if case["call"] == "answer":
        return {"bytes": float(m * (out * e + 4) + 4 * out + mask + n * (16 + 8 * case["top"])), "flops": 6.0 * m * out}
    if case["call"] == "push":
        return {"bytes": float(m * (out * e + 28) + n * out * e + 12 * out + mask), "flops": 10.0 * m * out}
    stored = 17 * ((d + BLOCK - 1) // BLOCK)
    if case["call"] == "keep4":
        return {"bytes": float(n * (2 * d * e + 2 * stored)), "flops": 4.0 * n * d}
    return {"bytes": float(n * d * e + 2 * n * stored + out * (stored + 4) + n * out * e), "flops": 2.0 * n * d * out}
