"""Workloads of the operators at the two ends of a trained layer stack, at the sizes of this repository's model shapes:

  embed     rows of an embedding table for tokens, times a factor (eagle3_embed), and the table's gradient (eagle3_embed_grad)
  norm      a branch added to the residual stream and the root-mean-square norm of the sum (eagle3_add_norm), the same in 8 bits with scales
            (eagle3_add_norm_codes), and the gradient (eagle3_add_norm_grad)
  distill   cross entropy of a student's logits against a teacher's largest ones (eagle3_distill), its gradient (eagle3_distill_grad), and both in one
            call (eagle3_distill_step)

`listed()` and `draw(rng)` give cases, `prepare(case, seed)` makes a case's inputs on the GPU, `run(state)` is one pass: in elementary torch
operations, or with `own` set through this package's entry points.  `work(case)` counts the bytes and operations that a pass cannot do
without, `exact(case, seed)` computes its results from the definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}
EPS = 1e-5                       # as in every shape
FP8_MOST, LEAST_SCALE = 448.0, 2.0 ** -100


def listed():
    return [
        # embeddings: the nodes of a draft tree onto the fp32 stream; a 70B-shaped prompt; the table's gradient of four training sequences of 2048 positions, some
        # of them padding; of a few fp32 rows of an odd width and a small vocabulary
        dict(name="embed-step", kind="embed", dtype="bf16", to="fp32", rows=60, dim=4096, vocab=128256, scale=1.0, padding=False, grad=False),
        dict(name="embed-prompt", kind="embed", dtype="bf16", to="bf16", rows=16384, dim=8192, vocab=128256, scale=1.0, padding=False, grad=False),
        dict(name="embed-grad", kind="embed", dtype="bf16", to="bf16", rows=8192, dim=4096, vocab=128256, scale=1.0, padding=True, grad=True),
        dict(name="embed-grad-small", kind="embed", dtype="fp32", to="fp32", rows=1021, dim=251, vocab=2048, scale=16.0, padding=True, grad=True),
        # norms: a decoding step of four sequences, a 70B-shaped branch onto the fp32 stream; a 70B-shaped prompt in bf16; 2048 rows in 8 bits for a product
        # with a scale to each 128 columns; the gradient of 8191 training positions, the stream's own gradient in fp32
        dict(name="norm-step", kind="norm", form="forward", dtype="bf16", stream="fp32", added=True, rows=4, dim=8192, group=0, packed=False),
        dict(name="norm-prompt", kind="norm", form="forward", dtype="bf16", stream="bf16", added=True, rows=16384, dim=8192, group=0, packed=False),
        dict(name="norm-codes", kind="norm", form="codes", dtype="bf16", stream="bf16", added=True, rows=2048, dim=8192, group=128, packed=False),
        dict(name="norm-grad", kind="norm", form="grad", dtype="bf16", stream="fp32", added=True, rows=8191, dim=4096, group=0, packed=False),
        # distillation: the loss alone of a few held-out positions over the whole vocabulary; its gradient for an odd number of positions and of draft tokens, half of
        # them a prompt's; a draft model's training step, the teacher's 64 largest logits mapped to the draft vocabulary; a step over the whole
        # vocabulary with the teacher's probabilities as they were (what is not among its 128 largest is left out)
        dict(name="distill-loss", kind="distill", form="loss", dtype="bf16", rows=16, vocab=128256, k=32, mapped=0, tail=True, temperature=1.0, masked=False),
        dict(name="distill-grad", kind="distill", form="grad", dtype="bf16", rows=2047, vocab=31999, k=10, mapped=0, tail=False, temperature=2.0, masked=True),
        dict(name="distill-draft", kind="distill", form="step", dtype="fp32", rows=2048, vocab=32000, k=64, mapped=128256, tail=False, temperature=1.0, masked=False),
        dict(name="distill-full", kind="distill", form="step", dtype="bf16", rows=2047, vocab=128256, k=128, mapped=0, tail=True, temperature=1.0, masked=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw(rng):
    kind, dtype = rng.choice(["embed", "norm", "distill"]), rng.choice(["bf16", "bf16", "fp32"])
    rows = _log(rng, 1, 16384)
    dim = rng.choice([256, 1000, 4096, 8192, _log(rng, 64, 8192), _log(rng, 64, 8192) | 1])
    vocab = rng.choice([2048, 32000, 128256, _log(rng, 500, 130000), _log(rng, 500, 130000) | 1])
    if kind == "embed":
        return dict(kind=kind, dtype=dtype, to=rng.choice(["bf16", "fp32"]), rows=rows, dim=dim, vocab=vocab, scale=rng.choice([1.0, 1.0, 16.0, 0.125]),
                    padding=rng.random() < 0.5, grad=rng.random() < 0.6)
    if kind == "norm":
        form, added = rng.choice(["forward", "codes", "grad", "grad"]), rng.random() < 0.75
        return dict(kind=kind, form=form, dtype=dtype, stream=rng.choice([dtype, "fp32"]) if added else dtype, added=added, rows=rows, dim=dim,
                    group=rng.choice([0, 128]) if form == "codes" else 0, packed=rng.random() < 0.3)
    return dict(kind=kind, form=rng.choice(["loss", "grad", "step", "step"]), dtype=dtype, rows=rows, vocab=vocab, k=_log(rng, 1, 256),
                mapped=rng.choice([0, 0, 4 * vocab]), tail=rng.random() < 0.4, temperature=rng.choice([1.0, 1.0, 0.7, 2.0]), masked=rng.random() < 0.3)


def draw(rng):
    """A case of the ranges above whose work, and whose plain form's, is that of the listed ones."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw(rng)
        plain = case["rows"] * case.get("vocab", case.get("dim", 0)) if case["kind"] != "embed" else case["vocab"] * case["dim"]     # elements of its 32-bit arrays
        if work(case)["bytes"] <= 0.9 * most and plain <= 600e6:
            return case


# ---------------------------------------------------------------- inputs
def _tokens(g, case):
    """Tokens as frequent as words are (the n-th most frequent one about 1 / n of the time), their ids in no order; -1 where there is padding."""
    V, R = case["vocab"], case["rows"]
    rank = ((V + 1) ** torch.rand(R, generator=g, device=DEV, dtype=torch.float64)).long().sub_(1).clamp_(0, V - 1)
    tokens = torch.randperm(V, generator=g, device=DEV)[rank].to(torch.int32)
    return torch.where(torch.rand(R, generator=g, device=DEV) < 0.1, torch.full_like(tokens, -1), tokens) if case["padding"] else tokens


def _rows(g, case, dtype):
    """[rows, dim], dense or the second half of rows twice as long."""
    R, d = case["rows"], case["dim"]
    return torch.randn(R, 2 * d, generator=g, device=DEV).to(dtype)[:, d:] if case["packed"] else torch.randn(R, d, generator=g, device=DEV).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, dt, R = case["kind"], DTYPES[case["dtype"]], case["rows"]
    st = {"kind": kind, "case": case}
    if kind == "embed":
        V, d = case["vocab"], case["dim"]
        st["tokens"] = _tokens(g, case)
        if case["grad"]:
            st["dy"] = (1e-3 * torch.randn(R, d, generator=g, device=DEV)).to(DTYPES[case["to"]])
        else:
            st["table"] = torch.randn(V, d, generator=g, device=DEV, dtype=torch.bfloat16).to(dt)
        return st
    if kind == "norm":
        h_dt = DTYPES[case["stream"]]
        st["gain"] = (1 + 0.1 * torch.randn(case["dim"], generator=g, device=DEV)).to(dt)
        if case["form"] == "grad":
            st["dy"] = _rows(g, case, dt)
            st["h"] = (3 * _rows(g, case, torch.float32)).to(h_dt)
            st["dh"] = _rows(g, case, h_dt) if case["added"] else None
        else:
            st["x"] = _rows(g, case, dt)
            st["residual"] = (3 * _rows(g, case, torch.float32)).to(h_dt) if case["added"] else None
        return st
    V, K = case["vocab"], min(case["k"], case["vocab"])
    z = 2.5 * torch.randn(R, V, generator=g, device=DEV)
    st["logits"] = z.to(dt)
    t = z.add_(torch.randn(R, V, generator=g, device=DEV))                 # the teacher: the student's opinion and more
    values, ids = t.topk(K, dim=1)
    st["t2d"] = None
    if case["mapped"]:                                                     # the teacher's vocabulary is larger than the student's
        M = case["mapped"]
        d2t = torch.randperm(M, generator=g, device=DEV)[:V].sort().values
        st["t2d"] = torch.full((M,), -1, dtype=torch.int32, device=DEV)
        st["t2d"][d2t] = torch.arange(V, dtype=torch.int32, device=DEV)
        other = torch.randint(0, M, ids.shape, generator=g, device=DEV)    # most of them not the student's
        ids = torch.where(torch.rand(ids.shape, generator=g, device=DEV) < 0.25, other, d2t[ids])
    st["ids"], st["values"] = ids.to(torch.int32), values
    st["lse"] = torch.logsumexp(t / case["temperature"], 1) if case["tail"] else None
    w = torch.full((R,), 1.0 / R, device=DEV)
    st["dloss"] = torch.where(torch.arange(R, device=DEV) < R // 2, torch.zeros_like(w), w) if case["masked"] else w
    if case["form"] == "grad":                                             # what the loss left for its backward pass: a row's largest logit and its sum
        s = st["logits"].float()
        m = s.amax(1)
        st["stats"] = torch.stack([m, ((s - m[:, None]) / case["temperature"]).exp_().double().sum(1).float()], 1)
    return st


# ---------------------------------------------------------------- one pass
def _embed(st):
    case, tok = st["case"], st["tokens"].long()
    V = case["vocab"]
    seen = (tok >= 0) & (tok < V)
    if case["grad"]:
        dy = torch.where(seen[:, None], st["dy"].float() * case["scale"], torch.zeros((), device=tok.device))
        return torch.zeros(V, case["dim"], device=tok.device).index_add_(0, tok.clamp(0, V - 1), dy).to(DTYPES[case["dtype"]])
    y = st["table"][tok.clamp(0, V - 1)].float() * case["scale"]
    return torch.where(seen[:, None], y, torch.zeros_like(y)).to(DTYPES[case["to"]])


def _norm(st):
    case = st["case"]
    gain = st["gain"].float()
    if case["form"] == "grad":
        h, gdy = st["h"].float(), st["dy"].float() * gain
        r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
        x = h * r
        dh = r * (gdy - x * (gdy * x).mean(1, keepdim=True))
        if st["dh"] is not None:
            dh = dh + st["dh"].float()
        return dh.to(st["dy"].dtype), dh.to(st["h"].dtype), (st["dy"].float() * x).sum(0).to(st["gain"].dtype)
    h = st["x"].float() if st["residual"] is None else st["x"].float() + st["residual"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * gain
    more = () if st["residual"] is None else (h.to(st["residual"].dtype),)
    if case["form"] == "forward":
        return (y.to(st["x"].dtype), *more)
    R, d = y.shape
    group = case["group"] or d
    y = torch.nn.functional.pad(y, (0, -d % group)).view(R, -1, group)
    scales = (y.abs().amax(2) / FP8_MOST).clamp(min=LEAST_SCALE)
    codes = (y / scales[..., None]).clamp(-FP8_MOST, FP8_MOST).to(torch.float8_e4m3fn)
    return (codes.view(torch.uint8).view(R, -1)[:, :d].contiguous().view(torch.float8_e4m3fn), scales, *more)


def _distill(st):
    case, T, V = st["case"], st["case"]["temperature"], st["case"]["vocab"]
    s = st["logits"].float()
    ids = st["ids"].long()
    if st["t2d"] is not None:
        ids = torch.where((ids >= 0) & (ids < len(st["t2d"])), st["t2d"].long()[ids.clamp(0, len(st["t2d"]) - 1)], -1)
    seen = (ids >= 0) & (ids < V)
    z = torch.where(seen, st["values"].float() / T, torch.full_like(st["values"], -math.inf))
    ids = ids.clamp(0, V - 1)
    if st["lse"] is not None:
        p = torch.exp(z - st["lse"][:, None])
    else:
        p = torch.exp(z - z.amax(1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
        p = p / p.sum(1, keepdim=True).clamp(min=1e-30)
    total = p.sum(1)
    if case["form"] == "grad":
        m, l = st["stats"].unbind(1)
        e = torch.exp((s - m[:, None]) / T)
    else:
        m = s.amax(1)
        e = torch.exp((s - m[:, None]) / T)
        l = e.sum(1)
        loss = total * l.log() + (p * (m[:, None] - s.gather(1, ids))).sum(1) / T
        if case["form"] == "loss":
            return loss, torch.stack([m, l], 1)
    g = st["dloss"] / T
    ds = (e * (g * total / l)[:, None]).scatter_add_(1, ids, -g[:, None] * p).to(st["logits"].dtype)
    return ds if case["form"] == "grad" else (loss, ds)


def run(state):
    st, kind, case = state, state["kind"], state["case"]
    if own:
        import paper_2503_01840_amd as E
        if kind == "embed":
            if case["grad"]:
                return E.eagle3_embed_grad(st["dy"], st["tokens"], case["vocab"], scale=case["scale"], dtype=DTYPES[case["dtype"]])
            return E.eagle3_embed(st["table"], st["tokens"], scale=case["scale"], dtype=DTYPES[case["to"]])
        if kind == "norm":
            if case["form"] == "grad":
                return E.eagle3_add_norm_grad(st["dy"], st["h"], st["gain"], EPS, dh=st["dh"])
            if case["form"] == "codes":
                return E.eagle3_add_norm_codes(st["x"], st["gain"], EPS, residual=st["residual"], group=case["group"])
            y = E.eagle3_add_norm(st["x"], st["gain"], EPS, residual=st["residual"])
            return y if case["added"] else (y,)
        teacher = dict(lse=st["lse"], t2d=st["t2d"], temperature=case["temperature"])
        if case["form"] == "loss":
            return E.eagle3_distill(st["logits"], st["ids"], st["values"], want_stats=True, **teacher)
        if case["form"] == "grad":
            return E.eagle3_distill_grad(st["dloss"], st["stats"], st["logits"], st["ids"], st["values"], **teacher)
        return E.eagle3_distill_step(st["dloss"], st["logits"], st["ids"], st["values"], **teacher)
    return (_embed if kind == "embed" else _norm if kind == "norm" else _distill)(st)


# ---------------------------------------------------------------- what a pass cannot do without
def _distinct(case):
    """How many different tokens _tokens gives, in the mean."""
    V = case["vocab"]
    n = torch.arange(1, V + 1, dtype=torch.float64)
    p = torch.log1p(1 / n) / math.log(V + 1)
    return float((1 - torch.exp(case["rows"] * torch.log1p(-p))).sum())


def work(case):
    kind, R, size = case["kind"], case["rows"], SIZE[case["dtype"]]
    if kind == "embed":
        d, V, to = case["dim"], case["vocab"], SIZE[case["to"]]
        live = 0.9 if case["padding"] else 1.0
        if case["grad"]:
            return {"bytes": int(live * R) * d * to + V * d * size + 4 * R, "flops": int(live * R) * d}
        return {"bytes": int(min(live * R, _distinct(case)) * d * size) + R * d * to + 4 * R, "flops": R * d}
    if kind == "norm":
        d, h = case["dim"], SIZE[case["stream"]]
        n, more = R * d, case["added"]
        if case["form"] == "grad":
            out = h + (size if size != h else 0)
            return {"bytes": n * (size + h + h * more + out) + 2 * d * size, "flops": 9 * n}
        y = size if case["form"] == "forward" else 1
        scales = 0 if case["form"] == "forward" else 4 * R * (-(-d // case["group"]) if case["group"] else 1)
        return {"bytes": n * (size + 2 * h * more + y) + scales + d * size, "flops": 5 * n}
    V, K = case["vocab"], min(case["k"], case["vocab"])
    live = R - R // 2 if case["masked"] and case["form"] == "grad" else R
    teacher = live * K * 8 + (4 * live if case["tail"] else 0) + (4 * min(case["mapped"], live * K))
    moved = {"loss": R * V, "grad": (live + R) * V, "step": 2 * R * V}[case["form"]]
    few = {"loss": 12 * R, "grad": 4 * R + 8 * live, "step": 8 * R}[case["form"]]
    return {"bytes": moved * size + teacher + few, "flops": {"loss": 3, "grad": 3, "step": 5}[case["form"]] * live * V}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "embed":
        V, d, tok = case["vocab"], case["dim"], st["tokens"].long()
        at = torch.nonzero((tok >= 0) & (tok < V))[:, 0]
        if not case["grad"]:
            y = torch.zeros(case["rows"], d, dtype=torch.float64, device=DEV)
            y[at] = st["table"][tok[at]].double() * case["scale"]
            return y
        # the sum over a token's rows: rows ordered by token, a running sum over blocks of columns, its differences at the ends of every token's rows
        order = tok[at].argsort(stable=True)
        ids, n = torch.unique_consecutive(tok[at][order], return_counts=True)
        out = torch.zeros(V, d, dtype=torch.float64, device=DEV)
        if len(ids):
            total = st["dy"][at][order].double().cumsum(0)
            total = total[n.cumsum(0) - 1]
            out[ids] = case["scale"] * torch.cat([total[:1], total[1:] - total[:-1]])
        return out
    if kind == "norm":
        d, gain = case["dim"], st["gain"].double()
        if case["form"] == "grad":
            h, dy = st["h"].double(), st["dy"].double()
            s = (h * h).sum(1, keepdim=True) / d + EPS
            # the product's derivative: y_i = g_i h_i s^(-1/2), ds / dh_j = 2 h_j / d
            dh = gain * dy / s.sqrt() - h * (dy * gain * h).sum(1, keepdim=True) / (d * s ** 1.5)
            dgain = (dy * h / s.sqrt()).sum(0)
            if st["dh"] is not None:
                dh = dh + st["dh"].double()
            return dh, dh, dgain
        h = st["x"].double()
        if st["residual"] is not None:
            h = h + st["residual"].double()
        y = gain * h / (h.pow(2).sum(1, keepdim=True) / d + EPS).sqrt()
        more = () if st["residual"] is None else (h,)
        if case["form"] == "forward":
            return (y, *more)
        group = case["group"] or d
        codes, scales = [], []
        for part in y.split(group, 1):
            scale = torch.maximum(part.abs().max(1).values / FP8_MOST, torch.full((case["rows"],), LEAST_SCALE, dtype=torch.float64, device=DEV))
            q = part / scale[:, None]
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)        # codes: the nearest values of the type, the even one at ties
            codes.append(torch.round(q / step) * step)
            scales.append(scale)
        return (torch.cat(codes, 1), torch.stack(scales, 1), *more)
    T, V, R = case["temperature"], case["vocab"], case["rows"]
    ids = st["ids"].long()
    if case["mapped"]:
        ids = st["t2d"].long()[ids]
    target = torch.zeros(R, ids.shape[1], dtype=torch.float64, device=DEV)
    weight = torch.where(ids >= 0, st["values"].double() / T, -math.inf)
    if st["lse"] is not None:
        target = torch.exp(weight - st["lse"].double()[:, None])
    else:
        target = torch.softmax(weight, 1).nan_to_num(0.0)                                       # rows whose every id is another vocabulary's: no targets
    ids = ids.clamp(min=0)
    losses, grads, stats = [], [], []
    for r0 in range(0, R, 512):                                                                 # some rows at a time, for the memory
        s = st["logits"][r0:r0 + 512].double() / T
        if case["form"] == "grad":
            m, l = st["stats"][r0:r0 + 512].double().unbind(1)
            logq = s - (m / T + l.log())[:, None]
        else:
            logq = torch.log_softmax(s, 1)
            m = s.amax(1)
            stats.append(torch.stack([m * T, torch.exp(torch.logsumexp(s, 1) - m)], 1))
        p, at = target[r0:r0 + 512], ids[r0:r0 + 512]
        losses.append(-(p * logq.gather(1, at)).sum(1))
        if case["form"] != "loss":
            dense = torch.zeros_like(s).scatter_add_(1, at, p)
            d = logq.exp_().mul_(p.sum(1, keepdim=True)).sub_(dense).mul_(st["dloss"][r0:r0 + 512, None].double() / T)
            grads.append(d.to(torch.float32) if R * V > 1 << 28 else d)
    if case["form"] == "loss":
        return torch.cat(losses), torch.cat(stats)
    return torch.cat(grads) if case["form"] == "grad" else (torch.cat(losses), torch.cat(grads))
