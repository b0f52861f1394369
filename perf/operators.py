"""Workloads of the operators around a paged key-value cache, at the sizes of this repository's model shapes:

  rope       rotary positions of queries and keys (eagle3_rope), and their gradient (eagle3_rope_grad)
  append     new keys and values written into the pages of their sequences, as they are or in 8 bits (eagle3_paged_append)
  read       rows of paged sequences read back into dense arrays (eagle3_paged_read)
  attention  one new token of every sequence over its paged keys and values (eagle3_paged_attention)

`listed()` and `draw(rng)` give cases, `prepare(case, seed)` makes a case's inputs on the GPU, `run(state)` is one pass: in elementary torch
operations, or with `own` set through this package's entry points.  `work(case)` counts the bytes and operations that a pass cannot do
without, `exact(case, seed)` computes its results from the definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
THETA = 5e5                      # as in the 8B and 70B shapes
PARTS = dict(factor=8.0, low=1.0, high=4.0, original_len=8192)     # contexts stretched eightfold over 8192 positions


def listed():
    return [
        # rotations: the rows of a decoding step of four sequences at far positions; a 70B-shaped prompt whose q and k lie in the product's
        # q|k|v rows; a training step's gradient, pairs of neighbours, half of each head, an odd number of rows
        dict(name="rope-step", kind="rope", dtype="bf16", rows=4, heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, scaling="parts",
             grad=False, packed=False, far=131072),
        dict(name="rope-prompt", kind="rope", dtype="bf16", rows=16384, heads=64, kv_heads=8, dim=128, rot=128, interleaved=False,
             scaling="parts", grad=False, packed=True, far=32768),
        dict(name="rope-grad", kind="rope", dtype="fp32", rows=2047, heads=32, kv_heads=8, dim=128, rot=64, interleaved=True,
             scaling="linear", grad=True, packed=False, far=2048),
        # writes: one row of each of 64 sequences, and a ragged batch of prompts, into 8 bits
        dict(name="append-step", kind="append", dtype="fp8", batch=64, rows=1, ragged=False, kv_heads=8, dim=128, page=64, packed=True),
        dict(name="append-prompts", kind="append", dtype="fp8", batch=7, rows=2048, ragged=True, kv_heads=8, dim=128, page=64, packed=True),
        # reads: prompts kept in 8 bits and wanted as a dense cache again; a few rows of small fp32 sequences in odd pages
        dict(name="read-prompts", kind="read", dtype="fp8", batch=16, rows=2048, ragged=True, kv_heads=8, dim=128, page=64, packed=False),
        dict(name="read-small", kind="read", dtype="fp32", batch=3, rows=77, ragged=True, kv_heads=4, dim=64, page=13, packed=False),
        # attention of the new token: a short 8B-shaped sequence; the ragged batch of 64 in 16 bits, and in 8 with three idle places;
        # a long 70B-shaped context in 8 bits; a tiny fp32 model with as many key heads as query heads
        dict(name="attention-short", kind="attention", dtype="bf16", batch=1, lo=517, hi=517, idle=0, heads=32, kv_heads=8, dim=128, page=16),
        dict(name="attention-batch", kind="attention", dtype="bf16", batch=64, lo=512, hi=2048, idle=0, heads=32, kv_heads=8, dim=128, page=16),
        dict(name="attention-batch-fp8", kind="attention", dtype="fp8", batch=64, lo=512, hi=2048, idle=3, heads=32, kv_heads=8, dim=128, page=64),
        dict(name="attention-long", kind="attention", dtype="fp8", batch=1, lo=131071, hi=131071, idle=0, heads=64, kv_heads=8, dim=128, page=64),
        dict(name="attention-tiny", kind="attention", dtype="fp32", batch=5, lo=1, hi=333, idle=0, heads=4, kv_heads=4, dim=64, page=32),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw(rng):
    kind = rng.choice(["rope", "append", "read", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "fp32"] if kind == "rope" else ["bf16", "fp8", "fp8", "fp32"])
    heads, kv_heads = rng.choice([(4, 4), (4, 2), (8, 1), (32, 8), (64, 8), (32, 32), (24, 1), (28, 4)])
    dim = rng.choice([64, 128])
    page = rng.choice([1, 7, 16, 16, 32, 64, 64, 100, 128, 256])
    if kind == "rope":
        return dict(kind=kind, dtype=dtype, rows=_log(rng, 1, 16384), heads=heads, kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim, dim // 2, dim - 6]),
                    interleaved=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "parts"]), grad=rng.random() < 0.4,
                    packed=rng.random() < 0.5, far=_log(rng, 128, 131072))
    batch = _log(rng, 1, 64)
    if kind == "attention":
        lo, hi = sorted((_log(rng, 1, 131072), _log(rng, 1, 131072)))
        return dict(kind=kind, dtype=dtype, batch=batch, lo=lo, hi=hi, idle=rng.choice([0, 0, 1]) if batch > 1 else 0, heads=heads, kv_heads=kv_heads,
                    dim=dim, page=page)
    return dict(kind=kind, dtype=dtype, batch=batch, rows=_log(rng, 1, 16384), ragged=rng.random() < 0.6, kv_heads=kv_heads, dim=dim, page=page,
                packed=rng.random() < 0.5)


def draw(rng):
    """A case of the ranges above whose work, and whose plain form's, is that of the listed ones."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw(rng)
        plain = case["batch"] * case["hi"] * case["kv_heads"] * case["dim"] * 4 if case["kind"] == "attention" else 0    # keys as the plain form holds them
        if work(case)["bytes"] <= 0.75 * most and plain <= 2 << 30:
            return case


def _lengths(n, lo, hi):
    """n lengths spread evenly over lo..hi."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _case_lengths(case):
    """Sequence lengths (attention) or rows of each sequence (append, read), before their order is shuffled."""
    if case["kind"] == "attention":
        return _lengths(case["batch"] - case["idle"], case["lo"], case["hi"]) + [0] * case["idle"]
    lo = (case["rows"] + 3) // 4 if case["ragged"] else case["rows"]
    return _lengths(case["batch"], lo, case["rows"])


# ---------------------------------------------------------------- inputs
def _frequencies(rot, scaling):
    """fp64 angle per position of every pair."""
    f = THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if scaling == "linear":
        return f / PARTS["factor"]
    if scaling == "parts":
        turns = PARTS["original_len"] * f / (2 * math.pi)
        w = ((turns - PARTS["low"]) / (PARTS["high"] - PARTS["low"])).clamp(0, 1)
        return f * (w + (1 - w) / PARTS["factor"])
    return f


def _rows(g, rows, heads, dim, dtype, packed, others):
    """[rows, heads, dim], dense or the first heads of rows that hold `others` more."""
    x = torch.randn(rows, heads + (others if packed else 0), dim, generator=g, device=DEV).to(dtype)
    return x[:, :heads]


def _exponents(x):
    """The smallest e >= -110 with |x| <= 448 * 2^e along the last dimension."""
    f, e = torch.frexp(x.float().abs().amax(-1))
    return (e - 9 + (f > 0.875)).clamp(min=-110)


def _codes(x):
    """x as 8-bit codes and the exponents of their scales, a scale for each row of the last dimension."""
    e = _exponents(x)
    scale = ((127 - e) << 23).to(torch.int32).view(torch.float32)          # 2^-e
    return (x.float() * scale[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(codes, exps):
    """The fp32 values of rows in 8 bits."""
    return codes.float() * (exps.to(torch.int32) << 23).view(torch.float32)[..., None]


def _take(pool, exps, at):
    """Rows of a cache as fp32 values."""
    if exps is None:
        return pool[at].float()
    return _values(pool.view(torch.uint8)[at].view(pool.dtype), exps[at])


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    st = {"kind": kind, "case": case}
    if kind == "rope":
        H, Hkv, d, T, dt = case["heads"], case["kv_heads"], case["dim"], case["rows"], DTYPES[case["dtype"]]
        x = _rows(g, T, H + Hkv, d, dt, case["packed"], Hkv)
        st["q"], st["k"] = (x[:, :H], x[:, H:]) if case["packed"] else (x[:, :H].contiguous(), x[:, H:].contiguous())
        first = int(torch.randint(0, max(1, case["far"] - T), (1,), generator=g, device=DEV))
        run_of_rows = torch.arange(T, device=DEV) + first if T > 64 else torch.randint(0, case["far"], (T,), generator=g, device=DEV)
        st["positions"] = run_of_rows.to(torch.int32)
        st["frequencies"] = _frequencies(case["rot"], case["scaling"])
        st["amplitude"] = 0.1 * math.log(PARTS["factor"]) + 1 if case["scaling"] == "parts" else 1.0
        if own:                                                            # the handle that a program keeps for its model
            import paper_2503_01840_amd as E
            st["rope"] = E.Rope(case["rot"], THETA, interleaved=case["interleaved"], scaling=case["scaling"], amplitude=st["amplitude"], device=DEV, **PARTS)
        return st
    # a pool with room for every sequence, its pages dealt out in random order
    Hkv, d, page, batch, dt = case["kv_heads"], case["dim"], case["page"], case["batch"], DTYPES[case["dtype"]]
    order = torch.randperm(batch, generator=g, device=DEV).cpu().tolist()
    lens = [_case_lengths(case)[i] for i in order]
    start = torch.randint(0, 2 * page, (batch,), generator=g, device=DEV).cpu().tolist() if kind != "attention" else [0] * batch
    used = [-(-(s + n) // page) for s, n in zip(start, lens)]
    room = [-(-n // page) + 2 for n in lens]                               # also for those that start late
    n_pages, max_pages = sum(room), max(room)
    free = torch.randperm(n_pages, generator=g, device=DEV).cpu()
    table = torch.zeros(batch, max_pages, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = free[at:at + n]
        at += n
    st["page_table"] = table.to(DEV)
    for n in ("k", "v"):
        pool = torch.randn(n_pages, page, Hkv, d, generator=g, device=DEV)
        st[n], st[n + "_exp"] = _codes(pool.bfloat16()) if case["dtype"] == "fp8" else (pool.to(dt), None)
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    st["start"] = torch.tensor(start, dtype=torch.int32, device=DEV)
    rows_dt = torch.bfloat16 if case["dtype"] == "fp8" else dt
    if kind == "attention":
        st["q"] = (2 * torch.randn(batch, case["heads"], d, generator=g, device=DEV)).to(rows_dt)
        st["max_len"] = case["hi"]
    else:
        st["n_rows"] = n_rows = sum(lens)
        st["first_row"] = st["lens"].cumsum(0, dtype=torch.int32) - st["lens"]
        x = _rows(g, n_rows, 2 * Hkv, d, rows_dt, case["packed"], 4 * Hkv)
        if kind == "append":
            st["k_new"], st["v_new"] = (x[:, :Hkv], x[:, Hkv:]) if case["packed"] else (x[:, :Hkv].contiguous(), x[:, Hkv:].contiguous())
        else:
            st["out"] = tuple(torch.zeros(n_rows, Hkv, d, dtype=rows_dt, device=DEV) for _ in range(2))
    if own:                                                                # the cache as a program holds it
        import paper_2503_01840_amd as E
        st["cache"] = E.PagedKVCache(st["k"], st["v"], st["page_table"], st["k_exp"], st["v_exp"])
    return st


# ---------------------------------------------------------------- one pass
def _rotate(x, st, sign):
    """x [rows, heads, dim] rotated in its first `rot` dimensions."""
    case = st["case"]
    rot = case["rot"]
    angle = sign * st["positions"].double()[:, None, None] * st["frequencies"]
    cos, sin = ((st["amplitude"] * t).float() for t in (angle.cos(), angle.sin()))
    y = x.float().clone()
    if case["interleaved"]:
        a, b = x[..., 0:rot:2].float(), x[..., 1:rot:2].float()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :rot // 2].float(), x[..., rot // 2:rot].float()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return y.to(x.dtype)


def _places(st):
    """Page and offset of every row of the sequences' rows, in order."""
    lens = st["lens"].long()
    seq = torch.repeat_interleave(torch.arange(len(lens), device=lens.device), lens, output_size=st["n_rows"])
    row = torch.arange(len(seq), device=lens.device) - st["first_row"].long()[seq]
    pos = st["start"].long()[seq] + row
    page = st["case"]["page"]
    return st["page_table"].long()[seq, pos // page], pos % page


def _attend(st):
    q, table, lens = st["q"].float(), st["page_table"].long(), st["lens"].long()
    B, H, d = q.shape
    page, Hkv = st["case"]["page"], st["case"]["kv_heads"]
    pos = torch.arange(st["max_len"], device=q.device)
    pages, off = table[:, pos // page], (pos % page).expand(B, -1)                           # [B, L]
    k, v = (_take(st[n], st[n + "_exp"], (pages, off)).transpose(1, 2).contiguous() for n in ("k", "v"))
    seen = (pos < lens[:, None])[:, None, None]                                              # [B, 1, 1, L]
    s = torch.matmul(q.view(B, Hkv, H // Hkv, d), k.transpose(2, 3).contiguous()) / math.sqrt(d)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    m = s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(seen.transpose(2, 3), v, torch.zeros_like(v))) / l.clamp(min=1e-30)
    return o.reshape(B, H, d).to(st["q"].dtype), (m + l.log()).reshape(B, H)


def run(state):
    st, kind, case = state, state["kind"], state["case"]
    if own:
        import paper_2503_01840_amd as E
        if kind == "rope":
            turn = E.eagle3_rope_grad if case["grad"] else E.eagle3_rope
            return turn(st["rope"], st["positions"], st["q"], st["k"])
        if kind == "append":
            E.eagle3_paged_append(st["cache"], st["k_new"], st["v_new"], st["start"], st["lens"], rows=case["rows"], row_start=st["first_row"])
            return {n: st[n] for n in ("k", "v", "k_exp", "v_exp")}
        if kind == "read":
            return E.eagle3_paged_read(st["cache"], st["start"], st["lens"], rows=case["rows"], row_start=st["first_row"], out=st["out"])
        return E.eagle3_paged_attention(st["cache"], st["q"], st["lens"], st["max_len"], want_lse=True)
    if kind == "rope":
        sign = -1 if case["grad"] else 1
        return _rotate(st["q"], st, sign), _rotate(st["k"], st, sign)
    if kind == "attention":
        return _attend(st)
    at = _places(st)
    for n in ("k", "v"):
        if kind == "read":
            st["out"][n == "v"][:] = _take(st[n], st[n + "_exp"], at)
        elif case["dtype"] == "fp8":
            codes, st[n + "_exp"][at] = _codes(st[n + "_new"])
            st[n].view(torch.uint8)[at] = codes.view(torch.uint8)
        else:
            st[n][at] = st[n + "_new"]
    return st["out"] if kind == "read" else {n: st[n] for n in ("k", "v", "k_exp", "v_exp")}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, d = case["kind"], case["dim"]
    size = {"bf16": 2, "fp32": 4, "fp8": 1}[case["dtype"]]
    if kind == "rope":
        n = case["rows"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * n * d * size + 4 * case["rows"], "flops": 3 * n * case["rot"]}
    total = sum(_case_lengths(case))
    dense, cached = (2, 1) if case["dtype"] == "fp8" else (size, size)
    cached_row = case["kv_heads"] * (d * cached + (1 if case["dtype"] == "fp8" else 0))
    if kind == "attention":
        H, B = case["heads"], case["batch"]
        return {"bytes": 2 * total * cached_row + 2 * B * H * d * dense + 4 * B * H, "flops": 4 * total * H * d}
    return {"bytes": 2 * total * (cached_row + case["kv_heads"] * d * dense), "flops": 2 * total * case["kv_heads"] * d}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        # each pair as a complex number, times A e^{i t}
        rot, T = case["rot"], case["rows"]
        t = st["positions"].double()[:, None] * st["frequencies"] * (-1 if case["grad"] else 1)
        turn = torch.polar(torch.full_like(t, st["amplitude"]), t)[:, None]
        outs = []
        for x in (st["q"].double(), st["k"].double()):
            shape = x.shape[:2] + ((rot // 2, 2) if case["interleaved"] else (2, rot // 2))
            pair = x[..., :rot].reshape(shape)
            pair = pair if case["interleaved"] else pair.transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            z = z if case["interleaved"] else z.transpose(2, 3)
            outs.append(torch.cat([z.reshape(T, -1, rot), x[..., rot:]], -1))
        return tuple(outs)

    def value(x, at):
        rows = st[x].flatten(0, 1)
        if case["dtype"] != "fp8":
            return rows[at].double()
        return rows.float()[at].double() * torch.exp2(st[x + "_exp"].flatten(0, 1)[at].double() - 127)[..., None]

    table, page, lens, start = st["page_table"].cpu(), case["page"], st["lens"].cpu().tolist(), st["start"].cpu().tolist()

    def rows_of(b, first, n):
        pos = torch.arange(first, first + n)
        return (table[b, pos // page].long() * page + pos % page).to(DEV)

    if kind == "attention":
        Hkv, H, d = case["kv_heads"], case["heads"], case["dim"]
        out = torch.zeros(case["batch"], H, d, dtype=torch.float64, device=DEV)
        lse = torch.full((case["batch"], H), -math.inf, dtype=torch.float64, device=DEV)
        for b, n in enumerate(lens):
            if n == 0:
                continue
            at = rows_of(b, 0, n)
            k, v = (value(x, at) for x in ("k", "v"))
            for h in range(Hkv):
                heads = slice(h * H // Hkv, (h + 1) * H // Hkv)
                s = st["q"][b, heads].double() @ k[:, h].T.contiguous() * d ** -0.5
                lse[b, heads] = torch.logsumexp(s, 1)
                out[b, heads] = torch.exp(s - lse[b, heads, None]) @ v[:, h]
        return out, lse
    if kind == "read":
        outs = []
        for x in ("k", "v"):
            outs.append(value(x, torch.cat([rows_of(b, s, n) for b, (s, n) in enumerate(zip(start, lens))])))
        return tuple(outs)
    # append: whole pools; 8-bit codes as the nearest values of the type, the even one at ties
    at = torch.cat([rows_of(b, s, n) for b, (s, n) in enumerate(zip(start, lens))])
    outs = {"k_exp": None, "v_exp": None}
    for x in ("k", "v"):
        new = st[x + "_new"].double()
        if case["dtype"] == "fp8":
            e = torch.ceil(torch.log2(new.abs().amax(-1) / 448)).clamp(min=-110)
            new = new / torch.exp2(e)[..., None]
            step = torch.exp2(torch.floor(torch.log2(new.abs().clamp(min=2.0 ** -6))) - 3)
            new = torch.round(new / step) * step
        pool = st[x].double().flatten(0, 1)
        pool[at] = new
        outs[x] = pool.view(st[x].shape)
    return outs
