"""Attention of single tokens over paged caches on the GPU against the definition in 64 bits, and the operators around a paged cache together."""
import math

import numpy as np
import pytest
import torch

import eagle3_synth as S
import paper_2503_01840_amd as E
import pipeline as PL
from test_gpu_edges import SMALL
from test_gpu_paged import DEV, ROW, i32, make_cache, raw, value

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def _rows(c, which):
    """A pool as fp64 slots [n_slots, Hkv, d]."""
    pool, exps = raw(getattr(c, which)), raw(getattr(c, which + "_exp"))
    x = value(pool, exps) if exps is not None else pool.double()
    return x.flatten(0, 1)


def _check(c, table, q, lens, got, lse, scale=None):
    """Every head of every sequence.  Of a sequence whose keys give |scale q_i k_i| sums of at most a: scores are off by es = (d + 2) 2^-24 a
    (sums of d products in 32 bits), their maximum and logarithm by as much again; weights by 2 es, 2^-16 (bf16 cache: two terms of
    8 bits) and a few units of exp2; their sums, and joined parts', by a unit for every key."""
    K, V = _rows(c, "k"), _rows(c, "v")
    B, H, d = q.shape
    Hkv, page = K.shape[1], c.k.shape[1]
    q64 = q.cpu().double()
    scale = d ** -0.5 if scale is None else scale
    for b, n in enumerate(lens):
        if n == 0:
            assert bool((got[b] == 0).all()) and bool((lse[b] == -INF).all())
            continue
        pos = torch.arange(n)
        at = table[b].long()[pos // page] * page + pos % page
        k, v = K[at].repeat_interleave(H // Hkv, 1), V[at].repeat_interleave(H // Hkv, 1)         # [n, H, d]
        s = scale * (q64[b] * k).sum(-1)
        a = (abs(scale) * (q64[b].abs() * k.abs()).sum(-1)).amax(0)                               # [H]
        ref_lse = torch.logsumexp(s, 0)
        p = torch.exp(s - ref_lse)
        ref = (p[..., None] * v).sum(0)
        es = (d + 2) * 2.0 ** -24 * a
        weight = 4 * es + 2.0 ** -16 * (q.dtype == torch.bfloat16) + (n + 64) * 2.0 ** -24
        tol = weight[:, None] * (p[..., None] * v.abs()).sum(0) * 2 + 1e-30
        if q.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (ref.abs() + tol)
        err = (got[b].cpu().double() - ref).abs()
        assert bool((err <= tol).all()), (b, n, float((err / tol).max()))
        lse_err = (lse[b].cpu().double() - ref_lse).abs()
        assert bool((lse_err <= 2 * es + (n + 64) * 2.0 ** -24 + 2.0 ** -21 * ref_lse.abs()).all()), (b, n, float(lse_err.max()))


def _run(dtype, H, Hkv, d, page, lens, seed, max_len=None, q_scale=2.0, scale=None, packed=False):
    g = torch.Generator().manual_seed(seed)
    max_pages = -(-max(max(lens), max_len or 1) // page) + 1
    c, table = make_cache(dtype, len(lens), max_pages, page, Hkv, d, g)
    if dtype == "fp8":                                       # values of ordinary size: exponents around those of a normal row
        for e in (c.k_exp, c.v_exp):
            e.sub_(118).clamp_(-5, 5).add_(119)
        signs = torch.randint(0, 2, c.k.shape, generator=g, dtype=torch.uint8).to(DEV) << 7
        c.k.view(torch.uint8).bitwise_or_(signs)
        c.v.view(torch.uint8).bitwise_or_(signs.flip(0))
    x = (q_scale * torch.randn(len(lens), H * (2 if packed else 1), d, generator=g)).to(ROW[dtype]).to(DEV)
    q = x[:, :H]
    n = i32(lens).to(DEV)
    out, lse = E.eagle3_paged_attention(c, q, n, max_len or max(max(lens), 1), scale=scale, want_lse=True)
    _check(c, table, q, lens, out, lse, scale)
    assert torch.equal(out, E.eagle3_paged_attention(c, q, n, max_len or max(max(lens), 1), scale=scale))
    return c, table, q, n, out, lse


HEADS = [(4, 4), (8, 1), (32, 8), (6, 2), (24, 1), (40, 2), (64, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", HEADS)
def test_head_layouts(dtype, d, H, Hkv):
    _run(dtype, H, Hkv, d, 16, [1, 77, 0, 300, 33], H + d)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("page", [1, 2, 7, 16, 31, 64, 100, 256])
def test_page_sizes_and_lengths_around_tiles(dtype, page):
    _run(dtype, 8, 2, 128, page, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513], page)


@pytest.mark.parametrize("dtype,H,Hkv,d,lens", [("bf16", 32, 8, 128, [5000]), ("fp8", 64, 8, 128, [20011]), ("fp32", 4, 4, 64, [9001, 3]),
                                                ("bf16", 8, 8, 64, [1, 12001, 0, 700]), ("fp8", 4, 1, 64, [30000, 1]), ("fp8", 16, 1, 128, [40003]),
                                                ("fp32", 32, 1, 128, [4097, 4096]), ("bf16", 2, 1, 128, [1023, 1024, 1025, 2047, 2048, 2049])])
def test_long_sequences(dtype, H, Hkv, d, lens):
    _run(dtype, H, Hkv, d, 64, lens, lens[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("B,bound", [(1, 4096), (3, 100000), (64, 2048), (200, 600)])
def test_bounds_ahead_of_the_lengths(dtype, B, bound):
    """A host bound above every length, as a program keeps it; lengths are clamped to it."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 500, (B,), generator=g).tolist()
    lens[0] = 499
    max_pages = -(-bound // 16)
    c, table = make_cache(dtype, B, 40, 16, 2, 64, g)
    wide = torch.zeros(B, max_pages, dtype=torch.int32)
    wide[:, :min(40, max_pages)] = table[:, :max_pages]
    if dtype == "fp8":
        for e in (c.k_exp, c.v_exp):
            e.clamp_(117, 120)
    c = E.PagedKVCache(c.k, c.v, wide.to(DEV), c.k_exp, c.v_exp)
    q = torch.randn(B, 4, 64, generator=g).to(ROW[dtype]).to(DEV)
    out, lse = E.eagle3_paged_attention(c, q, i32(lens).to(DEV), bound, want_lse=True)
    _check(c, wide, q, lens, out, lse)
    more = i32([n if i % 2 else 2 ** 30 for i, n in enumerate(lens)]).to(DEV)        # clamped to a bound of 300
    less = i32([-5 if n % 3 == 0 else n for n in lens]).to(DEV)
    out, lse = E.eagle3_paged_attention(c, q, more, 300, want_lse=True)
    _check(c, wide, q, [min(n, 300) if i % 2 else 300 for i, n in enumerate(lens)], out, lse)
    out, lse = E.eagle3_paged_attention(c, q, less, 500, want_lse=True)
    _check(c, wide, q, [0 if n % 3 == 0 else n for n in lens], out, lse)


# more than 16 query heads to a KV head: two products of each operand, in parts and whole, in pages of either kind; a last tile of 1, 8, 16 heads
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("H,Hkv,d,page,lens", [(24, 1, 128, 16, [40000, 0, 30001]), (17, 1, 64, 20, [70001]), (64, 2, 64, 48, [20000, 17000]), (33, 1, 128, 24, [66000]),
                                               (96, 4, 64, 16, [700, 0, 33] * 28), (32, 1, 128, 7, [700, 16, 31] * 33)])
def test_many_query_heads_to_a_kv_head(dtype, H, Hkv, d, page, lens):
    _run(dtype, H, Hkv, d, page, lens, H)


# enough keys for a range to every wavefront, in pages of whole blocks of 16 keys and in others
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("page", [48, 20])
def test_ranges_of_wavefronts(dtype, page):
    _run(dtype, 16, 16, 64, page, [26000, 0, 25011], page)


# batches of more than one look at 64 lengths, with idle places: ranges of a workgroup, of a wavefront, and a workgroup to each sequence
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("B,hi", [(65, 1500), (130, 1500), (300, 1500), (1100, 1100)])
def test_many_ragged_sequences(dtype, B, hi):
    g = torch.Generator().manual_seed(B)
    lens = [n if n % 5 else 0 for n in (torch.rand(B, generator=g) ** 3 * hi).int().tolist()]
    lens[0], lens[63], lens[64], lens[-1] = 0, hi, 1, hi - 1
    _run(dtype, 4, 2, 64, 16 if B % 2 else 24, lens, B, max_len=hi + 17)


def test_scales_and_packed_queries():
    for scale in (0.0, -0.3, 1.0, 0.01):
        _run("bf16", 8, 2, 128, 16, [40, 700], 5, q_scale=1.0, scale=scale, packed=True)
        _run("fp32", 8, 2, 64, 16, [40, 700], 6, q_scale=1.0, scale=scale, packed=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_scores_that_grow_and_that_tower(dtype):
    """Keys whose scores rise along the sequence (the running maximum moves at every tile), fall, or hold one peak among very low ones."""
    g = torch.Generator().manual_seed(11)
    n, d = 2000, 128
    for shape in ("rise", "fall", "peak", "low"):
        c, table = make_cache(dtype, 1, -(-n // 16), 16, 1, d, g)
        ramp = {"rise": torch.linspace(-60, 60, n), "fall": torch.linspace(60, -60, n), "peak": torch.full((n,), -300.0), "low": torch.full((n,), -1e30)}[shape]
        if shape == "peak":
            ramp[1234] = 250.0
        k = torch.zeros(n, 1, d)
        k[:, 0, 0] = ramp
        k[:, 0, 1:] = 0.01 * torch.randn(n, d - 1, generator=g) * (shape != "low")
        v = torch.randn(n, 1, d, generator=g)
        E.eagle3_paged_append(c, k.to(ROW[dtype]).to(DEV), v.to(ROW[dtype]).to(DEV), i32([0]).to(DEV))
        q = torch.zeros(1, 4, d)
        q[..., 0] = d ** 0.5
        q = q.to(ROW[dtype]).to(DEV)
        out, lse = E.eagle3_paged_attention(c, q, i32([n]).to(DEV), n, want_lse=True)
        assert bool(torch.isfinite(out).all())
        _check(c, table, q, [n], out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 40, 64, 777])
def test_what_is_behind_a_sequence_does_not_reach_it(dtype, n):
    """NaN and infinities in every slot that no visible token has: behind the length in the last page, in other pages, in other sequences."""
    g = torch.Generator().manual_seed(n)
    for page in (1, 16, 100):
        max_pages = -(-n // page) + 2
        c, table = make_cache(dtype, 2, max_pages, page, 2, 128, g)
        clean = [t.clone() for t in (c.k, c.v)]
        seen = torch.zeros(c.k.shape[0], page, dtype=torch.bool)
        pos = torch.arange(n)
        seen[table[0].long()[pos // page], pos % page] = True
        q = torch.randn(2, 8, 128, generator=g).to(ROW[dtype]).to(DEV)
        lens = i32([n, 0]).to(DEV)
        want = E.eagle3_paged_attention(c, q, lens, max_pages * page, want_lse=True)
        for bad in (NAN, INF, -INF, torch.finfo(ROW[dtype]).min):
            for t in (c.k, c.v):
                t[~seen.to(DEV)] = bad
            got = E.eagle3_paged_attention(c, q, lens, max_pages * page, want_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        c.k.copy_(clean[0]), c.v.copy_(clean[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("n", [1, 33, 700, 9000])
def test_a_bad_token_reaches_its_own_sequence_and_head_only(dtype, n):
    g = torch.Generator().manual_seed(n + 1)
    for where, bad in (("k", NAN), ("v", NAN), ("v", INF)):
        c, table = make_cache(dtype, 3, -(-n // 32) + 1, 32, 2, 128, g)
        x = [torch.randn(3 * n, 2, 128, generator=g).to(ROW[dtype]).to(DEV) for _ in range(2)]
        x[where == "v"][n + n // 2, 1, 5:9] = bad                 # sequence 1, its middle token, KV head 1
        E.eagle3_paged_append(c, x[0], x[1], i32([0, 0, 0]).to(DEV))
        q = torch.randn(3, 8, 128, generator=g).to(ROW[dtype]).to(DEV)
        out, lse = E.eagle3_paged_attention(c, q, i32([n, n, n]).to(DEV), n, want_lse=True)
        want = torch.ones_like(out, dtype=torch.bool)
        want[1, 4:] = False
        if where == "v":
            want[1, 4:, :5] = want[1, 4:, 9:] = True
        assert torch.equal(torch.isfinite(out), want)
        if bad == INF and dtype != "fp8":
            assert bool((out[1, 4:, 5:9] == INF).all())
        assert bool(torch.isfinite(lse[[0, 2]]).all()) and bool(torch.isfinite(lse[1, :4]).all())


def test_pages_outside_the_pool_are_clamped():
    """Page numbers a program never set: the results are finite garbage for that sequence, and right for the others."""
    c, table, q, n, out, _ = _run("bf16", 8, 2, 128, 16, [100, 200, 300], 3)
    table[1] = i32([-1, 2 ** 31 - 1, c.k.shape[0], -2 ** 31] * 10)[:table.shape[1]]
    c.page_table.copy_(table)
    got = E.eagle3_paged_attention(c, q, n, 300)
    assert torch.equal(got[[0, 2]], out[[0, 2]]) and bool(torch.isfinite(got).all())


def test_parts_of_a_context_join_through_their_logarithms():
    """A context attended to in two pieces (its first 640 tokens, and the rest under a table that starts there)."""
    c, table, q, n, out, lse = _run("bf16", 32, 8, 128, 64, [1500], 12)
    rest = E.PagedKVCache(c.k, c.v, c.page_table[:, 10:].contiguous())
    o1, l1 = E.eagle3_paged_attention(c, q, i32([640]).to(DEV), 640, want_lse=True)
    o2, l2 = E.eagle3_paged_attention(rest, q, i32([860]).to(DEV), 860, want_lse=True)
    joint = torch.logaddexp(l1, l2)
    both = (l1 - joint).exp()[..., None] * o1.float() + (l2 - joint).exp()[..., None] * o2.float()
    assert bool(((joint - lse).abs() < 1e-4).all())
    # each piece rounded to bf16 (2^-8 of it), the whole too
    mag = o1.float().abs() + o2.float().abs() + out.float().abs()
    assert bool(((both - out.float()).abs() <= 2.0 ** -8 * mag + 1e-3 * mag + 1e-6).all())


def test_captured_steps_replay_with_new_lengths():
    """Rotation, append and attention in one graph; every replay against the eager calls, with eager work and other calls between them."""
    g = torch.Generator().manual_seed(21)
    B, H, Hkv, d, page, bound = 3, 8, 2, 128, 16, 4000
    caches = [make_cache("fp8", B, bound // page, page, Hkv, d, torch.Generator().manual_seed(22))[0] for _ in range(2)]
    for c in caches:
        for e in (c.k_exp, c.v_exp):
            e.clamp_(117, 120)
    rope = E.Rope(d, 5e5, device=DEV)
    start = i32([0, 1500, 37]).to(DEV)
    lens = start + 1
    qkv = torch.randn(B, H + 2 * Hkv, d, generator=g).bfloat16().to(DEV)

    def step(c):
        q, k = E.eagle3_rope(rope, start, qkv[:, :H], qkv[:, H:H + Hkv])
        E.eagle3_paged_append(c, k, qkv[:, H + Hkv:].contiguous(), start)
        return E.eagle3_paged_attention(c, q, lens, bound, want_lse=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(caches[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):                                        # two graphs, that share what the allocator gives them
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            o = step(caches[0])
        graphs.append(gr), outs.append(o)
    for i in range(6):
        qkv.copy_(torch.randn(B, H + 2 * Hkv, d, generator=g).bfloat16())
        want = step(caches[1])
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        for a, b in zip(outs[i % 2], want):
            assert torch.equal(a, b), i
        assert torch.equal(caches[0].k.view(torch.uint8), caches[1].k.view(torch.uint8)) or i == 0
        start += 7
        lens += 7
        caches[0].k.view(torch.uint8).copy_(caches[1].k.view(torch.uint8))
        (torch.randn(1000, device=DEV) * 2).sum()


def test_two_streams_at_once():
    """Calls on two streams with their own outputs: workspaces are the call's own."""
    c, table, q, n, out, _ = _run("bf16", 32, 8, 128, 16, [3000, 1], 31)
    q2 = torch.randn_like(q)
    want = E.eagle3_paged_attention(c, q2, n, 3000)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(E.eagle3_paged_attention(c, (q, q2)[i], n, 3000))
    torch.cuda.synchronize()
    assert all(torch.equal(t, out) for t in got[0]) and all(torch.equal(t, want) for t in got[1])


def test_calls_go_to_the_tensors_gpu(monkeypatch):
    """With another GPU current the call changes over to the tensors' own and back (one GPU here: the current one's number is what is pretended)."""
    from paper_2503_01840_amd import binding as Bd
    c, table, q, n, out, _ = _run("bf16", 8, 2, 128, 16, [100, 200], 40)
    seen = []
    real = torch.cuda.device

    class Device(real):
        def __init__(self, d):
            seen.append(d)
            super().__init__(d)
    monkeypatch.setattr(Bd, "_current_gpu", lambda: 5)
    monkeypatch.setattr(torch.cuda, "device", Device)
    assert torch.equal(E.eagle3_paged_attention(c, q, n, 200), out) and seen == [q.device.index]


def test_binding_refuses_what_does_not_fit():
    c, table, q, n, out, _ = _run("bf16", 8, 2, 128, 16, [100, 200], 41)
    bad = [lambda: E.eagle3_paged_attention(c, q.float(), n, 200), lambda: E.eagle3_paged_attention(c, q[:1], n, 200),
           lambda: E.eagle3_paged_attention(c, q, n.long(), 200), lambda: E.eagle3_paged_attention(c, q, n[:1], 200),
           lambda: E.eagle3_paged_attention(c, q[..., :64], n, 200), lambda: E.eagle3_paged_attention(c, q, n, 200, out=out.float()),
           lambda: E.eagle3_paged_attention(c, q.cpu(), n, 200)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: E.eagle3_paged_attention(c, q[:, :7].contiguous(), n, 200), lambda: E.eagle3_paged_attention(c, q, n, 0),
                 lambda: E.eagle3_paged_attention(c, q, n, 10 ** 6)):
        with pytest.raises(E.Eagle3Error):
            call()


# ---------------------------------------------------------------- together, and with the framework's own calls
def _decode_layers(W, shape, tok, rope, caches, start, lens, bound):
    """One token of each sequence through the target's layers, its attention over pages; products and norms by torch in fp32."""
    rms = lambda x, w: x * torch.rsqrt((x * x).mean(-1, keepdim=True) + shape.rms_eps) * w
    H, Hkv, d = shape.n_heads, shape.n_kv_heads, shape.head_dim
    x = W["embed"][tok.long()]
    for w, c in zip(W["layers"], caches):
        y = rms(x, w["norm_attn"])
        qkv = torch.cat([y @ w[n].T for n in ("wq", "wk", "wv")], 1).view(len(tok), H + 2 * Hkv, d)
        E.eagle3_rope(rope, start, qkv[:, :H], qkv[:, H:H + Hkv], out=(qkv[:, :H], qkv[:, H:H + Hkv]))
        E.eagle3_paged_append(c, qkv[:, H:H + Hkv], qkv[:, H + Hkv:], start)
        o = E.eagle3_paged_attention(c, qkv[:, :H], lens, bound)
        x = x + o.reshape(len(tok), -1) @ w["wo"].T
        y = rms(x, w["norm_mlp"])
        x = x + (torch.nn.functional.silu(y @ w["w_gate"].T) * (y @ w["w_up"].T)) @ w["w_down"].T
    return rms(x, W["final_norm"]) @ W["lm_head"].T


def _prompt(shape, W, T, B):
    """Contexts of T prompt tokens of B sequences in contiguous caches, by eagle3_prefill."""
    ctx = E.Eagle3Context(shape, max_batch=B, max_nodes=8, max_depth=2, max_topk=2, max_new=4, device=DEV)
    ctx.set_weights(W["target"], W["draft"])
    cap, Hkv, d = T + 16, shape.n_kv_heads, shape.head_dim
    z = lambda n: torch.zeros(n, Hkv, d, dtype=ctx.storage_dtype, device=DEV)
    ks, vs = [z(B * cap) for _ in range(shape.n_layers)], [z(B * cap) for _ in range(shape.n_layers)]
    dk, dv = z(cap), z(cap)
    logits = []
    for b in range(B):
        toks = S.uniform_ints(S.SEED + b, S.TensorIds.PREFIX_TOK, (T,), 0, shape.vocab).int().to(DEV)
        kv = E.KVCache(ks, vs, i32([b * cap, (b + 1) * cap]).to(DEV), i32([0]).to(DEV), 0)
        logits.append(E.eagle3_prefill(ctx, toks, kv, E.KVCache([dk], [dv], i32([0, cap]).to(DEV), i32([0]).to(DEV), 0))[1])
    return ctx, ks, vs, cap, torch.stack(logits)


def test_decoding_over_pages_is_the_framework_s_decoding():
    """fp32: contexts of eagle3_prefill moved into pages, then four plain decoding steps: logits as eagle3_tree_verify of one node gives them."""
    shape, T, B, page = S.get_shape("c1"), 70, 3, 8
    W = PL.device_weights(shape, device=DEV)
    ctx, ks, vs, cap, logits = _prompt(shape, W, T, B)
    base = torch.arange(B, dtype=torch.int32, device=DEV) * cap
    indptr = torch.arange(B + 1, dtype=torch.int32, device=DEV) * cap
    zero, plen = torch.zeros(B, dtype=torch.int32, device=DEV), torch.full((B,), T, dtype=torch.int32, device=DEV)
    caches = []
    for k, v in zip(ks, vs):
        c, _ = make_cache("fp32", B, -(-cap // page), page, shape.n_kv_heads, shape.head_dim, torch.Generator().manual_seed(1))
        E.eagle3_paged_append(c, k, v, zero, plen, rows=T, row_start=base)
        caches.append(c)
    rope = E.Rope(shape.head_dim, shape.rope_theta, device=DEV)
    tok = logits.argmax(1).int()
    for i in range(4):
        kv = E.KVCache(ks, vs, indptr, plen + i, T + i)
        want = E.eagle3_tree_verify(ctx, tok[:, None].contiguous(), torch.full((B, 1), -1, dtype=torch.int32, device=DEV), kv)[0][:, 0]
        got = _decode_layers(W["target"], shape, tok, rope, caches, plen + i, plen + i + 1, T + 16)
        assert float((got - want).abs().max()) < 1e-4, i                    # both fp32 over four layers of exact kernels
        tok = want.argmax(1).int()
    # and back into contiguous caches: what the framework has written itself
    for l, c in enumerate(caches):
        k, v = torch.zeros_like(ks[l]), torch.zeros_like(vs[l])
        E.eagle3_paged_read(c, zero, plen + 4, rows=T + 4, row_start=base, out=(k, v))
        assert float((k - ks[l]).abs().max()) < 1e-4 and float((v - vs[l]).abs().max()) < 1e-4
        prompt = torch.cat([torch.arange(T) + b * cap for b in range(B)]).to(DEV)
        assert torch.equal(k[prompt], ks[l][prompt]) and torch.equal(v[prompt], vs[l][prompt])


def test_a_tree_is_verified_over_a_context_that_was_in_pages():
    """bf16: a context kept in pages and read back gives the tree's logits bit for bit; kept in 8 bits, those over the quantised context."""
    shape, T, N = SMALL, 200, 8
    W = PL.device_weights(shape, device=DEV)
    ctx, ks, vs, cap, _ = _prompt(shape, W, T, 1)
    parents = torch.as_tensor(S.random_tree(S.SEED, 3, N, 4, 2)[0], dtype=torch.int32, device=DEV)[None]
    toks = S.uniform_ints(S.SEED, S.TensorIds.TREE_TOK, (1, N), 0, shape.vocab).int().to(DEV)
    verify = lambda k, v: E.eagle3_tree_verify(ctx, toks, parents, E.KVCache(k, v, i32([0, cap]).to(DEV), i32([T]).to(DEV), T))[0]
    want = verify([t.clone() for t in ks], [t.clone() for t in vs])
    for dtype in ("bf16", "fp8"):
        rk, rv, qk, qv = [], [], [], []
        for k, v in zip(ks, vs):
            c, _ = make_cache(dtype, 1, -(-T // 16), 16, shape.n_kv_heads, shape.head_dim, torch.Generator().manual_seed(2))
            E.eagle3_paged_append(c, k[:T], v[:T], i32([0]).to(DEV))
            out = (torch.zeros_like(k), torch.zeros_like(v))
            E.eagle3_paged_read(c, None, i32([T]).to(DEV), rows=T, row_start=i32([0]).to(DEV), out=out)
            rk.append(out[0]), rv.append(out[1])
            for t, l, o in ((k, qk, out[0]), (v, qv, out[1])):
                from test_gpu_paged import quantised
                l.append(torch.cat([value(*quantised(t[:T].cpu())).to(t.dtype).to(DEV), torch.zeros_like(t[T:])]) if dtype == "fp8" else t.clone())
                assert torch.equal(o[:T], l[-1][:T])
        got = verify(rk, rv)
        assert torch.equal(got, verify(qk, qv))
        assert dtype == "fp8" or torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("H", [4, 24])
@pytest.mark.parametrize("bound", [300, 5000, 70000])
def test_weights_keep_what_a_cancelling_sum_needs(dtype, H, bound):
    """Dimension i is the difference of two weights w1, w2 that a factor of 2^(2^-13) parts, and nothing else.  Scores are exact in 32 bits (few significant bits,
    and a scale that is 1 in units of log2), so a weight is off by one unit of exp2, 2^-23, and by what its split into bf16 terms loses: terms of 8, 8 and 8 bits
    cut, cut and rounded leave 2^-24, and a first remainder is kept up by 2^-24 of its term, 2^-23 together.  Six additions to a sum of up to w1 are off by 2^-23 of
    it at most.  In all (2 * 2 + 6) 2^-23 w1, and the output's rounding.  Weights of 16 bits would be off by up to 2 * 2^-16."""
    d, n, scale = 128, 257, float(np.float32(np.log(2.0)))
    assert np.float32(scale) * np.float32(1.4426950408889634) == 1
    g = torch.Generator().manual_seed(H)
    c, table = make_cache(dtype, 1, -(-bound // 16), 16, 1, d, g)
    k, v = torch.zeros(n, 1, d), torch.zeros(n, 1, d)
    k[0, 0, 0] = 1                                             # the maximum, without a value
    coarse = -torch.randint(8, 16, (d, 3), generator=g) / 8
    for i in range(2):
        k[1 + i::2, 0, :3] = coarse
        v[torch.arange(1 + i, n, 2), 0, torch.arange(d)] = 1.0 - 2 * i
    k[2::2, 0, 3] = -1
    q = torch.zeros(1, H, d)
    q[0, :, 0] = 1
    q[0, :, 1:3] = (0.1 + 0.4 * torch.rand(H, 2, generator=g)).bfloat16().float()
    q[..., 3] = 2.0 ** -13
    E.eagle3_paged_append(c, k.bfloat16().to(DEV), v.bfloat16().to(DEV), i32([0]).to(DEV))
    out = E.eagle3_paged_attention(c, q.bfloat16().to(DEV), i32([n]).to(DEV), bound, scale=scale)[0].cpu().double()
    assert torch.equal(_rows(c, "k")[table[0].long()[torch.arange(n) // 16] * 16 + torch.arange(n) % 16], k.double())
    p = torch.softmax(scale * (q[0].double() @ k[:, 0].double().T), 1)
    ref = p[:, 1::2] - p[:, 2::2]
    tol = 10 * 2.0 ** -23 * p[:, 1::2]
    tol = tol + 2.0 ** -8 * (ref + tol)
    assert bool(((out - ref).abs() <= tol).all()), float(((out - ref).abs() / tol).max())


# a workgroup to a sequence, ranges, and two products of each operand in either way
@pytest.mark.parametrize("H,Hkv,B,bound", [(8, 2, 2, 704), (8, 2, 2, 5000), (48, 1, 100, 704), (48, 1, 2, 40000)])
@pytest.mark.parametrize("page", [1, 16, 100])
@pytest.mark.parametrize("n", [1, 40, 64, 700])
def test_what_is_behind_a_sequence_in_8_bits_does_not_reach_it(H, Hkv, B, bound, page, n):
    """NaN codes and the largest ones under exponent bytes of 0, 254 and 255 (an infinite scale) in every slot that no visible token has."""
    g = torch.Generator().manual_seed(n + page)
    c, table = make_cache("fp8", B, -(-n // page) + 2, page, Hkv, 128, g)
    for e in (c.k_exp, c.v_exp):
        e.clamp_(117, 120)
    wide = torch.zeros(B, max(-(-bound // page), table.shape[1]), dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    c = E.PagedKVCache(c.k, c.v, wide.to(DEV), c.k_exp, c.v_exp)
    seen = torch.zeros(c.k.shape[0], page, dtype=torch.bool)
    pos = torch.arange(n)
    seen[table[0].long()[pos // page], pos % page] = True
    unseen = ~seen.to(DEV)
    q = torch.randn(B, H, 128, generator=g).bfloat16().to(DEV)
    lens = [n] + [0] * (B - 1)
    want = E.eagle3_paged_attention(c, q, i32(lens).to(DEV), bound, want_lse=True)
    _check(c, wide, q, lens, *want)
    for code in (0x7F, 0xFF, 0x7E, 0xFE):
        for exp in (0, 254, 255):
            for t in (c.k, c.v):
                t.view(torch.uint8)[unseen] = code
            for t in (c.k_exp, c.v_exp):
                t[unseen] = exp
            got = E.eagle3_paged_attention(c, q, i32(lens).to(DEV), bound, want_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (code, exp)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("up", [105, -99])
@pytest.mark.parametrize("bound", [4000, 700])
def test_values_of_any_magnitude(dtype, up, bound):
    """Values times a power of two give results times it.  Up: bit for bit as long as the number of tokens times the largest, 4 * 2^105, is below 2^120; scores rise by
    less than 2^8 within a workgroup's reach, so that weights are as large as they may be.  Down: weights times an 8-bit row's scale, at least 2^-8 * 2^-107, are held in
    bf16 terms of multiples of 2^-133, which takes less than 2^-18 of a weight (weights of 2^-8 count 1 / 256); the output's two roundings may fall apart by a step, 2^-7."""
    n, d = bound, 128
    g = torch.Generator().manual_seed(bound)
    k = torch.zeros(n, 1, d)
    k[:, 0, 0] = torch.linspace(0, 7 * math.log(2.0), n)
    v = torch.randn(n, 1, d, generator=g).clamp(-4, 4)
    q = torch.zeros(1, 4, d)
    q[..., 0] = d ** 0.5
    q = q.to(ROW[dtype]).to(DEV)
    outs = []
    for scale in (1.0, 2.0 ** up):
        c, table = make_cache(dtype, 1, -(-n // 16), 16, 1, d, torch.Generator().manual_seed(5))
        E.eagle3_paged_append(c, k.to(ROW[dtype]).to(DEV), (v * scale).to(ROW[dtype]).to(DEV), i32([0]).to(DEV))
        out, lse = E.eagle3_paged_attention(c, q, i32([n]).to(DEV), n, want_lse=True)
        if scale == 1.0:
            _check(c, table, q, [n], out, lse)
        outs.append(out.double())
    assert bool(torch.isfinite(outs[1]).all())
    if up > 0:
        assert torch.equal(outs[1], outs[0] * 2.0 ** up)
    else:
        err = (outs[1] * 2.0 ** -up - outs[0]).abs()
        assert bool((err <= 2.0 ** -7 * outs[0].abs() + 2.0 ** -18 * 4).all()), float(err.max())
