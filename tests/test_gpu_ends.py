"""Embeddings, norms and distillation together: a draft model's training step, plain decoding beside the framework's own, streams and GPUs."""
import pytest
import torch

import eagle3_synth as S
import paper_2503_01840_amd as E
import pipeline as PL
from test_gpu_paged import DEV, make_cache
from test_gpu_paged_attention import _prompt

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32
EPS = 1e-5


class _Draft:
    """One layer of the draft model's kind: norms of a token's embedding and of a feature side by side, a product, the sum's norm, a gated product, the last norm, the head."""

    def __init__(self, g, vocab, draft_vocab, k):
        n = lambda *shape, s=1.0: s * torch.randn(*shape, generator=g, dtype=torch.float64)
        self.w = dict(table=n(vocab, k), g_embed=1 + n(k, s=0.1), g_feat=1 + n(k, s=0.1), mix=n(k, 2 * k, s=(2 * k) ** -0.5), g_mid=1 + n(k, s=0.1),
                      up=n(2 * k, k, s=k ** -0.5), down=n(k, 2 * k, s=(2 * k) ** -0.5), g_last=1 + n(k, s=0.1), head=n(draft_vocab, k, s=2 * k ** -0.5))

    def on(self, device, dtype):
        return {n: t.to(device=device, dtype=dtype, copy=True).requires_grad_() for n, t in self.w.items()}


def _forward(w, tok, feat, norm, embed):
    x = torch.cat([norm(embed(w["table"], tok), w["g_embed"], None), norm(feat, w["g_feat"], None)], 1)
    a = x @ w["mix"].T
    y, h = norm(a, w["g_mid"], feat)
    b = torch.nn.functional.silu(y @ w["up"].T) @ w["down"].T
    y, h = norm(b, w["g_last"], h)
    return y @ w["head"].T, h


def _plain(x, gain, residual):
    h = x if residual is None else x + residual
    y = gain * h / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    return y if residual is None else (y, h)


def _own(x, gain, residual):
    return E.eagle3_add_norm(x, gain, EPS, residual=residual)


def _batch(g, rows, vocab, draft_vocab, k, K):
    tok = torch.randint(-1, vocab, (rows,), generator=g, dtype=torch.int32)
    feat = torch.randn(rows, k, generator=g, dtype=torch.float64)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:K] for _ in range(rows)]).to(torch.int32)
    values = 2 * torch.randn(rows, K, generator=g, dtype=torch.float64)
    t2d = torch.full((vocab,), -1, dtype=torch.int32)
    t2d[torch.randperm(vocab, generator=g)[:draft_vocab]] = torch.arange(draft_vocab, dtype=torch.int32)
    weight = torch.where(torch.arange(rows) < rows // 3, 0.0, 1.0 / rows).double()             # a prompt's positions teach nothing
    return tok, feat, ids, values.float(), t2d, weight


def _reference(model, tok, feat, ids, values, t2d, weight):
    """Loss and gradients in 64 bits by autograd."""
    w = model.on("cpu", torch.float64)
    embed = lambda table, t: torch.where((t >= 0)[:, None], table[t.long().clamp(min=0)], 0.0)
    logits, h = _forward(w, tok, feat, _plain, embed)
    at = t2d.long()[ids.long()]
    z = torch.where(at >= 0, values.double(), -torch.inf)
    p = torch.softmax(z, 1).nan_to_num(0.0)
    loss = -(torch.where(at >= 0, p, 0.0) * torch.log_softmax(logits, 1).gather(1, at.clamp(min=0))).sum(1)
    total = (loss * weight).sum() + 0.01 * (h * h).mean()
    total.backward()
    return loss.detach(), float(total.detach()), {n: t.grad for n, t in w.items()}


SIZES = (70, 300, 120, 48, 24)                               # rows, vocabulary, draft vocabulary, width, teacher's entries


def test_a_training_step_of_a_draft():
    """Loss and every gradient in fp32 against autograd in 64 bits: products of 48 to 120 terms and sums over 70 rows in 32 bits through four layers stay within 1e-5 of the
    largest entries (each is off by some 2^-24 sqrt(120), about 1e-6 after seven of them)."""
    rows, vocab, draft_vocab, k, K = SIZES
    g = torch.Generator().manual_seed(0)
    model = _Draft(g, vocab, draft_vocab, k)
    tok, feat, ids, values, t2d, weight = _batch(g, rows, vocab, draft_vocab, k, K)
    want_loss, want_total, want = _reference(model, tok, feat, ids, values, t2d, weight)
    w = model.on(DEV, FP32)
    tok, ids, values, t2d = (t.to(DEV) for t in (tok, ids, values, t2d))
    feat, weight = feat.float().to(DEV), weight.float().to(DEV)
    logits, h = _forward(w, tok, feat, _own, E.eagle3_embed)
    loss = E.eagle3_distill(logits, ids, values, t2d=t2d)
    total = (loss * weight).sum() + 0.01 * (h * h).mean()
    total.backward()
    assert float((loss.detach().cpu().double() - want_loss).abs().max()) <= 1e-5 * float(want_loss.max())
    assert abs(float(total.detach()) - want_total) <= 1e-5 * abs(want_total)
    for n, t in w.items():
        assert float((t.grad.cpu().double() - want[n]).abs().max()) <= 1e-5 * float(want[n].abs().max()), n
    # the same gradients from loss and gradient in one call
    logits2, h2 = _forward(w, tok, feat, _own, E.eagle3_embed)
    loss2, d_logits = E.eagle3_distill_step(weight, logits2.detach(), ids, values, t2d=t2d)
    grads = torch.autograd.grad((logits2, 0.01 * (h2 * h2).mean()), list(w.values()), (d_logits, torch.ones((), device=DEV)))
    for (n, t), got in zip(w.items(), grads):
        assert float((t.grad - got).abs().max()) <= 1e-6 * float(t.grad.abs().max()), n


def test_a_captured_training_step_replays():
    """Forward and backward pass in one graph, other batches and weights at every replay, against eager steps."""
    rows, vocab, draft_vocab, k, K = SIZES
    g = torch.Generator().manual_seed(1)
    w = _Draft(g, vocab, draft_vocab, k).on(DEV, FP32)
    batch = [t.to(DEV) if t.dtype != torch.float64 else t.float().to(DEV) for t in _batch(g, rows, vocab, draft_vocab, k, K)]

    def step():
        tok, feat, ids, values, t2d, weight = batch
        logits, h = _forward(w, tok, feat, _own, E.eagle3_embed)
        loss = E.eagle3_distill(logits, ids, values, t2d=t2d)
        return [loss.detach(), *torch.autograd.grad((loss, h), list(w.values()), (weight, 0.01 * h.detach()))]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        with torch.no_grad():
            for t, new in zip(batch, _batch(g, rows, vocab, draft_vocab, k, K)):
                t.copy_(new)
            for t in w.values():
                t.mul_(1.01)
        graph.replay()
        torch.cuda.synchronize()
        got_now = [t.clone() for t in got]
        want = step()
        for a, b in zip(got_now, want):
            assert float((a - b).abs().max()) <= 1e-5 * float(b.abs().max()), i
        (torch.randn(1000, device=DEV) * 2).sum()


def _decode(W, shape, tok, rope, caches, start, lens, bound):
    """One token of each sequence through the target's layers by the calls that stand alone; products by torch in fp32."""
    H, Hkv, d = shape.n_heads, shape.n_kv_heads, shape.head_dim
    x = E.eagle3_embed(W["embed"], tok)
    branch = torch.zeros_like(x)
    for w, c in zip(W["layers"], caches):
        y, x = E.eagle3_add_norm(branch, w["norm_attn"], shape.rms_eps, residual=x)
        qkv = torch.cat([y @ w[n].T for n in ("wq", "wk", "wv")], 1).view(len(tok), H + 2 * Hkv, d)
        E.eagle3_rope(rope, start, qkv[:, :H], qkv[:, H:H + Hkv], out=(qkv[:, :H], qkv[:, H:H + Hkv]))
        E.eagle3_paged_append(c, qkv[:, H:H + Hkv], qkv[:, H + Hkv:], start)
        o = E.eagle3_paged_attention(c, qkv[:, :H], lens, bound)
        y, _ = E.eagle3_add_norm(o.reshape(len(tok), -1) @ w["wo"].T, w["norm_mlp"], shape.rms_eps, residual=x, out=(None, x))
        branch = (torch.nn.functional.silu(y @ w["w_gate"].T) * (y @ w["w_up"].T)) @ w["w_down"].T
    return E.eagle3_add_norm(branch, W["final_norm"], shape.rms_eps, residual=x)[0] @ W["lm_head"].T


def test_decoding_by_these_calls_is_the_framework_s_decoding():
    """fp32: contexts of eagle3_prefill moved into pages, then plain decoding steps: logits as eagle3_tree_verify of one node gives them (1e-4, the bound of the
    fp32 configuration).  The loss of these logits against their own 32 largest ones is these entries' part of the distribution's entropy."""
    shape, T, B, page = S.get_shape("c1"), 37, 2, 16
    W = PL.device_weights(shape, device=DEV)
    context, ks, vs, cap, logits = _prompt(shape, W, T, B)
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
        want = E.eagle3_tree_verify(context, tok[:, None].contiguous(), torch.full((B, 1), -1, dtype=torch.int32, device=DEV), kv)[0][:, 0]
        got = _decode(W["target"], shape, tok, rope, caches, plen + i, plen + i + 1, T + 16)
        assert float((got - want).abs().max()) < 1e-4, i
        values, ids = got.topk(32, 1)
        p = torch.softmax(got.double(), 1).gather(1, ids)
        loss = E.eagle3_distill(got, ids.int(), values.contiguous(), lse=torch.logsumexp(got, 1))
        assert float((loss.double() + (p * p.log()).sum(1)).abs().max()) <= 1e-5, i
        gain, group = torch.ones(shape.vocab, device=DEV), 128
        codes, scales = E.eagle3_add_norm_codes(got, gain, shape.rms_eps, group=group)
        step = scales.repeat_interleave(group, 1)[:, :shape.vocab]
        y = E.eagle3_add_norm(got, gain, shape.rms_eps)
        assert bool(((codes.float() * step - y).abs() <= 2.0 ** -4 * y.abs() + 2.0 ** -9 * step).all()), i
        tok = want.argmax(1).int()


def _calls(g, device=DEV):
    """Every call with inputs of its own: (name, function of nothing)."""
    rows, vocab, dim, V, K = 200, 500, 136, 40000, 12
    r = lambda *shape: torch.randn(*shape, generator=g).to(device)
    tok = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).to(device)
    ids = torch.randint(0, V, (5, K), generator=g, dtype=torch.int32).to(device)
    table, x, res, gain, logits, values, dloss = r(vocab, dim), r(rows, dim), r(rows, dim), r(dim), r(5, 2 * V), r(5, K), r(5)
    stats = E.eagle3_distill(logits[:, :V], ids, values, want_stats=True)[1]
    return {
        "embed": lambda: (E.eagle3_embed(table, tok),), "embed_grad": lambda: (E.eagle3_embed_grad(x, tok, vocab),), "norm": lambda: E.eagle3_add_norm(x, gain, EPS, residual=res),
        "codes": lambda: E.eagle3_add_norm_codes(x, gain, EPS, residual=res), "norm_grad": lambda: E.eagle3_add_norm_grad(x, res, gain, EPS, dh=x),
        "distill": lambda: (E.eagle3_distill(logits, ids, values),), "distill_grad": lambda: (E.eagle3_distill_grad(dloss, stats, logits[:, :V], ids, values),),
        "step": lambda: E.eagle3_distill_step(dloss, logits, ids, values),
    }


def _same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def test_calls_on_several_streams_at_once():
    """Workspaces are a call's own: two streams with other inputs each, many calls deep, give what each gives alone."""
    both = [_calls(torch.Generator().manual_seed(s)) for s in (3, 4)]
    want = [{n: f() for n, f in calls.items()} for calls in both]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append({n: f() for n, f in both[i].items()})
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            for n in run:
                assert _same(run[n], want[i][n]), n


def test_calls_go_to_the_tensors_gpu(monkeypatch):
    """With another GPU current the calls change over to the tensors' own and back (one GPU here: the current one's number is what is pretended)."""
    from paper_2503_01840_amd import binding as Bd
    calls = _calls(torch.Generator().manual_seed(5))
    want = {n: f() for n, f in calls.items()}
    seen = []
    real = torch.cuda.device

    class Device(real):
        def __init__(self, d):
            seen.append(d)
            super().__init__(d)
    monkeypatch.setattr(Bd, "_current_gpu", lambda: 5)
    monkeypatch.setattr(torch.cuda, "device", Device)
    for n, f in calls.items():
        seen.clear()
        assert _same(f(), want[n]) and seen == [0], n


def test_calls_under_graphs_that_share_a_pool():
    """Two captured graphs, their workspaces from one pool, replayed in turn: the second's are not the first's results."""
    both = [_calls(torch.Generator().manual_seed(s)) for s in (6, 7)]
    want = [{n: f() for n, f in calls.items()} for calls in both]
    pool = torch.cuda.graph_pool_handle()
    graphs, got = [], []
    for calls in both:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            got.append({n: f() for n, f in calls.items()})
        graphs.append(graph)
    for _ in range(3):
        for i in (0, 1):
            graphs[i].replay()
            torch.cuda.synchronize()
            for n in got[i]:
                assert _same(got[i][n], want[i][n]), n


def test_offsets_past_32_bits():
    """Tables and rows whose last bytes lie more than 2^32 behind their first: 8.6 GB each."""
    vocab, dim = 1050000, 4096
    g = torch.Generator().manual_seed(8)
    tok = torch.tensor([0, vocab - 1, 5, 524288, 1048576, vocab - 1, -1], dtype=torch.int32, device=DEV)
    dy = torch.randn(7, dim, generator=g).to(DEV)
    table = E.eagle3_embed_grad(dy, tok, vocab, dtype=BF16)
    assert torch.equal(E.eagle3_embed(table, tok, dtype=FP32), torch.stack([dy[0], dy[1] + dy[5], dy[2], dy[3], dy[4], dy[1] + dy[5], 0 * dy[6]]).to(BF16).float())
    assert int(table.count_nonzero(1).ne(0).sum()) == 5                       # and zeros everywhere else
    x = table.view(5, -1)[:, :2 * dim]                                        # rows 1.7e9 bytes apart
    x.copy_(torch.randn(5, 2 * dim, generator=g))
    gain = torch.ones(dim, device=DEV)
    dense = x.contiguous()
    assert torch.equal(E.eagle3_add_norm(x[:, :dim], gain, EPS), E.eagle3_add_norm(dense[:, :dim], gain, EPS))
    ids, values = torch.randint(0, dim, (5, 6), generator=g, dtype=torch.int32).to(DEV), torch.randn(5, 6, generator=g).to(DEV)
    weight = torch.ones(5, device=DEV)
    want = E.eagle3_distill_step(weight, dense[:, :dim], ids, values)
    got = E.eagle3_distill_step(weight, x[:, :dim], ids, values, out=x[:, dim:])
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], x[:, dim:])
    assert torch.equal(x[:, :dim], dense[:, :dim])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_teacher_that_says_one_token_a_thousand_times(dtype):
    """1024 entries of one token, and of two in turn: the weights of a token are added up, whatever entries they stand in."""
    V = 700
    g = torch.Generator().manual_seed(9)
    logits, values = torch.randn(3, V, generator=g).to(dtype).to(DEV), torch.randn(3, 1024, generator=g).to(DEV)
    ids = torch.full((3, 1024), 17, dtype=torch.int32, device=DEV)
    ids[1, ::2] = 18
    ids[2] = torch.randint(0, 4, (1024,), generator=g, dtype=torch.int32).to(DEV)
    loss, grad = E.eagle3_distill_step(torch.ones(3, device=DEV), logits, ids, values)
    p = torch.zeros(3, V, dtype=torch.float64, device=DEV).scatter_add_(1, ids.long(), torch.softmax(values.double(), 1))
    x = logits.double()
    # weights: each off by 10 steps of 2^-24 or so, added one behind the other: 1024 of them, 2^-14 at most
    assert float((loss.double() + (p * torch.log_softmax(x, 1)).sum(1)).abs().max()) <= 2.0 ** -14 * 12
    want = torch.softmax(x, 1) - p
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    assert bool(((grad.double() - want).abs() <= 2.0 ** -14 * (p + torch.softmax(x, 1)) + half * want.abs()).all())
