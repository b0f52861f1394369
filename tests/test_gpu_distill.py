"""Distillation's loss and gradient on the GPU against the definition in 64 bits, and the gradient against differences."""
import math

import pytest
import torch

import paper_2503_01840_amd as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32
U = 2.0 ** -24                                               # half a step of fp32


def _targets(V, ids, values, lse, t2d, T):
    """Weights [rows, k] and the student's ids, on the CPU in 64 bits."""
    ids, z = ids.long().cpu(), values.double().cpu() / T
    if t2d is not None:
        t2d = t2d.long().cpu()
        ids = torch.where((ids >= 0) & (ids < len(t2d)), t2d[ids.clamp(0, len(t2d) - 1)], -1)
    seen = (ids >= 0) & (ids < V)
    z = torch.where(seen, z, -math.inf)
    if lse is not None:
        p = torch.exp(z - lse.double().cpu()[:, None])
    else:
        p = torch.softmax(z, 1)
        p = torch.where((z > -math.inf).any(1, keepdim=True) | z.isnan().any(1, keepdim=True), p, 0.0)
    return p, ids.clamp(0, V - 1), z


def _reference(logits, ids, values, lse, t2d, T, dloss):
    """Loss, gradient, and what their errors are measured by."""
    x = logits.double().cpu() / T
    V = x.shape[1]
    p, at, z = _targets(V, ids, values, lse, t2d, T)
    m = x.amax(1, keepdim=True)
    s = torch.exp(x - m).sum(1, keepdim=True)
    logq = x - m - s.log()
    P = p.sum(1, keepdim=True)
    loss = -torch.where(p > 0, p * logq.gather(1, at), 0.0).sum(1)
    dense = torch.zeros_like(x).scatter_add_(1, at, p)
    g = (dloss.double().cpu() / T)[:, None]
    grad = g * (P * logq.exp() - dense)
    # Sum: exponents off by 3 U of their size (difference, factor, product) and the exponential by 2 U; a thread rescales its sum once for 16 values, 8 times
    # in a row that registers hold and V / 8192 times in a longer one, between threads 6 + 15 times, each by 3 U more; it adds up to V / 1024 values in a chain, 32 where V is below
    # 16384, and 22 sums: 3 (8 + 21) + 32 + 22 or 3 (8 + V / 8192 + 21) + V / 1024 + 22 steps, less than 4 (V / 2048 + 22) + 60 at every V.  Weights: exponents off by 2 U of theirs, the exponential 2 U, a sum of
    # k terms, a quotient.
    spread = (m - x.amin(1, keepdim=True)).clamp(max=104)     # what is further below has no part in the sum
    rel_s = (3 * spread + 4 * (V / 2048 + 22) + 60) * U
    zs = torch.where(z > -math.inf, z, z.amax(1, keepdim=True))
    zs = torch.where((z > -math.inf).any(1, keepdim=True), zs, 0.0)                # a row without targets: exact zeros, no weight to be off
    top = zs.amax(1, keepdim=True)
    rel_p = (2 * ((top - zs).amax(1, keepdim=True) if lse is None else zs.abs().amax(1, keepdim=True) + lse.double().cpu().abs()[:, None]) + 2 * p.shape[1] + 8) * U
    away = torch.where(p > 0, p * (m - x.gather(1, at)), 0.0).sum(1, keepdim=True)
    loss_err = P * (rel_s + s.log() * (rel_p + 4 * U)) + away * (rel_p + (p.shape[1] + 4) * U)
    q = P * logq.exp()
    grad_err = g.abs() * (q * (rel_s + rel_p + 3 * (m - x).clamp(max=104) * U + 6 * U) + dense * (rel_p + (p.shape[1] + 4) * U)) + 2.0 ** -126
    return loss, grad, loss_err[:, 0], grad_err, m[:, 0] * T, s[:, 0], rel_s[:, 0]


def _check(got, want, err, dtype=FP32):
    bound = err + (2.0 ** -8 if dtype == BF16 else U) * (want.abs() + err)
    bad = ~((got.double().cpu() - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), float((got.double().cpu() - want).abs()[bad].max()))


def _case(g, rows, V, k, dtype, tail, mapped, T):
    x = (3 * torch.randn(rows, V, generator=g)).to(dtype)
    values = 3 + 2 * torch.randn(rows, k, generator=g)
    t2d = None
    if mapped:
        M = 3 * V + 1
        t2d = torch.full((M,), -1, dtype=torch.int32)
        t2d[torch.randperm(M, generator=g)[:V]] = torch.arange(V, dtype=torch.int32)
        t2d[M - 1] = V                                        # stands for a token that there is not
        ids = torch.randint(-1, M + 1, (rows, k), generator=g, dtype=torch.int32)
    else:
        ids = torch.randint(0, V, (rows, k), generator=g, dtype=torch.int32)      # the same one twice where k is near V
    if rows > 2:
        ids[1] = -1                                           # a row without targets
        values[2, k // 2:] = -math.inf
    lse = torch.logsumexp(values.double() / T, 1).float() + 0.3 if tail else None
    move = lambda t: None if t is None else t.to(DEV)
    return [move(t) for t in (x, ids, values, lse, t2d)]


CASES = [  # rows, vocabulary, k, tail, mapped, temperature
    (1, 1, 1, False, False, 1.0), (3, 2, 3, True, False, 2.0), (5, 31, 4, False, True, 0.7), (4, 1000, 64, False, False, 1.0), (1030, 72, 5, True, True, 1.0),
    (2, 8191, 1024, False, False, 1.0), (16, 32000, 32, True, False, 1.0), (3, 128256, 128, False, True, 1.0), (1025, 2047, 10, False, False, 3.0), (1100, 8200, 40, True, False, 1.0),
    (7, 20011, 256, False, True, 1.0), (1024, 32001, 16, False, False, 1.0), (1, 300007, 300, True, False, 1.0), (1024, 40960, 8, False, True, 1.3),
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", CASES)
def test_loss_and_gradient(case, dtype):
    rows, V, k, tail, mapped, T = case
    g = torch.Generator().manual_seed(rows + V)
    x, ids, values, lse, t2d = _case(g, rows, V, k, dtype, tail, mapped, T)
    dloss = torch.randn(rows, generator=g)
    dloss[rows // 2] = 0.0 if rows > 3 else 1.5
    dloss = dloss.to(DEV)
    teacher = dict(lse=lse, t2d=t2d, temperature=T)
    loss, stats = E.eagle3_distill(x, ids, values, want_stats=True, **teacher)
    grad = E.eagle3_distill_grad(dloss, stats, x, ids, values, **teacher)
    T = float(torch.tensor(T, dtype=FP32))
    want, want_grad, err, grad_err, m, s, rel = _reference(x, ids, values, lse, t2d, T, dloss)
    _check(loss, want, err)
    assert torch.equal(stats[:, 0].cpu().double(), x.double().amax(1).cpu())
    assert bool(((stats[:, 1].double().cpu() - s).abs() <= s * rel).all())
    _check(grad, want_grad, grad_err, dtype)
    assert torch.equal(loss, E.eagle3_distill(x, ids, values, **teacher)) and torch.equal(grad, E.eagle3_distill_grad(dloss, stats, x, ids, values, **teacher))
    for out in (None, x.clone()):                             # in one call; over the logits
        again, got = E.eagle3_distill_step(dloss, x if out is None else out, ids, values, out=out, **teacher)
        _check(again, want, err)
        _check(got, want_grad, grad_err, dtype)
    over = x.clone()
    assert E.eagle3_distill_grad(dloss, stats, over, ids, values, out=over, **teacher) is over and torch.equal(over, grad)
    none = torch.nonzero(torch.all(torch.zeros_like(want_grad) == want_grad, 1))[:, 0]
    assert bool((grad[none.to(DEV)] == 0).all()) and bool((got[none.to(DEV)] == 0).all())


@pytest.mark.parametrize("rows,V,k,dtype,tail,mapped", [(64, 70001, 40, FP32, False, False), (66, 98304, 1024, FP32, True, True), (65, 128256, 1024, FP32, True, False), (67, 131071, 128, BF16, True, False),
                                                        (64, 140001, 300, BF16, False, True), (65, 210003, 1024, BF16, True, False)])
def test_long_rows_in_one_launch(rows, V, k, dtype, tail, mapped):
    """Rows that are not worked on in parts and have more pieces than a workgroup's registers hold (16384): up to 24576 of them stay in LDS behind the teacher's tables, of which the largest are among
    these, and what is behind is read twice; and rows of 16 bits just below the first line."""
    test_loss_and_gradient((rows, V, k, tail, mapped, 1.0), dtype)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,V", [(3, 1001), (5, 40003), (1025, 1003), (1024, 33001)])
def test_rows_that_lie_apart(rows, V, dtype):
    """Logits and gradients as parts of longer rows, at any distance from a multiple of 16 bytes: the same bits, and nothing else is written."""
    g = torch.Generator().manual_seed(V)
    x, ids, values, lse, t2d = _case(g, rows, V, 9, dtype, True, False, 1.0)
    dloss = torch.randn(rows, generator=g).to(DEV)
    loss, stats = E.eagle3_distill(x, ids, values, lse, want_stats=True)
    want = E.eagle3_distill_grad(dloss, stats, x, ids, values, lse)
    ref = _reference(x, ids, values, lse, None, 1.0, dloss)
    for off, out_off, width in ((0, 0, V + 7), (1, 1, V + 13), (3, 6, V + 16), (5, 0, V + 9)):
        wide = torch.full((rows, width), 30.0, dtype=dtype, device=DEV)
        view = wide[:, off:off + V]
        view.copy_(x)
        around = torch.full((rows, width), 30.0, dtype=dtype, device=DEV)
        out = around[:, out_off:out_off + V]
        got_loss, got_stats = E.eagle3_distill(view, ids, values, lse, want_stats=True)
        _check(got_loss, ref[0], ref[2])
        assert torch.equal(got_stats[:, 0], stats[:, 0])
        assert E.eagle3_distill_grad(dloss, stats, view, ids, values, lse, out=out) is out and torch.equal(out, want)
        assert bool((around[:, :out_off] == 30).all()) and bool((around[:, out_off + V:] == 30).all())
        around.fill_(30)
        got_loss, _ = E.eagle3_distill_step(dloss, view, ids, values, lse, out=out)
        _check(got_loss, ref[0], ref[2])
        _check(out, ref[1], ref[3], dtype)
        assert bool((around[:, :out_off] == 30).all()) and bool((around[:, out_off + V:] == 30).all())
        E.eagle3_distill_step(dloss, view, ids, values, lse, out=view)
        assert torch.equal(view, out if off == out_off else view) and bool((wide[:, :off] == 30).all()) and bool((wide[:, off + V:] == 30).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,V", [(3, 1001), (5, 40003), (1025, 1003), (64, 70003)])
def test_gradients_over_logits_that_start_anywhere(rows, V, dtype):
    """Over the logits, at any distance from a multiple of 16 bytes, against the definition: in one call, and from the stats."""
    g = torch.Generator().manual_seed(V + 1)
    x, ids, values, lse, _ = _case(g, rows, V, 9, dtype, True, False, 1.0)
    dloss = torch.randn(rows, generator=g).to(DEV)
    ref = _reference(x, ids, values, lse, None, 1.0, dloss)
    _, stats = E.eagle3_distill(x, ids, values, lse, want_stats=True)
    for off, width in ((0, V + 7), (1, V + 13), (3, V + 16), (5, V + 9), (7, V + 8)):
        for call in (lambda o: E.eagle3_distill_step(dloss, o, ids, values, lse, out=o)[1], lambda o: E.eagle3_distill_grad(dloss, stats, o, ids, values, lse, out=o)):
            wide = torch.full((rows, width), 30.0, dtype=dtype, device=DEV)
            view = wide[:, off:off + V]
            view.copy_(x)
            assert call(view) is view
            _check(view, ref[1], ref[3], dtype)
            assert bool((wide[:, :off] == 30).all()) and bool((wide[:, off + V:] == 30).all())


@pytest.mark.parametrize("rows,V", [(8, 300), (8, 50000), (1032, 9000)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_masked_infinite_and_missing_values(rows, V, dtype):
    g = torch.Generator().manual_seed(V)
    k = 6
    x, ids, values, _, _ = _case(g, rows, V, k, dtype, False, False, 1.0)
    ids[:] = torch.arange(k, dtype=torch.int32, device=DEV) * 7 % V
    values[:] = torch.randn(rows, k, generator=g).to(DEV)
    lowest = torch.finfo(dtype).min
    x[0, 100:] = -math.inf                                    # a mask that leaves the teacher's tokens
    x[1, 50:] = lowest
    x[2, 0], values[2, 0] = -math.inf, -math.inf              # no weight where there is no probability
    x[3, 0] = -math.inf                                       # a weight where there is none: the loss is infinite
    x[4] = -math.inf
    x[5] = math.nan
    x[6, V - 1] = math.nan
    x[7] = -math.inf
    ids[5], values[7] = -1, -math.inf                         # rows without weights, whatever their logits are
    dloss = torch.ones(rows, device=DEV)
    loss, stats = E.eagle3_distill(x, ids, values, want_stats=True)
    grad = E.eagle3_distill_grad(dloss, stats, x, ids, values)
    step_loss, step_grad = E.eagle3_distill_step(dloss, x, ids, values)
    for l, d in ((loss.cpu(), grad.cpu()), (step_loss.cpu(), step_grad.cpu())):
        fine = [0, 1, 2] + list(range(8, rows))
        ref = _reference(x[fine], ids[fine], values[fine], None, None, 1.0, dloss[fine])
        _check(l[fine], ref[0], ref[2])
        _check(d[fine], ref[1], ref[3], dtype)
        assert bool((d[0, 100:] == 0).all()) and bool((d[1, 50:] == 0).all())
        assert l[3] == math.inf and bool(torch.isfinite(d[3]).all()) and d[3, 0] < 0
        assert bool(l[[4, 6]].isnan().all()) and bool(d[[4, 6]].isnan().all())
        assert bool((l[[5, 7]] == 0).all()) and bool((d[[5, 7]] == 0).all())
    # what the teacher does not know: NaN stays in its row; a dloss of 0 hides a row
    values[0, 1] = math.nan
    dloss[4] = 0
    loss, stats = E.eagle3_distill(x, ids, values, want_stats=True)
    grad = E.eagle3_distill_grad(dloss, stats, x, ids, values)
    _, step_grad = E.eagle3_distill_step(dloss, x, ids, values)
    for d in (grad, step_grad):
        assert bool(d[0].isnan().any()) and bool((d[4] == 0).all()) and bool(torch.isfinite(d[1]).all())
    assert bool(loss[0].isnan()) and bool(torch.isfinite(loss[1]))


def test_autograd_and_differences():
    g = torch.Generator().manual_seed(6)
    rows, V, k = 40, 300, 12
    x, ids, values, lse, t2d = _case(g, rows, V, k, FP32, False, True, 1.5)
    x.requires_grad_()
    w = torch.randn(rows, generator=g).to(DEV)
    loss, stats = E.eagle3_distill(x, ids, values, lse, t2d, 1.5, want_stats=True)
    assert loss.requires_grad and not stats.requires_grad
    loss.backward(w)
    assert torch.equal(x.grad, E.eagle3_distill_grad(w, stats, x.detach(), ids, values, lse, t2d, 1.5))
    # central differences, step 2^-6 along u: a softmax's third derivative is below 2 |u|^3 of a row's weight, losses are off by some 40 U of their size
    u, e = torch.randn(rows, V, generator=g).to(DEV), 2.0 ** -6
    f = lambda s: E.eagle3_distill(x.detach() + s * e * u, ids, values, lse, t2d, 1.5).double()
    d = ((f(1) - f(-1)) * w.double()).sum() / (2 * e)
    along = (x.grad.double() * u.double()).sum()
    assert abs(float(d - along)) <= float(w.abs().sum()) * (2 * 4.0 ** 3 * e * e + 40 * U * float(loss.detach().max()) / e)
    # an expanded gradient, as of a mean
    x.grad = None
    E.eagle3_distill(x, ids, values, lse, t2d, 1.5).mean().backward()
    assert torch.equal(x.grad, E.eagle3_distill_grad(torch.full((rows,), 1 / rows, device=DEV), stats, x.detach(), ids, values, lse, t2d, 1.5))
    # both in one call for logits that require a gradient: nothing is recorded, and not over them
    both = E.eagle3_distill_step(torch.full((rows,), 1 / rows, device=DEV), x, ids, values, lse, t2d, 1.5)
    assert not both[1].requires_grad
    for call in (lambda o: E.eagle3_distill_step(w, x, ids, values, out=o), lambda o: E.eagle3_distill_grad(w, stats, x, ids, values, out=o)):
        with pytest.raises(ValueError):
            call(x)
    with pytest.raises(ValueError):
        E.eagle3_distill(x, ids, values.clone().requires_grad_())


def test_captured_losses_replay():
    """Rows in parts and whole, other logits and teachers at every replay, against eager calls."""
    g = torch.Generator().manual_seed(7)
    for rows, V in ((6, 40000), (1030, 700)):
        x, ids, values, lse, _ = _case(g, rows, V, 20, BF16, True, False, 1.0)
        dloss = torch.randn(rows, generator=g).to(DEV)

        def step():
            loss, stats = E.eagle3_distill(x, ids, values, lse, want_stats=True)
            return (loss, E.eagle3_distill_grad(dloss, stats, x, ids, values, lse), *E.eagle3_distill_step(dloss, x, ids, values, lse))

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for i in range(4):
            x.copy_(torch.randn(rows, V, generator=g))
            ids.copy_(torch.randint(0, V, (rows, 20), generator=g, dtype=torch.int32))
            graph.replay()
            want = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i
            (torch.randn(1000, device=DEV) * 2).sum()
