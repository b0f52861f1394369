"""Rotary positions and their gradient on the GPU against the formula in 64 bits, and the gradient against differences."""
import math

import pytest
import torch

import paper_2503_01840_amd as E
from oracle import eagle3_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _reference(x, positions, rot, theta, interleaved, scaling, amplitude, sign, factor=8.0, low=1.0, high=4.0, original=8192.0):
    """(result, sum of the magnitudes of a pair) in 64 bits."""
    x = x.double().cpu()
    f = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        w = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * (w + (1 - w) / factor)
    t = positions.double().cpu()[:, None, None] * f
    ia = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    a, b = x[..., ia], x[..., ib]
    y, mag = x.clone(), torch.zeros_like(x)
    y[..., ia] = amplitude * (a * t.cos() - sign * b * t.sin())
    y[..., ib] = amplitude * (b * t.cos() + sign * a * t.sin())
    mag[..., ia] = mag[..., ib] = abs(amplitude) * (a.abs() + b.abs())
    return y, mag


def _bound(y, mag, dtype):
    """Angle: the fraction of a turn and its double in 32 bits (pi 2^-25 + pi 2^-25), sine and cosine to 2 units of 2^-24, times the amplitude,
    products and sum to half a unit each: 2^-24 (pi + 2 + 0.5 + 1) < 7 * 2^-24 of the pair's magnitudes; one rounding to bf16."""
    return 7 * 2.0 ** -24 * mag + (2.0 ** -8 * (y.abs() + 7 * 2.0 ** -24 * mag) if dtype == torch.bfloat16 else 0) + 1e-37


def _check(got, x, rope_args, positions, sign):
    y, mag = _reference(x, positions, *rope_args, sign)
    err = (got.double().cpu() - y).abs()
    assert bool((err <= _bound(y, mag, x.dtype)).all()), float((err - _bound(y, mag, x.dtype)).max())


CASES = [  # rows, H, Hkv, d, rot, interleaved, scaling
    (1, 1, 1, 2, 2, False, "none"), (1, 32, 8, 128, 128, False, "parts"), (3, 4, 2, 64, 64, True, "linear"), (65, 3, 1, 80, 40, False, "none"),
    (7, 5, 5, 128, 122, False, "parts"), (130, 8, 2, 128, 64, True, "parts"), (33, 2, 1, 256, 256, True, "none"), (5, 1, 1, 1024, 512, False, "linear"),
    (515, 28, 4, 128, 128, False, "none"), (9, 4, 4, 66, 34, True, "none"), (257, 6, 2, 64, 16, False, "none"), (2, 64, 8, 128, 128, True, "linear"),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES)
def test_rope_and_gradient_follow_the_formula(case, dtype):
    rows, H, Hkv, d, rot, inter, scaling = case
    g = torch.Generator().manual_seed(rows + d)
    amplitude = 1.2079441541679836 if scaling == "parts" else 1.0
    rope = E.Rope(rot, 5e5, interleaved=inter, scaling=scaling, factor=8.0, amplitude=amplitude, device=DEV)
    args = (rot, 5e5, inter, scaling, amplitude)
    q, k = (torch.randn(rows, h, d, generator=g).to(dtype).to(DEV) for h in (H, Hkv))
    pos = torch.randint(-50, 131072, (rows,), generator=g, dtype=torch.int32)
    pos[0] = 0
    pos[-1] = 2 ** 24 + 1 if rows > 2 else 131071
    p = pos.to(DEV)
    keep = q.clone(), k.clone()
    for call, sign in ((E.eagle3_rope, 1), (E.eagle3_rope_grad, -1)):
        got = call(rope, p, q, k)
        _check(got[0], q, args, pos, sign)
        _check(got[1], k, args, pos, sign)
        alone, into = call(rope, p, q), torch.zeros_like(q)
        assert torch.equal(alone, got[0]) and call(rope, p, q, out=into) is into and torch.equal(into, alone)
    assert torch.equal(q, keep[0]) and torch.equal(k, keep[1])
    # parts of longer rows, in place: the same bits, and the rest of the rows as it was
    both = torch.randn(rows, H + 2 * Hkv, d, generator=g).to(dtype).to(DEV)
    was = both.clone()
    qv, kv = both[:, :H], both[:, H:H + Hkv]
    want = E.eagle3_rope(rope, p, qv.contiguous(), kv.contiguous())
    E.eagle3_rope(rope, p, qv, kv, out=(qv, kv))
    assert torch.equal(qv, want[0]) and torch.equal(kv, want[1]) and torch.equal(both[:, H + Hkv:], was[:, H + Hkv:])


# rows at addresses and distances that allow no wide loads
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,extra", [(1, 0), (0, 1), (2, 6), (8, 8), (4, 4)])
def test_rope_at_odd_addresses(dtype, offset, extra):
    rows, H, Hkv, d = 19, 4, 2, 128
    g = torch.Generator().manual_seed(offset)
    stride = H * d + extra
    flat = torch.randn(offset + rows * stride + 64, generator=g).to(dtype).to(DEV)
    q = flat.as_strided((rows, H, d), (stride, d, 1), offset)
    k = torch.randn(rows, Hkv, d, generator=g).to(dtype).to(DEV)
    out = torch.full((offset + rows * stride + 64,), 3.0, dtype=dtype, device=DEV)
    qo = out.as_strided((rows, H, d), (stride, d, 1), offset)
    pos = torch.randint(0, 5000, (rows,), generator=g, dtype=torch.int32)
    for inter in (False, True):
        rope = E.Rope(d, 1e4, interleaved=inter, device=DEV)
        want = E.eagle3_rope(rope, pos.to(DEV), q.contiguous(), k)
        out.fill_(3.0)
        got = E.eagle3_rope(rope, pos.to(DEV), q, k, out=(qo, None))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        qo.fill_(3.0)
        assert bool((out == 3.0).all()), "only the rows are written"


def test_rope_is_the_framework_s_rotation():
    """The oracle's (half layout, unscaled) rotation of queries and keys."""
    rows, H, d = 40, 4, 64
    x = torch.randn(rows, H, d, generator=torch.Generator().manual_seed(1))
    pos = torch.arange(rows, dtype=torch.int32) + 1000
    got = E.eagle3_rope(E.Rope(d, 1e4, device=DEV), pos.to(DEV), x.to(DEV)).cpu().double()
    ref = torch.from_numpy(O.rope(x.double().numpy(), pos.numpy(), 1e4))
    assert bool(((got - ref).abs() <= 7 * 2.0 ** -24 * 2 * x.abs().max()).all())


@pytest.mark.parametrize("inter", [False, True])
def test_gradient_against_differences(inter):
    """The map is linear: <w, rope(x + e) - rope(x)> = <rope_grad(w), e> up to the roundings of the four products' terms."""
    rows, H, d, rot = 11, 3, 64, 48
    g = torch.Generator().manual_seed(4)
    x, e, w = (torch.randn(rows, H, d, generator=g).to(DEV) for _ in range(3))
    pos = torch.randint(0, 131072, (rows,), generator=g, dtype=torch.int32).to(DEV)
    rope = E.Rope(rot, 5e5, interleaved=inter, scaling="parts", factor=8.0, amplitude=1.25, device=DEV)
    diff = (E.eagle3_rope(rope, pos, x + e).double() - E.eagle3_rope(rope, pos, x).double())
    left, right = (w.double() * diff).sum((1, 2)), (E.eagle3_rope_grad(rope, pos, w).double() * e.double()).sum((1, 2))
    # each rotated value is off by 7 units of 2^-24 of its pair (|pair| < 1.25 * 2 * 5 * 2), x + e by half a unit of 8; weights below 5
    bound = H * d * 5 * (2 * 7 * 2.0 ** -24 * 1.25 * 20 + 1.25 * 2 * 2.0 ** -24 * 8 + 7 * 2.0 ** -24 * 1.25 * 10)
    assert float((left - right).abs().max()) <= bound < 0.1 * float(left.abs().max())


@pytest.mark.parametrize("inter", [False, True])
def test_gradient_as_a_backward_pass(inter):
    """In a torch.autograd.Function: the gradients that torch finds for the same formula in elementary operations."""
    rows, H, Hkv, d, rot = 9, 4, 2, 64, 64
    g = torch.Generator().manual_seed(6)
    rope = E.Rope(rot, 1e4, interleaved=inter, amplitude=1.5, device=DEV)
    pos = torch.randint(0, 4096, (rows,), generator=g, dtype=torch.int32).to(DEV)

    class Rotate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k):
            return E.eagle3_rope(rope, pos, q, k)

        @staticmethod
        def backward(ctx, dq, dk):
            return E.eagle3_rope_grad(rope, pos, dq.contiguous(), dk.contiguous())

    leaves = [torch.randn(rows, h, d, generator=g).to(DEV).requires_grad_() for h in (H, Hkv)]
    w = [torch.randn(rows, h, d, generator=g).to(DEV) for h in (H, Hkv)]
    (sum((a * b).sum() for a, b in zip(Rotate.apply(*leaves), w))).backward()
    t = pos.double()[:, None, None] * 1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    for x, weight in zip(leaves, w):
        y = x.detach().double().requires_grad_()
        a, b = (y[..., 0::2], y[..., 1::2]) if inter else (y[..., :rot // 2], y[..., rot // 2:])
        ra, rb = 1.5 * (a * t.cos() - b * t.sin()), 1.5 * (b * t.cos() + a * t.sin())
        wa, wb = (weight[..., 0::2], weight[..., 1::2]) if inter else (weight[..., :rot // 2], weight[..., rot // 2:])
        (ra * wa + rb * wb).sum().backward()
        assert bool(((x.grad - y.grad).abs() <= 7 * 2.0 ** -24 * 1.5 * 2 * float(weight.abs().max())).all())


def test_nan_and_infinity_stay_in_their_pair():
    rows, H, d, rot = 4, 2, 128, 64
    x = torch.ones(rows, H, d, dtype=torch.bfloat16)
    x[1, 0, 3], x[2, 1, 40], x[3, 0, 100] = float("nan"), float("inf"), float("nan")
    rope = E.Rope(rot, 1e4, device=DEV)
    y = E.eagle3_rope(rope, torch.arange(rows, dtype=torch.int32, device=DEV), x.to(DEV)).cpu()
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, 0, [3, 35]] = True
    want[2, 1, [8, 40]] = True
    want[3, 0, 100] = True
    assert torch.equal(bad, want)


def test_large_prompt_and_one_row_agree():
    """The rows of a prompt of 5000 one by one: the same bits."""
    g = torch.Generator().manual_seed(9)
    T, H, d = 5000, 8, 128
    q = torch.randn(T, H, d, generator=g).bfloat16().to(DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    rope = E.Rope(d, 5e5, device=DEV)
    y = E.eagle3_rope(rope, pos, q)
    for i in (0, 1, 63, 64, 2500, 4998, 4999):
        assert torch.equal(E.eagle3_rope(rope, pos[i:i + 1], q[i:i + 1])[0], y[i])


def test_binding_refuses_what_does_not_fit():
    rope = E.Rope(64, 1e4, device=DEV)
    q, pos = torch.zeros(3, 2, 64, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        E.eagle3_rope(rope, pos.long(), q)
    with pytest.raises(ValueError):
        E.eagle3_rope(rope, pos[:2], q)
    with pytest.raises(ValueError):
        E.eagle3_rope(rope, pos, q.half())
    with pytest.raises(ValueError):
        E.eagle3_rope(rope, pos, q.transpose(0, 1))
    with pytest.raises(ValueError):
        E.eagle3_rope(rope, pos, q, q.bfloat16())
    with pytest.raises(ValueError):
        E.eagle3_rope(rope, pos.cpu(), q)
    with pytest.raises(ValueError):
        E.eagle3_rope(rope, pos, q[..., ::2])
    with pytest.raises(E.Eagle3Error):
        E.eagle3_rope(E.Rope(128, 1e4, device=DEV), pos, q)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("alone", [False, True])
def test_gradients_are_recorded_where_they_are_wanted(inter, alone):
    """The gradients of leaves through the call itself are the bits of eagle3_rope_grad, and those of the gradients' gradients of eagle3_rope."""
    rows, H, Hkv, d, rot = 9, 4, 2, 64, 48
    g = torch.Generator().manual_seed(7)
    rope = E.Rope(rot, 1e4, interleaved=inter, amplitude=1.5, device=DEV)
    pos = torch.randint(0, 4096, (rows,), generator=g, dtype=torch.int32).to(DEV)
    heads = (H,) if alone else (H, Hkv)
    x = [torch.randn(rows, h, d, generator=g).to(DEV).requires_grad_() for h in heads]
    w = [torch.randn(rows, h, d, generator=g).to(DEV).requires_grad_() for h in heads]
    tup = lambda y: y if isinstance(y, tuple) else (y,)
    y = tup(E.eagle3_rope(rope, pos, *x))
    with torch.no_grad():
        plain, back = tup(E.eagle3_rope(rope, pos, *x)), tup(E.eagle3_rope_grad(rope, pos, *w))
    assert all(torch.equal(a, b) and a.requires_grad and not b.requires_grad for a, b in zip(y, plain))
    dx = torch.autograd.grad(y, x, w, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(dx, back))
    u = [torch.randn_like(t) for t in x]
    with torch.no_grad():
        again = tup(E.eagle3_rope(rope, pos, *u))
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(dx, w, u), again))
    # expanded gradients (of a sum); and of one of the two tensors only, the other's result unused
    sum(t.sum() for t in tup(E.eagle3_rope(rope, pos, *x))).backward()
    ones = tup(E.eagle3_rope_grad(rope, pos, *[torch.ones_like(t) for t in x]))
    assert all(torch.equal(t.grad, o) for t, o in zip(x, ones))
    if not alone:
        x[0].grad = None
        q, _ = E.eagle3_rope(rope, pos, x[0], x[1].detach())
        q.backward(w[0].detach())
        assert torch.equal(x[0].grad, back[0])
    # positions that move on before the backward pass would give other gradients
    y = tup(E.eagle3_rope(rope, pos, *x))
    pos += 1
    with pytest.raises(RuntimeError):
        y[0].sum().backward()


def test_results_are_not_written_over_where_gradients_are_recorded():
    rope = E.Rope(64, 1e4, device=DEV)
    q, pos = torch.ones(3, 2, 64, device=DEV), torch.arange(3, dtype=torch.int32, device=DEV)
    leaf = q.clone().requires_grad_()
    product = leaf * 2
    for call in (E.eagle3_rope, E.eagle3_rope_grad):
        for x, k, out in ((product, None, product), (q, None, leaf), (q, product, (None, product)), (q, product, (q, None))):
            with pytest.raises(ValueError):
                call(rope, pos, x, k, out=out)
    with torch.no_grad():
        want = E.eagle3_rope(rope, pos, product)
        assert E.eagle3_rope(rope, pos, product, out=product) is product and torch.equal(product, want)
    x = q.clone()
    assert E.eagle3_rope(rope, pos, x, out=x) is x and not x.requires_grad


# A wavefront has up to 8192 / rows (at least one) parts of a row's pieces and takes 256 of them a round, 512 single elements: 584 pieces in three rounds (bf16) or
# 1168 in five, 1168 or 2336 between neighbours, 4891 elements in ten; 3000 rows in two parts of 320 or 640; rows whose heads
# are copied by half
MANY_ROUNDS = [(4100, 64, 9, 128, 128, False), (4100, 64, 9, 128, 128, True), (4100, 64, 9, 128, 122, False), (4100, 64, 9, 128, 122, True), (3000, 64, 9, 128, 128, False),
               (4097, 64, 9, 128, 64, False)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,H,Hkv,d,rot,inter", MANY_ROUNDS)
def test_many_rows_of_many_heads(dtype, rows, H, Hkv, d, rot, inter):
    """The bits of 250 rows at a time, whose pieces lie within one round; some rows against the formula; in place too."""
    g = torch.Generator(device=DEV).manual_seed(rows + rot)
    rope = E.Rope(rot, 5e5, interleaved=inter, scaling="linear", amplitude=1.25, device=DEV, factor=8.0)
    x = torch.randn(rows, H + Hkv, d, generator=g, device=DEV).to(dtype)
    q, k = x[:, :H], x[:, H:]
    pos = torch.randint(-50, 131072, (rows,), generator=g, device=DEV, dtype=torch.int32)
    for call, sign in ((E.eagle3_rope, 1), (E.eagle3_rope_grad, -1)):
        got = call(rope, pos, q, k)
        few = [call(rope, pos[i:i + 250], q[i:i + 250], k[i:i + 250]) for i in range(0, rows, 250)]
        for i in range(2):
            assert torch.equal(got[i], torch.cat([f[i] for f in few]))
        at = [0, 1, 2, 3, rows // 2, rows - 2, rows - 1]
        for y, t in zip(got, (q, k)):
            _check(y[at], t[at], (rot, 5e5, inter, "linear", 1.25), pos[at], sign)
        both = x.clone()
        call(rope, pos, both[:, :H], both[:, H:], out=(both[:, :H], both[:, H:]))
        assert torch.equal(both[:, :H], got[0]) and torch.equal(both[:, H:], got[1])


def test_a_captured_step_with_its_gradients_replays():
    """Forward and backward pass in one graph, replayed with other inputs and positions, against the eager calls."""
    rows, H, Hkv, d = 65, 4, 2, 64
    g = torch.Generator().manual_seed(8)
    rope = E.Rope(d, 1e4, device=DEV)
    pos = torch.arange(rows, dtype=torch.int32, device=DEV)
    x = [torch.randn(rows, h, d, generator=g).to(DEV).requires_grad_() for h in (H, Hkv)]
    w = [torch.randn(rows, h, d, generator=g).to(DEV) for h in (H, Hkv)]

    def step():
        y = E.eagle3_rope(rope, pos, *x)
        return [t.detach() for t in y], torch.autograd.grad(y, x, w)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = step()
    for i in range(4):
        with torch.no_grad():
            for t in x + w:
                t.copy_(torch.randn(t.shape, generator=g))
            pos += 100
            want, grads = E.eagle3_rope(rope, pos, *x), E.eagle3_rope_grad(rope, pos, *w)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(list(y) + list(dx), list(want) + list(grads))), i
        (torch.randn(1000, device=DEV) * 2).sum()
