"""What the calls of embeddings, norms and distillation refuse, through the C ABI with addresses that are never dereferenced, and through the binding with tensors
that are on no GPU: nothing is enqueued (there is no GPU here)."""
import ctypes as C
import math
import os

import pytest
import torch

import paper_2503_01840_amd as E
from paper_2503_01840_amd import binding as Bd

AT = 1 << 20                                                 # an address


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(E.LIB_PATH):
        from paper_2503_01840_amd.build import build_library
        build_library()
    return E.lib()


def _args(base, over):
    v = dict(base)
    assert set(over) <= set(v), over
    v.update(over)
    return list(v.values()) + [None]


EMBED = dict(dtype=1, rows=2, dim=64, vocab=10, table=AT, tokens=AT, scale=1.0, out_dtype=0, out=AT, stride=64)


@pytest.mark.parametrize("over,code", [(dict(table=None), -1), (dict(tokens=None), -1), (dict(out=None), -1), (dict(dtype=2), -2), (dict(out_dtype=-1), -2), (dict(rows=0), -2),
                                       (dict(rows=1 << 24), -2), (dict(dim=0), -2), (dict(dim=65537, stride=1 << 20), -2), (dict(vocab=0), -2), (dict(stride=63), -2),
                                       (dict(stride=1 << 40), -2), (dict(table=AT + 1), -2), (dict(out=AT + 2), -2)])
def test_embeddings(L, over, code):
    assert L.eagle3_embed(*_args(EMBED, over)) == code


EMBED_GRAD = dict(dtype=1, rows=200, dim=64, vocab=10, dy=AT, stride=64, tokens=AT, scale=1.0, add=0, out_dtype=0, d_table=AT, ws=AT, size=1 << 40)


@pytest.mark.parametrize("over,code", [(dict(dy=None), -1), (dict(tokens=None), -1), (dict(d_table=None), -1), (dict(dtype=2), -2), (dict(out_dtype=3), -2), (dict(rows=0), -2),
                                       (dict(rows=1 << 22), -2), (dict(dim=0), -2), (dict(dim=65537, stride=1 << 20), -2), (dict(rows=1 << 21, dim=1 << 15, stride=1 << 15), -2),
                                       (dict(vocab=0), -2), (dict(vocab=1 << 27), -2), (dict(vocab=1 << 26, dim=128, stride=128), -2), (dict(stride=63), -2), (dict(dy=AT + 1), -2), (dict(d_table=AT + 2), -2),
                                       (dict(ws=None), -3), (dict(ws=AT + 128), -3), (dict(size=1000), -3)])
def test_gradients_of_embeddings(L, over, code):
    assert L.eagle3_embed_grad(*_args(EMBED_GRAD, over)) == code


NORM = dict(rows=2, dim=64, x_dtype=1, x=AT, xs=64, sum_dtype=0, res=AT, rs=64, h=AT + 4096, hs=64, gain_dtype=1, gain=AT, eps=1e-5, out_dtype=1, out=AT + 8192, os=64)
BAD_NORMS = [(dict(x=None), -1), (dict(gain=None), -1), (dict(h=None), -1), (dict(res=None), -1), (dict(x_dtype=2), -2), (dict(gain_dtype=2), -2), (dict(sum_dtype=2), -2),
             (dict(sum_dtype=1, x_dtype=0), -2), (dict(rows=0), -2), (dict(rows=1 << 24), -2), (dict(dim=0), -2), (dict(dim=16385), -2), (dict(eps=-1e-6), -2), (dict(eps=math.nan), -2),
             (dict(xs=63), -2), (dict(rs=63), -2), (dict(hs=63), -2), (dict(xs=1 << 40), -2), (dict(x=AT + 1), -2), (dict(res=AT + 2), -2), (dict(gain=AT + 1), -2),
             (dict(h=AT, hs=65), -2)]


@pytest.mark.parametrize("over,code", BAD_NORMS + [(dict(out=None), -1), (dict(out_dtype=2), -2), (dict(os=63), -2), (dict(out=AT + 1), -2), (dict(out=AT, out_dtype=0), -2),
                                                   (dict(out=AT, os=65), -2)])
def test_norms(L, over, code):
    assert L.eagle3_add_norm(*_args(NORM, over)) == code


CODES = {**{n: v for n, v in NORM.items() if n not in ("out_dtype", "out", "os")}, "group": 128, "codes": AT, "cs": 64, "scales": AT}


@pytest.mark.parametrize("over,code", BAD_NORMS + [(dict(codes=None), -1), (dict(scales=None), -1), (dict(group=64), -2), (dict(group=-1), -2), (dict(cs=63), -2), (dict(scales=AT + 2), -2)])
def test_norms_in_8_bits(L, over, code):
    assert L.eagle3_add_norm_codes(*_args(CODES, over)) == code


NORM_GRAD = dict(rows=2, dim=64, dy_dtype=1, dy=AT, dys=64, sum_dtype=0, h=AT, hs=64, dh=AT, dhs=64, gain_dtype=1, gain=AT, eps=1e-5, d_sum=AT + 4096, dss=64, x_dtype=1, dx=AT + 8192,
                 dxs=64, d_gain=AT, ws=AT, size=1 << 30)


@pytest.mark.parametrize("over,code", [(dict(dy=None), -1), (dict(h=None), -1), (dict(gain=None), -1), (dict(d_sum=None, dx=None), -1), (dict(dy_dtype=2), -2), (dict(sum_dtype=2), -2),
                                       (dict(gain_dtype=2), -2), (dict(x_dtype=2), -2), (dict(sum_dtype=1, x_dtype=0), -2), (dict(rows=0), -2), (dict(rows=1 << 24), -2), (dict(dim=0), -2),
                                       (dict(dim=16385), -2), (dict(eps=-1.0), -2), (dict(dys=63), -2), (dict(hs=63), -2), (dict(dhs=63), -2), (dict(dss=63), -2), (dict(dxs=63), -2),
                                       (dict(dy=AT + 1), -2), (dict(h=AT + 2), -2), (dict(dh=AT + 2), -2), (dict(d_sum=AT + 2), -2), (dict(dx=AT + 1), -2), (dict(d_gain=AT + 1), -2),
                                       (dict(d_sum=AT, dss=65), -2), (dict(ws=None), -3), (dict(ws=AT + 16), -3), (dict(size=511), -3)])
def test_gradients_of_norms(L, over, code):
    assert L.eagle3_add_norm_grad(*_args(NORM_GRAD, over)) == code


def test_results_over_each_other(L):
    """Norm and sum, codes and sum, and the two gradients, in rows of one buffer: refused where a byte is written by both."""
    apart = dict(h=AT + 65536, out=AT + 131072)
    for over in (dict(out=AT + 65536), dict(out=AT + 65536, out_dtype=0), dict(out=AT + 65536 + 64, out_dtype=0), dict(out=AT + 65536 - 4, out_dtype=0), dict(out=AT + 65536 + 192, out_dtype=0),
                 dict(out=AT + 65536 + 256, out_dtype=0), dict(out=AT + 65536, os=70), dict(rows=1, out=AT + 65536 + 252, hs=99), dict(rows=1, out=AT + 65536 - 126, os=99)):
        assert L.eagle3_add_norm(*_args(NORM, {**apart, **over})) == -2, over
    for over in (dict(codes=AT + 65536), dict(codes=AT + 65536, cs=256), dict(codes=AT + 65536 + 255, cs=256), dict(codes=AT + 65536 - 63, cs=256), dict(rows=1, codes=AT + 65536 + 255)):
        assert L.eagle3_add_norm_codes(*_args(CODES, {"h": AT + 65536, **over})) == -2, over
    # every place of dx around d_sum against the bytes themselves; without a workspace nothing is enqueued in any case
    size = {0: 4, 1: 2}
    for rows, stride in ((1, 5), (2, 3), (2, 7), (3, 5)):
        for sum_t, x_t in ((0, 0), (1, 1), (0, 1)):
            for x_stride in {stride, stride * size[sum_t] // size[x_t]}:
                if x_stride < 3:
                    continue
                bytes_of = lambda at, s, t: {at + r * s * size[t] + b for r in range(rows) for b in range(3 * size[t])}
                for off in range(-40, 42, 2 if x_t else 4):
                    both = dict(rows=rows, dim=3, dys=3, hs=3, dh=None, sum_dtype=sum_t, d_sum=AT + 65536, dss=stride, x_dtype=x_t, dx=AT + 65536 + off, dxs=x_stride, ws=None)
                    meet = bool(bytes_of(0, stride, sum_t) & bytes_of(off, x_stride, x_t))
                    if rows > 1 and stride * size[sum_t] != x_stride * size[x_t]:
                        meet = off == 0                       # rows not equally far apart: known by their beginning only
                    same = off == 0 and sum_t == x_t and stride == x_stride
                    assert L.eagle3_add_norm_grad(*_args(NORM_GRAD, both)) == (-2 if meet and not same else -3), both


def _teacher(**over):
    v = dict(ids=AT, values=AT, lse=None, t2d=None, n_t2d=0, k=4, temperature=1.0)
    v.update(over)
    return Bd.Teacher(*v.values())


HEAD = dict(dtype=1, rows=2, vocab=1000, logits=AT, stride=1000, teacher=None)
CALLS = {"eagle3_distill": {**HEAD, "loss": AT, "stats": None, "ws": AT, "size": 1 << 40},
         "eagle3_distill_grad": {**HEAD, "stats": AT, "dloss": AT, "out": AT + 8192, "os": 1000},
         "eagle3_distill_step": {**HEAD, "dloss": AT, "loss": AT, "out": AT + 8192, "os": 1000, "ws": AT, "size": 1 << 40}}


@pytest.mark.parametrize("call", CALLS)
def test_distillation(L, call):
    f = getattr(L, call)
    for over, code in [(dict(ids=None), -1), (dict(values=None), -1), (dict(k=0), -2), (dict(k=1025), -2), (dict(t2d=AT), -2), (dict(temperature=0.0), -2), (dict(temperature=-1.0), -2),
                       (dict(temperature=math.inf), -2), (dict(temperature=math.nan), -2), (dict(temperature=1e-39), -2)]:
        assert f(*_args(CALLS[call], dict(teacher=_teacher(**over)))) == code, over
    wrong = [(dict(teacher=None), -1), (dict(logits=None), -1), (dict(dtype=2), -2), (dict(rows=0), -2), (dict(rows=1 << 24), -2), (dict(vocab=0), -2),
             (dict(vocab=1 << 27, stride=1 << 27), -2), (dict(stride=999), -2), (dict(stride=1 << 40), -2), (dict(logits=AT + 1), -2), (dict(loss=None), -1), (dict(dloss=None), -1), (dict(out=None), -1),
             (dict(os=999), -2), (dict(out=AT + 1), -2), (dict(out=AT, os=1001), -2), (dict(stats=AT + 4), -2)]
    for over, code in wrong:
        if set(over) <= set(CALLS[call]):
            assert f(*_args(CALLS[call], {"teacher": _teacher(), **over})) == code, over
    if call == "eagle3_distill_grad":
        assert f(*_args(CALLS[call], dict(teacher=_teacher(), stats=None))) == -1


def test_workspaces(L):
    n = C.c_size_t(5)
    assert L.eagle3_embed_grad_workspace(10, 10, 10, None) == L.eagle3_add_norm_grad_workspace(10, 10, None) == L.eagle3_distill_workspace(10, 10, None) == -1
    assert L.eagle3_embed_grad_workspace(0, 10, 10, n) == L.eagle3_add_norm_grad_workspace(10, 16385, n) == L.eagle3_distill_workspace(10, 0, n) == -2 and n.value == 5
    assert L.eagle3_distill_workspace(1, 1 << 26, n) == 0
    if n.value:                                               # few long rows are worked on in parts
        for ws, size in ((None, n.value), (AT, n.value - 1), (AT + 128, n.value)):
            for call in ("eagle3_distill", "eagle3_distill_step"):
                over = dict(teacher=_teacher(), rows=1, vocab=1 << 26, stride=1 << 26, ws=ws, size=size)
                if "os" in CALLS[call]:
                    over["os"] = 1 << 26
                assert getattr(L, call)(*_args(CALLS[call], over)) == -3
    # every size has one: no overflow, whole lines
    for rows, dim in ((1, 1), (33, 7), ((1 << 22) - 1, 16383), (4097, 65536)):
        assert L.eagle3_embed_grad_workspace(rows, dim, 10, n) == 0 and n.value >= 16 * rows and n.value % 256 == 0
    for rows, dim in ((1, 1), (511, 16384), ((1 << 24) - 1, 16384)):
        assert L.eagle3_add_norm_grad_workspace(rows, dim, n) == 0 and n.value >= 4 * min(rows, 512) * dim and n.value % 256 == 0


def test_the_binding_wants_tensors_on_a_gpu(L):
    x, tok = torch.zeros(4, 16), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: E.eagle3_embed(x, tok), lambda: E.eagle3_embed_grad(x, tok, 9), lambda: E.eagle3_add_norm(x, x[0], 1e-5), lambda: E.eagle3_add_norm_codes(x, x[0], 1e-5),
                 lambda: E.eagle3_add_norm_grad(x, x, x[0], 1e-5), lambda: E.eagle3_distill(x, tok[:, None], x[:, :1]), lambda: E.eagle3_distill_grad(x[:, 0], x[:, :2], x, tok[:, None], x[:, :1]),
                 lambda: E.eagle3_distill_step(x[:, 0], x, tok[:, None], x[:, :1])):
        with pytest.raises(ValueError):
            call()


@pytest.fixture()
def sent(L, monkeypatch):
    """What would be launched, with tensors on the CPU in the place of the GPU's."""
    got = []
    monkeypatch.setattr(Bd, "_on", lambda gpu, call, *args: got.append(args))
    monkeypatch.setattr(Bd, "_gpu_of", lambda t, what: -1)
    return got


def test_what_tensors_have_to_be(sent):
    z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype)
    i = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    x, gain, tok = z(4, 16), z(16), i(4)
    half, b16 = z(4, 16, dtype=torch.float16), z(4, 16, dtype=torch.bfloat16)
    bad = [
        lambda: E.eagle3_embed(z(9, 32)[:, :16], tok), lambda: E.eagle3_embed(z(9, 16, dtype=torch.float16), tok), lambda: E.eagle3_embed(z(9, 16), tok.long()),
        lambda: E.eagle3_embed(z(9, 16), i(2, 2)), lambda: E.eagle3_embed(z(9, 16), i(8)[::2]), lambda: E.eagle3_embed(z(9, 16), tok, out=z(4, 15)), lambda: E.eagle3_embed(z(9, 16), tok, out=z(16, 4).t()),
        lambda: E.eagle3_embed(z(9, 16), tok, dtype=torch.float16), lambda: E.eagle3_embed(z(9, 16), tok, dtype=torch.bfloat16, out=x),
        lambda: E.eagle3_embed_grad(x, i(5), 9), lambda: E.eagle3_embed_grad(z(1, 16).expand(4, 16), tok, 9), lambda: E.eagle3_embed_grad(x, tok, 9, accumulate=True),
        lambda: E.eagle3_embed_grad(x, tok, 9, out=z(9, 32)[:, :16]), lambda: E.eagle3_embed_grad(x, tok, 9, out=z(8, 16)), lambda: E.eagle3_embed_grad(x, tok, 9, out=z(9, 16).requires_grad_()),
        lambda: E.eagle3_add_norm(half, gain, 1e-5), lambda: E.eagle3_add_norm(x, z(15), 1e-5), lambda: E.eagle3_add_norm(x, z(32)[::2], 1e-5), lambda: E.eagle3_add_norm(x, gain, 1e-5, residual=b16),
        lambda: E.eagle3_add_norm(x, gain, 1e-5, residual=z(4, 15)), lambda: E.eagle3_add_norm(x, gain, 1e-5, out=(x, x)), lambda: E.eagle3_add_norm(b16, gain, 1e-5, residual=x, out=(None, b16)),
        lambda: E.eagle3_add_norm(x, gain, 1e-5, dtype=torch.float8_e4m3fn), lambda: E.eagle3_add_norm(z(2, 4, 16), gain, 1e-5), lambda: E.eagle3_add_norm(x.t(), z(4), 1e-5),
        lambda: E.eagle3_add_norm_codes(x, gain, 1e-5, out=x), lambda: E.eagle3_add_norm_grad(x, z(4, 15), gain, 1e-5), lambda: E.eagle3_add_norm_grad(x, b16, gain, 1e-5),
        lambda: E.eagle3_add_norm_grad(x, x, gain, 1e-5, dh=b16), lambda: E.eagle3_add_norm_grad(x, x, gain, 1e-5, x_dtype=torch.float16),
        lambda: E.eagle3_distill(x, i(4, 3).long(), z(4, 3)), lambda: E.eagle3_distill(x, i(4, 3), z(4, 3, dtype=torch.bfloat16)), lambda: E.eagle3_distill(x, i(5, 3), z(5, 3)),
        lambda: E.eagle3_distill(x, i(4, 3), z(4, 2)), lambda: E.eagle3_distill(x, i(4, 3), z(4, 3), lse=z(3)), lambda: E.eagle3_distill(x, i(4, 3), z(4, 3), t2d=i(7, 2)),
        lambda: E.eagle3_distill(x, i(4, 3), z(4, 3), t2d=z(7)), lambda: E.eagle3_distill(half, i(4, 3), z(4, 3)), lambda: E.eagle3_distill(x, i(4, 3), z(4, 3).requires_grad_()),
        lambda: E.eagle3_distill_step(z(3), x, i(4, 3), z(4, 3)), lambda: E.eagle3_distill_step(z(4), x, i(4, 3), z(4, 3), out=b16), lambda: E.eagle3_distill_grad(z(4), z(4), x, i(4, 3), z(4, 3)),
        lambda: E.eagle3_distill_grad(z(4), z(4, 2), x, i(4, 3), z(4, 3), out=z(4, 17)),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert not sent
    # rows any distance apart, one row of any distance
    E.eagle3_add_norm(z(4, 40)[:, 3:19], gain, 1e-5, residual=z(4, 20)[:, :16])
    assert sent[-1][4] == 40 and sent[-1][7] == 20
    E.eagle3_distill_step(z(1), z(9, 50)[::9, :16], i(1, 3), z(1, 3))
    assert sent[-1][4] == 16


def test_what_is_written_over_is_known_to_a_backward_pass(sent):
    """A result written over what a recorded call keeps for its gradient: the backward pass says so."""
    ids, values = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    logits = torch.zeros(4, 16).requires_grad_()
    loss = E.eagle3_distill(logits, ids, values).sum()
    E.eagle3_distill_step(torch.ones(4), logits.detach(), ids, values, out=logits.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    gain = torch.ones(16).requires_grad_()
    y, h = E.eagle3_add_norm(torch.zeros(4, 16), gain, 1e-5, residual=torch.zeros(4, 16))
    E.eagle3_add_norm(torch.zeros(4, 16), gain.detach(), 1e-5, residual=h.detach(), out=(None, h.detach()))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    x, at = torch.zeros(4, 16), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: E.eagle3_embed(x, at, out=x), lambda: E.eagle3_embed_grad(x, at, 4, out=x), lambda: E.eagle3_add_norm(x, x[0], 1e-5, out=x),
                 lambda: E.eagle3_add_norm_codes(x, x[0], 1e-5, residual=x, out=x), lambda: E.eagle3_distill_grad(x[:, 0].contiguous(), torch.zeros(4, 2), x, ids, values, out=x)):
        before = x._version
        call()
        assert x._version == before + 1


def _recorded_calls(mark):
    """Each input of the calls that are recorded, and what is written through `out`, as `mark` gives it."""
    z = lambda *shape: torch.zeros(*shape)
    x, gain, table, tok, ids, values = z(4, 16), z(16), z(9, 16), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32), z(4, 2)
    return [lambda: E.eagle3_embed(mark(table), tok), lambda: E.eagle3_embed(mark(table), tok, 2.0, torch.bfloat16), lambda: E.eagle3_embed(mark(table), tok, out=z(4, 16)),
            lambda: E.eagle3_embed(table, tok, out=mark(x)), lambda: E.eagle3_add_norm(mark(x), gain, 1e-5), lambda: E.eagle3_add_norm(x, mark(gain), 1e-5),
            lambda: E.eagle3_add_norm(x, gain, 1e-5, residual=mark(z(4, 16))), lambda: E.eagle3_add_norm(mark(x), gain, 1e-5, out=z(4, 16)), lambda: E.eagle3_distill(mark(x), ids, values),
            lambda: E.eagle3_distill(x, ids, mark(values)), lambda: E.eagle3_distill(x, ids, values, lse=mark(z(4))), lambda: E.eagle3_distill(mark(x), ids, values, want_stats=True)]


def test_forward_mode_derivatives_are_refused(sent):
    """A dual tensor would come back without its tangent: derivatives of 0, with no error."""
    from torch.autograd import forward_ad
    dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))
    for call in _recorded_calls(dual):
        for mode in (torch.enable_grad, torch.no_grad):       # tangents are carried on in either
            with forward_ad.dual_level(), mode(), pytest.raises(ValueError, match="forward-mode"):
                call()
    for call in (lambda t: E.eagle3_embed(t, torch.zeros(4, dtype=torch.int32)), lambda t: E.eagle3_add_norm(t, torch.ones(16), 1e-5),
                 lambda t: E.eagle3_distill(t, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))):
        with pytest.raises(Exception):
            torch.func.jvp(call, (torch.zeros(4, 16),), (torch.ones(4, 16),))
    q = torch.zeros(4, 2, 16)
    for call in (E.eagle3_rope, E.eagle3_rope_grad):
        for args in (lambda: (dual(q),), lambda: (q, dual(q)), lambda: (q, None, dual(q)), lambda: (q, q, (q.clone(), dual(q)))):
            with forward_ad.dual_level(), pytest.raises(ValueError, match="forward-mode"):
                call(None, torch.zeros(4, dtype=torch.int32), *args())
    assert not sent
    # an open level does no harm to other tensors, and a dual tensor none behind it
    with forward_ad.dual_level():
        kept = dual(torch.zeros(4, 16))
        for call in _recorded_calls(lambda t: t):
            call()
    E.eagle3_add_norm(kept, torch.ones(16), 1e-5)
    assert len(sent) == 13
