"""The table of rotary angles (host code): plain, linear and by-parts scaling against the formulas in higher precision, and refusals."""
import ctypes as C
import os
from fractions import Fraction

import pytest
import torch

import paper_2503_01840_amd as E


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(E.LIB_PATH):
        from paper_2503_01840_amd.build import build_library
        build_library()
    return E.lib()


def _turns(L, rot, theta, scaling=0, factor=1.0, low=1.0, high=4.0, original=8192.0):
    out = torch.full((max(rot, 2) // 2,), -7.0, dtype=torch.float64)
    rc = L.eagle3_rope_turns(rot, theta, scaling, factor, low, high, original, out.data_ptr())
    return rc, out


@pytest.mark.parametrize("rot", [2, 6, 64, 122, 128])
@pytest.mark.parametrize("theta", [1e4, 5e5])
def test_turns_follow_their_formulas(L, rot, theta):
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    plain = torch.exp(-i / rot * torch.log(torch.tensor(theta, dtype=torch.float64))) / (2 * torch.pi)
    rc, got = _turns(L, rot, theta)
    assert rc == 0 and torch.allclose(got, plain, rtol=1e-13, atol=0)
    assert float(got[0]) == float(Fraction(1) / Fraction(6.283185307179586))                  # pair 0: one radian per position
    rc, got = _turns(L, rot, theta, 1, factor=4.0)
    assert rc == 0 and torch.allclose(got, plain / 4, rtol=1e-13, atol=0)
    rc, got = _turns(L, rot, theta, 2, factor=8.0, low=1.0, high=4.0, original=8192.0)
    want = []
    for f in plain.tolist():
        r = 8192.0 * f
        if r <= 1.0:
            want.append(f / 8)
        elif r >= 4.0:
            want.append(f)
        else:                                                # between them, linear in the number of turns
            w = (r - 1.0) / 3.0
            want.append(f * w + f / 8 * (1 - w))
    assert rc == 0 and torch.allclose(got, torch.tensor(want, dtype=torch.float64), rtol=1e-12, atol=0)


def test_parts_leaves_fast_pairs_and_stretches_slow_ones(L):
    _, plain = _turns(L, 128, 5e5)
    _, got = _turns(L, 128, 5e5, 2, factor=8.0)
    assert got[0] == plain[0] and abs(float(got[-1] / plain[-1]) - 1 / 8) < 1e-12
    mid = (got < plain * 0.999) & (got > plain / 8 * 1.001)
    assert bool(mid.any()), "some pairs lie between the two"


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("args", [(0, 1e4), (3, 1e4), (-2, 1e4), (64, 0.0), (64, -1.0), (64, NAN), (64, INF), (64, 1e4, 3), (64, 1e4, -1),
                                  (64, 1e4, 1, 0.0), (64, 1e4, 1, NAN), (64, 1e4, 2, 8.0, 4.0, 4.0), (64, 1e4, 2, 8.0, NAN, 4.0),
                                  (64, 1e4, 2, 8.0, 1.0, INF), (64, 1e4, 2, 8.0, 1.0, 4.0, 0.0), (64, 1e4, 2, 8.0, 1.0, 4.0, INF)])
def test_turns_without_a_meaning_are_refused(L, args):
    rc, out = _turns(L, *args)
    assert rc == -2 and bool((out == -7.0).all())


def test_turns_need_a_place(L):
    assert L.eagle3_rope_turns(64, 1e4, 0, 1.0, 1.0, 4.0, 1.0, None) == -1
    with pytest.raises(ValueError):
        E.Rope(64, 1e4, scaling="cubic")
    with pytest.raises(ValueError):
        E.Rope(63, 1e4)
    with pytest.raises(ValueError):
        E.Rope(64, 1e4, device="cpu")


@pytest.mark.parametrize("args", [(64, 1e4, 1, 5e-324, 1, 4, 8192), (64, 1e4, 2, 5e-324, 1, 4, 8192), (128, 5e-324, 0, 1, 1, 4, 8192), (64, 1e-300, 1, 1e-100, 1, 4, 8192),
                                  (2, 1e4, 1, 1e-300, 1, 4, 8192)])
def test_turns_that_no_number_holds_are_refused(L, args):
    """Parameters each in range whose turns are not, or not times the farthest position: every rotated value would be NaN."""
    out = torch.full((args[0] // 2,), 7.0, dtype=torch.float64)
    assert L.eagle3_rope_turns(*args, out.data_ptr()) == -2
    assert bool((out == 7).all())
