"""Infinite states and gradients go the way of the formulas with every length of sequence: behind gates that are open far enough, f times infinity is infinity.
In dG, which multiplies and subtracts them, what they reach is infinite or NaN.  Nothing else changes."""
import numpy as np
import pytest

from test_gpu_scan import Problem, _torch

pytestmark = pytest.mark.gpu


def _others(x, b, ch, H):
    """x without channel ch of sequence b (of every gate)."""
    keep = np.ones(x.shape, bool)
    keep[b, ..., ch::H] = False
    return x[keep]


@pytest.mark.parametrize("B,T,H", [(3, 1, 5), (3, 4, 9), (2, 3, 3), (2, 5, 66), (2, 60, 9), (2, 128, 70), (3, 200, 66), (2, 600, 70)])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("where", ["c0", "dc_last", "dh"])
def test_what_an_infinite_value_reaches(B, T, H, reverse, where):
    torch, _, _ = _torch()
    p = Problem(B, T, H, reverse=reverse, seed=T)
    p.G[:, :, :H] += 3                                       # a product of 600 gates far above fp32's smallest number
    p.G[:, ::3, :H] *= -0.5 if T < 10 else 1                 # few steps: closed ones too
    clean, b, ch, t = p.run(), 1, H - 2, T // 2
    if where == "dh":
        p.dh[b, t, ch] = float("inf")
    else:
        getattr(p, where)[b, ch] = -float("inf")
    got = p.run()
    for k in got:
        assert np.array_equal(_others(got[k], b, ch, H), _others(clean[k], b, ch, H)), k
    if where == "c0":
        assert (got["h"][b, :, ch] == -np.inf).all() and got["c_last"][b, ch] == -np.inf and got["dc0"][b, ch] == clean["dc0"][b, ch]
        assert not np.isfinite(got["dG"][b, :, [ch, 2 * H + ch]]).any()
        return
    assert all(np.array_equal(got[k], clean[k]) for k in ("h", "c_last"))
    assert got["dc0"][b, ch] == (np.inf if where == "dh" else -np.inf)
    behind = slice(0, T) if where == "dc_last" else slice(t, T) if reverse else slice(0, t + 1)
    assert not np.isfinite(got["dG"][b, behind][:, [ch, H + ch]]).any()
    ahead = slice(0, 0) if where == "dc_last" else slice(0, t) if reverse else slice(t + 1, T)
    assert np.array_equal(got["dG"][b, ahead, ch::H], clean["dG"][b, ahead, ch::H])
