"""Long float32 recurrences against the float64 oracle with an error that forgets as the recurrence does: a state that is exchanged between warps and blocks in fewer bits, or
a tile's end that is left out, shows in every channel but the slowest ones.

Derivation, with s = 2^-24.  A step rounds its state twice, by at most s times its magnitude M (the recurrence of absolute values); it is run twice, once composed from zero
and once from the state in front.  The composed map rounds u, A and C twice each a step, all of which later steps make smaller by a.  A warp has at least 4 steps; behind them its
map is composed with the block's (3 roundings of u, 3 of C or A), the block's with the cluster's states (2), the state with the warps' maps (2): 10 in 4 steps, less than 3 a
step.  Together 2 * 2 + 4 + 3 = 11 roundings: 12 s (M_i + M_{i-1}) a step.  b is off by 2^-20 relative (power 2^-22, quotient 2^-22, composition), which moves the state by that
times b (|x| + M), uncoupled b M.  So e_i = a_i e_{i-1} + 12 s (M_i + M_{i-1}) + 2^-20 b_i (|x_i| + M_{i-1})."""
import numpy as np
import pytest

from oracle import operators as orc
from test_gpu_operators import HALF, _close, _np, _recurrence_case, _torch

pytestmark = pytest.mark.gpu
S, GATE = 2.0 ** -24, 2.0 ** -20


def _forgotten(a, added, lengths, backwards):
    """e_i = a_i e_{i-1} + added_i over each sequence's steps (from the last one where backwards); behind the last one too.  [B, T, D], [B, D]"""
    B, T, D = a.shape
    out, cur = np.zeros((B, T, D)), np.zeros((B, D))
    for i in (range(T - 1, -1, -1) if backwards else range(T)):
        on = (np.asarray(lengths) > i)[:, None]
        cur = np.where(on, a[:, i] * cur + added[:, i], cur)
        out[:, i] = cur
    return out, cur


@pytest.mark.parametrize("coupled", [True, False])
@pytest.mark.parametrize("B,T,D,kw", [(1, 24001, 64, {}), (2, 12000, 72, dict(ragged=True)), (1, 2049, 34, {}), (2, 9000, 33, dict(ragged=True)), (75, 290, 72, dict(layout="time")),
                                      (3, 3000, 328, dict(ragged=True)), (300, 70, 64, dict(ragged=True))])
def test_float32_errors_are_forgotten_with_the_state(B, T, D, kw, coupled):
    torch, b, _ = _torch()
    c = _recurrence_case(B, T, D, "f32", seed=31, **kw)
    y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], lengths=c["t_len"], coupled=coupled)
    ref, refT, mag, magT = orc.recurrence_forward(c["x"], c["gate"], c["y0"], c["lengths"], coupled)
    beta, a = orc.sigmoid(c["gate"])
    M0 = np.concatenate([np.abs(c["y0"])[:, None], mag[:, :-1]], 1)
    e, eT = _forgotten(a, 12 * S * (mag + M0) + GATE * beta * ((np.abs(c["x"]) if coupled else 0) + M0), c["lengths"], False)
    _close(_np(y), ref, np.where(mag > 0, e, 0) + HALF["f32"] * np.abs(ref), "y")
    _close(_np(yT), refT, eT, "yT")

    dy = torch.empty_like(y).copy_(c["t_dy"])
    got = b.recurrence_backward(c["t_x"], c["t_gate"], y, dy, dL_dyT=c["t_dyT"], y0=c["t_y0"], lengths=c["t_len"], coupled=coupled)
    traj = _np(y)
    dx, dg, dy0, lmag, rmag = orc.recurrence_backward(c["x"], c["gate"], traj, c["dy"], c["dyT"], c["y0"], c["lengths"], coupled)
    # r in front of a step: a (dy + r), of magnitude a lmag; what is added is rounded at the magnitude lmag
    r, r0 = _forgotten(a, 24 * S * lmag + GATE * beta * lmag, c["lengths"], True)
    behind = np.concatenate([r[:, 1:], np.zeros((B, 1, D))], 1)                 # of r behind step i, which l takes in
    behind[np.arange(T)[None] >= np.asarray(c["lengths"])[:, None] - 1] = 0     # (dyT is exact)
    el = (behind + (S + GATE) * lmag) * (np.arange(T)[None] < np.asarray(c["lengths"])[:, None])[..., None]
    before = np.concatenate([c["y0"][:, None], traj[:, :-1]], 1)
    _close(_np(got[0]), dx, (beta if coupled else 1.0) * el + HALF["f32"] * np.abs(dx), "dx")
    _close(_np(got[1]), dg, a * beta * (np.abs(c["x"]) + np.abs(before) if coupled else np.abs(before)) * el + HALF["f32"] * np.abs(dg), "dgate")
    _close(_np(got[2]), dy0, r0 + 0 * rmag, "dy0")
