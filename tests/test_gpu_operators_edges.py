"""Sequence and residual operators on the GPU at their edges: gates whose slope is near the smallest normal number, states that are infinite, what lies behind the lengths, results over inputs.

Tolerances as in test_gpu_operators.py."""
import numpy as np
import pytest

from oracle import operators as orc
from test_gpu_operators import E, _check_residual, _close, _np, _recurrence_case, _recurrence_error, _residual_case, _stored, _torch, _up

pytestmark = pytest.mark.gpu

FAR = [-40.0, -46.0, -50.0, -51.0, -52.0, -60.0, -75.0, -86.0, -100.0, -np.inf]


@pytest.mark.parametrize("T", [1, 40, 1300, 5000])
@pytest.mark.parametrize("D", [48, 33])
@pytest.mark.parametrize("coupled", [True, False])
def test_recurrence_gradients_of_bfloat16_gates_far_below_zero(T, D, coupled):
    # The slope b (1 - b) of these gates is 1e-18 to 1e-38, an ordinary bfloat16 number.  Relative error of b and of the slope: the power's argument is rounded (86 * 2^-24
    # = 2^-17.6), the power, the quotient and three products 2^-21 together: below 2^-16.  Below 2^-126 b counts as zero: off by that times the other factors.
    torch, b, _ = _torch()
    rng = np.random.default_rng(17)
    c = _recurrence_case(2, T, D, "bf16", gate=rng.choice(FAR + [30.0, np.inf, 0.0], size=(2, T, D)))
    y = _up(rng.normal(size=(2, T, D)), torch.bfloat16)
    got = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"], coupled=coupled)
    _check_far(c, _np(y), got, coupled)


@pytest.mark.parametrize("T", [1, 40, 5000])
def test_recurrence_gradients_of_float16_gates_far_below_zero(T):
    # The same where a large adjoint brings the gradients into float16's range (steps that forget nothing hand it on unchanged)
    torch, b, _ = _torch()
    rng = np.random.default_rng(18)
    c = _recurrence_case(2, T, 48, "f16", gate=rng.choice([-50.0, -51.0, -52.0, -60.0, -100.0, -np.inf], size=(2, T, 48)))
    c["dyT"], c["dy"] = c["dyT"] * 2.0 ** 72, 0 * c["dy"]
    y = _up(rng.normal(size=(2, T, 48)), torch.float16)
    got = b.recurrence_backward(c["t_x"], c["t_gate"], y, None, dL_dyT=_up(c["dyT"]), y0=c["t_y0"])
    _check_far(c, _np(y), got, True)


def _check_far(c, y, got, coupled):
    dx, dg, dy0, lmag, rmag = orc.recurrence_backward(c["x"], c["gate"], y, c["dy"], c["dyT"], c["y0"], c["lengths"], coupled)
    T = y.shape[1]
    err = _recurrence_error(T, np.concatenate([lmag, np.abs(c["dyT"])[:, None]], 1))
    b, a = orc.sigmoid(c["gate"])
    before = np.concatenate([c["y0"][:, None], y[:, :-1]], 1)
    other = np.abs(c["x"]) + np.abs(before) if coupled else np.abs(before)
    el = err + 2.0 ** -16 * lmag
    _close(_np(got[0]), dx, _stored(dx, c["low"], b * el + 2.0 ** -126 * lmag if coupled else el), "dx")
    _close(_np(got[1]), dg, _stored(dg, c["low"], other * (a * b * el + 2.0 ** -126 * lmag)), "dgate")
    _close(_np(got[2]), dy0, err[:, 0], "dy0")


@pytest.mark.parametrize("M,D", [(40, 64), (9, 785), (6, 2048), (5, 4096)])
def test_residual_gradients_of_bfloat16_gates_far_below_zero(M, D):
    torch, b, _ = _torch()
    c = _residual_case(M, D, "bf16")
    g = np.random.default_rng(19).choice(FAR + [0.0, 30.0, np.inf], size=(M, D))
    c["t_gate"] = _up(g, torch.bfloat16)
    c["gate"] = _np(c["t_gate"])
    step = b.ResidualStep(D, low="bf16", h=0.3, site=21)
    w = dict(gate=c["t_gate"], w_post=c["t_w_post"], scale=c["t_scale"], w_pre=c["t_w_pre"])
    got = step.forward(c["t_y"], c["t_u"], **w)
    grads = step.backward(got[0], c["t_u"], got[2], dL_dy=c["t_dy"], dL_dz=c["t_dz"], **w)
    h, eps = float(np.float32(0.3)), float(np.float32(1e-5))
    _check_residual(c, ("rms", "rms"), h, got, {**grads, "dscale": None, "dw_post": None}, eps=eps)
    # The weights' sums may have such gates alone: beside the relative error, sigmoids below 2^-126 count as zero and are off by that times the other factors
    y1 = _np(got[0])
    ref = orc.residual_backward(y1, c["u"], c["gate"], c["w_post"], c["scale"], c["w_pre"], h, "rms", "rms", eps, c["factors"], c["dy"], c["dz"])
    n2, _, ry = orc.norm(y1, "rms", eps)
    dzw = np.abs(c["dz"] * c["w_pre"])
    amag = np.abs(c["dy"]) + ry[:, None] * (dzw + np.abs(n2) * (dzw * np.abs(n2)).mean(1, keepdims=True))
    mag = h * amag * np.abs(orc.norm(c["u"], "rms", eps)[0])
    sig = orc.sigmoid(c["gate"])[0]
    for key, w in (("dscale", c["w_post"]), ("dw_post", c["scale"])):
        _close(_np(grads[key]), ref[key], (mag * np.abs(w) * ((4 * E + M * 2.0 ** -24) * sig + 2.0 ** -126)).sum(0), key)


@pytest.mark.parametrize("B,T,D,low,layout", [(80, 300, 64, "bf16", "plain"), (75, 290, 72, "f32", "time"), (20, 700, 200, "f16", "half"), (300, 20, 64, "bf16", "plain"),
                                              (2, 4500, 40, "f16", "plain"), (3, 3000, 328, "bf16", "time"), (2, 12000, 72, "f32", "half"), (3, 23000, 40, "f16", "plain")])
@pytest.mark.parametrize("coupled", [True, False])
def test_recurrence_uses_nothing_behind_the_lengths_where_tiles_are_copied(B, T, D, low, layout, coupled):
    # Blocks by themselves and clusters: NaN behind the lengths changes no result, given outputs stay as they are there
    torch, b, _ = _torch()
    c = _recurrence_case(B, T, D, low, layout=layout)
    lengths = [(T, 0, 1, T // 2, T - 1, T // 3 + 5, 16, 17)[s % 8] for s in range(B)][::-1]
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
    kw = dict(y0=c["t_y0"], lengths=n, coupled=coupled)

    def copied(t):
        return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device).copy_(t)

    y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], **kw)
    traj, dy = copied(c["t_x"]).copy_(y), copied(c["t_dy"])
    ref = b.recurrence_backward(c["t_x"], c["t_gate"], traj, dy, dL_dyT=c["t_dyT"], **kw)
    off = torch.arange(T, device="cuda:0")[None, :, None] >= n[:, None, None]
    dirty = [copied(t).masked_fill_(off, float("nan")) for t in (c["t_x"], c["t_gate"], traj, dy)]
    out = copied(c["t_x"]).fill_(7.0)
    _, got = b.recurrence_forward(dirty[0], dirty[1], y=out, **kw)
    assert torch.equal(got, yT) and torch.equal(out, torch.where(off, torch.full_like(y, 7.0), y))
    dx, dg, flag = copied(out).fill_(5.0), copied(out).fill_(6.0), torch.zeros(1, dtype=torch.int32, device="cuda:0")
    _, _, dy0 = b.recurrence_backward(*dirty, dL_dyT=c["t_dyT"], dL_dx=dx, dL_dgate=dg, flag=flag, **kw)
    assert torch.equal(dx, torch.where(off, torch.full_like(y, 5.0), ref[0])) and torch.equal(dg, torch.where(off, torch.full_like(y, 6.0), ref[1]))
    assert torch.equal(dy0, ref[2]) and int(flag) == 0


@pytest.mark.parametrize("T,D,low", [(9, 34, "bf16"), (9, 33, "f16"), (12, 35, "f32"), (20, 63, "bf16")])
def test_recurrence_in_place_where_a_warp_runs_alone(T, D, low):
    # So many sequences that each gets one warp, whose last lanes run its last channels again: results over x, gate, dL_dy and the states, with lengths and without
    torch, b, _ = _torch()
    B = 5000
    rng = np.random.default_rng(4)
    _, _, dt = _torch()
    x, gate, dy = (_up(rng.normal(size=(B, T, D)), dt[low]) for _ in range(3))
    y0, dyT = _up(rng.normal(size=(B, D))), _up(rng.normal(size=(B, D)))
    for n in (None, torch.arange(B, dtype=torch.int32, device="cuda:0") % (T + 1)):
        y, yT = b.recurrence_forward(x, gate, y0=y0, lengths=n)
        ref = b.recurrence_backward(x, gate, y, dy, dL_dyT=dyT, y0=y0, lengths=n)
        over, state = x.clone(), y0.clone()
        b.recurrence_forward(over, gate, y0=state, lengths=n, y=over, yT=state)
        off = torch.zeros_like(y, dtype=torch.bool) if n is None else torch.arange(T, device="cuda:0")[None, :, None] >= n[:, None, None]
        assert torch.equal(over, torch.where(off, x, y)) and torch.equal(state, yT)
        dx, dg, adjoint = dy.clone(), gate.clone(), dyT.clone()
        b.recurrence_backward(x, dg, y, dx, dL_dyT=adjoint, y0=y0, lengths=n, dL_dx=dx, dL_dgate=dg, dL_dy0=adjoint)
        assert torch.equal(dx, torch.where(off, dy, ref[0])) and torch.equal(dg, torch.where(off, gate, ref[1])) and torch.equal(adjoint, ref[2])


# alone in a warp, several warps with single and paired accesses, tiles staged in shared memory, clusters, clusters with a scanning warp
INF_SHAPES = [(3, 3, 48, "bf16"), (5, 9, 64, "bf16"), (5, 9, 33, "f32"), (4, 128, 64, "bf16"), (80, 300, 64, "bf16"), (80, 300, 64, "f32"), (1, 1100, 31, "f16"),
              (2, 2600, 40, "f32"), (2, 4500, 40, "bf16"), (1, 24001, 64, "bf16"), (300, 20, 64, "bf16"), (5000, 20, 64, "bf16"), (5000, 20, 63, "f32")]


def _ends(B, T):
    """Lengths that end in the middle of a tile, at its edge and nowhere."""
    return [(T, 0, 1, T // 2, T - 1, min(T, 8), min(T, 16), min(T, 17))[s % 8] for s in range(B)]


@pytest.mark.parametrize("B,T,D,low", INF_SHAPES)
@pytest.mark.parametrize("coupled", [True, False])
def test_recurrence_hands_on_a_state_that_is_infinite(B, T, D, low, coupled):
    # A state that becomes infinite with the last step is infinite in y and in yT, whatever runs behind it; with no step at all it is the initial state
    torch, b, _ = _torch()
    c = _recurrence_case(B, T, D, low)
    c["t_gate"].clamp_(min=-5)                                    # b x is infinite for an infinite x
    lengths = _ends(B, T)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
    clean, cleanT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], lengths=n, coupled=coupled)
    x, y0, y_ref, T_ref = c["t_x"].clone(), c["t_y0"].clone(), clean.clone(), cleanT.clone()
    for s, m in enumerate(lengths):
        for channel, value in ((1, float("inf")), (D - 1, float("-inf"))):
            if m > 0:
                x[s, m - 1, channel] = value
                y_ref[s, m - 1, channel] = value
            else:
                y0[s, channel] = value
            T_ref[s, channel] = value
    y, yT = b.recurrence_forward(x, c["t_gate"], y0=y0, lengths=n, coupled=coupled)
    assert torch.equal(y, y_ref) and torch.equal(yT, T_ref)


@pytest.mark.parametrize("B,T,D,low", INF_SHAPES)
@pytest.mark.parametrize("coupled", [True, False])
def test_recurrence_hands_back_an_adjoint_that_is_infinite(B, T, D, low, coupled):
    # It reaches the last step of the sequence, where b times it is infinite, unchanged; with no step at all it is the adjoint of the initial state
    torch, b, _ = _torch()
    c = _recurrence_case(B, T, D, low)
    c["t_gate"].clamp_(min=-5)
    lengths = _ends(B, T)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
    kw = dict(y0=c["t_y0"], lengths=n, coupled=coupled)
    y, _ = b.recurrence_forward(c["t_x"], c["t_gate"], **kw)
    clean = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], **kw)
    dyT = c["t_dyT"].clone()
    dyT[:, 1], dyT[:, D - 1] = float("inf"), float("-inf")
    dx, dg, dy0 = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=dyT, **kw)
    for s, m in enumerate(lengths):
        if m > 0:
            assert float(dx[s, m - 1, 1]) == float("inf") and float(dx[s, m - 1, D - 1]) == float("-inf"), (s, m)
        else:
            assert torch.equal(dy0[s], dyT[s])
    rest = [i for i in range(D) if i not in (1, D - 1)]
    for got, ref in zip((dx, dg, dy0), clean):
        assert torch.equal(got[..., rest], ref[..., rest])


def test_dropout_of_one_row_of_two_to_the_31_columns_less_one():
    # One row's groups are numbered like as many rows of eight columns
    torch, b, _ = _torch()
    n = (1 << 31) - 1
    words = torch.tensor([5, 6], dtype=torch.int64, device="cuda:0")
    row, eights = (torch.ones(n + 1, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    b.dropout(row[:n], 0.25, words, site=2, out=row[:n])
    b.dropout(eights.view(-1, 8), 0.25, words, site=2, out=eights.view(-1, 8))
    assert torch.equal(row[:n], eights[:n]) and float(row[n]) == 1


@pytest.mark.parametrize("M,D", [(50, 96), (700, 2048), (40, 785), (30, 4096)])
def test_residual_gradients_of_shared_weights_meet_in_one_buffer(M, D):
    # One weight in two or three places: its gradients are added to one buffer, in the order dw_post, dscale, dw_pre, the same bits every time
    torch, b, _ = _torch()
    c = _residual_case(M, D, "bf16")
    step = b.ResidualStep(D, low="bf16")
    for names in (("dw_post", "dw_pre"), ("dw_post", "dscale"), ("dw_post", "dscale", "dw_pre")):
        w = dict(gate=c["t_gate"], w_post=c["t_w_post"], scale=c["t_scale"], w_pre=c["t_w_pre"])
        y, z, stats = step.forward(c["t_y"], c["t_u"], **w)
        one = step.backward(y, c["t_u"], stats, dL_dy=c["t_dy"], dL_dz=c["t_dz"], **w)
        buffer = torch.ones(D, device="cuda:0")
        into = {k: buffer if k in names else torch.zeros(D, device="cuda:0") for k in ("dw_post", "dscale", "dw_pre")}
        got = step.backward(y, c["t_u"], stats, dL_dy=c["t_dy"], dL_dz=c["t_dz"], accumulate_into=into, **w)
        want = torch.ones(D, device="cuda:0")
        for k in ("dw_post", "dscale", "dw_pre"):
            if k in names:
                want += one[k]
            else:
                assert torch.equal(got[k], one[k])
        assert torch.equal(buffer, want)
