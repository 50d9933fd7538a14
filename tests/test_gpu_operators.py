"""Gated linear recurrence, residual step and dropout on the GPU against their float64 oracle.

Tolerances.  A value stored in a low format is off by half a step, HALF * |value| (fp16 also by half its smallest spacing, 2^-25).  In front of that
rounding stands float32 arithmetic, whose error is bounded through magnitudes: a result that is a sum of products is off by at most k 2^-24 times the sum of the
terms' absolute values, k the roundings a term passes through.  Exponentials, quotients and reciprocal roots of the device are within 2^-21 relative.
"""
import numpy as np
import pytest

from oracle import operators as orc

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # half a step: finfo.eps / 2
# Relative bounds end at the smallest normal number.  float16: results below 2^-14 are multiples of 2^-24, off by at most half of that.  float32 and bfloat16: a
# factor below 2^-126 (a gate of -100) is off by up to 2 spacings of 2^-149, times magnitudes below 2^13 that is 2^-135: covered by 2^-126.
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}


def _torch():
    import torch
    from paper_2510_23498_b200 import binding
    return torch, binding, {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _up(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda:0")
    return t if dtype is None else t.to(dtype)


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _close(got, ref, tol, what=""):
    got, err = np.asarray(got), np.abs(np.asarray(got) - ref)
    bad = ~(err <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g at %s (tolerance %g, value %g)" % (
        what, bad.sum(), bad.size, np.nanmax(np.where(bad, err, 0)), np.argwhere(bad)[0], np.broadcast_to(tol, err.shape)[tuple(np.argwhere(bad)[0])],
        ref[tuple(np.argwhere(bad)[0])])


def _stored(ref, low, err):
    """Tolerance of a stored value whose float32 error is `err`: half a step of the value itself, at most a step's half larger by that error."""
    return HALF[low] * (np.abs(ref) + err) + TINY[low] + err


# ------------------------------------------------------------------------------------------------ gated linear recurrence
def _layout(a, dtype, layout):
    """[B, T, D] on the device: contiguous, time-major, a slice of rows twice as long at an odd offset, or their first half."""
    torch, _, _ = _torch()
    t = _up(a, dtype)
    if layout == "time":
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "half":
        buf = torch.full((t.shape[0], t.shape[1], 2 * t.shape[2]), float("nan"), dtype=t.dtype, device=t.device)
        buf[..., :t.shape[2]] = t
        return buf[..., :t.shape[2]]
    if layout == "slice":
        buf = torch.full((t.shape[0], t.shape[1], 2 * t.shape[2] + 1), float("nan"), dtype=t.dtype, device=t.device)
        buf[..., 1:1 + t.shape[2]] = t
        return buf[..., 1:1 + t.shape[2]]
    return t


def _recurrence_case(B, T, D, low, seed=0, ragged=False, layout="plain", gate=None):
    torch, _, dt = _torch()
    rng = np.random.default_rng(seed)
    c = dict(low=low, x=_np(_up(rng.normal(size=(B, T, D)), dt[low])), y0=rng.normal(size=(B, D)).astype(np.float32).astype(np.float64))
    g = rng.normal(size=(B, T, D)) + np.linspace(1, -7, D) if gate is None else gate
    c["gate"] = _np(_up(g, dt[low]))
    c["dy"], c["dyT"] = _np(_up(rng.normal(size=(B, T, D)), dt[low])), rng.normal(size=(B, D)).astype(np.float32).astype(np.float64)
    c["lengths"] = np.full(B, T)
    if ragged:
        c["lengths"] = rng.integers(0, T + 1, size=B)
        c["lengths"][0] = T
        c["lengths"][-1] = 0
    c["t_x"], c["t_gate"], c["t_dy"] = (_layout(c[k], dt[low], layout) for k in ("x", "gate", "dy"))
    c["t_y0"], c["t_dyT"] = _up(c["y0"]), _up(c["dyT"])
    c["t_len"] = torch.tensor(c["lengths"], dtype=torch.int32, device="cuda:0") if ragged else None
    return c


# float32 error of the recurrences.  A step makes at most 6 roundings of values no larger than its magnitude, and its gate (exponential and quotient) is off by
# 2^-21 relative; the gates' errors add up with weights that sum to one (coupled: b_j times the product of the later a), or multiply the states' magnitudes once
# for each step that is remembered.  Every step may have been composed twice (once from zero, once from the state).  So 2 (6 T 2^-24 + 8 * 2^-24 T), with the
# largest magnitude of the channel: 28 T 2^-24.
def _recurrence_error(T, mag):
    return (28 * T + 32) * 2.0 ** -24 * mag.max(axis=1, keepdims=True)


def _check_forward(c, coupled, y=None, yT=None):
    ref, refT, mag, magT = orc.recurrence_forward(c["x"], c["gate"], c["y0"], c["lengths"], coupled)
    T = c["x"].shape[1]
    err = _recurrence_error(T, np.concatenate([mag, np.abs(c["y0"])[:, None]], 1))
    _close(_np(y), ref, _stored(ref, c["low"], err), "y")
    _close(_np(yT), refT, err[:, 0], "yT")


def _check_backward(c, coupled, y, got):
    dx, dg, dy0, lmag, rmag = orc.recurrence_backward(c["x"], c["gate"], y, c["dy"], c["dyT"], c["y0"], c["lengths"], coupled)
    T = c["x"].shape[1]
    err = _recurrence_error(T, np.concatenate([lmag, np.abs(c["dyT"])[:, None]], 1))
    b, a = orc.sigmoid(c["gate"])
    before = np.concatenate([c["y0"][:, None], y[:, :-1]], 1)
    on = (np.arange(T)[None] < c["lengths"][:, None])[..., None]
    slope = a * b * (np.abs(c["x"]) + np.abs(before) if coupled else np.abs(before)) * on
    # a gradient is the adjoint times factors with errors of 2^-20 in all
    ex = (b if coupled else 1.0) * (err + 2.0 ** -20 * lmag) * on
    eg = slope * (err + 2.0 ** -20 * lmag)
    _close(_np(got[0]), dx, _stored(dx, c["low"], ex), "dx")
    _close(_np(got[1]), dg, _stored(dg, c["low"], eg), "dgate")
    _close(_np(got[2]), dy0, err[:, 0], "dy0")


CASES = [
    # one token, one step at a time
    (1, 1, 1, "bf16", {}), (3, 1, 64, "f32", {}), (100, 1, 130, "f16", {}), (2, 2, 33, "bf16", {}), (3, 1, 64, "bf16", dict(layout="time")),
    # around the tiles of warps and blocks, one and two channels a lane
    (2, 8, 64, "bf16", {}), (2, 9, 66, "f16", {}), (2, 16, 32, "f32", {}), (2, 17, 65, "bf16", {}), (1, 129, 64, "bf16", {}), (5, 127, 130, "f16", dict(ragged=True)),
    # split over clusters, several rounds
    (1, 1100, 40, "bf16", {}), (1, 2049, 34, "f32", {}), (2, 1500, 31, "f16", dict(ragged=True)), (3, 700, 100, "bf16", dict(ragged=True, layout="time")),
    # tiles brought to shared memory ahead: blocks by themselves (enough channels in all), and clusters over several rounds
    (80, 300, 64, "bf16", dict(ragged=True)), (75, 290, 72, "f32", dict(layout="time")), (20, 700, 200, "f16", dict(ragged=True, layout="half")),
    (1, 5000, 64, "bf16", {}), (2, 4500, 40, "f16", dict(ragged=True)), (1, 2600, 72, "f32", dict(layout="half")), (3, 3000, 328, "bf16", dict(ragged=True, layout="time")),
    # clusters of more warps, for many rounds
    (1, 24001, 64, "bf16", {}), (2, 12000, 72, "f32", dict(ragged=True)), (3, 23000, 40, "f16", dict(ragged=True, layout="time")),
    # many short sequences
    (300, 5, 66, "bf16", dict(ragged=True)), (40, 33, 96, "f32", dict(ragged=True, layout="time")),
    # slices of wider rows at odd addresses
    (2, 150, 64, "bf16", dict(layout="slice")), (4, 40, 33, "f32", dict(ragged=True, layout="slice")),
]


@pytest.mark.parametrize("coupled", [True, False])
@pytest.mark.parametrize("B,T,D,low,kw", CASES)
def test_recurrence_against_the_oracle(B, T, D, low, kw, coupled):
    torch, b, dt = _torch()
    c = _recurrence_case(B, T, D, low, **kw)
    y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], lengths=c["t_len"], coupled=coupled)
    _check_forward(c, coupled, y, yT)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    dy = torch.empty_like(y).copy_(c["t_dy"])
    got = b.recurrence_backward(c["t_x"], c["t_gate"], y, dy, dL_dyT=c["t_dyT"], y0=c["t_y0"], lengths=c["t_len"], coupled=coupled, flag=flag)
    _check_backward(c, coupled, _np(y), got)
    assert int(flag) == 0
    # without what is optional: zero states and cotangents
    z = np.zeros_like(c["y0"])
    y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], lengths=c["t_len"], coupled=coupled)
    _check_forward({**c, "y0": z}, coupled, y, yT)
    got = b.recurrence_backward(c["t_x"], c["t_gate"], y, None, dL_dyT=c["t_dyT"], lengths=c["t_len"], coupled=coupled)
    _check_backward({**c, "y0": z, "dy": np.zeros_like(c["dy"])}, coupled, _np(y), got)


@pytest.mark.parametrize("T", [1, 40, 1300, 5000])
@pytest.mark.parametrize("coupled", [True, False])
def test_recurrence_with_extreme_gates(T, coupled):
    # Gates of infinity reset the state, of minus infinity keep it; 1e-6 a step is a memory of a million steps.  float32, both directions.
    rng = np.random.default_rng(8)
    g = rng.choice([0.0, np.inf, -np.inf, 30.0, -30.0, 100.0, -100.0, -13.8], size=(2, T, 48))
    g[:, :, :16] = -13.8
    c = _recurrence_case(2, T, 48, "f32", gate=g)
    c["y0"][1] *= 1000
    torch, b, _ = _torch()
    c["t_y0"] = _up(c["y0"])
    y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], coupled=coupled)
    _check_forward(c, coupled, y, yT)
    _check_backward(c, coupled, _np(y), b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"], coupled=coupled))


@pytest.mark.parametrize("low", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 50, 5000])
def test_recurrence_passes_on_what_is_not_a_number(low, T):
    # A NaN in one channel's gate or input reaches that channel's later states and earlier gradients, and no other channel
    torch, b, _ = _torch()
    c = _recurrence_case(2, T, 64, low)
    at = T // 2
    for name, channel in (("t_gate", 5), ("t_x", 40)):
        c[name][1, at, channel] = float("nan")
    y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"])
    want = torch.zeros_like(y, dtype=torch.bool)
    want[1, at:, 5] = want[1, at:, 40] = True
    assert torch.equal(y.isnan(), want) and torch.equal(yT.isnan(), want[:, -1])
    flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    dx, dg, dy0 = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], flag=flag)
    assert dx[1, :at + 1, 5].isnan().all() and dy0[1, 5].isnan() and not dx[0].isnan().any() and not dy0[0].isnan().any()
    assert not dx[1, at + 1:, 5].isnan().any() and not dx[1, :, 40].isnan().any() and dg[1, at, 40].isnan() and int(flag) == 1


def test_recurrence_takes_outputs_of_other_strides_and_alignment_than_its_inputs():
    # Inputs that bulk copies can read, outputs that they could not write: odd addresses, the other order of time and sequences
    torch, b, _ = _torch()
    for B, T, D, low in ((80, 300, 64, "bf16"), (1, 5000, 64, "f16"), (2, 2600, 64, "f32")):
        c = _recurrence_case(B, T, D, low)
        y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"])
        ref = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"])

        def odd(shape):
            return torch.empty(shape[0] * shape[1] * shape[2] + 1, dtype=y.dtype, device=y.device)[1:].view(shape)

        out, dx, dg = odd(y.shape), odd(y.shape), odd(y.shape)
        b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], y=out)
        b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"], dL_dx=dx, dL_dgate=dg)
        assert _same(out, y) and _same(dx, ref[0]) and _same(dg, ref[1])
        if B > 1:
            tm = torch.empty((T, B, D), dtype=y.dtype, device=y.device).transpose(0, 1)
            b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], y=tm)
            dy = torch.empty_like(tm).copy_(c["t_dy"])
            got = b.recurrence_backward(c["t_x"], c["t_gate"], tm, dy, dL_dyT=c["t_dyT"], y0=c["t_y0"])
            assert _same(tm, y) and _same(got[0], ref[0]) and _same(got[1], ref[1])


def _same(got, ref):
    """Equal up to what the order of a composition may change: 2^-6 of a 16-bit value, 2^-15 of a float32 one, where the largest are about 10."""
    tol = 2.0 ** -15 if got.dtype == ref.dtype and got.element_size() == 4 else 2.0 ** -6
    return bool(((got.float() - ref.float()).abs() <= tol * (ref.float().abs() + 1)).all())


def test_recurrence_slow_channels_keep_their_rate_over_long_sequences():
    # Constant gate and input: y_T = 1 - (1 - b)^T exactly.  b = 2e-5 over 60 000 steps: rounding a = 1 - b to 24 bits would change the rate by 1e-3.
    # Error: b to 2^-21 relative (times T b e^{-T b} < 0.37) and the states' roundings, at most 2^-24 each and forgotten after 1 / b = 5e4 steps: 5e4 * 2^-24 = 3e-3
    # if all had one sign; y rises steadily, so that its last bit does not round one way for more than a binade's part of the path.  Taken: a fifth of that bound.
    torch, b, _ = _torch()
    T, g = 60000, -10.8
    x, gate = torch.ones(1, T, 32, device="cuda:0"), torch.full((1, T, 32), g, device="cuda:0")
    _, yT = b.recurrence_forward(x, gate)
    beta = float(orc.sigmoid(np.float64(np.float32(g)))[0])
    assert np.abs(_np(yT) - (1 - (1 - beta) ** T)).max() < 6e-4


def test_recurrence_reads_and_writes_nothing_behind_the_lengths():
    torch, b, dt = _torch()
    c = _recurrence_case(6, 300, 34, "bf16", ragged=True)
    clean = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], lengths=c["t_len"])
    grads = b.recurrence_backward(c["t_x"], c["t_gate"], clean[0], c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"], lengths=c["t_len"])
    off = torch.arange(300, device="cuda:0")[None, :, None] >= c["t_len"][:, None, None]
    dirty = [torch.where(off, torch.full_like(t, float("nan")), t) for t in (c["t_x"], c["t_gate"], clean[0], c["t_dy"])]
    y = torch.full_like(clean[0], 7.0)
    b.recurrence_forward(dirty[0], dirty[1], y0=c["t_y0"], lengths=c["t_len"], y=y)
    assert torch.equal(y, torch.where(off, torch.full_like(y, 7.0), clean[0]))
    dx, dg = torch.full_like(y, 5.0), torch.full_like(y, 6.0)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    out = b.recurrence_backward(*dirty, dL_dyT=c["t_dyT"], y0=c["t_y0"], lengths=c["t_len"], dL_dx=dx, dL_dgate=dg, flag=flag)
    assert torch.equal(dx, torch.where(off, torch.full_like(y, 5.0), grads[0])) and torch.equal(dg, torch.where(off, torch.full_like(y, 6.0), grads[1]))
    assert torch.equal(out[2], grads[2]) and int(flag) == 0
    # lengths beyond the sequence and below zero are clamped
    wild = torch.tensor([10 ** 6, -5, 300, 0, 299, 1], dtype=torch.int32, device="cuda:0")
    tame = torch.tensor([300, 0, 300, 0, 299, 1], dtype=torch.int32, device="cuda:0")
    for p, q in zip(b.recurrence_forward(c["t_x"], c["t_gate"], lengths=wild), b.recurrence_forward(c["t_x"], c["t_gate"], lengths=tame)):
        assert torch.equal(p, q)


def test_recurrence_step_by_step_is_the_whole_sequence():
    # Serving: one token at a time with the state updated in place gives the sequence's trajectory, within the composition's float32 error
    torch, b, _ = _torch()
    c = _recurrence_case(7, 50, 96, "f32")
    state = c["t_y0"].clone()
    for t in range(50):
        y, out = b.recurrence_forward(c["t_x"][:, t:t + 1], c["t_gate"][:, t:t + 1], y0=state, yT=state)
        assert out is state and torch.equal(y[:, 0], state)
    _check_forward({**c, "x": c["x"], "lengths": np.full(7, 50)}, True, b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"])[0], state)


def test_recurrence_in_place_and_over_its_inputs():
    torch, b, _ = _torch()
    for T in (1, 5, 700):
        c = _recurrence_case(3, T, 64, "bf16")
        y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"])
        x = c["t_x"].clone()
        b.recurrence_forward(x, c["t_gate"], y0=c["t_y0"], y=x)
        assert torch.equal(x, y)
        ref = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"])
        dy, g, dyT = c["t_dy"].clone(), c["t_gate"].clone(), c["t_dyT"].clone()
        b.recurrence_backward(c["t_x"], g, y, dy, dL_dyT=dyT, y0=c["t_y0"], dL_dx=dy, dL_dgate=g, dL_dy0=dyT)
        assert torch.equal(dy, ref[0]) and torch.equal(g, ref[1]) and torch.equal(dyT, ref[2])


@pytest.mark.parametrize("T,D,n", [(9000, 64, 1), (9000, 64, 33), (9000, 30, 500), (20000, 65, 7), (20000, 65, 0)])
def test_recurrence_state_in_place_where_blocks_share_a_sequence(T, D, n):
    # Few steps of a long sequence: the first block writes the state while the others have no steps to read for
    torch, b, _ = _torch()
    c = _recurrence_case(2, T, D, "bf16")
    lengths = torch.tensor([n, T], dtype=torch.int32, device="cuda:0")
    y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"], lengths=lengths)
    ref = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"], lengths=lengths)
    state, adjoint = c["t_y0"].clone(), c["t_dyT"].clone()
    assert torch.equal(b.recurrence_forward(c["t_x"], c["t_gate"], y0=state, yT=state, lengths=lengths)[0], y)
    assert torch.equal(state, yT)
    got = b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=adjoint, y0=c["t_y0"], lengths=lengths, dL_dy0=adjoint)
    assert all(torch.equal(p, q) for p, q in zip(got, ref))


def test_recurrence_flags_gradients_that_overflow():
    torch, b, _ = _torch()
    c = _recurrence_case(2, 200, 34, "f16")
    y, _ = b.recurrence_forward(c["t_x"], c["t_gate"])
    flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    dyT = torch.zeros_like(c["t_dyT"])
    dyT[1, 33] = 1e9
    b.recurrence_backward(c["t_x"], c["t_gate"], y, None, dL_dyT=dyT, coupled=False, flag=flag)
    assert int(flag) == 1


def test_recurrence_beyond_two_to_the_31_elements():
    # 2^25 + 77 steps of 64 channels.  A reset near the end makes what follows independent of the rest: the last steps against the oracle.
    torch, b, _ = _torch()
    T, D, n = (1 << 25) + 77, 64, 90
    rng = np.random.default_rng(2)
    x, g = torch.zeros(1, T, D, dtype=torch.bfloat16, device="cuda:0"), torch.zeros(1, T, D, dtype=torch.bfloat16, device="cuda:0")
    tail = rng.normal(size=(2, 1, n, D))
    tail[1, 0, 0] = np.inf
    x[0, T - n:], g[0, T - n:] = (_up(t[0], torch.bfloat16) for t in tail)
    c = dict(low="bf16", x=_np(x[:, T - n:]), gate=_np(g[:, T - n:]), y0=np.zeros((1, D)), lengths=[n])
    y, yT = b.recurrence_forward(x, g, y=x)
    _check_forward(c, True, y[:, T - n:], yT)
    assert float(y[0, :T - n].abs().max()) == 0


# ------------------------------------------------------------------------------------------------ residual step
def _residual_case(M, D, low, gated=True, weights=True, p=0.0, seed=0, layout="plain"):
    torch, b, dt = _torch()
    rng = np.random.default_rng(seed)
    c = dict(low=low, p=p, gated=gated)
    c["y"] = (2 * rng.normal(size=(M, D))).astype(np.float32).astype(np.float64)
    c["dy"] = rng.normal(size=(M, D)).astype(np.float32).astype(np.float64)
    for k in ("u", "gate", "dz"):
        c[k] = _np(_up(rng.normal(size=(M, D)) + 0.25, dt[low]))
    for k in ("w_post", "scale", "w_pre"):
        c[k] = (rng.normal(size=D) * 0.1 + 1).astype(np.float32).astype(np.float64) if weights else np.ones(D)
        c["t_" + k] = _up(c[k]) if weights else None
    if M > 1:
        c["u"][M // 2] = 0                     # a row of nothing
    for k in ("y", "dy", "u", "gate", "dz"):
        c["t_" + k] = _layout(c[k][None], torch.float32 if k in ("y", "dy") else dt[low], layout)[0]
    if not gated:
        c["gate"] = c["t_gate"] = None
    c["t_rng"] = torch.tensor([(5 << 40) + 77, (1 << 33) + 12], dtype=torch.int64, device="cuda:0") if p > 0 else None
    c["factors"] = orc.drop_factors(M, D, p, (5 << 40) + 77, 12, 21) if p > 0 else np.ones((M, D))
    return c


# float32 error of the step.  A mean over D elements is summed 8 at a time in a thread, then in a tree of at most 11 levels: 20 roundings, 2^-19 relative to the mean of
# absolute values; reciprocal root, gate and the products behind it: 2^-20.  Together 2^-18 of each term's magnitude, where a normalised value's magnitude is
# (|v| + |mean|) rstd.
E = 2.0 ** -18


def _check_residual(c, kinds, h, got, grads=None, scale_exp=0, eps=1e-5):
    post, pre = kinds
    low = c["low"]
    args = (c["w_post"], c["scale"], c["w_pre"], h, post, pre, eps, c["factors"])
    y1, z, stats = orc.residual_forward(c["y"], c["u"], c["gate"], *args)
    n, mu, ru = orc.norm(c["u"], post, eps)
    nmag = (np.abs(c["u"]) + np.abs(mu)[:, None]) * ru[:, None]
    sig, cosig = orc.sigmoid(c["gate"]) if c["gate"] is not None else (1.0, 0.0)
    ey = E * (np.abs(c["y"]) + np.abs(h * c["scale"] * c["w_post"] * c["factors"]) * nmag * sig)
    y_new, z_got, st = _np(got[0]), _np(got[1]), _np(got[2])
    _close(y_new, y1, ey, "y'")
    _, my, ry = orc.norm(y_new, pre, eps)
    n2 = (y_new - my[:, None]) * ry[:, None]
    n2mag = (np.abs(y_new) + np.abs(my)[:, None]) * ry[:, None]
    ez = E * np.abs(c["w_pre"]) * n2mag
    _close(z_got, n2 * c["w_pre"], _stored(n2 * c["w_pre"], low, ez), "z")
    ref = np.stack([mu, ru, my, ry], 1)
    _close(st, ref, E * (np.abs(ref) + np.stack([np.abs(c["u"]).mean(1), 0 * mu, np.abs(y_new).mean(1), 0 * mu], 1)), "stats")
    if grads is None:
        return
    g = orc.residual_backward(y_new, c["u"], c["gate"], *args, c["dy"], c["dz"])
    dzw = np.abs(c["dz"] * c["w_pre"])
    amag = np.abs(c["dy"]) + ry[:, None] * (dzw + n2mag * (dzw * n2mag).mean(1, keepdims=True) + dzw.mean(1, keepdims=True))
    _close(_np(grads["dy"]), g["dy"], 2 * E * amag, "dy")
    t = h * amag * c["factors"]
    tv = np.abs(t * c["w_post"]) * nmag * sig
    # sums over rows: one product after another in a thread, then the blocks' sums: at most M roundings
    col = (4 * E + len(c["y"]) * 2.0 ** -24)
    _close(_np(grads["dw_pre"]) if grads["dw_pre"] is not None else g["dw_pre"], g["dw_pre"], col * (np.abs(c["dz"]) * n2mag).sum(0), "dw_pre")
    _close(_np(grads["dscale"]) if grads["dscale"] is not None else g["dscale"], g["dscale"], col * tv.sum(0), "dscale")
    ts = np.abs(t * c["scale"])
    _close(_np(grads["dw_post"]) if grads["dw_post"] is not None else g["dw_post"], g["dw_post"], col * (ts * sig * nmag).sum(0), "dw_post")
    S = 2.0 ** scale_exp
    if c["gate"] is not None:
        eg = S * 4 * E * np.abs(c["scale"]) * tv * cosig
        _close(_np(grads["dgate"]), S * g["dgate"], _stored(S * g["dgate"], low, eg), "dgate")
    tw = ts * sig * np.abs(c["w_post"])
    eu = S * 4 * E * ru[:, None] * (tw + nmag * (tw * nmag).mean(1, keepdims=True) + tw.mean(1, keepdims=True))
    _close(_np(grads["du"]), S * g["du"], _stored(S * g["du"], low, eu), "du")


RES = [
    (1, 1, "f32", ("rms", "rms"), {}), (5, 8, "bf16", ("rms", "rms"), dict(p=0.3)), (9, 13, "f16", ("meanvar", "meanvar"), dict(p=0.3)),
    (37, 256, "bf16", ("rms", "rms"), dict(p=0.1)), (20, 257, "f32", ("meanvar", "rms"), {}), (70, 300, "bf16", ("rms", "none"), dict(gated=False)),
    (33, 512, "f16", ("none", "rms"), dict(p=0.5)), (600, 64, "bf16", ("rms", "rms"), dict(weights=False)), (11, 785, "f32", ("meanvar", "meanvar"), dict(p=0.1)),
    (500, 1024, "bf16", ("rms", "rms"), {}), (7, 2048, "f16", ("rms", "meanvar"), dict(gated=False, p=0.25)), (5, 4096, "bf16", ("meanvar", "meanvar"), {}),
    (4, 4097, "f32", ("rms", "rms"), {}), (6, 8192, "bf16", ("rms", "rms"), dict(p=0.1)), (3, 16384, "f16", ("meanvar", "rms"), {}),
    (3, 12300, "bf16", ("rms", "meanvar"), dict(weights=False)), (40, 4104, "bf16", ("meanvar", "rms"), dict(p=0.2)), (9, 6000, "f32", ("rms", "rms"), {}),
    # more rows than run at once: every block goes through several
    (2000, 1024, "bf16", ("rms", "rms"), dict(p=0.1)), (1500, 2048, "f16", ("meanvar", "rms"), {}), (9000, 64, "bf16", ("rms", "meanvar"), {}),
    (700, 4096, "bf16", ("rms", "rms"), dict(p=0.1)), (1200, 785, "f32", ("rms", "rms"), {}), (5000, 40, "f32", ("meanvar", "meanvar"), dict(gated=False)),
    (12, 64, "bf16", ("rms", "rms"), dict(layout="slice")), (12, 1001, "f16", ("rms", "rms"), dict(layout="slice", p=0.2)),
]


@pytest.mark.parametrize("M,D,low,kinds,kw", RES)
def test_residual_step_against_the_oracle(M, D, low, kinds, kw):
    torch, b, _ = _torch()
    c = _residual_case(M, D, low, **kw)
    step = b.ResidualStep(D, low=low, post_norm=kinds[0], pre_norm=kinds[1], h=0.3, p=c["p"], site=21)
    w = dict(gate=c["t_gate"], w_post=c["t_w_post"], scale=c["t_scale"], w_pre=c["t_w_pre"], rng=c["t_rng"])
    got = step.forward(c["t_y"], c["t_u"], **w)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    dy = torch.empty_strided(c["t_y"].shape, c["t_y"].stride(), device="cuda:0").copy_(c["t_dy"])
    grads = step.backward(got[0], c["t_u"], got[2], dL_dy=dy, dL_dz=c["t_dz"], flag=flag, **w)
    _check_residual(c, kinds, float(np.float32(0.3)), got, grads, eps=float(np.float32(1e-5)))
    assert int(flag) == 0


def test_residual_step_scaled_adjoints_and_accumulation():
    # With S = 2^6 the low cotangents come in and go out scaled, everything in float32 is as without; weight gradients are added to
    torch, b, _ = _torch()
    c = _residual_case(50, 96, "bf16")
    step = b.ResidualStep(96, low="bf16")
    w = dict(gate=c["t_gate"], w_post=c["t_w_post"], scale=c["t_scale"], w_pre=c["t_w_pre"])
    y, z, stats = step.forward(c["t_y"], c["t_u"], **w)
    one = step.backward(y, c["t_u"], stats, dL_dy=c["t_dy"], dL_dz=c["t_dz"], **w)
    acc = {k: one[k].clone() for k in ("dw_post", "dscale", "dw_pre")}
    two = step.backward(y, c["t_u"], stats, dL_dy=c["t_dy"], dL_dz=c["t_dz"] * 64, scale_exp=6, accumulate_into=acc, **w)
    assert torch.equal(two["dy"], one["dy"]) and torch.equal(two["du"], one["du"] * 64) and torch.equal(two["dgate"], one["dgate"] * 64)
    assert two["dscale"] is acc["dscale"] and all(torch.equal(acc[k], 2 * one[k]) for k in acc)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    f16 = b.ResidualStep(96, low="f16")
    f16.backward(y, c["t_u"].half(), stats, dL_dy=c["t_dy"] * 1e6, flag=flag, **{**w, "gate": c["t_gate"].half()})
    assert int(flag) == 1


def test_residual_step_without_block_or_without_next_input():
    torch, b, _ = _torch()
    c = _residual_case(10, 200, "bf16")
    step = b.ResidualStep(200, low="bf16", h=0.5)
    y, z, stats = step.forward(c["t_y"], w_pre=c["t_w_pre"])                        # the norm in front of the first block
    assert y is c["t_y"]
    n, _, _ = orc.norm(c["y"], "rms", 1e-5)
    ref = n * c["w_pre"]
    _close(_np(z), ref, _stored(ref, "bf16", E * np.abs(ref)), "z")
    g = step.backward(y, None, stats, dL_dy=c["t_dy"], dL_dz=c["t_dz"], w_pre=c["t_w_pre"])
    ref = orc.residual_backward(c["y"], None, None, None, None, c["w_pre"], 0.5, "rms", "rms", 1e-5, None, c["dy"], c["dz"])
    _close(_np(g["dy"]), ref["dy"], 1e-5 * (1 + np.abs(ref["dy"])), "dy")
    assert g["du"] is None and g["dgate"] is None
    y2, none, stats = step.forward(c["t_y"], c["t_u"], want_z=False)                # behind the last block
    assert none is None
    g = step.backward(y2, c["t_u"], stats, dL_dy=c["t_dy"], want_weights=False)
    assert torch.equal(g["dy"], c["t_dy"]) and g["dw_post"] is None
    full = step.forward(c["t_y"].clone(), c["t_u"], y_out=None)
    inplace = c["t_y"].clone()
    out = step.forward(inplace, c["t_u"], y_out=inplace)
    assert out[0] is inplace and torch.equal(inplace, full[0]) and torch.equal(out[1], full[1])


@pytest.mark.parametrize("D", [64, 785, 2048, 4096])
def test_residual_step_over_its_own_inputs(D):
    # y' over y; dL_dy over dL_dy', dL_du over u and dL_dgate over gate, through the C entry points
    import ctypes as C
    torch, b, _ = _torch()
    M = 1000
    c = _residual_case(M, D, "bf16")
    w = dict(gate=c["t_gate"], w_post=c["t_w_post"], scale=c["t_scale"], w_pre=c["t_w_pre"])
    step = b.ResidualStep(D, low="bf16", h=0.5)
    y, z, stats = step.forward(c["t_y"], c["t_u"], **w)
    ref = step.backward(y, c["t_u"], stats, dL_dy=c["t_dy"], dL_dz=c["t_dz"], **w)
    inplace = c["t_y"].clone()
    got = step.forward(inplace, c["t_u"], y_out=inplace, **w)
    assert torch.equal(inplace, y) and torch.equal(got[1], z) and torch.equal(got[2], stats)
    lib = b.load_library()
    desc = step._desc(D, D, D, D)
    a, u, g = c["t_dy"].clone(), c["t_u"].clone(), c["t_gate"].clone()
    grads = [torch.empty(D, device="cuda:0") for _ in range(3)]
    n = lib.mpode_residual_workspace_bytes(desc, M)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda:0")
    at = [t.data_ptr() for t in (y, u, g, w["w_post"], w["scale"], w["w_pre"])] + [None] + [t.data_ptr() for t in (stats, a, c["t_dz"])]
    st = lib.mpode_residual_backward(desc, torch.cuda.current_stream().cuda_stream, M, *at, 0, a.data_ptr(), u.data_ptr(), g.data_ptr(),
                                     *[t.data_ptr() for t in grads], 0, None, ws.data_ptr(), n)
    assert st == b.OK
    assert torch.equal(a, ref["dy"]) and torch.equal(u, ref["du"]) and torch.equal(g, ref["dgate"])
    assert all(torch.equal(x, ref[k]) for x, k in zip(grads, ("dw_post", "dscale", "dw_pre")))


def test_residual_step_passes_on_what_is_not_a_number():
    torch, b, _ = _torch()
    for D in (64, 200, 2048, 4096):
        c = _residual_case(40, D, "bf16")
        step = b.ResidualStep(D, low="bf16")
        c["t_u"][7, 3] = float("nan")
        c["t_u"][9, 5] = float("inf")
        y, z, stats = step.forward(c["t_y"], c["t_u"], gate=c["t_gate"])
        clean = torch.ones(40, dtype=torch.bool, device="cuda:0")
        clean[7] = clean[9] = False
        assert y[7].isnan().all() and z[7].isnan().all() and z[9].isnan().any() and not y[clean].isnan().any() and not z[clean].isnan().any()
        flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
        g = step.backward(y, c["t_u"], stats, dL_dy=c["t_dy"], dL_dz=c["t_dz"], gate=c["t_gate"], flag=flag)
        assert g["du"][7].isnan().all() and not g["du"][clean].isnan().any() and int(flag) == 1


# ------------------------------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("M,D,low,p", [(1, 1, "f32", 0.5), (3, 8, "bf16", 0.1), (7, 13, "f16", 0.25), (40, 256, "bf16", 0.999), (5, 785, "f32", 0.1), (4, 64, "f16", 0.0),
                                       (4, 64, "f16", 1.0)])
@pytest.mark.parametrize("layout", ["plain", "slice"])
def test_dropout_against_the_oracle(M, D, low, p, layout):
    torch, b, dt = _torch()
    rng = np.random.default_rng(1)
    x = _np(_up(rng.normal(size=(M, D)), dt[low]))
    t = _layout(x[None], dt[low], layout)[0]
    words = torch.tensor([-3, (7 << 32) + 5], dtype=torch.int64, device="cuda:0")
    out = b.dropout(t, p, words, site=2 ** 32 - 1)
    f = orc.drop_factors(M, D, p, (1 << 64) - 3, 5, 2 ** 32 - 1) if p < 1 else np.zeros((M, D))
    ref = x * f
    assert ((_np(out) == 0) == (ref == 0)).all()
    _close(_np(out), ref, _stored(ref, low, 2.0 ** -23 * np.abs(ref)), "dropout")           # (the factor and the product are rounded to float32)
    same = t.clone() if layout == "plain" else t
    b.dropout(same, p, words, site=2 ** 32 - 1, out=same)
    assert torch.equal(same, out)


def test_dropout_zeroes_what_is_not_finite_and_flags_what_it_keeps():
    torch, b, _ = _torch()
    words = torch.tensor([1, 2], dtype=torch.int64, device="cuda:0")
    x = torch.full((64, 64), float("nan"), dtype=torch.float16, device="cuda:0")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    out = b.dropout(x, 0.5, words, flag=flag)
    f = orc.drop_factors(64, 64, 0.5, 1, 2, 0)
    assert (np.isnan(_np(out)) == (f > 0)).all() and int(flag) == 1


def test_dropout_counts_groups_beyond_32_bits():
    torch, b, _ = _torch()
    rows = (1 << 32) + 5
    x = torch.ones(rows, 1, dtype=torch.bfloat16, device="cuda:0")
    words = torch.tensor([11, 13], dtype=torch.int64, device="cuda:0")
    b.dropout(x, 0.5, words, site=4, out=x)
    assert (_np(x[-5:]) == orc.drop_factors(5, 1, 0.5, 11, 13, 4, first_row=rows - 5)).all()
    assert (_np(x[:300]) == orc.drop_factors(300, 1, 0.5, 11, 13, 4)).all()


# ------------------------------------------------------------------------------------------------ together
def _network(b, torch, par, y, words, low, lengths, grads_at=None):
    """Two residual blocks (projection, recurrence over the sequence, dropout, projection) around the float32 state [B, T, D], forward and backward."""
    B, T, D = y.shape
    step = b.ResidualStep(D, low=low, h=0.5, p=0.2, site=1)
    flat = y.reshape(B * T, D)
    tape = []
    state, z, stats = step.forward(flat, w_pre=par["w_pre0"])
    tape.append((state, stats))
    for k in range(2):
        both = (z @ par["win%d" % k]).view(B, T, 2 * D)
        x, gate = both[..., :D], both[..., D:]
        r, _ = b.recurrence_forward(x, gate, lengths=lengths)
        rd = b.dropout(r, 0.1, words, site=10 + k)
        u = rd.view(B * T, D) @ par["wout%d" % k]
        new, z2, stats = step.forward(state, u, gate=z, w_post=par["w_post%d" % k], scale=par["scale%d" % k], w_pre=par["w_pre%d" % (k + 1)], rng=words)
        tape.append((z, x, gate, r, rd, u, new, stats))
        state, z = new, z2
    if grads_at is None:
        return state, z
    a, dz = grads_at
    g = {}
    for k in (1, 0):
        zin, x, gate, r, rd, u, new, stats = tape[k + 1]
        s = step.backward(new, u, stats, dL_dy=a, dL_dz=dz, gate=zin, w_post=par["w_post%d" % k], scale=par["scale%d" % k], w_pre=par["w_pre%d" % (k + 1)], rng=words)
        a = s["dy"]
        g["w_post%d" % k], g["scale%d" % k], g["w_pre%d" % (k + 1)] = s["dw_post"], s["dscale"], s["dw_pre"]
        g["wout%d" % k] = rd.view(B * T, D).float().t() @ s["du"].float()
        dr = b.dropout((s["du"] @ par["wout%d" % k].t()).view(B, T, D), 0.1, words, site=10 + k)
        dboth = torch.zeros(B, T, 2 * D, dtype=x.dtype, device=x.device)
        b.recurrence_backward(x, gate, r, dr, lengths=lengths, dL_dx=dboth[..., :D], dL_dgate=dboth[..., D:])
        dboth = dboth.view(B * T, 2 * D)
        g["win%d" % k] = zin.float().t() @ dboth.float()
        dz = dboth @ par["win%d" % k].t() + s["dgate"]
    state0, stats0 = tape[0]
    s = step.backward(state0, None, stats0, dL_dy=a, dL_dz=dz, w_pre=par["w_pre0"])
    g["w_pre0"], g["y"] = s["dw_pre"], s["dy"]
    return state, z, g


def _network_exact(torch, par, y, f_step, f_drop, lengths):
    """The same network in float64 with torch's differentiation, written step by step."""
    B, T, D = y.shape

    def norm(v):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-5)

    state, z = y, norm(y) * par["w_pre0"]
    for k in range(2):
        both = z @ par["win%d" % k]
        x, b = both[..., :D], torch.sigmoid(both[..., D:])
        rows, cur = [], torch.zeros(B, D, dtype=torch.float64)
        for t in range(T):
            on = (lengths > t)[:, None]
            cur = torch.where(on, cur + b[:, t] * (x[:, t] - cur), cur)
            rows.append(torch.where(on, cur, torch.zeros_like(cur)))
        u = (torch.stack(rows, 1) * f_drop[k]) @ par["wout%d" % k]
        state = state + 0.5 * par["scale%d" % k] * f_step * torch.sigmoid(z) * norm(u) * par["w_post%d" % k]
        z = norm(state) * par["w_pre%d" % (k + 1)]
    return state, z


def test_the_operators_together_train_a_residual_sequence_network():
    # float32 network against float64 differentiation.  Its products are float32 too (TF32 off by default): errors of 2^-22 of sums of 48 terms, through two blocks
    # whose norms divide by values near one; 2e-5 of each gradient's largest entry leaves a factor of ten over 2 * 48 * 2^-24 * 8 operations.
    torch, b, _ = _torch()
    rng = np.random.default_rng(12)
    B, T, D = 3, 21, 48
    par = {}
    for k in range(2):
        par["win%d" % k], par["wout%d" % k] = rng.normal(size=(D, 2 * D)) / D ** 0.5, rng.normal(size=(D, D)) / D ** 0.5
        par["w_post%d" % k], par["scale%d" % k] = 1 + 0.1 * rng.normal(size=D), 1 + 0.1 * rng.normal(size=D)
    for k in range(3):
        par["w_pre%d" % k] = 1 + 0.1 * rng.normal(size=D)
    par = {k: v.astype(np.float32).astype(np.float64) for k, v in par.items()}
    y0, wy, wz = (rng.normal(size=(B, T, D)).astype(np.float32).astype(np.float64) for _ in range(3))
    lengths = np.array([21, 9, 0])
    dev = {k: _up(v) for k, v in par.items()}
    words = torch.tensor([21, 4], dtype=torch.int64, device="cuda:0")
    len_t = torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
    cots = (_up(wy).view(B * T, D), _up(wz).view(B * T, D))
    state, z, g = _network(b, torch, dev, _up(y0), words, "f32", len_t, cots)

    f_step = torch.from_numpy(orc.drop_factors(B * T, D, 0.2, 21, 4, 1).reshape(B, T, D))
    f_drop = [torch.from_numpy(orc.drop_factors(B * T, D, 0.1, 21, 4, 10 + k).reshape(B, T, D)) for k in range(2)]
    leaves = {k: torch.from_numpy(v).requires_grad_() for k, v in par.items()}
    y_leaf = torch.from_numpy(y0).requires_grad_()
    es, ez = _network_exact(torch, leaves, y_leaf, f_step, f_drop, torch.from_numpy(lengths))
    ((es * torch.from_numpy(wy)).sum() + (ez * torch.from_numpy(wz)).sum()).backward()
    ref = {**{k: v.grad.numpy() for k, v in leaves.items()}, "y": y_leaf.grad.numpy().reshape(B * T, D)}
    for name, got, want in [("state", state, es.detach().numpy().reshape(B * T, D)), ("z", z, ez.detach().numpy().reshape(B * T, D))] + [(k, g[k], ref[k]) for k in ref]:
        assert np.abs(_np(got) - want).max() <= 2e-5 * max(np.abs(want).max(), 1), name
    # the same bits again
    again = _network(b, torch, dev, _up(y0), words, "f32", len_t, cots)
    assert torch.equal(again[0], state) and all(torch.equal(again[2][k], g[k]) for k in g)


def test_captured_and_replayed_on_another_stream_with_new_inputs():
    # One graph of the whole network, forward and backward; replays read the inputs, parameters and {seed, step} that the buffers hold then, while
    # eager calls of the same operators run on another stream
    torch, b, _ = _torch()
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    B, T, D = 2, 300, 64

    def rand(*s):
        return torch.randn(*s, generator=gen, device="cuda:0")

    par = {}
    for k in range(2):
        par["win%d" % k], par["wout%d" % k] = (rand(D, 2 * D) / 8).bfloat16(), (rand(D, D) / 8).bfloat16()
        par["w_post%d" % k], par["scale%d" % k] = 1 + 0.1 * rand(D), 1 + 0.1 * rand(D)
    for k in range(3):
        par["w_pre%d" % k] = 1 + 0.1 * rand(D)
    y, words = rand(B, T, D), torch.tensor([1, 1], dtype=torch.int64, device="cuda:0")
    lengths = torch.tensor([T, 100], dtype=torch.int32, device="cuda:0")
    cots = (rand(B * T, D), rand(B * T, D).bfloat16())
    eager = _network(b, torch, par, y, words, "bf16", lengths, cots)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = _network(b, torch, par, y, words, "bf16", lengths, cots)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], eager[0]) and all(torch.equal(out[2][k], eager[2][k]) for k in eager[2])
    y.copy_(rand(B, T, D))
    words.copy_(torch.tensor([1, 2], dtype=torch.int64))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.replay()
    new = _network(b, torch, par, y, words, "bf16", lengths, cots)
    torch.cuda.synchronize()
    assert not torch.equal(new[0], eager[0])
    assert torch.equal(out[0], new[0]) and all(torch.equal(out[2][k], new[2][k]) for k in new[2])


def test_calls_on_two_streams_at_once():
    # Each operator on two streams, queued alternately with different inputs: the same bits as one after the other
    torch, b, _ = _torch()
    work = []
    for seed in (1, 2):
        long, batch, rows = _recurrence_case(1, 6000, 128, "bf16", seed=seed), _recurrence_case(90, 300, 64, "bf16", seed=seed), _residual_case(900, 4096, "bf16", seed=seed)
        step = b.ResidualStep(4096, low="bf16")
        w = dict(gate=rows["t_gate"], w_post=rows["t_w_post"], scale=rows["t_scale"], w_pre=rows["t_w_pre"])

        def run(long=long, batch=batch, rows=rows, step=step, w=w):
            out = []
            for c in (long, batch):
                y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"])
                out += [y, yT, *b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"])]
            y, z, stats = step.forward(rows["t_y"], rows["t_u"], **w)
            g = step.backward(y, rows["t_u"], stats, dL_dy=rows["t_dy"], dL_dz=rows["t_dz"], **w)
            return out + [y, z, stats] + [g[k] for k in sorted(g)]

        work.append(run)
    alone = [run() for run in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(4):
        together = []
        for run, s in zip(work, streams):
            with torch.cuda.stream(s):
                together.append(run())
        torch.cuda.synchronize()
        for x, y in zip(alone, together):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


def test_calls_from_several_host_threads_at_once():
    # Sizes of one kernel that need different amounts of shared memory, each from its own thread on its own stream
    import threading
    torch, b, _ = _torch()
    cases = [_recurrence_case(B, T, D, "bf16") for B, T, D in ((300, 160, 64), (2500, 160, 64), (1, 9000, 64), (1, 9000, 72))]

    def run(c):
        y, yT = b.recurrence_forward(c["t_x"], c["t_gate"], y0=c["t_y0"])
        return [y, yT, *b.recurrence_backward(c["t_x"], c["t_gate"], y, c["t_dy"], dL_dyT=c["t_dyT"], y0=c["t_y0"])]

    alone = [run(c) for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(300):
                    got = run(cases[i])
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(p, q) for p, q in zip(got, alone[i])):
                    wrong.append("values of case %d" % i)
        except Exception as e:
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def test_operators_work_on_empty_batches():
    torch, b, _ = _torch()
    x = torch.zeros(0, 5, 8, dtype=torch.bfloat16, device="cuda:0")
    y, yT = b.recurrence_forward(x, x)
    assert y.shape == x.shape and yT.shape == (0, 8)
    x = torch.zeros(3, 0, 8, dtype=torch.bfloat16, device="cuda:0")
    y0 = torch.randn(3, 8, device="cuda:0")
    y, yT = b.recurrence_forward(x, x, y0=y0)
    assert torch.equal(yT, y0)
    assert torch.equal(b.recurrence_backward(x, x, y, y, dL_dyT=y0)[2], y0)
    s = b.ResidualStep(8)
    e, w = torch.zeros(0, 8, device="cuda:0"), torch.ones(8, device="cuda:0")
    y1, z, st = s.forward(e, e.bfloat16(), w_post=w)
    g = s.backward(y1, e.bfloat16(), st, dL_dy=e, dL_dz=z, w_post=w)
    assert z.shape == (0, 8) and torch.equal(g["dw_post"], torch.zeros(8, device="cuda:0"))
    assert b.dropout(torch.zeros(0, 8, device="cuda:0"), 0.5, torch.zeros(2, dtype=torch.int64, device="cuda:0")).shape == (0, 8)
