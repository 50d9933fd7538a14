"""Sequence and residual operators on the CPU: pins of their float64 oracle (finite differences, published generator vectors) and the argument checks of the
C entry points, which are taken before anything is queued and need no device."""
import ctypes as C

import numpy as np
import pytest

from oracle import operators as orc


def _fd(f, args, name, w, eps=1e-6):
    """Central differences of <w, f(args)> in every entry of args[name]."""
    base = args[name]
    out = np.zeros_like(base)
    for i in np.ndindex(base.shape):
        hi, lo = base.copy(), base.copy()
        hi[i] += eps
        lo[i] -= eps
        out[i] = (w(f(**{**args, name: hi})) - w(f(**{**args, name: lo}))) / (2 * eps)
    return out


@pytest.mark.parametrize("coupled", [True, False])
def test_recurrence_gradients_are_those_of_central_differences(coupled):
    rng = np.random.default_rng(3)
    B, T, D = 3, 5, 2
    args = dict(x=rng.normal(size=(B, T, D)), gate=rng.normal(size=(B, T, D)), y0=rng.normal(size=(B, D)), lengths=[5, 0, 3], coupled=coupled)
    wy, wT = rng.normal(size=(B, T, D)), rng.normal(size=(B, D))
    for s, n in enumerate(args["lengths"]):
        wy[s, n:] = 0
    y = orc.recurrence_forward(**args)[0]
    dx, dg, dy0, _, _ = orc.recurrence_backward(args["x"], args["gate"], y, wy, wT, args["y0"], args["lengths"], coupled)

    def w(out):
        return (wy * out[0]).sum() + (wT * out[1]).sum()

    for name, g in (("x", dx), ("gate", dg), ("y0", dy0)):
        assert np.allclose(g, _fd(orc.recurrence_forward, args, name, w), rtol=1e-7, atol=1e-8), name


def test_coupled_recurrence_is_the_implicit_euler_step_of_the_relaxation_equation():
    # (y_i - y_{i-1}) / h = lambda (x - y_i) with gate = log(h lambda), on a grid of unequal steps
    rng = np.random.default_rng(4)
    h, lam, x = rng.uniform(0.1, 2, (1, 6, 1)), rng.uniform(0.1, 3, (1, 6, 4)), rng.normal(size=(1, 6, 4))
    y = orc.recurrence_forward(x, np.log(h * lam), np.ones((1, 4)), [6], True)[0]
    before = np.concatenate([np.ones((1, 1, 4)), y[:, :-1]], 1)
    assert np.allclose((y - before) / h, lam * (x - y), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("post,pre,gated,dropped", [("rms", "rms", True, True), ("meanvar", "meanvar", True, False), ("none", "meanvar", False, True),
                                                   ("rms", "none", False, False)])
def test_residual_gradients_are_those_of_central_differences(post, pre, gated, dropped):
    rng = np.random.default_rng(5)
    M, D = 3, 9
    args = dict(y=rng.normal(size=(M, D)), u=rng.normal(size=(M, D)), gate=rng.normal(size=(M, D)) if gated else None, w_post=rng.normal(size=D),
                scale=rng.normal(size=D), w_pre=rng.normal(size=D), h=0.3, post=post, pre=pre, eps=1e-2,
                factors=orc.drop_factors(M, D, 0.3, 7, 8, 9) if dropped else np.ones((M, D)))
    dy, dz = rng.normal(size=(M, D)), rng.normal(size=(M, D))
    y_new = orc.residual_forward(**args)[0]
    g = orc.residual_backward(y_new, args["u"], args["gate"], args["w_post"], args["scale"], args["w_pre"], 0.3, post, pre, 1e-2, args["factors"], dy, dz)

    def w(out):
        return (dy * out[0]).sum() + (dz * out[1]).sum()

    for name, key in (("y", "dy"), ("u", "du"), ("gate", "dgate"), ("w_post", "dw_post"), ("scale", "dscale"), ("w_pre", "dw_pre")):
        if args[name] is not None:
            assert np.allclose(g[key], _fd(orc.residual_forward, args, name, w), rtol=1e-6, atol=1e-7), name


def test_generator_gives_the_published_vectors():
    # Known answers of Philox4x32-10 that its authors publish with the paper
    assert orc.philox4x32([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert orc.philox4x32([0xffffffff] * 4, [0xffffffff] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def test_dropout_keeps_the_stated_share_and_the_mean():
    f = orc.drop_factors(64, 100, 0.25, 1, 2, 3)
    kept = (f > 0).mean()
    assert abs(kept - 0.75) < 5 * np.sqrt(0.25 * 0.75 / f.size) and np.allclose(f[f > 0], 4 / 3)
    assert (f == orc.drop_factors(64, 100, 0.25, 1, 2, 3)).all()
    assert (f != orc.drop_factors(64, 100, 0.25, 1, 2, 4)).any() and (f != orc.drop_factors(64, 100, 0.25, 1, 3, 3)).any()


# ------------------------------------------------------------------------------------------------ refusals (no device: nothing is queued, no address is followed)
AT = [(1 << 40) + (i << 30) for i in range(20)]


def _recurrence(lib, direction="forward", at=None, **kw):
    from paper_2510_23498_b200 import binding
    f = dict(low=1, n_seq=2, n_steps=3, width=8, coupled=1)
    f.update(kw)
    p = dict(enumerate(AT))
    p.update(at or {})
    d = binding.RecurrenceDesc(**f)
    if direction == "forward":
        return lib.mpode_recurrence_forward(C.byref(d), None, *[p[i] for i in range(6)])
    return lib.mpode_recurrence_backward(C.byref(d), None, *[p[i] for i in range(11)])


def test_recurrence_refuses_bad_arguments():
    from paper_2510_23498_b200 import binding as b
    lib = b.load_library()
    bad = [dict(low=3), dict(n_seq=-1), dict(n_steps=-1), dict(width=0), dict(in_step_stride=7), dict(out_step_stride=7), dict(in_seq_stride=4),
           dict(in_seq_stride=8, in_step_stride=8), dict(in_seq_stride=23), dict(out_seq_stride=8, out_step_stride=15),
           dict(at={0: None}), dict(at={1: None}), dict(at={4: None}), dict(at={0: AT[0] + 1}), dict(at={2: AT[2] + 2}), dict(at={3: AT[3] + 1})]
    for kw in bad:
        assert _recurrence(lib, **kw) == b.ERR_INVALID_ARG, kw
        assert b"recurrence" in lib.mpode_operator_error()
    for kw in bad[:10] + [dict(at={0: None}), dict(at={1: None}), dict(at={4: None}), dict(at={7: None}), dict(at={8: None}), dict(at={10: AT[10] + 2})]:
        assert _recurrence(lib, "backward", **kw) == b.ERR_INVALID_ARG, kw
    assert _recurrence(lib, n_seq=1 << 30, width=1 << 20) == b.ERR_UNSUPPORTED
    assert _recurrence(lib, n_seq=1, in_step_stride=1 << 27) == b.ERR_UNSUPPORTED        # 16 steps beyond 4 GB
    assert lib.mpode_recurrence_forward(None, None, *AT[:6]) == b.ERR_INVALID_ARG
    assert _recurrence(lib, n_seq=0, at={i: None for i in range(6)}) == b.OK            # nothing to do


def test_recurrence_refuses_outputs_over_inputs_of_other_strides_and_strides_beyond_64_bits():
    from paper_2510_23498_b200 import binding as b
    lib = b.load_library()
    for kw in (dict(at={4: AT[0]}, in_step_stride=16, in_seq_stride=48), dict(at={4: AT[0]}, in_step_stride=16, in_seq_stride=8), dict(at={4: AT[1]}, out_seq_stride=32),
               dict(n_seq=(1 << 20) + 1, in_seq_stride=1 << 44, in_step_stride=1 << 22, n_steps=(1 << 30) + 1)):
        assert _recurrence(lib, **kw) == b.ERR_INVALID_ARG, kw
        assert b"recurrence" in lib.mpode_operator_error()
    for i in (7, 8):
        assert _recurrence(lib, "backward", at={i: AT[5]}, out_seq_stride=32) == b.ERR_INVALID_ARG


def _residual(lib, direction="forward", rows=4, at=None, scale_exp=0, nbytes=1 << 30, **kw):
    from paper_2510_23498_b200 import binding
    f = dict(low=1, width=64, post_norm=1, pre_norm=1, eps=1e-5, h=1.0, p_drop=0.0)
    f.update(kw)
    p = dict(enumerate(AT))
    p.update(at or {})
    d = binding.ResidualDesc(**f)
    if direction == "forward":
        return lib.mpode_residual_forward(C.byref(d), None, rows, *[p[i] for i in range(10)])
    return lib.mpode_residual_backward(C.byref(d), None, rows, *[p[i] for i in range(10)], scale_exp, *[p[i] for i in range(10, 16)], 0, p[16], p[17], nbytes)


def test_residual_step_refuses_bad_arguments():
    from paper_2510_23498_b200 import binding as b
    lib = b.load_library()
    both = [dict(low=-1), dict(width=0), dict(rows=-1), dict(post_norm=3), dict(pre_norm=-1), dict(eps=0.0), dict(eps=float("nan")), dict(p_drop=1.5),
            dict(p_drop=float("nan")), dict(ld_y=63), dict(ld_u=63), dict(ld_gate=1), dict(ld_z=63), dict(at={1: AT[1] + 1}), dict(at={0: AT[0] + 2})]
    for kw in both + [dict(at={0: None}), dict(at={7: None}), dict(at={1: None}), dict(at={1: None, 2: None, 8: None}), dict(at={9: AT[9] + 8}),
                      dict(p_drop=0.1, at={6: None}), dict(p_drop=0.1, at={6: AT[6] + 4})]:
        assert _residual(lib, **kw) == b.ERR_INVALID_ARG, kw
        assert lib.mpode_operator_error()
    for kw in both + [dict(at={10: None}), dict(at={11: None}), dict(at={12: None}), dict(at={0: None}), dict(at={1: None}), dict(at={2: None}),
                      dict(at={7: None}), dict(scale_exp=101), dict(scale_exp=-101), dict(at={17: None}), dict(at={17: AT[17] + 128}), dict(at={13: AT[13] + 2})]:
        assert _residual(lib, "backward", **kw) == b.ERR_INVALID_ARG, kw
    assert _residual(lib, "backward", nbytes=16) == b.ERR_WORKSPACE_TOO_SMALL
    assert _residual(lib, width=16385) == b.ERR_UNSUPPORTED
    assert _residual(lib, rows=0, at={i: None for i in range(10)}) == b.OK
    bad = b.ResidualDesc(1, 0, 1, 1, 1e-5, 1.0, 0.0)
    assert lib.mpode_residual_workspace_bytes(C.byref(bad), 4) == 0


def test_dropout_refuses_bad_arguments():
    from paper_2510_23498_b200 import binding as b
    lib = b.load_library()

    def call(low=1, rows=4, width=16, x=AT[0], ld_x=0, out=AT[1], ld_out=0, p=0.5, rng=AT[2], flag=AT[3]):
        return lib.mpode_dropout(low, None, rows, width, x, ld_x, out, ld_out, p, rng, 0, flag)

    for kw in (dict(low=5), dict(rows=-1), dict(width=0), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(ld_x=15), dict(ld_out=8), dict(x=None),
               dict(out=None), dict(rng=None), dict(rng=AT[2] + 4), dict(x=AT[0] + 1), dict(flag=AT[3] + 1), dict(out=AT[0], ld_x=32)):
        assert call(**kw) == b.ERR_INVALID_ARG, kw
    assert call(rows=1 << 41) == b.ERR_UNSUPPORTED
    assert call(rows=0, x=None, out=None, rng=None) == b.OK


def test_tensors_that_do_not_fit_are_refused_by_the_binding():
    import torch
    from paper_2510_23498_b200 import binding as b
    x = torch.zeros(2, 3, 8, dtype=torch.bfloat16)
    calls = [lambda: b.recurrence_forward(x, x),                                                # not on a CUDA device
             lambda: b.recurrence_forward(x[0], x[0]),
             lambda: b.recurrence_forward(x, x.float()),
             lambda: b.recurrence_forward(x.double(), x.double()),
             lambda: b.recurrence_forward(x, x.transpose(0, 1).contiguous().transpose(0, 1)),   # strides of x and gate differ
             lambda: b.recurrence_forward(x[:, :1].expand(2, 3, 8), x),
             lambda: b.recurrence_forward(x, x, y0=torch.zeros(2, 7)),
             lambda: b.recurrence_forward(x, x, lengths=torch.zeros(2, dtype=torch.int64)),
             lambda: b.recurrence_backward(x, x, x, x, dL_dx=x.clone()),                        # dL_dx without dL_dgate
             lambda: b.recurrence_backward(x, x, x, x, dL_dyT=torch.zeros(2, 8, dtype=torch.float64)),
             lambda: b.ResidualStep(8).forward(torch.zeros(3, 8), torch.zeros(3, 8)),           # u is not bf16
             lambda: b.ResidualStep(8).forward(torch.zeros(3, 8), w_pre=torch.zeros(9)),
             lambda: b.ResidualStep(8).forward(torch.zeros(3, 1).expand(3, 8)),
             lambda: b.dropout(x, 0.5, torch.zeros(2, dtype=torch.int32)),
             lambda: b.dropout(x, 0.5, torch.zeros(2, dtype=torch.int64))]
    for i, f in enumerate(calls):
        with pytest.raises(b.MpodeError):
            f()
            raise AssertionError(i)
