"""Sequence and residual operators as a user's program calls them, as a list of cases that can be timed and compared.

Three operators of a residual sequence block whose depth is the time of an ODE:

  recurrence  y_i = y_{i-1} + b_i (x_i - y_{i-1}) with b = sigmoid(gate) along a sequence (coupled), or y_i = (1 - b_i) y_{i-1} + x_i;
              forward returns the stored trajectory and the final state, backward the gradients of x, gate and the initial state
  residual    one step of the float32 state around a block that the caller evaluates: y' = y + h s drop(sigmoid(gate) N_post(u)) and the
              next block's input z = N_pre(y'); backward returns the adjoint of y, the cotangents of u and gate and the weights' gradients
  dropout     zero with probability p, the rest scaled by 1 / (1 - p), the mask from a counter-based generator

`run` with own = False is the plain form in elementary torch operations, with own = True the library's entry points.
"""
import math

import numpy as np
import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def _rec(name, **kw):
    c = dict(name=name, op="recurrence", train=False, seqs=1, steps=1, width=1, low="bf16", coupled=True, ragged=False, time_major=False)
    c.update(kw)
    return c


def _res(name, **kw):
    c = dict(name=name, op="residual", train=False, rows=1, width=1, low="bf16", norm="rms", gated=True, p=0.0)
    c.update(kw)
    return c


def _drop(name, **kw):
    c = dict(name=name, op="dropout", rows=1, width=1, low="bf16", p=0.1)
    c.update(kw)
    return c


def listed():
    return [
        # serving one token of each of 100 sequences: latency of a single step with the state carried along
        _rec("recurrence_step", seqs=100, steps=1, width=1024),
        # one long sequence read at once: few channels, the time axis has to be split
        _rec("recurrence_long", seqs=1, steps=65536, width=1024),
        # training on a batch of ordinary length, both directions
        _rec("recurrence_forward", seqs=8, steps=4096, width=2048),
        _rec("recurrence_backward", train=True, seqs=8, steps=4096, width=2048),
        # a padded batch with an odd width, states gated by the caller (uncoupled), float16
        _rec("recurrence_ragged_backward", train=True, seqs=37, steps=1000, width=785, low="f16", coupled=False, ragged=True),
        # serving a small batch: one row for each sequence
        _res("residual_step", rows=37, width=2048),
        # training: 8192 tokens, gate and dropout fused, both directions
        _res("residual_forward", rows=8192, width=2048, p=0.1),
        _res("residual_backward", train=True, rows=8192, width=2048, p=0.1),
        # float32 mode, an odd width and mean/variance norms
        _res("residual_f32_backward", train=True, rows=1000, width=785, low="f32", norm="meanvar"),
        # a wide state
        _res("residual_wide_backward", train=True, rows=4096, width=8192),
        # dropout alone: a toy network's layer, and a training batch
        _drop("dropout_small", rows=512, width=32, low="f16"),
        _drop("dropout_large", rows=8192, width=8192),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly multiples of 8, as people choose them, now and then an odd width."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, (w + 4) // 8 * 8)


def draw(rng):
    op = rng.choice(["recurrence", "recurrence", "residual", "residual", "dropout"])
    low = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "recurrence":
        c = _rec("", train=rng.random() < 0.5, seqs=_log_int(rng, 1, 256), steps=rng.choice([1, _log_int(rng, 2, 65536), _log_int(rng, 2, 65536)]),
                 width=_width(rng, 16, 4096), low=low, coupled=rng.random() < 0.7, ragged=rng.random() < 0.4, time_major=rng.random() < 0.3)
        while c["seqs"] * c["steps"] * c["width"] > 1 << 25:
            key = "seqs" if c["seqs"] > 1 else "steps"
            c[key] = max(1, c[key] * 2 // 3)
    elif op == "residual":
        c = _res("", train=rng.random() < 0.6, rows=_log_int(rng, 1, 16384), width=_width(rng, 32, 8192), low=low,
                 norm=rng.choice(["rms", "rms", "meanvar"]), gated=rng.random() < 0.7, p=rng.choice([0.0, 0.0, 0.1, 0.25]))
        while c["rows"] * c["width"] > 1 << 24:
            c["rows"] = max(1, c["rows"] * 2 // 3)
    else:
        c = _drop("", rows=_log_int(rng, 1, 16384), width=_width(rng, 16, 8192), low=low, p=rng.choice([0.05, 0.1, 0.25, 0.5]))
        while c["rows"] * c["width"] > 1 << 25:
            c["rows"] = max(1, c["rows"] * 2 // 3)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ what a program has in hand
def _normal(gen, shape, dtype=torch.float32, scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale + mean).to(dtype)


def _lengths(B, T):
    """From the full length down to nothing in equal steps (the order comes from the seed)."""
    return (torch.arange(B, 0, -1) * T // B if B < 2 else torch.arange(B - 1, -1, -1) * T // (B - 1)).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 17)
    low = DTYPE[case["low"]]
    s = dict(case=case, low=low)
    if case["op"] == "recurrence":
        B, T, D = case["seqs"], case["steps"], case["width"]

        def rows(t):         # [B, T, D], or a view of that shape of a [T, B, D] buffer
            return t.transpose(0, 1).contiguous().transpose(0, 1) if case["time_major"] else t
        # channels with memories from a few steps to about a thousand, the gates moving with the input
        bias = torch.linspace(1.0, -7.0, D, device="cuda")
        s["x"] = rows(_normal(gen, (B, T, D), low))
        s["gate"] = rows((torch.randn((B, T, D), generator=gen, device="cuda") + bias).to(low))
        s["y0"] = _normal(gen, (B, D))
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = _lengths(B, T).to("cuda")[torch.randperm(B, generator=gen, device="cuda")]
        if case["train"]:
            s["y"] = rows(_recurrence_forward(s)[0])
            s["dy"] = rows(_normal(gen, (B, T, D), low))
            s["dyT"] = _normal(gen, (B, D))
    elif case["op"] == "residual":
        M, D = case["rows"], case["width"]
        s["h"] = 0.5
        s["y"] = _normal(gen, (M, D), scale=2.0)
        s["u"] = _normal(gen, (M, D), low, mean=0.25)
        s["gate"] = _normal(gen, (M, D), low, mean=0.5) if case["gated"] else None
        s["w_post"] = _normal(gen, (D,), scale=0.1, mean=1.0)
        s["w_pre"] = _normal(gen, (D,), scale=0.1, mean=1.0)
        s["scale"] = _normal(gen, (D,), scale=0.1, mean=0.5)
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=gen, device="cuda", dtype=torch.int64) if case["p"] > 0 else None
        if case["train"]:
            s["y"], _, s["stats"] = _residual_forward(s)       # the state behind the step, as the forward pass left it
            s["dy"] = _normal(gen, (M, D))
            s["dz"] = _normal(gen, (M, D), low)
        if own:
            from paper_2510_23498_b200 import binding
            s["step"] = binding.ResidualStep(D, low=case["low"], post_norm=case["norm"], pre_norm=case["norm"], eps=EPS, h=s["h"], p=case["p"], site=3)
    else:
        M, D = case["rows"], case["width"]
        s["x"] = _normal(gen, (M, D), low)
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=gen, device="cuda", dtype=torch.int64)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _scan(C, u):
    """Inclusive composition along dim 1 of the maps y -> y + u - C y, by doubling the distance."""
    k, T = 1, C.shape[1]
    while k < T:
        Cr, ur = C[:, k:], u[:, k:]
        Cl, ul = C[:, :-k], u[:, :-k]
        u = torch.cat([u[:, :k], ur + (ul - Cr * ul)], 1)
        C = torch.cat([C[:, :k], Cl + Cr * (1 - Cl)], 1)
        k *= 2
    return C, u


def _valid(s):
    if s["lengths"] is None:
        return None
    return (torch.arange(s["x"].shape[1], device="cuda")[None] < s["lengths"][:, None])[..., None]


def _recurrence_forward(s):
    c = s["case"]
    x, g = s["x"].float(), s["gate"].float()
    b = 1 / (1 + torch.exp(-g))
    u = b * x if c["coupled"] else x
    m = _valid(s)
    if m is not None:
        b, u = torch.where(m, b, torch.zeros_like(b)), torch.where(m, u, torch.zeros_like(u))
    C, u = _scan(b, u)
    y = u + (1 - C) * s["y0"][:, None]
    yT = y[:, -1].clone()
    if m is not None:
        y = torch.where(m, y, torch.zeros_like(y))
    return y.to(s["low"]), yT


def _recurrence_backward(s):
    c = s["case"]
    x, g, y, dy = s["x"].float(), s["gate"].float(), s["y"].float(), s["dy"].float()
    e = torch.exp(-g.abs())
    small, big = e / (1 + e), 1 / (1 + e)
    b, keep = torch.where(g < 0, small, big), torch.where(g < 0, big, small)
    before = torch.cat([s["y0"][:, None], y[:, :-1]], 1)
    m = _valid(s)
    if m is not None:
        zero = torch.zeros_like(b)
        b, keep, dy = torch.where(m, b, zero), torch.where(m, keep, zero + 1), torch.where(m, dy, zero)
    C, u = _scan(b.flip(1), (keep * dy).flip(1))
    r = u + (1 - C) * s["dyT"][:, None]                 # what reaches the state before step T-1, T-2, ..., 0
    lam = dy + torch.cat([s["dyT"][:, None], r[:, :-1]], 1).flip(1)
    dx = b * lam if c["coupled"] else lam
    dg = lam * (x - before if c["coupled"] else -before) * (small * big)
    if m is not None:
        dx, dg = torch.where(m, dx, zero), torch.where(m, dg, zero)
    return dx.to(s["low"]), dg.to(s["low"]), r[:, -1].clone()


def _philox(n_groups, rng, site):
    """Philox4x32-10 (Salmon et al. 2011) of the counters (group, group >> 32, step, site), key = the seed: four int64 tensors of 32-bit words."""
    mask = 0xffffffff
    i = torch.arange(n_groups, device="cuda", dtype=torch.int64)
    seed, step = rng[0], rng[1]
    w = [i & mask, i >> 32, (step & mask).expand(n_groups), torch.full_like(i, site)]
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        p0, p1 = w[0] * 0xD2511F53, w[2] * 0xCD9E8D57
        w = [((p1 >> 32) & mask) ^ w[1] ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ w[3] ^ k1, p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return w


def _threshold(p):
    return int(p * 65536 + 0.5)


def _mask(rows, width, rng, site, p):
    """Kept elements: 16 bits each, eight neighbours of a row from one counter."""
    groups = (width + 7) // 8
    w = torch.stack(_philox(rows * groups, rng, site), -1)
    bits = torch.stack([w & 0xffff, w >> 16], -1).reshape(rows, groups * 8)[:, :width]
    return bits >= _threshold(p)


def _apply_mask(v, keep, p):
    return torch.where(keep, v * (65536.0 / (65536 - _threshold(p))), torch.zeros_like(v))


def _norm(v, kind):
    mean = v.mean(1, keepdim=True) if kind == "meanvar" else torch.zeros_like(v[:, :1])
    d = v - mean
    rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    return d * rstd, mean, rstd


def _norm_back(dn, n, rstd, kind):
    out = dn - n * (dn * n).mean(1, keepdim=True)
    if kind == "meanvar":
        out = out - dn.mean(1, keepdim=True)
    return out * rstd


def _residual_forward(s):
    c = s["case"]
    n, mu, ru = _norm(s["u"].float(), c["norm"])
    v = n * s["w_post"]
    if s["gate"] is not None:
        v = v / (1 + torch.exp(-s["gate"].float()))
    if c["p"] > 0:
        v = _apply_mask(v, _mask(c["rows"], c["width"], s["rng"], 3, c["p"]), c["p"])
    y = s["y"] + s["h"] * s["scale"] * v
    z, my, ry = _norm(y, c["norm"])
    return y, (z * s["w_pre"]).to(s["low"]), torch.cat([mu, ru, my, ry], 1)


def _residual_backward(s):
    c, h = s["case"], s["h"]
    z, _, ry = _norm(s["y"], c["norm"])
    dz = s["dz"].float()
    dw_pre = (dz * z).sum(0)
    a = s["dy"] + _norm_back(dz * s["w_pre"], z, ry, c["norm"])
    n, _, ru = _norm(s["u"].float(), c["norm"])
    v = n * s["w_post"]
    keep = _mask(c["rows"], c["width"], s["rng"], 3, c["p"]) if c["p"] > 0 else None
    t = _apply_mask(a, keep, c["p"]) if keep is not None else a        # the mask is the same factor in both directions
    sig = 1 / (1 + torch.exp(-s["gate"].float())) if s["gate"] is not None else None
    dscale = h * (t * (v * sig if sig is not None else v)).sum(0)
    t = h * s["scale"] * t
    dgate = (t * v * sig * (1 - sig)).to(s["low"]) if sig is not None else None
    if sig is not None:
        t = t * sig
    dw_post = (t * n).sum(0)
    du = _norm_back(t * s["w_post"], n, ru, c["norm"]).to(s["low"])
    out = dict(dy=a, du=du, dw_post=dw_post, dscale=dscale, dw_pre=dw_pre)
    if dgate is not None:
        out["dgate"] = dgate
    return out


def _dropout(s):
    c = s["case"]
    return _apply_mask(s["x"].float(), _mask(c["rows"], c["width"], s["rng"], 5, c["p"]), c["p"]).to(s["low"])


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2510_23498_b200 import binding
        if c["op"] == "recurrence" and not c["train"]:
            return binding.recurrence_forward(s["x"], s["gate"], y0=s["y0"], lengths=s["lengths"], coupled=c["coupled"])
        if c["op"] == "recurrence":
            return binding.recurrence_backward(s["x"], s["gate"], s["y"], s["dy"], dL_dyT=s["dyT"], y0=s["y0"], lengths=s["lengths"],
                                               coupled=c["coupled"])
        if c["op"] == "residual" and not c["train"]:
            return s["step"].forward(s["y"], s["u"], gate=s["gate"], w_post=s["w_post"], scale=s["scale"], w_pre=s["w_pre"], rng=s["rng"])
        if c["op"] == "residual":
            g = s["step"].backward(s["y"], s["u"], s["stats"], dL_dy=s["dy"], dL_dz=s["dz"], gate=s["gate"], w_post=s["w_post"], scale=s["scale"],
                                   w_pre=s["w_pre"], rng=s["rng"])
            names = ["dy", "du", "dw_post", "dscale", "dw_pre"] + (["dgate"] if c["gated"] else [])
            return {k: g[k] for k in names}
        return binding.dropout(s["x"], c["p"], s["rng"], site=5)
    if c["op"] == "recurrence":
        return _recurrence_backward(s) if c["train"] else _recurrence_forward(s)
    if c["op"] == "residual":
        return _residual_backward(s) if c["train"] else _residual_forward(s)
    return _dropout(s)


# ------------------------------------------------------------------------------------------------ least work
def work(case):
    es = 4 if case["low"] == "f32" else 2
    if case["op"] == "recurrence":
        n, w = case["seqs"] * case["steps"] * case["width"], case["seqs"] * case["width"]
        read = int(_lengths(case["seqs"], case["steps"]).sum()) * case["width"] if case["ragged"] else n
        if case["train"]:          # x, gate, y, dy in; dx, dgate out; y0, dyT in, dy0 out
            inputs = 4 if case["coupled"] else 3      # the uncoupled form's gradients do not depend on x
            return {"bytes": es * (inputs * read + 2 * n) + 12 * w, "flops": 24 * read}
        return {"bytes": es * (2 * read + n) + 8 * w, "flops": 10 * read}
    n, w = case["rows"] * case["width"], case["width"]
    if case["op"] == "residual":
        low = 2 if case["gated"] else 1
        if case["train"]:          # y, dy, dz, u, gate, stats in; dy, du, dgate out; three weights in, three gradients out
            return {"bytes": n * (12 + es * (1 + 2 * low)) + 16 * case["rows"] + 24 * w, "flops": 50 * n}
        return {"bytes": n * (8 + es * (1 + low)) + 16 * case["rows"] + 12 * w, "flops": 25 * n}
    return {"bytes": 2 * es * n, "flops": 14 * n}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_mask(rows, width, rng, site, p):
    """The generator again, in numpy's unsigned integers."""
    seed, step = int(rng[0]), int(rng[1])
    groups = (width + 7) // 8
    ctr = np.zeros((4, rows * groups), dtype=np.uint64)
    idx = np.arange(rows * groups, dtype=np.uint64)
    full, half = np.uint64(0xffffffff), np.uint64(32)
    ctr[0], ctr[1], ctr[2], ctr[3] = idx & full, idx >> half, step & 0xffffffff, site
    key = [seed & 0xffffffff, (seed >> 32) & 0xffffffff]
    for _ in range(10):
        a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = np.stack([(b >> half) ^ ctr[1] ^ np.uint64(key[0]), b & full, (a >> half) ^ ctr[3] ^ np.uint64(key[1]), a & full])
        key = [(key[0] + 0x9E3779B9) & 0xffffffff, (key[1] + 0xBB67AE85) & 0xffffffff]
    bits = np.ascontiguousarray(ctr.T.astype("<u4")).view("<u2").reshape(rows, groups * 8)[:, :width]
    return torch.from_numpy((bits >= _threshold(p))).to("cuda")


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "recurrence":
        T = case["steps"]
        x, b, y0 = s["x"].to(f64), torch.sigmoid(s["gate"].to(f64)), s["y0"].to(f64)
        n = s["lengths"] if s["lengths"] is not None else torch.full((case["seqs"],), T, device="cuda")
        on = torch.arange(T, device="cuda")[:, None, None] < n[None, :, None]                # [T, B, 1]
        if not case["train"]:
            y, rows = y0, torch.zeros_like(x)
            for i in range(T):
                new = (1 - b[:, i]) * y + (b[:, i] * x[:, i] if case["coupled"] else x[:, i])
                y = torch.where(on[i], new, y)
                rows[:, i] = torch.where(on[i], new, 0.0)
            return rows, y
        dy, before = s["dy"].to(f64), torch.cat([y0[:, None], s["y"].to(f64)[:, :-1]], 1)
        r, dx, dg = s["dyT"].to(f64), torch.zeros_like(x), torch.zeros_like(x)
        one_minus = torch.sigmoid(-s["gate"].to(f64))
        for i in range(T - 1, -1, -1):
            lam = r + dy[:, i]
            slope = b[:, i] * one_minus[:, i]
            if case["coupled"]:
                gx, gg = b[:, i] * lam, lam * slope * (x[:, i] - before[:, i])
            else:
                gx, gg = lam, -lam * slope * before[:, i]
            dx[:, i], dg[:, i] = torch.where(on[i], gx, 0.0), torch.where(on[i], gg, 0.0)
            r = torch.where(on[i], one_minus[:, i] * lam, r)
        return dx, dg, r
    M, D, p = case["rows"], case["width"], case["p"]
    if case["op"] == "dropout":
        keep = _exact_mask(M, D, s["rng"], 5, p)
        return torch.where(keep, s["x"].to(f64) * (65536.0 / (65536 - _threshold(p))), 0.0)

    def normed(v):
        mean = v.mean(1) if case["norm"] == "meanvar" else torch.zeros(M, device="cuda", dtype=f64)
        rstd = (((v - mean[:, None]) ** 2).sum(1) / D + EPS) ** -0.5
        return (v - mean[:, None]) * rstd[:, None], mean, rstd

    factor = s["h"] * _exact_mask(M, D, s["rng"], 3, p).to(f64) * (65536.0 / (65536 - _threshold(p))) if p > 0 else s["h"]
    leaf = {k: s[k].to(f64).requires_grad_(case["train"]) for k in ("u", "gate", "w_post", "scale", "w_pre", "y") if s[k] is not None}
    n, mu, ru = normed(leaf["u"])
    v = n * leaf["w_post"] * leaf["scale"] * factor
    if case["gated"]:
        v = v * torch.sigmoid(leaf["gate"])
    if not case["train"]:
        y = leaf["y"] + v
        z, my, ry = normed(y)
        return y, z * leaf["w_pre"], torch.stack([mu, ru, my, ry], 1)
    z = normed(leaf["y"])[0] * leaf["w_pre"]
    gy, gw = torch.autograd.grad(z, [leaf["y"], leaf["w_pre"]], s["dz"].to(f64))
    a = s["dy"].to(f64) + gy
    names = ["u", "w_post", "scale"] + (["gate"] if case["gated"] else [])
    grads = dict(zip(names, torch.autograd.grad(v, [leaf[k] for k in names], a)))
    out = dict(dy=a, du=grads["u"], dw_post=grads["w_post"], dscale=grads["scale"], dw_pre=gw)
    if case["gated"]:
        out["dgate"] = grads["gate"]
    return out
