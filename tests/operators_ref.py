"""The operators of sequence models written out in 64 bits, with bounds for what float32 arithmetic and one
rounding to the storage type may add.  Plain torch on the CPU or the GPU; nothing of the library is used.

U is half a step of float32.  A bound counts roundings: a sum of terms t_k along a chain of at most K
additions is off by at most K U sum |t_k|, a product or a quotient by U relative, the native
exponential and reciprocal by two U each (one unit in the last place), and the stored result by half a
step of its type."""
import math

import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# what a type's smallest numbers are apart, halved
TINY = {torch.float32: 2.0 ** -140, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
BLOCK = 32


def stored(bound, value, dtype):
    """A bound for a result computed to within `bound` and rounded once to `dtype`."""
    return bound + HALF_STEP[dtype] * (value.abs() + bound) + TINY[dtype]


def close(name, got, want, bound):
    g, w = got.double().to(want.device), want
    err = (g - w).abs()
    bad = ~((err <= bound) | (torch.isnan(g) & torch.isnan(w)) | ((g == w) & torch.isinf(w)))
    if bad.any():
        at = bad.nonzero()[:4].tolist()
        worst = float((err / bound).nan_to_num(math.inf)[bad].max())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds, worst {worst:.3g} times its bound, first at {at}: "
                             f"got {g[bad][:4].tolist()}, want {w[bad][:4].tolist()}")


# ------------------------------------------------------------------ layer normalisation

def norm_chain(cols):
    """Additions that a row's sum passes through: a thread's own elements (at most 32, or one per vector of a
    long row), 6 across a wavefront, 16 wavefronts."""
    return 64 + cols // 1024


def layer_norm(x, w, b, eps, dtype):
    """y, mean, rstd, n and the bounds of y, mean, rstd (relative) and n."""
    x = x.double()
    cols = x.shape[-1]
    mean = x.mean(-1, keepdim=True)
    var = ((x - mean) ** 2).mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    n = (x - mean) * rstd
    K = norm_chain(cols)
    e_mean = K * U * x.abs().mean(-1, keepdim=True) + U * mean.abs()
    # the sum of squares about a mean that is off by e is larger by e^2, each term rounded three times; the root halves
    e_rstd = (K + 8) * U + 0.5 * (e_mean * rstd) ** 2
    e_n = (e_mean + 2 * U * (x - mean).abs()) * rstd * (1 + e_rstd) + n.abs() * (e_rstd + 2 * U)
    w = torch.ones(cols, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(cols, dtype=torch.float64, device=x.device) if b is None else b.double()
    y = n * w + b
    e_y = w.abs() * e_n + U * (y.abs() + (n * w).abs())
    return dict(y=y, mean=mean[..., 0], rstd=rstd[..., 0], n=n, e_n=e_n, e_y=stored(e_y, y, dtype),
                e_mean=e_mean[..., 0] + TINY[torch.float32], e_rstd=(e_rstd * rstd)[..., 0])


def layer_norm_grad(dy, w, n, rstd, e_n, dtype, param_dtype):
    """dx, dweight, dbias and their bounds; n and rstd as the kernel reads them, n to within e_n.  Leading axes are rows."""
    cols = dy.shape[-1]
    dy, n = dy.double().reshape(-1, cols), n.double().reshape(-1, cols)
    e_n = torch.zeros_like(n) + e_n if not torch.is_tensor(e_n) else e_n.reshape(-1, cols)
    r = rstd.double().reshape(-1, 1)
    w = torch.ones(cols, dtype=torch.float64, device=dy.device) if w is None else w.double()
    g = dy * w
    rows = max(1, dy.shape[0])
    m1, m2 = g.mean(-1, keepdim=True), (g * n).mean(-1, keepdim=True)
    dx = r * (g - m1 - n * m2)
    K = norm_chain(cols)
    e1 = (K + 2) * U * g.abs().mean(-1, keepdim=True)
    e2 = (K + 3) * U * (g * n).abs().mean(-1, keepdim=True) + (g.abs() * e_n).mean(-1, keepdim=True)
    e_dx = r * (e1 + n.abs() * e2 + m2.abs() * e_n + 3 * U * (g.abs() + m1.abs() + (n * m2).abs())) + U * dx.abs()
    # a column's sum: rows of a workgroup one after the other, its threads' sums, and the workgroups' partials
    D = 200 + rows // 256
    dw, db = (dy * n).sum(0), dy.sum(0)
    e_dw = D * U * (dy * n).abs().sum(0) + (dy.abs() * e_n).sum(0)
    e_db = D * U * dy.abs().sum(0)
    return dict(dx=dx, dw=dw, db=db, e_dx=stored(e_dx, dx, dtype), e_dw=stored(e_dw, dw, param_dtype), e_db=stored(e_db, db, param_dtype))


# ------------------------------------------------------------------ 8 bits

def pow2(k):
    """2^k from its bits: the GPU's 64-bit exp2, and with it torch's ldexp and 2.0 ** k, is off by a unit in the last
    place at some whole numbers (-19, -9, -4 among them)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def e4m3_step(q):
    """What neighbouring e4m3 values around q are apart."""
    return pow2(torch.frexp(q.abs().clamp_min(2.0 ** -6))[1] - 4)


def keep8(x, kind):
    """Codes (as whole numbers of int8, or e4m3 values), scale bytes and the values they stand for."""
    x = x.double()
    cols = x.shape[-1]
    full = torch.nn.functional.pad(x, (0, -cols % BLOCK)).reshape(*x.shape[:-1], -1, BLOCK)
    top = full.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(full).all(-1, keepdim=True)
    most = 127.0 if kind == "i8" else 448.0
    k = torch.full_like(top, -126)
    for p in range(-125, 129):                        # the smallest power that reaches the largest magnitude
        k = torch.where(torch.nan_to_num(top, 0, 0) > most * 2.0 ** (p - 1), float(p), k)
    unit = pow2(k)
    q = torch.where(finite, full / unit, 0.0)
    if kind == "i8":
        code = torch.round(q)
    else:
        code = torch.round(q / e4m3_step(q)) * e4m3_step(q)
    byte = torch.where(finite, k + 127, 255.0)
    value = torch.where(finite, code * unit, math.nan)
    flat = lambda t: t.reshape(*x.shape[:-1], -1)[..., :cols]
    return flat(code), byte[..., 0].to(torch.uint8), flat(value), flat(unit.expand_as(full))


ACTS = {
    "identity": (lambda x: x, lambda x: torch.ones_like(x) + 0 * x),
    "relu": (lambda x: torch.where(x > 0, x, 0 * x), lambda x: torch.where(x > 0, 1.0, 0 * x)),
    "tanh": (torch.tanh, lambda x: 1 / torch.cosh(x) ** 2),
    "sigmoid": (torch.sigmoid, lambda x: torch.sigmoid(x) * torch.sigmoid(-x)),
    "silu": (lambda x: x * torch.sigmoid(x), lambda x: torch.sigmoid(x) * (1 + x * torch.sigmoid(-x))),
    "gelu": (lambda x: x * 0.5 * torch.erfc(-x / math.sqrt(2)),
             lambda x: 0.5 * torch.erfc(-x / math.sqrt(2)) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)),
}


def act_bounds(act, x):
    """Bounds for the value and the slope in float32.  The sigmoid's exponential has its argument rounded: |x| U and |x| U
    for the constant's rounding, two units each for the exponential and the reciprocal, one addition; tanh and erf to within
    two units in the last place of a number of at most one (4 U); the density's argument is rounded three times."""
    a = x.abs()
    rel = (2 * a + 6) * U                                   # of sigmoid(x), sigmoid(-x)
    p, m = torch.sigmoid(x), torch.sigmoid(-x)
    if act in ("identity", "relu"):
        return 0 * a, 0 * a
    if act == "tanh":
        return 4 * U + 0 * a, 10 * U + 0 * a
    if act == "sigmoid":
        return rel * p, (2 * rel + U) * p * m
    if act == "silu":
        return (rel + U) * a * p, (rel + U) * p + (2 * rel + 3 * U) * a * p * m
    density = torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return a * 6 * U, 6 * U + a * density * (4 * x * x + 8) * U


def act_relative_bounds(act, x):
    """Bounds for tanh's slope and for gelu's value and slope that hold far from zero, where they are small themselves.
    tanh: 4 f (1 - f), f = sigmoid(2 x), each factor as in `act_bounds`.  gelu: the argument of erfc(z) / 2, z = -x / sqrt 2, may be
    rounded twice, z erfc'(z) / erfc(z) is at most 2 z^2 + 2 = x^2 + 2 in size, 16 units in the last place for erfc itself,
    and two products follow; the density as in `act_bounds`, its own two units among them."""
    a = x.abs()
    if act == "tanh":
        return None, ACTS[act][1](x) * (2 * (4 * a + 6) + 2) * U
    below = 0.5 * torch.erfc(-x / math.sqrt(2)) * (2 * x * x + 4 + 32 + 2) * U
    density = torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    slope = ACTS[act][1](x).abs()
    return a * below, below + a * density * (4 * x * x + 8) * U + slope * U


# float32 gates, relative, over all of float32's range: e = exp(-u) is off by its native unit (2 U) and a correction's rounding, 1 + e by U,
# its reciprocal by U and what one Newton step leaves; 1 - f = e f by another product
GATE = 8 * U


# ------------------------------------------------------------------ recurrence

def recurrence(u, v, w, h0, lengths, dtype):
    """h, last and their bounds.  The maps of a run of steps are composed before they are applied: every product and sum of
    the composition is counted at the step whose factor it rounds, with the magnitude M that the state would have if nothing cancelled."""
    u, v = u.double(), v.double()
    B, T, D = u.shape
    f, g = torch.sigmoid(u), torch.sigmoid(-u)
    i = g if w is None else torch.sigmoid(w.double())
    au, aw = u.abs(), u.abs() if w is None else w.double().abs()
    rf, ri = ((2 * au + 3) * g + 4) * U, (2 * aw + 8) * U
    h = torch.zeros(B, D, dtype=torch.float64, device=u.device) if h0 is None else h0.double()
    M, E = h.abs(), torch.zeros_like(h)
    n = torch.full((B, 1), T, device=u.device) if lengths is None else lengths.to(torch.int64).clamp(0, T)[:, None]
    hs, es = torch.zeros_like(u), torch.zeros_like(u)
    for t in range(T):
        on = n > t
        nM = f[:, t] * M + i[:, t] * v[:, t].abs()
        nE = f[:, t] * E + f[:, t] * M * (rf[:, t] + 4 * U) + i[:, t] * v[:, t].abs() * (ri[:, t] + 4 * U)
        nh = f[:, t] * h + i[:, t] * v[:, t]
        h, M, E = torch.where(on, nh, h), torch.where(on, nM, M), torch.where(on, nE, E)
        hs[:, t], es[:, t] = nh, nE
    valid = (torch.arange(T, device=u.device)[None, :] < n)[:, :, None].expand(B, T, D)
    return dict(h=hs, last=h, e_h=stored(2 * es, hs, dtype), e_last=2 * E + TINY[torch.float32], valid=valid)


def recurrence_grad(u, v, w, h, h0, dh, dlast, lengths, dtype):
    """du, dv, dw, dh0 and their bounds; h as it is stored."""
    u, v, dh, h = u.double(), v.double(), dh.double(), h.double()
    B, T, D = u.shape
    f, g = torch.sigmoid(u), torch.sigmoid(-u)
    i, j = (g, f) if w is None else (torch.sigmoid(w.double()), torch.sigmoid(-w.double()))
    au, aw = u.abs(), u.abs() if w is None else w.double().abs()
    rf, rg = ((2 * au + 3) * g + 4) * U, (2 * au + 8) * U
    ri, rj = (2 * aw + 8) * U, (2 * aw + 8) * U
    zero = torch.zeros(B, D, dtype=torch.float64, device=u.device)
    h0 = zero if h0 is None else h0.double()
    s = zero if dlast is None else dlast.double()
    M, E = s.abs(), torch.zeros_like(s)
    n = torch.full((B, 1), T, device=u.device) if lengths is None else lengths.to(torch.int64).clamp(0, T)[:, None]
    out = {k: torch.zeros_like(u) for k in ("du", "dv", "dw", "e_du", "e_dv", "e_dw")}
    for t in range(T - 1, -1, -1):
        on = n > t
        G, MG = dh[:, t] + s, dh[:, t].abs() + M
        EG = E + 4 * U * MG
        before = h[:, t - 1] if t else h0
        vt, ft, gt, it, jt = v[:, t], f[:, t], g[:, t], i[:, t], j[:, t]
        past = before - vt if w is None else before
        out["dv"][:, t], out["e_dv"][:, t] = G * it, 2 * EG * it + G.abs() * it * (ri[:, t] + 2 * U)
        out["du"][:, t] = G * past * ft * gt
        mag = before.abs() + vt.abs() if w is None else before.abs()
        out["e_du"][:, t] = 2 * EG * past.abs() * ft * gt + G.abs() * (past.abs() * (rf[:, t] + rg[:, t] + 4 * U) + U * mag) * ft * gt
        out["dw"][:, t] = G * vt * it * jt
        out["e_dw"][:, t] = 2 * EG * vt.abs() * it * jt + out["dw"][:, t].abs() * (ri[:, t] + rj[:, t] + 4 * U)
        s, M = torch.where(on, ft * G, s), torch.where(on, ft * MG, M)
        E = torch.where(on, ft * (EG + MG * (rf[:, t] + 3 * U)), E)
    out["dh0"], out["e_dh0"] = s, 2 * E + TINY[torch.float32]
    for k in ("du", "dv", "dw"):
        out["e_" + k] = stored(out["e_" + k], out[k], dtype)
    out["valid"] = (torch.arange(T, device=u.device)[None, :] < n)[:, :, None].expand(B, T, D)
    return out
