"""The operators over a vocabulary written out in 64 bits, with bounds for what float32 arithmetic and one rounding to the storage
type may add.  Plain torch on the CPU or the GPU; nothing of the library is used.

U is half a step of float32.  With t_j = scale (x_j - peak), a term exp(t_j) of a sum is formed about a point on the way to the peak that
is at most 2^8 (5.6 in natural units) off it or behind it, and moved there: the way is at most |t_j| + 12 long.  The difference, the product
and the rounded factor (itself a product) put 4 U of that into the exponent, each move (one for 5.5 units of the way, and two) three
more roundings; the native exponential is off by two.  Additions are CHAIN long.  A logarithm is off by two U of itself."""
import math

import torch

from tests.operators_ref import U, close, stored  # noqa: F401

INF = float("inf")
NOTHING = 2.0 ** -125                    # the native exponential is zero below 2^-126; the rest of its exponent is at most one power of two
MOST = 2.0 ** 128 - 2.0 ** 103          # the largest float32 and half a step


def chain(cols):
    """Additions that a row's sum passes through: a thread's own (one of 256, or of 64 up to 2048 logits), 6 across a
    wavefront, 16 wavefronts, 64 parts."""
    return 100 + cols // 256


def sound(out):
    """Bounds where there is a number to be near to: elsewhere results are what they are (an infinity, a NaN, the zeros of padding)."""
    for n in [n for n in out if n.startswith("e_")]:
        if n[2:] in out:
            # (results are float32: what that does not reach is an infinity)
            out[n[2:]] = torch.where(out[n[2:]].abs() > MOST, out[n[2:]].sign() * INF, out[n[2:]])
            out[n] = torch.where(torch.isfinite(out[n]) & torch.isfinite(out[n[2:]]), out[n], 0.0)
    return out


def softmax_stats(x, scale):
    """Of rows of logits in 64 bits: live rows (a finite logit, and nothing that is not), t, p, peak, logsum, entropy and the bounds of the last two,
    and the relative bound of a saved exponential."""
    x = x.double()
    cols = x.shape[-1]
    bad = (torch.isnan(x) | (x == INF)).any(-1)
    peak = torch.where(torch.isnan(x), -INF, x).amax(-1)
    none = (peak == -INF) & ~bad
    ref = torch.where(torch.isfinite(peak), peak, 0.0).unsqueeze(-1)
    t = (x - ref) * scale
    e = torch.exp(t)
    s = e.sum(-1)
    logsum = torch.log(s)
    p = torch.where(none.unsqueeze(-1), 0.0, e / s.unsqueeze(-1))
    at = t.abs().clamp_max(800.0)
    et = U * (4 * (at + 12) + 3 * (at / 5.5 + 2) + 4 + chain(cols))
    e_s = (p * et).sum(-1)
    e_logsum = e_s + U * (2 * logsum.abs() + 1)
    tt = torch.where(p > 0, t, 0.0)
    w = (p * tt).sum(-1)
    entropy = torch.where(none, 0.0, logsum - w)
    e_w = (p * (at + 12) * (et + 4 * U)).sum(-1)
    e_entropy = e_logsum + e_w + w.abs() * (e_s + 4 * U) + 2 * U * (entropy.abs() + logsum.abs())
    nan = math.nan
    return dict(bad=bad, none=none, peak=torch.where(bad, nan, peak), t=t, p=p, logsum=torch.where(bad, nan, logsum),
                entropy=torch.where(bad, nan, entropy), e_logsum=e_logsum, e_entropy=e_entropy)


def log_p(st, t):
    """log p of logits whose t is given, and its bound."""
    logsum = st["logsum"].unsqueeze(-1)
    value = torch.where(st["none"].unsqueeze(-1), -INF, t - logsum)
    return value, st["e_logsum"].unsqueeze(-1) + 3 * U * torch.where(torch.isfinite(t), t.abs(), 0.0) + U * torch.where(
        torch.isfinite(value), value.abs(), 0.0) + 2.0 ** -140


def top(x, k):
    """The places of the k largest logits of each row, by value, then by place; -1 where there is none."""
    x = x.double().reshape(-1, x.shape[-1])
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :k]
    there = x.gather(1, order) > -INF
    out = torch.full((x.shape[0], k), -1, dtype=torch.int64, device=x.device)
    out[:, :order.shape[1]] = torch.where(there, order, -1)
    return out


def token_logprobs(x, tokens, scale, k=0):
    """All results and their bounds (e_...), rows flattened."""
    cols = x.shape[-1]
    x = x.reshape(-1, cols)
    st = softmax_stats(x, scale)
    rows = x.shape[0]
    pad = torch.zeros(rows, dtype=torch.bool, device=x.device)
    out = {n: st[n] for n in ("peak", "logsum", "entropy", "e_logsum", "e_entropy")}
    out["e_peak"] = torch.zeros(rows, dtype=torch.float64, device=x.device)
    if tokens is not None:
        tokens = tokens.reshape(-1).long()
        pad = (tokens < 0) | (tokens >= cols)
        value, bound = log_p(st, st["t"].gather(1, torch.where(pad, 0, tokens).unsqueeze(1)))
        out["logprob"], out["e_logprob"] = torch.where(st["bad"], math.nan, value[:, 0]), bound[:, 0]
    for n in ("peak", "logsum", "entropy", "logprob"):
        if n in out:
            out[n] = torch.where(pad, 0.0, out[n])
    if k:
        index = top(x, k)
        gone = (index < 0) | pad.unsqueeze(1) | st["bad"].unsqueeze(1)
        value, bound = log_p(st, st["t"].gather(1, index.clamp_min(0)))
        value = torch.where(st["bad"].unsqueeze(1) & ~pad.unsqueeze(1), math.nan, torch.where(gone, -INF, value))
        out.update(top_indices=torch.where(gone, -1, index), top_values=value, e_top_values=bound)
    return sound(out)


def _exponent(x, peak, logsum, scale):
    """log p from saved statistics (as they were stored), and the relative bound of its exponential in float32."""
    none = (peak == -INF).unsqueeze(-1)
    peak, logsum = peak.double().unsqueeze(-1), logsum.double().unsqueeze(-1)
    t = (x.double() - torch.where(none, 0.0, peak)) * scale
    logp = torch.where(none, -INF, t - logsum)
    off = torch.where(none, 0.0, logsum)
    rel = U * (5 * t.abs().clamp_max(800.0) + 4 * off.abs() + 2 * logp.abs().clamp_max(800.0) + 4)
    return logp, rel


def token_logprobs_grad(x, tokens, dlogprob, dentropy, peak, logsum, entropy, scale, dtype):
    cols = x.shape[-1]
    x = x.reshape(-1, cols)
    flat = lambda v: None if v is None else v.reshape(-1).double()
    dlogprob, dentropy, peak, logsum, entropy = (flat(v) for v in (dlogprob, dentropy, peak, logsum, entropy))
    logp, rel = _exponent(x, peak, logsum, scale)
    p = torch.exp(logp)
    dx, bound = torch.zeros_like(p), torch.zeros_like(p)
    pad = (peak == -INF)
    if tokens is not None:
        tokens = tokens.reshape(-1).long()
        outside = (tokens < 0) | (tokens >= cols)
        pad = pad | outside
        hot = torch.zeros_like(p).scatter_(1, torch.where(outside, 0, tokens).unsqueeze(1), 1.0)
    if dlogprob is not None:
        g = dlogprob.unsqueeze(1)
        dx += g * (hot - p)
        bound += g.abs() * (p * (rel + 6 * U) + 4 * U * hot + NOTHING)
    if dentropy is not None:
        h, H = dentropy.unsqueeze(1), entropy.unsqueeze(1)
        lp = torch.where(p > 0, logp, 0.0)
        dx -= h * p * (lp + H)
        bound += h.abs() * (p * ((lp.abs() + H.abs()) * (rel + 8 * U) + rel) + NOTHING * (130 + H.abs()))
    dx, bound = dx * scale, bound * scale
    dx = torch.where(pad.unsqueeze(1), 0.0, dx)
    bound = torch.where(pad.unsqueeze(1), 0.0, bound + 2 * U * dx.abs())
    return dx, stored(bound, dx, dtype)


def teacher(values, indices, cols, tail, teacher_scale):
    """q, log q, truth of the entries that exist, q_t, and the bounds of q (relative), log q and q_t."""
    k = values.shape[-1]
    v = values.reshape(-1, k).double() * teacher_scale
    index = indices.reshape(-1, k).long()
    there = (index >= 0) & (index < cols)
    v = torch.where(there, v, -INF)
    a = torch.where(torch.isfinite(v), v.abs(), 0.0)
    if tail:
        q, logq = torch.exp(v), v
        e_q, e_logq = U * (2 * a + 4), U * (a + 1)
        rest = (1 - q.sum(1)).clamp_min(0)
        e_rest = (q * (e_q + 16 * U)).sum(1) + 2 * U
        return q, logq, there, rest, e_q, e_logq, e_rest
    some = torch.isfinite(v).any(1, keepdim=True)
    m = torch.where(some, v.amax(1, keepdim=True), 0.0)
    # (a value that is not finite makes the row NaN)
    m = torch.where(torch.isfinite(m), m, 0.0)
    e = torch.exp(v - m)
    s = torch.where(some, e.sum(1, keepdim=True), 1.0)
    q, logq = e / s, v - m - torch.log(s)
    e_q = U * (4 * a + 2 * m.abs() + 24 + 2 * logq.abs().clamp_max(800.0))
    return q, logq, there, None, e_q, e_q, None


def outside(indices, there, cols):
    """Truth of the logits that no entry names."""
    rows = there.shape[0]
    rest = torch.ones((rows, cols + 1), dtype=torch.bool, device=there.device)
    rest.scatter_(1, torch.where(there, indices.reshape(rows, -1).long(), cols), False)
    return rest[:, :cols]


def distill(x, values, indices, scale, teacher_scale, tail):
    cols = x.shape[-1]
    x = x.reshape(-1, cols).double()
    q, logq, there, rest_q, e_q, e_logq, e_rest = teacher(values, indices, cols, tail, teacher_scale)
    index = indices.reshape(there.shape).long()
    st = softmax_stats(x, scale)
    logp, e_logp = log_p(st, st["t"].gather(1, torch.where(there, index, 0)))
    term = torch.where(q > 0, q * (logq - logp), 0.0)
    fine = torch.where(torch.isfinite(logq - logp), logq - logp, 0.0).abs()
    loss = term.sum(1)
    e_loss = (q * (fine * (e_q + 14 * U) + e_logq + e_logp)).sum(1)
    out = {n: st[n] for n in ("peak", "logsum", "e_logsum")}
    out["e_peak"] = torch.zeros_like(loss)
    if tail:
        free = outside(indices, there, cols)
        sub = softmax_stats(torch.where(free, x, -INF), scale)
        far = torch.where(sub["none"] | st["none"], 0.0, sub["peak"] - st["peak"]) * scale
        out["tail"] = torch.where(sub["none"], -INF, far + sub["logsum"])
        out["e_tail"] = sub["e_logsum"] + 3 * U * far.abs() + U * torch.where(sub["none"], 0.0, out["tail"]).abs()
        # (the sum over the entries and the tail's, joined: the whole row's bound holds for that too)
        logpt = torch.where(sub["none"] | st["none"], -INF, out["tail"] - st["logsum"])
        counts = logpt >= -126 * math.log(2)
        lq = torch.log(torch.maximum(rest_q, e_rest))
        use = torch.where(counts, rest_q, 0.0)
        loss = loss + torch.where(use > 0, use * (torch.log(use) - logpt), 0.0)
        span = torch.where(counts, (lq - logpt).abs() + 1, 0.0)
        e_loss = e_loss + span * e_rest + torch.where(use > 0, use * (out["e_tail"] + st["e_logsum"] + 6 * U * span), 0.0)
        out["counts"] = counts
    live = there.any(1)
    zero = lambda v: torch.where(live, v, 0.0)
    out["loss"], out["e_loss"] = torch.where(st["bad"], math.nan, loss), e_loss + 4 * U * torch.where(torch.isfinite(loss), loss.abs(), 0.0)
    for n in ("loss", "peak", "logsum", "tail"):
        if n in out:
            out[n] = zero(torch.where(st["bad"], math.nan, out[n]) if n == "tail" else out[n])
    return sound(out)


def distill_grad(x, values, indices, peak, logsum, tail, dloss, scale, teacher_scale, dtype):
    """From the statistics as they were stored."""
    cols = x.shape[-1]
    x = x.reshape(-1, cols)
    rows = x.shape[0]
    peak, logsum = peak.reshape(-1).double(), logsum.reshape(-1).double()
    q, logq, there, rest_q, e_q, e_logq, e_rest = teacher(values, indices, cols, tail is not None, teacher_scale)
    index = torch.where(there, indices.reshape(there.shape).long(), cols)
    logp, rel = _exponent(x, peak, logsum, scale)
    p = torch.exp(logp)
    scatter = lambda v: torch.zeros((rows, cols + 1), dtype=torch.float64, device=x.device).scatter_add_(1, index, torch.where(there, v, 0.0))[:, :cols]
    hit, e_hit = scatter(q), scatter(q * (e_q + 8 * U))
    w = torch.ones(rows, dtype=torch.float64, device=x.device) if dloss is None else dloss.reshape(-1).double()
    w = (w * scale).unsqueeze(1)
    mass = (q.sum(1) if tail is not None else (q > 0).any(1).double()).unsqueeze(1)
    e_mass = (q * (e_q + 16 * U)).sum(1, keepdim=True) if tail is not None else 0.0
    if tail is None:
        dx = mass * p - hit
        bound = p * mass * (rel + 6 * U) + e_hit + NOTHING
    else:
        tail = tail.reshape(-1).double()
        logpt = torch.where((tail == -INF) | (peak == -INF), -INF, tail - logsum)
        counts = (logpt >= -126 * math.log(2)).unsqueeze(1)
        free = outside(indices, there, cols)
        rest = torch.where(counts, rest_q.unsqueeze(1), 0.0)
        e_r = torch.where(counts, e_rest.unsqueeze(1), 0.0)
        mass = mass + rest
        part = torch.where(counts & free, torch.exp(logp - torch.where(counts[:, 0], logpt, 0.0).unsqueeze(1)), 0.0)        # p / p_t
        pt = torch.where(counts, torch.exp(logpt).unsqueeze(1), 0.0)
        dx = mass * p - torch.where(free, rest * part, hit)
        rel_t = rel + 4 * U * (tail.abs().clamp_max(800.0) + logsum.abs().clamp_max(800.0)).nan_to_num(800.0, 800.0, 800.0).unsqueeze(1)
        # behind the entries: p / p_t (m p_t - q_t)
        inner = (mass * pt - rest).abs() * rel_t + mass * pt * (rel_t + 6 * U) + pt * (e_mass + e_r) + e_r + 2 * U * rest
        bound = torch.where(free & counts, part * inner + 6 * U * part * (mass * pt + rest), p * (mass * (rel + 6 * U) + e_mass + e_r) + e_hit) + NOTHING
    live = there.any(1, keepdim=True)
    dx = torch.where(live, dx * w, 0.0)
    bound = torch.where(live, bound * w.abs(), 0.0) + 4 * U * dx.abs()
    return dx, stored(bound, dx, dtype)
