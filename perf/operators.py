"""The operators of language models that this library offers beside its expressions, at the sizes they meet.

Families and their declared ranges (`draw` spreads over all of each, odd sizes among them):

  norm        layer normalisation forward with its statistics, 1..65536 rows of 16..16384
  norm_grad   its backward pass with the gradients of scale and shift
  norm_step   both, the normalised rows kept in 8 bits in between (16-bit types)
  act_step    an activation and its backward pass, its argument kept in 8 bits in between
  keep        a tensor written in 8 bits and read back, 1..65536 rows of 1..16384
  rec         the gated linear recurrence over 1..65536 steps of 1..64 sequences of 1..4096 channels,
              whole or ragged, with the input gate tied to the forget gate or of its own
  rec_grad    its backward pass

The formulas, for a row x of `cols` elements:  m = mean(x), r = 1/sqrt(mean((x - m)^2) + eps), n = (x - m) r,
y = n w + b; with g = dy w:  dx = r (g - mean(g) - n mean(g n)), dw = sum over rows of dy n, db = sum of dy.
8 bits: blocks of 32 along a row share a power of two, the smallest 2^k, k >= -126, with max|x| 2^-k <= 127
(int8) or 448 (e4m3); an element stands for 2^k times its code, x 2^-k rounded to nearest, ties to even.
Recurrence over t, channel by channel:  f = sigmoid(u), i = sigmoid(w) or 1 - f,  h_t = f_t h_(t-1) + i_t v_t.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


def listed():
    return [
        # serving, one token of each of eight sequences: latency
        {"name": "norm_8x4096_bf16", "op": "norm", "dtype": "bf16", "params": "bf16", "rows": 8, "cols": 4096},
        # a training step's activations: mixed precision, float32 scale and shift
        {"name": "norm_16384x4096_bf16", "op": "norm", "dtype": "bf16", "params": "f32", "rows": 16384, "cols": 4096},
        # ... and their backward pass
        {"name": "norm_grad_16384x4096_bf16", "op": "norm_grad", "dtype": "bf16", "params": "f32", "rows": 16384, "cols": 4096},
        # rows of odd length, of which no two begin on the same alignment
        {"name": "norm_grad_4099x1001_f16", "op": "norm_grad", "dtype": "f16", "params": "f16", "rows": 4099, "cols": 1001},
        # a step that keeps a byte instead of two for each activation
        {"name": "norm_step_8192x2048_bf16_i8", "op": "norm_step", "dtype": "bf16", "params": "bf16", "codes": "i8", "rows": 8192, "cols": 2048},
        # the widest activations of a step, kept in a byte each
        {"name": "act_silu_8192x8192_bf16_i8", "op": "act_step", "dtype": "bf16", "codes": "i8", "act": "silu", "rows": 8192, "cols": 8192},
        # rows that end inside a block of 32
        {"name": "keep_5001x1003_bf16_e4m3", "op": "keep", "dtype": "bf16", "codes": "e4m3", "rows": 5001, "cols": 1003},
        # serving, one token of each of 64 sequences: latency
        {"name": "rec_64x1x2048_bf16", "op": "rec", "dtype": "bf16", "batch": 64, "steps": 1, "channels": 2048, "tied": True, "ragged": False},
        # a training step
        {"name": "rec_8x4096x2048_bf16", "op": "rec", "dtype": "bf16", "batch": 8, "steps": 4096, "channels": 2048, "tied": True, "ragged": False},
        # ... and its backward pass
        {"name": "rec_grad_8x4096x2048_bf16", "op": "rec_grad", "dtype": "bf16", "batch": 8, "steps": 4096, "channels": 2048, "tied": True,
         "ragged": False},
        # one long document: few channels, many steps
        {"name": "rec_1x65536x1024_f32", "op": "rec", "dtype": "f32", "batch": 1, "steps": 65536, "channels": 1024, "tied": True, "ragged": False},
        # a padded batch of odd sizes, an input gate of its own
        {"name": "rec_grad_5x1237x1000_f16_ragged", "op": "rec_grad", "dtype": "f16", "batch": 5, "steps": 1237, "channels": 1000, "tied": False,
         "ragged": True},
    ]


MOST = 1 << 25      # elements of a drawn case


def draw(rng):
    def size(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))

    op = rng.choice(["norm", "norm_grad", "norm_step", "act_step", "keep", "rec", "rec_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("rec", "rec_grad"):
        channels, batch = size(1, 4096), size(1, 64)
        steps = size(1, max(1, min(65536, MOST // (channels * batch))))
        return {"op": op, "dtype": dtype, "batch": batch, "steps": steps, "channels": channels, "tied": rng.random() < 0.6,
                "ragged": rng.random() < 0.4}
    # (rows of two elements have no gradient but rounding: a normalised pair is always 1 and -1)
    cols = size(16 if op.startswith("norm") else 1, 16384)
    case = {"op": op, "dtype": dtype, "rows": size(1, min(65536, MOST // cols)), "cols": cols}
    if op == "norm_step" and dtype == "f32":
        case["dtype"] = "bf16"
    if op.startswith("norm"):
        case["params"] = case["dtype"] if op == "norm_step" else rng.choice([dtype, "f32"])
    if op in ("norm_step", "act_step", "keep"):
        case["codes"] = rng.choice(["i8", "e4m3"])
    if op == "act_step":
        case["act"] = rng.choice(["relu", "tanh", "sigmoid", "silu", "gelu"])
    return case


def work(case):
    size = _SIZE[case["dtype"]]
    if "steps" in case:
        # (a ragged batch: lengths are spread evenly, `_lengths` below)
        n = case["batch"] * case["steps"] * case["channels"] * (0.5 if case["ragged"] else 1.0)
        state = 4 * case["batch"] * case["channels"]
        gates = 1 if case["tied"] else 2
        if case["op"] == "rec":
            return {"bytes": (gates + 2) * n * size + 2 * state, "flops": (8 if case["tied"] else 12) * n}
        return {"bytes": (2 * gates + 4) * n * size + 3 * state, "flops": (16 if case["tied"] else 22) * n}
    n = case["rows"] * case["cols"]
    params = case["cols"] * _SIZE[case.get("params", "f32")]
    kept = n + case["rows"] * ((case["cols"] + 31) // 32)
    stats = 4 * case["rows"]
    return {
        "norm": {"bytes": 2 * n * size + 2 * params + 2 * stats, "flops": 8 * n},
        "norm_grad": {"bytes": 3 * n * size + 3 * params + 2 * stats, "flops": 14 * n},
        # forward: x, y, 8 bits; backward: dy, 8 bits, dx
        "norm_step": {"bytes": 4 * n * size + 2 * kept + 5 * params + 3 * stats, "flops": 26 * n},
        "act_step": {"bytes": 4 * n * size + 2 * kept, "flops": 24 * n},
        "keep": {"bytes": 2 * n * size + 2 * kept, "flops": 6 * n},
    }[case["op"]]


# ---------------------------------------------------------------------------------- inputs

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _inputs(case, seed):
    """The tensors of a case, made from the seed alone."""
    dev, dt = _device(), _TORCH[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, mean=0.0, std=1.0, dtype=dt):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).mul_(std).add_(mean).to(dtype)

    s = {"case": case}
    if "steps" in case:
        b, t, c = case["batch"], case["steps"], case["channels"]
        # forget gates of a trained model: most near one, so that states carry far
        s["u"] = normal(b, t, c, mean=2.0, std=1.5)
        s["v"] = normal(b, t, c)
        s["w"] = None if case["tied"] else normal(b, t, c)
        s["h0"] = normal(b, c, dtype=torch.float32)
        s["lengths"] = _lengths(case, g, dev) if case["ragged"] else None
        if case["op"] == "rec_grad":
            s["dh"] = normal(b, t, c)
            s["dlast"] = normal(b, c, dtype=torch.float32)
        return s
    rows, cols = case["rows"], case["cols"]
    if case["op"].startswith("norm"):
        pt = _TORCH[case["params"]]
        # activations away from zero, as behind a residual sum
        s["x"] = normal(rows, cols, mean=0.3, std=1.7)
        s["weight"] = normal(cols, mean=1.0, std=0.2, dtype=pt)
        s["bias"] = normal(cols, std=0.2, dtype=pt)
    else:
        s["x"] = normal(rows, cols, std=1.5)
    if case["op"] in ("norm_grad", "norm_step", "act_step"):
        s["dy"] = normal(rows, cols)
    return s


def _lengths(case, g, dev):
    """Sequence lengths spread evenly from 0 to all steps, in an order of the seed's own."""
    b = case["batch"]
    even = torch.arange(b, device=dev, dtype=torch.float64).add_(0.5).mul_(case["steps"] / b).round_().to(torch.int32)
    return even[torch.randperm(b, generator=g, device=dev)].contiguous()


def prepare(case, seed):
    s = _inputs(case, seed)
    dev = s["x"].device if "x" in s else s["u"].device
    # what a program keeps in hand besides: saved values of the forward pass, results' memory
    if "steps" in case:
        b, c = case["batch"], case["channels"]
        if case["op"] == "rec_grad":
            s["h"] = _rec(s)["h"]
            s.update(du=torch.zeros_like(s["u"]), dv=torch.zeros_like(s["u"]), dw=None if case["tied"] else torch.zeros_like(s["u"]),
                     dh0=torch.empty_like(s["h0"]))
        else:
            s.update(h=torch.zeros_like(s["u"]), last=torch.empty_like(s["h0"]))
        return s
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "norm_grad":
        s["mean"], s["rstd"] = _stats(s["x"].float())
    elif case["op"].startswith("norm"):
        s["mean"], s["rstd"] = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
    if "codes" in case:
        s["codes"] = torch.empty((rows, cols), device=dev, dtype=torch.int8 if case["codes"] == "i8" else torch.float8_e4m3fn)
        s["scales"] = torch.empty((rows, (cols + 31) // 32), device=dev, dtype=torch.uint8)
    s["out"] = torch.empty_like(s["x"])
    if case["op"] in ("norm_grad", "norm_step"):
        s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
    if "dy" in s:
        s["dx"] = torch.empty_like(s["x"])
    return s


# ---------------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if own:
        return _run_own(s)
    if "steps" in case:
        return _rec_grad(s) if case["op"] == "rec_grad" else _rec(s)
    dt = s["x"].dtype
    if case["op"] == "norm":
        y, mean, rstd, _ = _norm(s)
        return {"y": y, "mean": mean, "rstd": rstd}
    if case["op"] == "norm_grad":
        n = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        return _norm_grad(s, n, s["rstd"])
    if case["op"] == "norm_step":
        y, _, rstd, n = _norm(s)
        kept, power = _pack(n, case["codes"])
        return {"y": y, **_norm_grad(s, _unpack(kept, power, n.shape), rstd)}
    x = s["x"].float()
    kept, power = _pack(x, case["codes"])
    x8 = _unpack(kept, power, x.shape)
    if case["op"] == "keep":
        return {"x": x8.to(dt)}
    return {"y": _act(case["act"], x).to(dt), "dx": (s["dy"].float() * _slope(case["act"], x8)).to(dt)}


def _stats(x):
    mean = x.sum(1) / x.shape[1]
    centred = x - mean[:, None]
    return mean, 1.0 / torch.sqrt((centred * centred).sum(1) / x.shape[1] + EPS)


def _norm(s):
    x = s["x"].float()
    mean, rstd = _stats(x)
    n = (x - mean[:, None]) * rstd[:, None]
    return (n * s["weight"].float() + s["bias"].float()).to(s["x"].dtype), mean, rstd, n


def _norm_grad(s, n, rstd):
    dy, w = s["dy"].float(), s["weight"]
    g = dy * w.float()
    cols = g.shape[1]
    dx = (g - g.sum(1, keepdim=True) / cols - n * ((g * n).sum(1, keepdim=True) / cols)) * rstd[:, None]
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * n).sum(0).to(w.dtype), "dbias": dy.sum(0).to(w.dtype)}


def _pack(x, codes):
    """Codes (as float32 whole numbers or e4m3 values) and the powers of two of blocks of 32 along a row."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    padded = torch.zeros((rows, blocks * 32), dtype=x.dtype, device=x.device)
    padded[:, :cols] = x
    padded = padded.view(rows, blocks, 32)
    part, power = torch.frexp(padded.abs().amax(2))      # the largest magnitude is part * 2^power, part in [1/2, 1)
    if codes == "i8":
        power = torch.where(part > 127 / 128, power - 6, power - 7)
    else:
        power = torch.where(part > 448 / 512, power - 8, power - 9)
    power = power.clamp_min(-126)[:, :, None]
    scaled = padded * _pow2(-power)
    if codes == "i8":
        return scaled.round().to(torch.int8), power
    return scaled.to(torch.float8_e4m3fn), power


def _unpack(kept, power, shape):
    rows, cols = shape
    return (kept.float() * _pow2(power)).view(rows, -1)[:, :cols]


def _pow2(k):
    """2^k from its bits (torch's ldexp multiplies by exp2(k), which is not a power of two to the bit everywhere)."""
    return ((k + 127) << 23).to(torch.int32).view(torch.float32)


def _act(act, x):
    if act == "relu":
        return x.clamp_min(0)
    if act == "tanh":
        return torch.tanh(x)
    if act == "sigmoid":
        return torch.sigmoid(x)
    if act == "silu":
        return x * torch.sigmoid(x)
    return x * (0.5 * (1 + torch.erf(x * math.sqrt(0.5))))


def _slope(act, x):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "tanh":
        t = torch.tanh(x)
        return 1 - t * t
    p = torch.sigmoid(x)
    if act == "sigmoid":
        return p * (1 - p)
    if act == "silu":
        return p * (1 + x * (1 - p))
    return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))


def _scan(a, b):
    """h_t = a_t h_(t-1) + b_t along dimension 1, by doubling: after the k-th step an element holds the
    composition of the 2^k steps up to it."""
    k = 1
    while k < a.shape[1]:
        b = torch.cat((b[:, :k], torch.addcmul(b[:, k:], a[:, k:], b[:, :-k])), 1)
        a = torch.cat((a[:, :k], a[:, k:] * a[:, :-k]), 1)
        k *= 2
    return b


def _gates(s):
    u = s["u"].float()
    return torch.sigmoid(u), torch.sigmoid(-u) if s["w"] is None else torch.sigmoid(s["w"].float())


def _valid(s):
    """[batch, steps, 1]: the steps before the sequence's length (None: all of them)."""
    if s["lengths"] is None:
        return None
    return torch.arange(s["u"].shape[1], device=s["u"].device)[None, :, None] < s["lengths"][:, None, None]


def _rec(s):
    f, i = _gates(s)
    b = i * s["v"].float()
    ok = _valid(s)
    if ok is not None:      # steps behind the length leave the state as it is
        f, b = torch.where(ok, f, 1.0), torch.where(ok, b, 0.0)
    b[:, 0] += f[:, 0] * s["h0"]
    h = _scan(f, b)
    last = h[:, -1].contiguous()
    if ok is not None:
        h = torch.where(ok, h, 0.0)
    return {"h": h.to(s["u"].dtype), "last": last}


def _rec_grad(s):
    f, i = _gates(s)
    dh, v, dt = s["dh"].float(), s["v"].float(), s["u"].dtype
    ok = _valid(s)
    carry = f
    if ok is not None:
        carry, dh = torch.where(ok, f, 1.0), torch.where(ok, dh, 0.0)
    # backwards in time: g_t = dh_t + f_(t+1) g_(t+1), from the gradient of the last state
    a = torch.cat((torch.ones_like(carry[:, :1]), carry[:, 1:].flip(1)), 1)
    b = dh.flip(1)
    b[:, 0] += s["dlast"]
    g = _scan(a, b).flip(1)
    before = torch.cat((s["h0"][:, None], s["h"][:, :-1].float()), 1)
    slope = torch.sigmoid(s["u"].float()) * torch.sigmoid(-s["u"].float())
    out = {"dh0": carry[:, 0] * g[:, 0]}
    if s["w"] is None:
        out["du"] = g * slope * (before - v)
    else:
        out["du"] = g * slope * before
        out["dw"] = g * v * i * torch.sigmoid(-s["w"].float())
    out["dv"] = g * i
    for k in ("du", "dv", "dw"):
        if k in out:
            out[k] = (out[k] if ok is None else torch.where(ok, out[k], 0.0)).to(dt)
    return out


def _run_own(s):
    """The same passes through the library, on the caller's stream.  Calls are bound to their tensors
    once, as a program does that calls them many times."""
    from paper_1605_02688_amd import ewf
    case = s["case"]
    if "calls" not in s:
        s["calls"] = _bind(ewf, s)
    stream = torch.cuda.current_stream().cuda_stream
    for call in s["calls"]:
        call.launch(stream)
    if case["op"] == "rec":
        return {"h": s["h"], "last": s["last"]}
    if case["op"] == "rec_grad":
        out = {"dh0": s["dh0"], "du": s["du"], "dv": s["dv"]}
        return out if case["tied"] else {**out, "dw": s["dw"]}
    if case["op"] == "norm":
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
    if case["op"] == "norm_grad":
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if case["op"] == "norm_step":
        return {"y": s["out"], "dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if case["op"] == "keep":
        return {"x": s["out"]}
    return {"y": s["out"], "dx": s["dx"]}


def _bind(ewf, s):
    case = s["case"]
    kept = dict(codes=s["codes"], scales=s["scales"]) if "codes" in case else {}

    def bound(fn, *args, **kw):
        nbytes = fn.workspace_bytes(*args, **kw)
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
        return fn.bind(*args, workspace=work, **kw)

    if case["op"] == "rec":
        return [bound(ewf.recurrence, s["u"], s["v"], s["h"], w=s["w"], h0=s["h0"], last=s["last"], lengths=s["lengths"])]
    if case["op"] == "rec_grad":
        return [bound(ewf.recurrence_grad, s["u"], s["v"], s["h"], s["dh"], s["du"], s["dv"], w=s["w"], dw=s["dw"], h0=s["h0"],
                      dh0=s["dh0"], dlast=s["dlast"], lengths=s["lengths"])]
    if case["op"] == "keep":
        return [bound(ewf.keep8, s["x"], s["codes"], s["scales"]), bound(ewf.read8, s["codes"], s["scales"], s["out"])]
    if case["op"] == "act_step":
        return [bound(ewf.activation, case["act"], s["x"], s["out"], **kept),
                bound(ewf.activation_grad, case["act"], s["dy"], s["dx"], **kept)]
    forward = bound(ewf.layer_norm, s["x"], s["weight"], s["bias"], s["out"], mean=s["mean"], rstd=s["rstd"], eps=EPS, **kept) \
        if case["op"] != "norm_grad" else None
    if case["op"] == "norm":
        return [forward]
    source = kept or dict(x=s["x"], mean=s["mean"])
    backward = bound(ewf.layer_norm_grad, s["dy"], s["weight"], s["rstd"], s["dx"], dweight=s["dweight"], dbias=s["dbias"], **source)
    return [backward] if case["op"] == "norm_grad" else [forward, backward]


# ---------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    if "steps" in case:
        return _exact_rec(case, s)
    x = s["x"].double()
    if not case["op"].startswith("norm"):
        x8 = _exact_kept(x, case["codes"])
        if case["op"] == "keep":
            return {"x": x8}
        y, _ = _exact_act(case["act"], x)
        return {"y": y, "dx": s["dy"].double() * _exact_act(case["act"], x8)[1]}
    w, b = s["weight"].double(), s["bias"].double()
    var, mean = torch.var_mean(x, 1, correction=0)
    dev = torch.sqrt(var + EPS)
    n = (x - mean.unsqueeze(1)) / dev.unsqueeze(1)
    y = torch.addcmul(b, n, w)
    if case["op"] == "norm":
        return {"y": y, "mean": mean, "rstd": 1 / dev}
    if case["op"] == "norm_step":
        n = _exact_kept(n, case["codes"])
    dy = s["dy"].double()
    g = dy * w
    along = torch.mean(g * n, 1, keepdim=True)
    out = {"dx": (g - torch.mean(g, 1, keepdim=True) - along * n) / dev.unsqueeze(1), "dweight": torch.sum(dy * n, 0), "dbias": torch.sum(dy, 0)}
    return out if case["op"] == "norm_grad" else {"y": y, **out}


def _exact_kept(x, codes):
    """The values that 8 bits stand for: the grid's spacing at each element, from the block's power of two."""
    rows, cols = x.shape
    full = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, 32)
    top = full.abs().max(2, keepdim=True).values
    most = 127.0 if codes == "i8" else 448.0
    def pow2(k):            # from its bits: the GPU's 64-bit exp2 is off by a unit in the last place at some whole numbers
        return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)

    unit = pow2(torch.frexp((top / most).clamp_min(2.0 ** -140))[1] - 2)
    for _ in range(3):
        unit = torch.where(top > most * unit, 2 * unit, unit)
    unit = unit.clamp_min(2.0 ** -126)
    q = full / unit
    if codes == "e4m3":     # three bits behind the leading one, and a smallest spacing of 2^-9
        grid = pow2(torch.frexp(q.abs().clamp_min(2.0 ** -6))[1] - 4)
        q = torch.round(q / grid) * grid
    else:
        q = torch.round(q)
    return (q * unit).reshape(rows, -1)[:, :cols]


def _exact_act(act, x):
    """An activation and its derivative."""
    if act == "relu":
        return torch.where(x > 0, x, 0.0), torch.where(x > 0, 1.0, 0.0).to(x.dtype)
    if act == "tanh":
        return torch.tanh(x), 1 / torch.cosh(x) ** 2
    p = 1 / (1 + torch.exp(-x))
    if act == "sigmoid":
        return p, p / (1 + torch.exp(x))
    if act == "silu":
        return x * p, p + x * p / (1 + torch.exp(x))
    cdf = 0.5 * torch.erfc(-x / math.sqrt(2))
    return x * cdf, cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def _exact_rec(case, s):
    """Step by step, as the recurrence is written."""
    steps = case["steps"]
    u, v = s["u"].double(), s["v"].double()
    f = 1 / (1 + torch.exp(-u))
    i = 1 - f if case["tied"] else 1 / (1 + torch.exp(-s["w"].double()))
    live = torch.full((case["batch"], 1), steps, device=u.device) if s["lengths"] is None else s["lengths"][:, None]
    h = s["h0"].double()
    states = torch.zeros_like(u)
    inputs = i * v
    for t in range(steps):
        h = torch.where(live > t, torch.addcmul(inputs[:, t], f[:, t], h), h)
        states[:, t] = torch.where(live > t, h, 0.0)
    if case["op"] == "rec":
        return {"h": states, "last": h}
    # the backward pass reads the states as the forward pass stored them
    states = states.to(s["u"].dtype).double()
    g = s["dlast"].double()
    dh = s["dh"].double()
    du, dv, dw = torch.zeros_like(u), torch.zeros_like(u), torch.zeros_like(u)
    for t in range(steps - 1, -1, -1):
        on = live > t
        total = g + dh[:, t]
        before = states[:, t - 1] if t else s["h0"].double()
        past = before - v[:, t] if case["tied"] else before
        du[:, t] = torch.where(on, total * past * f[:, t] * (1 - f[:, t]), 0.0)
        dv[:, t] = torch.where(on, total * i[:, t], 0.0)
        if not case["tied"]:
            dw[:, t] = torch.where(on, total * v[:, t] * i[:, t] * (1 - i[:, t]), 0.0)
        g = torch.where(on, total * f[:, t], g)
    out = {"dh0": g, "du": du, "dv": dv}
    return out if case["tied"] else {**out, "dw": dw}
