"""The operators over a vocabulary that this library offers beside its expressions, at the sizes they meet.

Families and their declared ranges (`draw` spreads over all of each, odd sizes among them):

  logp          log probabilities of given tokens, with entropy and 0..128 top alternatives,
                1..16384 rows of 256..262144 logits, all rows given or a quarter of them padding
  logp_grad     the gradient of log probabilities and entropies
  distill       the loss against a teacher's 1..128 top logits
  distill_step  the loss and its gradient in one call
  distill_grad  the gradient from what the loss's call has saved

The formulas, for a row x of logits and a scale c (one over the temperature):
  peak = max x,  e_j = exp(c (x_j - peak)),  logsum = log sum e,  log p_j = c (x_j - peak) - logsum,
  entropy = - sum p_j log p_j;  alternatives: the largest log p_j, ties to the lowest index.
  With g and h the gradients of log p_token and of the entropy:
  dx_j = c (g ([j = token] - p_j) - h p_j (log p_j + entropy)).
A row whose token lies outside the vocabulary is padding: results 0, no alternatives, gradient 0.
Alternatives that do not exist (logits of minus infinity, fewer logits than asked for) are -infinity at index -1.

Distillation from entries (i_k, v_k), k < K; entries with an index outside the vocabulary do not exist:
  q = softmax(c' v),  loss = sum_k q_k (log q_k - log p_(i_k)),  dx_j = c w (p_j - sum of the q_k with i_k = j);
with a tail, v are log probabilities, q_k = exp(c' v_k), and the rest of the vocabulary is one class more:
  q_t = max(0, 1 - sum q),  p_t = sum of p over the rest,  loss = ... + q_t (log q_t - log p_t),
  dx_j = c w (m p_j - q_t p_j / p_t),  m = q_t + sum q, in the rest; c w (m p_j - q_k) at the entries;
a tail with p_t < 2^-126 does not count (q_t = 0).  A row without entries is padding.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
INF = float("inf")


def listed():
    return [
        # serving, the next token of eight sequences with twenty alternatives each: latency
        {"name": "logp_8x50257_bf16_top20", "op": "logp", "dtype": "bf16", "rows": 8, "vocab": 50257, "top": 20, "scale": 1.0, "ragged": False,
         "masked": False},
        # ... of one sequence over a long vocabulary, tempered, a part of the vocabulary forbidden
        {"name": "logp_1x131072_f32_top5", "op": "logp", "dtype": "f32", "rows": 1, "vocab": 131072, "top": 5, "scale": 1.25, "ragged": False,
         "masked": True},
        # scoring the tokens of a batch of the language model's vocabulary of ten thousand words
        {"name": "logp_1280x10000_f32", "op": "logp", "dtype": "f32", "rows": 1280, "vocab": 10000, "top": 0, "scale": 1.0, "ragged": False,
         "masked": False},
        # scoring a sub-word vocabulary: rows of odd length
        {"name": "logp_4096x50257_bf16", "op": "logp", "dtype": "bf16", "rows": 4096, "vocab": 50257, "top": 0, "scale": 1.0, "ragged": False,
         "masked": False},
        # a teacher's pass over a batch: what distillation reads
        {"name": "logp_2048x131072_bf16_top64", "op": "logp", "dtype": "bf16", "rows": 2048, "vocab": 131072, "top": 64, "scale": 1.0, "ragged": False,
         "masked": False},
        # training on log probabilities with an entropy term
        {"name": "logp_grad_4096x50257_bf16", "op": "logp_grad", "dtype": "bf16", "rows": 4096, "vocab": 50257, "scale": 1.0, "entropy": True,
         "ragged": False, "masked": False},
        # ... a padded batch of odd sizes without one, tempered
        {"name": "logp_grad_1001x33279_f16_ragged", "op": "logp_grad", "dtype": "f16", "rows": 1001, "vocab": 33279, "scale": 0.7, "entropy": False,
         "ragged": True, "masked": False},
        # a few tokens' training step: latency
        {"name": "distill_step_64x10000_bf16_k8", "op": "distill_step", "dtype": "bf16", "rows": 64, "vocab": 10000, "top": 8, "scale": 1.0,
         "tail": False, "ragged": False, "masked": False},
        # a batch's training step on the long vocabulary, the teacher's remainder as one class
        {"name": "distill_step_2048x131072_bf16_k64_tail", "op": "distill_step", "dtype": "bf16", "rows": 2048, "vocab": 131072, "top": 64,
         "scale": 1.0, "tail": True, "ragged": False, "masked": False},
        # ... in float32 over rows of odd length, tempered
        {"name": "distill_step_1280x50257_f32_k20", "op": "distill_step", "dtype": "f32", "rows": 1280, "vocab": 50257, "top": 20, "scale": 0.5,
         "tail": False, "ragged": False, "masked": False},
        # the loss alone, as for a held-out batch: odd sizes, padding, fewer entries in some rows
        {"name": "distill_777x10007_f16_k7_ragged", "op": "distill", "dtype": "f16", "rows": 777, "vocab": 10007, "top": 7, "scale": 1.0,
         "tail": True, "ragged": True, "masked": False},
        # the gradient alone, weights known after the loss
        {"name": "distill_grad_4096x32768_bf16_k32", "op": "distill_grad", "dtype": "bf16", "rows": 4096, "vocab": 32768, "top": 32, "scale": 1.0,
         "tail": True, "ragged": False, "masked": True},
    ]


MOST = 1 << 26      # logits of a drawn case


def draw(rng):
    def size(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))

    op = rng.choice(["logp", "logp", "logp_grad", "distill", "distill_step", "distill_grad"])
    vocab = size(256, 262144)
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "rows": size(1, min(16384, MOST // vocab)), "vocab": vocab,
            "scale": rng.choice([1.0, 1.0, 0.5, 0.7, 1.25]), "ragged": rng.random() < 0.3, "masked": rng.random() < 0.3}
    if op == "logp":
        case["top"] = 0 if rng.random() < 0.3 else size(1, 128)
    elif op == "logp_grad":
        case["entropy"] = rng.random() < 0.5
    else:
        case["top"] = size(1, 128)
        case["tail"] = rng.random() < 0.5
    return case


def _padding(case):
    """Rows of a ragged batch that hold no token."""
    return case["rows"] // 4 if case["ragged"] else 0


def work(case):
    rows, vocab, size = case["rows"], case["vocab"], _SIZE[case["dtype"]]
    live = rows - _padding(case)
    read, write = live * vocab * size, rows * vocab * size
    top = case.get("top", 0)
    n = live * vocab
    # logits once; a row's words: token, three results or their gradients; entries of eight bytes
    return {
        "logp": {"bytes": read + rows * (20 + 8 * top), "flops": 7 * n},
        "logp_grad": {"bytes": read + write + rows * 24, "flops": (9 if case.get("entropy") else 5) * n},
        "distill": {"bytes": read + rows * (16 + 8 * top), "flops": 5 * n},
        "distill_step": {"bytes": read + write + rows * (20 + 8 * top), "flops": 9 * n},
        "distill_grad": {"bytes": read + write + rows * (16 + 8 * top), "flops": 5 * n},
    }[case["op"]]


# ---------------------------------------------------------------------------------- inputs

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _inputs(case, seed):
    """The tensors of a case, made from the seed alone."""
    dev, dt = _device(), _TORCH[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    # a trained model's logits: most far below a few likely tokens
    x = torch.randn((rows, vocab), generator=g, device=dev).mul_(2.0).sub_(1.0)
    likely = torch.randint(0, vocab, (rows, 8), generator=g, device=dev)
    x.scatter_add_(1, likely, torch.rand((rows, 8), generator=g, device=dev).mul_(8.0).add_(2.0))
    allowed = vocab - (max(1, vocab // 50) if case["masked"] else 0)
    if case["masked"]:      # the end of a padded vocabulary
        x[:, allowed:] = -INF
    s = {"case": case, "logits": x.to(dt)}
    padding = torch.randperm(rows, generator=g, device=dev) < _padding(case)
    if case["op"].startswith("logp"):
        # tokens that were drawn from the model are likely ones; a few are not
        pick = torch.randint(0, 8, (rows, 1), generator=g, device=dev)
        token = torch.where(torch.rand(rows, generator=g, device=dev) < 0.9, likely.gather(1, pick)[:, 0],
                            torch.randint(0, allowed, (rows,), generator=g, device=dev))
        s["tokens"] = torch.where(padding, -1, token.clamp_max(allowed - 1)).to(torch.int32)
        if case["op"] == "logp_grad":
            s["dlogprob"] = torch.randn(rows, generator=g, device=dev)
            s["dentropy"] = torch.randn(rows, generator=g, device=dev).mul_(0.1) if case["entropy"] else None
        return s
    # the teacher: near the student, and surer
    k = case["top"]
    x.mul_(1.1).add_(torch.randn((rows, vocab), generator=g, device=dev), alpha=0.7)
    value, index = torch.topk(x, k, 1)
    if case["tail"]:
        value = (value - torch.logsumexp(x, 1, keepdim=True))
    if case["ragged"]:      # and rows with fewer entries than others
        count = torch.randint(1, k + 1, (rows, 1), generator=g, device=dev)
        index = torch.where((torch.arange(k, device=dev) < count) & ~padding[:, None], index, -1)
    index = torch.where(value == -INF, -1, index)
    s["teacher_values"], s["teacher_indices"] = value.contiguous(), index.to(torch.int32).contiguous()
    if case["op"] != "distill":
        # the mean over the batch; float16 training scales its loss up against underflow
        s["dloss"] = torch.rand(rows, generator=g, device=dev).add_(0.5).div_(1 if dt == torch.float16 else rows)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    rows, dev = case["rows"], s["logits"].device

    def column():
        return torch.empty(rows, device=dev)

    # what a program keeps in hand besides: saved values of the forward pass, results' memory
    if case["op"] == "logp":
        s.update(logprob=column(), peak=column(), logsum=column(), entropy=column())
        if case["top"]:
            s["top_values"] = torch.empty((rows, case["top"]), device=dev)
            s["top_indices"] = torch.empty((rows, case["top"]), device=dev, dtype=torch.int32)
        return s
    if case["op"] == "logp_grad":
        saved = _logp(s, False)
        s.update(peak=saved["peak"], logsum=saved["logsum"], entropy=saved["entropy"])
    elif case["op"] == "distill_grad":
        saved = _distill(s)
        s.update(peak=saved["peak"], logsum=saved["logsum"], tail=saved.get("tail"))
    else:
        s.update(loss=column(), peak=column(), logsum=column(), tail=column() if case["tail"] else None)
    if case["op"] != "distill":
        s["dlogits"] = torch.empty_like(s["logits"])
    return s


# ---------------------------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "logp":
        return _logp(s, True)
    if op == "logp_grad":
        return _logp_grad(s)
    if op == "distill_grad":
        return {"dlogits": _distill_grad(s, s["peak"], s["logsum"], s["tail"])}
    out = _distill(s)
    if op == "distill_step":
        out["dlogits"] = _distill_grad(s, out["peak"], out["logsum"], out.get("tail"))
    return out


def _logp(s, with_top):
    case, x = s["case"], s["logits"].float()
    live = s["tokens"] >= 0
    peak = x.amax(1)
    t = (x - peak[:, None]) * case["scale"]
    e = torch.exp(t)
    total = e.sum(1)
    logsum = torch.log(total)
    entropy = logsum - (e * t.clamp_min(-1e4)).sum(1) / total
    token = s["tokens"].clamp_min(0).long()[:, None]
    out = {"logprob": t.gather(1, token)[:, 0] - logsum, "peak": peak, "logsum": logsum, "entropy": entropy}
    out = {k: torch.where(live, v, 0.0) for k, v in out.items()}
    if with_top and case["top"]:
        value, index = _top(x, case["top"])
        value = (value - peak[:, None]) * case["scale"] - logsum[:, None]
        there = live[:, None] & (index >= 0)
        out["top_values"], out["top_indices"] = torch.where(there, value, -INF), torch.where(there, index, -1)
    return out


def _top(x, k):
    """The k largest of each row, the lowest index first among equals: one whole number ranks value and place."""
    rows, cols = x.shape
    bits = (x + 0.0).view(torch.int32)
    rank = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
    rank += 0xFFFFFFFF - torch.arange(cols, device=x.device)
    index = 0xFFFFFFFF - (torch.topk(rank, min(k, cols), 1).values & 0xFFFFFFFF)
    value = x.gather(1, index)
    index = torch.where(value == -INF, -1, index)
    if k > cols:
        value = torch.cat((value, torch.full((rows, k - cols), -INF, device=x.device)), 1)
        index = torch.cat((index, torch.full((rows, k - cols), -1, device=x.device)), 1)
    return value, index.to(torch.int32)


def _logp_grad(s):
    case, x = s["case"], s["logits"].float()
    live = (s["tokens"] >= 0)[:, None]
    t = (x - s["peak"][:, None]) * case["scale"]
    logp = t - s["logsum"][:, None]
    p = torch.exp(logp)
    g = s["dlogprob"][:, None]
    dx = -g * p
    dx.scatter_add_(1, s["tokens"].clamp_min(0).long()[:, None], g.clone())
    if s["dentropy"] is not None:
        dx -= s["dentropy"][:, None] * p * (logp.clamp_min(-1e4) + s["entropy"][:, None])
    return {"dlogits": torch.where(live, dx * case["scale"], 0.0).to(s["logits"].dtype)}


def _teacher(s):
    """q, log q, entries that exist, the tail's q, the sum of all."""
    value = s["teacher_values"].float()
    there = s["teacher_indices"] >= 0
    value = torch.where(there, value, -INF)
    if s["case"]["tail"]:
        q = torch.exp(value)
        tail = (1.0 - q.sum(1)).clamp_min(0.0)
        return q, value, there, tail, tail + q.sum(1)
    value = value * s["case"]["scale"]
    some = there.any(1, keepdim=True)
    top = torch.where(some, value.amax(1, keepdim=True), 0.0)
    e = torch.exp(value - top)
    total = torch.where(some, e.sum(1, keepdim=True), 1.0)
    return e / total, value - top - torch.log(total), there, None, some[:, 0].float()


def _outside(s, there):
    """Truth of every logit that no entry names."""
    rows, vocab = s["logits"].shape
    rest = torch.ones((rows, vocab + 1), dtype=torch.bool, device=there.device)
    rest.scatter_(1, torch.where(there, s["teacher_indices"].long(), vocab), False)
    return rest[:, :vocab]


def _distill(s):
    case, x = s["case"], s["logits"].float()
    q, logq, there, tail_q, _ = _teacher(s)
    live = there.any(1)
    peak = x.amax(1)
    t = (x - peak[:, None]) * case["scale"]
    logsum = torch.log(torch.exp(t).sum(1))
    logp = t.gather(1, s["teacher_indices"].clamp_min(0).long()) - logsum[:, None]
    loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1)
    out = {"peak": peak, "logsum": logsum}
    if case["tail"]:
        t = torch.where(_outside(s, there), t, -INF)
        top = t.amax(1)
        top = torch.where(top > -INF, top, 0.0)
        out["tail"] = top + torch.log(torch.exp(t - top[:, None]).sum(1))
        logp = out["tail"] - logsum
        counts = (logp >= -126 * math.log(2)) & (tail_q > 0)
        loss = loss + torch.where(counts, tail_q * (torch.log(tail_q) - logp), 0.0)
    return {k: torch.where(live, v, 0.0) for k, v in {"loss": loss, **out}.items()}


def _distill_grad(s, peak, logsum, tail):
    case, x = s["case"], s["logits"].float()
    q, _, there, tail_q, total = _teacher(s)
    live = there.any(1, keepdim=True)
    logp = (x - peak[:, None]) * case["scale"] - logsum[:, None]
    index = torch.where(there, s["teacher_indices"], 0).long()
    if case["tail"]:
        counts = tail - logsum >= -126 * math.log(2)
        total = torch.where(counts, total, total - tail_q)
        rest = torch.where(_outside(s, there) & counts[:, None], tail_q[:, None] * torch.exp(logp - (tail - logsum)[:, None]), 0.0)
        dx = total[:, None] * torch.exp(logp) - rest
    else:
        dx = total[:, None] * torch.exp(logp)
    dx.scatter_add_(1, index, torch.where(there, -q, 0.0))
    return torch.where(live, dx * (case["scale"] * s["dloss"])[:, None], 0.0).to(s["logits"].dtype)


def _run_own(s):
    """The same passes through the library, on the caller's stream.  Calls are bound to their tensors
    once, as a program does that calls them many times."""
    from paper_1605_02688_amd import ewf
    if "call" not in s:
        s["call"], s["results"] = _bind(ewf, s)
    s["call"].launch(torch.cuda.current_stream().cuda_stream)
    return s["results"]


def _bind(ewf, s):
    case = s["case"]
    scale = case["scale"]

    def bound(names, fn, *args, **kw):
        nbytes = fn.workspace_bytes(*args, **kw)
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
        return fn.bind(*args, workspace=work, **kw), {n: s[n] for n in names if s.get(n) is not None}

    if case["op"] == "logp":
        return bound(("logprob", "peak", "logsum", "entropy", "top_values", "top_indices"), ewf.token_logprobs, s["logits"], s["tokens"],
                     s["logprob"], peak=s["peak"], logsum=s["logsum"], entropy=s["entropy"], top_values=s.get("top_values"),
                     top_indices=s.get("top_indices"), scale=scale)
    if case["op"] == "logp_grad":
        return bound(("dlogits",), ewf.token_logprobs_grad, s["logits"], s["tokens"], s["dlogprob"], s["dlogits"], peak=s["peak"],
                     logsum=s["logsum"], entropy=s["entropy"] if case["entropy"] else None, dentropy=s["dentropy"], scale=scale)
    teacher = dict(scale=scale, teacher_scale=1.0 if case["tail"] else scale)
    if case["op"] == "distill_grad":
        return bound(("dlogits",), ewf.distill_grad, s["logits"], s["teacher_values"], s["teacher_indices"], s["dlogits"], peak=s["peak"],
                     logsum=s["logsum"], tail=s["tail"], dloss=s["dloss"], **teacher)
    step = dict(dlogits=s["dlogits"], dloss=s["dloss"]) if case["op"] == "distill_step" else {}
    return bound(("loss", "peak", "logsum", "tail", "dlogits"), ewf.distill, s["logits"], s["teacher_values"], s["teacher_indices"], s["loss"],
                 peak=s["peak"], logsum=s["logsum"], tail=s["tail"], **step, **teacher)


# ---------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    c = case["scale"]
    x = s["logits"].double()
    logp = torch.log_softmax(x * c, 1)
    if case["op"].startswith("logp"):
        return _exact_logp(case, s, x, logp)
    return _exact_distill(case, s, x, logp)


def _exact_logp(case, s, x, logp):
    live = s["tokens"] >= 0
    at = torch.arange(case["rows"], device=x.device)[live], s["tokens"].long()[live]
    p = torch.softmax(x * case["scale"], 1)
    entropy = -torch.xlogy(p, p).sum(1) * live
    if case["op"] == "logp_grad":
        hot = torch.zeros_like(x)
        hot[at] = 1.0
        dx = s["dlogprob"].double().unsqueeze(1) * (hot - p)
        if case["entropy"]:
            dx = dx - s["dentropy"].double().unsqueeze(1) * (torch.xlogy(p, p) + p * entropy.unsqueeze(1))
        return {"dlogits": case["scale"] * dx * live.unsqueeze(1)}
    peak = x.max(1).values
    logprob = torch.zeros_like(peak)
    logprob[live] = logp[at]
    out = {"logprob": logprob, "peak": peak * live, "entropy": entropy,
           "logsum": (torch.logsumexp(x * case["scale"], 1) - peak * case["scale"]) * live}
    if case["top"]:
        best = torch.sort(logp, 1, descending=True).values if case["vocab"] <= 1024 else torch.topk(logp, min(case["top"], case["vocab"]), 1).values
        values = torch.full((case["rows"], case["top"]), -INF, dtype=torch.float64, device=x.device)
        n = min(case["top"], case["vocab"])
        values[live, :n] = best[live, :n]
        out["top_values"], out["top_indices"] = values, None
    return out


def _exact_distill(case, s, x, logp):
    rows, vocab = x.shape
    there = s["teacher_indices"] >= 0
    live = there.any(1)
    rank = s["teacher_values"].double() * (1.0 if case["tail"] else case["scale"])
    rank = rank.masked_fill(~there, -INF)
    if not case["tail"]:
        rank = torch.log_softmax(rank.masked_fill(~live.unsqueeze(1), 0.0), 1)
    # the teacher's probabilities in the vocabulary's own places, the last one for entries that do not exist
    place = s["teacher_indices"].long().masked_fill(~there, vocab)
    q = torch.zeros((rows, vocab + 1), dtype=torch.float64, device=x.device).scatter_add(1, place, torch.exp(rank))[:, :vocab]
    named = torch.zeros((rows, vocab + 1), dtype=torch.bool, device=x.device).scatter(1, place, True)[:, :vocab]
    p = torch.exp(logp)
    loss = (torch.xlogy(q, q) - torch.where(q > 0, q * logp, 0.0)).sum(1)
    grad = q.sum(1, keepdim=True) * p - q
    peak = x.max(1).values
    out = {"peak": peak * live, "logsum": (torch.logsumexp(x * case["scale"], 1) - peak * case["scale"]) * live}
    if case["tail"]:
        rest = torch.logsumexp(logp.masked_fill(named, -INF), 1)
        left = torch.where(rest >= math.log(2.0 ** -126), (1 - q.sum(1)).clamp_min(0), 0.0)
        loss = loss + torch.xlogy(left, left) - torch.where(left > 0, left * rest, 0.0)
        grad = grad + left.unsqueeze(1) * (p - torch.where(named, 0.0, torch.exp(logp - torch.where(rest > -INF, rest, 0.0).unsqueeze(1))))
        out["tail"] = torch.where(live, rest + out["logsum"], 0.0)
    dx = case["scale"] * s["dloss"].double().unsqueeze(1) * grad * live.unsqueeze(1) if case["op"] != "distill" else None
    if case["op"] == "distill_grad":
        return {"dlogits": dx}
    out = {"loss": loss * live, **out}
    return out if dx is None else {**out, "dlogits": dx}
