"""The operators over a vocabulary on the GPU against the formulas in 64 bits (tests/vocab_ref.py, which also derives the bounds): sizes around
every row shape, alignments, strides, masks, ties, padding, values that are not finite, calls in place, on other streams and in captured graphs."""
import math

import pytest
import torch

import tests.vocab_ref as ref
from paper_1605_02688_amd import ewf

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
INF = float("inf")


def stream():
    return torch.cuda.current_stream().cuda_stream


def say(*words):
    print("[case]", *words, flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def work_for(op, *args, **kw):
    n = op.workspace_bytes(*args, **kw)
    return torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda") if n else None


def run(op, *args, **kw):
    op(*args, workspace=work_for(op, *args, **kw), stream=stream(), **kw)


def logits_of(g, *shape, dtype=torch.float32, std=3.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def tokens_of(g, *shape, cols, padding=0.25):
    t = torch.randint(0, cols, shape, generator=g, device="cuda")
    gone = torch.rand(shape, generator=g, device="cuda") < padding
    far = torch.tensor([-1, cols, -100, 2 ** 31 - 1, -2 ** 31], device="cuda")[torch.randint(0, 5, shape, generator=g, device="cuda")]
    return torch.where(gone, far, t).to(torch.int32)


def scored(x, tokens, scale=1.0, k=0, entropy=True):
    """token_logprobs on x into fresh tensors (filled, so that what is not written shows)."""
    lead = x.shape[:-1]
    new = lambda *more, dtype=torch.float32: torch.full((*lead, *more), 77, dtype=dtype, device="cuda")
    out = dict(peak=new(), logsum=new())
    if entropy:
        out["entropy"] = new()
    if k:
        out.update(top_values=new(k), top_indices=new(k, dtype=torch.int32))
    logprob = None if tokens is None else new()
    run(ewf.token_logprobs, x, tokens, logprob, scale=scale, **out)
    if logprob is not None:
        out["logprob"] = logprob
    return out


def check_scored(x, tokens, out, scale=1.0, k=0):
    want = ref.token_logprobs(x, tokens, scale, k)
    for n, got in out.items():
        if n == "top_indices":
            assert torch.equal(got.reshape(want[n].shape).long(), want[n]), n
        else:
            ref.close(n, got.reshape(want[n].shape), want[n], want["e_" + n])


# sizes each side of: a vector, the threads of a row, what a workgroup ranks, the parts of a row
COLS = (1, 2, 3, 7, 8, 9, 15, 17, 33, 64, 100, 127, 128, 300, 511, 513, 1000, 1024, 1025, 2047, 2048, 2049, 2056, 4097, 8192, 10000, 16385, 33279, 50257,
        65537)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", COLS)
def test_token_logprobs(dtype, cols):
    for rows, k, scale in ((1, 0, 1.0), (5, 1, 0.7), (3, 20, 1.0), (67 if cols < 9000 else 9, 5, 1.25), (4, 128, 1.0)):
        say("token logprobs", dtype, rows, cols, k)
        g = gen(cols * 5 + rows)
        x = logits_of(g, rows, cols, dtype=DT[dtype])
        tokens = None if rows == 1 else tokens_of(g, rows, cols=cols)
        check_scored(x, tokens, scored(x, tokens, scale, k, entropy=k != 5), scale, k)


@pytest.mark.parametrize("dtype", sorted(DT))
def test_many_rows_and_few_long_ones(dtype):
    for rows, cols, k in ((700, 8200, 64), (300, 40001, 20), (2, 300001, 20), (1, 1000003, 128), (3, 600000, 0), (1, 262144, 5), (20000, 260, 3)):
        say("token logprobs", dtype, rows, cols, k)
        g = gen(cols + rows)
        x = logits_of(g, rows, cols, dtype=DT[dtype])
        tokens = tokens_of(g, rows, cols=cols)
        out = scored(x, tokens, 1.0, k)
        check_scored(x, tokens, out, 1.0, k)
        again = scored(x, tokens, 1.0, k)
        assert all(torch.equal(out[n], again[n]) for n in out)


@pytest.mark.parametrize("dtype", sorted(DT))
def test_ties_go_to_the_lowest_index(dtype):
    g = gen(3)
    for cols in (5, 200, 2048, 8191, 20000, 400001):
        for k in (1, 3, 20, 128):
            say("ties", dtype, cols, k)
            rows = [torch.zeros(cols), torch.full((cols,), -3.0), torch.arange(cols) * (2.0 ** -7), torch.arange(cols).flip(0) * (2.0 ** -7),
                    torch.randint(0, 3, (cols,)).float(), torch.where(torch.arange(cols) % 2 == 0, 0.0, -0.0),
                    (torch.arange(cols) % 2048 < 100).float(), (torch.arange(cols) % 8192 < 300).float() * (torch.arange(cols) % 7).float(),
                    torch.where(torch.arange(cols) % 16 == 3, 1.0, -INF)]
            x = torch.stack(rows).cuda().to(DT[dtype])
            check_scored(x, None, scored(x, None, 1.0, k), 1.0, k)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", (3, 100, 1000, 9001, 50257, 300000))
def test_masks_and_values_that_are_not_finite(dtype, cols):
    dt, g = DT[dtype], gen(cols)
    x = logits_of(g, 14, cols, dtype=dt)
    lowest = torch.finfo(dt).min
    x[0] = -INF
    x[1] = -INF
    x[1, cols // 2] = 1.0
    x[2, 1:] = -INF
    x[3] = lowest
    x[4, :] = lowest
    x[4, cols - 1] = 2.0
    x[5, cols // 3] = float("nan")
    x[6, cols - 1] = INF
    x[7, 0] = -INF
    x[8, :cols - 1] = -INF
    x[9] = float("nan")
    x[10, 0] = torch.finfo(dt).max
    x[11, :] = torch.finfo(dt).max
    x[12] = INF
    tokens = torch.randint(0, cols, (14,), generator=g, device="cuda").to(torch.int32)
    tokens[13] = -1
    x[13] = float("nan")                                    # padding: not read
    say("masks", dtype, cols)
    for k in (0, 4, 128):
        out = scored(x, tokens, 1.0, k)
        check_scored(x, tokens, out, 1.0, k)
    assert (out["top_indices"][[0, 5, 6, 9, 12, 13]] == -1).all() and out["entropy"][0] == 0 and out["logprob"][0] == -INF
    # gradients: nothing where there is no logit or no token, NaN where the row has one, and only there
    dx = torch.full_like(x, 77)
    dlogprob, dentropy = torch.randn(14, generator=g, device="cuda"), torch.randn(14, generator=g, device="cuda")
    run(ewf.token_logprobs_grad, x, tokens, dlogprob, dx, peak=out["peak"], logsum=out["logsum"], entropy=out["entropy"], dentropy=dentropy)
    assert (dx[[0, 13]] == 0).all() and torch.isnan(dx[[5, 6, 9, 12]]).all()
    fine = [1, 2, 3, 4, 7, 8, 10, 11]
    want, bound = ref.token_logprobs_grad(x[fine], tokens[fine], dlogprob[fine], dentropy[fine], out["peak"][fine], out["logsum"][fine],
                                          out["entropy"][fine], 1.0, dt)
    ref.close("dlogits", dx[fine], want, bound)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", COLS)
def test_token_logprobs_gradient(dtype, cols):
    dt = DT[dtype]
    for rows, scale in ((1, 1.0), (37 if cols < 9000 else 6, 0.7)):
        say("token logprobs gradient", dtype, rows, cols)
        g = gen(cols * 3 + rows)
        x = logits_of(g, rows, cols, dtype=dt)
        tokens = tokens_of(g, rows, cols=cols)
        out = scored(x, tokens, scale)
        dlogprob, dentropy = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
        for t, gp, ge in ((tokens, dlogprob, dentropy), (tokens, dlogprob, None), (tokens, None, dentropy), (None, None, dentropy)):
            dx = torch.full_like(x, 77)
            if t is None:
                out = scored(x, None, scale)
            run(ewf.token_logprobs_grad, x, t, gp, dx, peak=out["peak"], logsum=out["logsum"], entropy=out["entropy"] if ge is not None else None,
                dentropy=ge, scale=scale)
            want, bound = ref.token_logprobs_grad(x, t, gp, ge, out["peak"], out["logsum"], out["entropy"], scale, dt)
            ref.close("dlogits", dx, want, bound)
        # in place, and with a gradient that all rows share
        shared = torch.tensor([0.25], device="cuda").expand(rows)
        want, bound = ref.token_logprobs_grad(x, tokens, shared, None, out["peak"], out["logsum"], None, scale, dt)
        y = x.clone()
        run(ewf.token_logprobs_grad, y, tokens, shared, y, peak=out["peak"], logsum=out["logsum"], scale=scale)
        ref.close("dlogits", y, want, bound)


def entries_of(g, x, k, tail, dtype=torch.float32, ragged=False):
    """A teacher near x: its k likeliest tokens with values as a teacher's pass gives them; absent entries hold NaN."""
    rows, cols = x.shape
    y = torch.where(torch.isfinite(x.float()), x.float(), -20.0) * 0.9 + torch.randn(x.shape, generator=g, device="cuda")
    value, index = torch.topk(y, min(k, cols), 1)
    if tail:
        value = value - torch.logsumexp(y, 1, keepdim=True)
    if k > cols:
        value = torch.cat((value, value.new_full((rows, k - cols), math.nan)), 1)
        index = torch.cat((index, index.new_full((rows, k - cols), -1)), 1)
    if ragged:
        gone = torch.rand(value.shape, generator=g, device="cuda") < 0.3
        gone[:: 3] = True
        index = torch.where(gone, torch.where(torch.rand(value.shape, generator=g, device="cuda") < 0.5, -1, cols + 5), index)
        value = torch.where(gone, math.nan, value)
    order = torch.randperm(k, generator=g, device="cuda")
    return value[:, order].to(dtype).contiguous(), index[:, order].to(torch.int32).contiguous()


def distilled(x, values, indices, tail, scale=1.0, teacher_scale=1.0, dloss=None, gradient=True, into=None, keep=True):
    lead = x.shape[:-1]
    new = lambda: torch.full(lead, 77.0, device="cuda")
    out = dict(peak=new(), logsum=new()) if keep else {}
    if tail:
        out["tail"] = new()
    loss = new()
    dx = into if into is not None else torch.full_like(x, 77) if gradient else None
    run(ewf.distill, x, values, indices, loss, dlogits=dx, dloss=dloss if dx is not None else None, scale=scale, teacher_scale=teacher_scale, **out)
    return {**out, "loss": loss}, dx


def check_distilled(x, values, indices, tail, out, dx, scale, teacher_scale, dloss):
    want = ref.distill(x, values, indices, scale, teacher_scale, tail)
    for n, got in out.items():
        ref.close(n, got.reshape(-1), want[n], want["e_" + n])
    if dx is not None:
        w, bound = ref.distill_grad(x, values, indices, out["peak"], out["logsum"], out.get("tail"), dloss, scale, teacher_scale, dx.dtype)
        ref.close("dlogits", dx.reshape(w.shape), w, bound)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", COLS + (131072, 140003))
def test_distill(dtype, cols):
    dt = DT[dtype]
    for rows, k, tail, ragged, scale in ((1, 1, False, False, 1.0), (6, 20, True, True, 1.0), (7, 128, True, False, 0.7), (9, 64, False, True, 0.5)):
        say("distill", dtype, rows, cols, k, tail)
        g = gen(cols * 11 + k)
        x = logits_of(g, rows, cols, dtype=dt)
        values, indices = entries_of(g, x, k, tail, dt if k == 64 else torch.float32, ragged)
        dloss = torch.randn(rows, generator=g, device="cuda")
        ts = 1.0 if tail else scale
        out, _ = distilled(x, values, indices, tail, scale, ts, gradient=False)
        check_distilled(x, values, indices, tail, out, None, scale, ts, None)
        both, dx = distilled(x, values, indices, tail, scale, ts, dloss)
        check_distilled(x, values, indices, tail, both, dx, scale, ts, dloss)
        alone = torch.full_like(x, 77)
        run(ewf.distill_grad, x, values, indices, alone, peak=out["peak"], logsum=out["logsum"], tail=out.get("tail"), dloss=dloss, scale=scale,
            teacher_scale=ts)
        check_distilled(x, values, indices, tail, out, alone, scale, ts, dloss)
        # over the logits, with a weight that all rows share, and nothing kept
        shared = torch.tensor([0.5], device="cuda").expand(rows)
        y = x.clone()
        got, _ = distilled(y, values, indices, tail, scale, ts, shared, into=y, keep=False)
        assert torch.equal(got["loss"], both["loss"])
        check_distilled(x, values, indices, tail, both, y, scale, ts, shared)
        y = x.clone()
        run(ewf.distill_grad, y, values, indices, y, peak=out["peak"], logsum=out["logsum"], tail=out.get("tail"), dloss=dloss, scale=scale, teacher_scale=ts)
        assert torch.equal(y, alone)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", (9, 300, 5000, 20011, 150000))
def test_an_index_that_comes_twice(dtype, cols):
    dt, g = DT[dtype], gen(cols)
    x = logits_of(g, 6, cols, dtype=dt)
    for k in (4, 100):
        index = torch.randint(0, min(cols, 30), (6, k), generator=g, device="cuda").to(torch.int32)
        index[1] = 5                                         # all the same one
        index[2, ::2], index[2, 1::2] = cols - 1, 0          # on both edges
        values = torch.log_softmax(torch.randn(6, k, generator=g, device="cuda"), 1) - 0.3
        dloss = torch.randn(6, generator=g, device="cuda")
        for tail in (False, True):
            say("twice", dtype, cols, k, tail)
            out, dx = distilled(x, values, index, tail, dloss=dloss)
            check_distilled(x, values, index, tail, out, dx, 1.0, 1.0, dloss)
            again, dy = distilled(x, values, index, tail, dloss=dloss)
            assert torch.equal(dx, dy) and torch.equal(out["loss"], again["loss"])


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", (40, 1000, 9001, 150000))
def test_distill_masks_and_values_that_are_not_finite(dtype, cols):
    dt, g = DT[dtype], gen(cols)
    rows = 12
    x = logits_of(g, rows, cols, dtype=dt)
    for tail in (False, True):
        say("distill masks", dtype, cols, tail)
        values, indices = entries_of(g, x, 8, tail)
        y = x.clone()
        y[0] = -INF                                          # a student without a logit
        y[1] = -INF
        y[1].scatter_(0, indices[1].long(), torch.randn(8, device="cuda").to(dt))        # the entries alone: no tail
        y[2].scatter_(0, indices[2].long(), torch.full((8,), -INF, device="cuda").to(dt))  # all but the entries
        y[3, :] = torch.finfo(dt).min
        y[3].scatter_(0, indices[3].long(), torch.randn(8, device="cuda").to(dt))
        y[4, cols // 2] = float("nan")
        y[5, cols - 1] = INF
        y[6] = float("nan")                                  # padding
        indices[6] = -1
        values[6] = float("nan")
        values[7, 3] = -INF                                  # an entry of probability 0
        values[8] = -INF
        values[9, 2] = float("nan")
        indices[10, 1:] = -7
        dloss = torch.rand(rows, generator=g, device="cuda") + 0.5
        out, dx = distilled(y, values, indices, tail, dloss=dloss)
        fine = [1, 6, 7, 8, 10, 11] + ([] if tail and dt != torch.float16 else [3])
        pick = lambda t: None if t is None else t[fine]
        check_distilled(y[fine], values[fine], indices[fine], tail, {n: t[fine] for n, t in out.items()}, dx[fine], 1.0, 1.0, dloss[fine])
        assert out["loss"][0] == INF and out["loss"][2] == INF
        q = torch.exp(values.double()) if tail else torch.softmax(values.double(), 1)
        for r in (0, 2):                                     # p = 0 at the entries
            got = dx[r].double().gather(0, indices[r].long())
            want = -dloss[r].double() * q[r]
            ref.close("entries", got, want, ref.stored(60 * ref.U * want.abs(), want, dt))
        assert (dx[0].double().scatter(0, indices[0].long(), 0.0) == 0).all()
        assert torch.isnan(out["loss"][[4, 5]]).all() and torch.isnan(dx[[4, 5]]).all()
        assert (dx[6] == 0).all() and out["loss"][6] == 0
        assert torch.isnan(out["loss"][9])
        alone = torch.full_like(x, 77)
        run(ewf.distill_grad, y, values, indices, alone, peak=out["peak"], logsum=out["logsum"], tail=out.get("tail"), dloss=dloss)
        check_distilled(y[fine], values[fine], indices[fine], tail, {n: t[fine] for n, t in out.items()}, alone[fine], 1.0, 1.0, dloss[fine])
        assert torch.isnan(alone[[4, 5]]).all() and (alone[6] == 0).all()


@pytest.mark.parametrize("dtype", sorted(DT))
def test_strides_and_alignments(dtype):
    dt, g = DT[dtype], gen(9)
    for cols in (7, 130, 1001, 9000, 70001):
        for off in (0, 1, 3):
            say("strides", dtype, cols, off)
            pitch = cols + 13
            base = logits_of(g, 4, 3, pitch, dtype=dt)
            x = base.transpose(0, 1)[:, :, off:off + cols]               # [3, 4, cols]
            tokens = tokens_of(g, 4, 3, cols=cols).t()
            k = 6
            tv, ti = torch.full((3, 4, k + 2), 77.0, device="cuda"), torch.full((4, 3, k), 77, dtype=torch.int32, device="cuda").transpose(0, 1)
            logprob, peak, logsum, entropy = (torch.full((4, 3), 77.0, device="cuda").t() for _ in range(4))
            run(ewf.token_logprobs, x, tokens, logprob, peak=peak, logsum=logsum, entropy=entropy, top_values=tv[:, :, 1:k + 1], top_indices=ti)
            check_scored(x, tokens, dict(logprob=logprob, peak=peak, logsum=logsum, entropy=entropy, top_values=tv[:, :, 1:k + 1], top_indices=ti), 1.0, k)
            assert (tv[:, :, 0] == 77).all() and (tv[:, :, -1] == 77).all()
            room = torch.full((3, 4, cols + 9), 77.0, dtype=dt, device="cuda")
            dx = room[:, :, 5 - off:5 - off + cols]
            gp = torch.randn(3, 1, device="cuda").expand(3, 4)
            run(ewf.token_logprobs_grad, x, tokens, gp, dx, peak=peak, logsum=logsum)
            want, bound = ref.token_logprobs_grad(x, tokens, gp, None, peak, logsum, None, 1.0, dt)
            ref.close("dlogits", dx.reshape(want.shape), want, bound)
            assert (room[:, :, :5 - off] == 77).all() and (room[:, :, 5 - off + cols:] == 77).all()
            values, indices = entries_of(g, x.reshape(12, cols), k, True)
            values, indices = values.view(3, 4, k), indices.view(4, 3, k).transpose(0, 1)
            room.fill_(77.0)
            loss, tail = torch.full((3, 4), 77.0, device="cuda"), torch.full((3, 4), 77.0, device="cuda")
            run(ewf.distill, x, values, indices, loss, peak=peak, logsum=logsum, tail=tail, dlogits=dx, dloss=gp)
            check_distilled(x, values, indices, True, dict(loss=loss, peak=peak, logsum=logsum, tail=tail), dx, 1.0, 1.0, gp)
            assert (room[:, :, :5 - off] == 77).all() and (room[:, :, 5 - off + cols:] == 77).all()
            first = dx.clone()
            room.fill_(77.0)
            run(ewf.distill_grad, x, values, indices, dx, peak=peak, logsum=logsum, tail=tail, dloss=gp)
            check_distilled(x, values, indices, True, dict(loss=loss, peak=peak, logsum=logsum, tail=tail), dx, 1.0, 1.0, gp)
            assert (room[:, :, :5 - off] == 77).all() and (room[:, :, 5 - off + cols:] == 77).all()
            assert first.shape == dx.shape
