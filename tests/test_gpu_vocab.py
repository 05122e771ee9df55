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


@pytest.mark.parametrize("fill", (0x00, 0x01, 0x7F, 0xFF))
def test_whatever_a_workspace_holds(fill):
    # rows of padding among others, in every form that has a workspace
    g = gen(4)
    for dtype, rows, cols in (("bf16", 9, 140003), ("f32", 6, 300001), ("f16", 2, 400000), ("bf16", 30, 9000)):
        say("workspace", fill, dtype, rows, cols)
        x = logits_of(g, rows, cols, dtype=DT[dtype])
        values, index = entries_of(g, x, 20, True, ragged=True)
        index[0] = -1
        tokens = tokens_of(g, rows, cols=cols)
        filled = lambda op, *args, **kw: torch.full((max(16, op.workspace_bytes(*args, **kw)),), fill, dtype=torch.uint8, device="cuda")
        new = lambda *s, dtype=torch.float32: torch.full(s, 77, dtype=dtype, device="cuda")
        out = dict(peak=new(rows), logsum=new(rows), tail=new(rows))
        loss, dx, dy = new(rows), torch.full_like(x, 77), torch.full_like(x, 77)
        args, kw = (x, values, index, loss), dict(dlogits=dx, **out)
        ewf.distill(*args, workspace=filled(ewf.distill, *args, **kw), stream=stream(), **kw)
        check_distilled(x, values, index, True, dict(loss=loss, **out), dx, 1.0, 1.0, None)
        args, kw = (x, values, index, dy), out
        ewf.distill_grad(*args, workspace=filled(ewf.distill_grad, *args, **kw), stream=stream(), **kw)
        check_distilled(x, values, index, True, dict(loss=loss, **out), dy, 1.0, 1.0, None)
        scores = dict(peak=new(rows), logsum=new(rows), entropy=new(rows), top_values=new(rows, 9), top_indices=new(rows, 9, dtype=torch.int32))
        lp = new(rows)
        args = (x, tokens, lp)
        ewf.token_logprobs(*args, workspace=filled(ewf.token_logprobs, *args, **scores), stream=stream(), **scores)
        check_scored(x, tokens, dict(logprob=lp, **scores), 1.0, 9)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows,vectors", ((9001, 50), (9001, 101), (2200, 250), (9001, 251), (5003, 501), (4500, 1019), (1500, 1500), (1100, 3001), (700, 5000), (600, 7001), (301, 9001),
                                           (560, 12500)))
def test_more_rows_than_are_held_at_once(dtype, rows, vectors):
    # each kind of row in turn with the others: masked, padded, huge, not finite, named twice
    dt = DT[dtype]
    cols = vectors * 16 // dt.itemsize + 3
    for k, tail in ((20, True), (100, True), (64, False)):
        say("many", dtype, rows, cols, k, tail)
        g = gen(rows + cols + k)
        x = logits_of(g, rows, cols, dtype=dt)
        values, index = entries_of(g, x, k, tail, ragged=True)
        twice = torch.arange(rows, device="cuda") % 5 == 1
        index[twice, 3:7] = index[twice, 2:3]
        values[twice] -= 3.0
        x[2::7, : cols // 2] = -math.inf
        x[4::31, cols // 3] = math.nan
        x[6::41] = -math.inf
        x[8::37] *= 2000.0 if dtype == "f16" else 3e6
        dloss = torch.randn(rows, generator=g, device="cuda")
        out, dx = distilled(x, values, index, tail, dloss=dloss)
        # what the oracle does not have: a student's or a teacher's NaN, a student without a logit
        there = (index >= 0) & (index < cols)
        live, none = there.any(1), (x == -math.inf).all(1)
        nan = live & (torch.isnan(x).any(1) | ((there & torch.isnan(values)).any(1) & ~none))
        assert torch.isnan(out["loss"][nan]).all() and torch.isnan(dx[nan]).all()
        named = torch.zeros((rows, cols + 1), dtype=torch.bool, device="cuda").scatter_(1, torch.where(there, index, cols).long(), True)[:, :cols]
        assert (dx[none & live][~named[none & live]] == 0).all()
        assert ((out["loss"] == math.inf) | torch.isnan(out["loss"]))[none & live].all()
        fine = ~nan & ~(none & live)
        check_distilled(x[fine], values[fine], index[fine], tail, {n: t[fine] for n, t in out.items()}, dx[fine], 1.0, 1.0, dloss[fine])
        y = x.clone()
        again, _ = distilled(y, values, index, tail, dloss=dloss, into=y)
        assert torch.equal(torch.nan_to_num(y), torch.nan_to_num(dx)) and torch.equal(torch.nan_to_num(again["loss"]), torch.nan_to_num(out["loss"]))


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


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", (5, 300, 3000, 9001, 40000))
def test_logits_of_any_size(dtype, cols):
    dt, g = DT[dtype], gen(cols + 1)
    sizes = (1e-6, 1e-2, 50.0, 3e3, 2e4) if dtype == "f16" else (1e-30, 1e-3, 50.0, 3e3, 1e5, 3e6, 1e9, 1e20, 1e37)
    for scale in (1.0, 2.0 ** -20, 2.0 ** 20):
        say("sizes", dtype, cols, scale)
        x = torch.stack([torch.randn(cols, generator=g, device="cuda") * z + c * z for z in sizes for c in (0.0, 5.0, -5.0)]).to(dt)
        rows = x.shape[0]
        tokens = torch.randint(0, cols, (rows,), generator=g, device="cuda").to(torch.int32)
        tokens[::2] = x[::2].float().argmax(1).to(torch.int32)
        out = scored(x, tokens, scale, 3)
        check_scored(x, tokens, out, scale, 3)
        gp, ge = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
        dx = torch.full_like(x, 77)
        run(ewf.token_logprobs_grad, x, tokens, gp, dx, peak=out["peak"], logsum=out["logsum"], entropy=out["entropy"], dentropy=ge, scale=scale)
        want, bound = ref.token_logprobs_grad(x, tokens, gp, ge, out["peak"], out["logsum"], out["entropy"], scale, dt)
        # (a product that leaves the type is not what this is about)
        fine = want.abs() < 0.5 * torch.finfo(dt).max
        ref.close("dlogits", torch.where(fine, dx.double(), 0.0), torch.where(fine, want, 0.0), torch.where(fine, bound, 0.0))
        k = min(cols, 4)
        index = torch.topk(x.float(), k, 1).indices.to(torch.int32)
        index[:, 0] = tokens
        values = torch.log_softmax(torch.randn(rows, k, generator=g, device="cuda"), 1) - 0.5
        for tail in (False, True):
            for step in (True, False):
                got, dx = distilled(x, values, index, tail, scale=scale, gradient=step)
                if not step:
                    dx = torch.full_like(x, 77)
                    run(ewf.distill_grad, x, values, index, dx, peak=got["peak"], logsum=got["logsum"], tail=got.get("tail"), scale=scale)
                want, bound = ref.distill_grad(x, values, index, got["peak"], got["logsum"], got.get("tail"), None, scale, 1.0, dt)
                fine = want.abs() < 0.5 * torch.finfo(dt).max
                ref.close("dlogits", torch.where(fine, dx.double(), 0.0), torch.where(fine, want, 0.0), torch.where(fine, bound, 0.0))
                loss = ref.distill(x, values, index, scale, 1.0, tail)
                for n, v in got.items():
                    few = loss[n].abs() < 1e38
                    ref.close(n, torch.where(few, v.double(), 0.0), torch.where(few, loss[n], 0.0), torch.where(few, loss["e_" + n], 0.0))


@pytest.mark.parametrize("dtype", sorted(DT))
def test_one_row_alone(dtype):
    # rank 1: the rows' tensors have no axis
    for cols in (100, 5000, 70000):
        g = gen(cols)
        x = logits_of(g, cols, dtype=DT[dtype])
        token = torch.tensor(cols // 3, dtype=torch.int32, device="cuda")
        logprob, peak, logsum = (torch.full((), 77.0, device="cuda") for _ in range(3))
        tv, ti = torch.full((3,), 77.0, device="cuda"), torch.full((3,), 77, dtype=torch.int32, device="cuda")
        run(ewf.token_logprobs, x, token, logprob, peak=peak, logsum=logsum, top_values=tv, top_indices=ti)
        check_scored(x.view(1, -1), token.view(1), dict(logprob=logprob.view(1), peak=peak.view(1), logsum=logsum.view(1), top_values=tv.view(1, 3),
                                                        top_indices=ti.view(1, 3)), 1.0, 3)
        loss, dx = torch.full((), 77.0, device="cuda"), torch.empty_like(x)
        run(ewf.distill, x, tv, ti, loss, peak=peak, logsum=logsum, dlogits=dx)
        check_distilled(x.view(1, -1), tv.view(1, 3), ti.view(1, 3), False, dict(loss=loss.view(1), peak=peak.view(1), logsum=logsum.view(1)), dx.view(1, -1), 1.0,
                        1.0, None)


# ------------------------------------------------------------------ streams, graphs, several calls at once

def vocab_calls(g):
    """One bound call of every operator and form on tensors of its own: [(call, results)]."""
    made = []

    def bound(op, results, *args, **kw):
        made.append((op.bind(*args, workspace=work_for(op, *args, **kw), **kw), results))

    new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda")
    for rows, cols, dt, k in ((300, 5001, torch.bfloat16, 7), (2, 300000, torch.float32, 20), (40, 700, torch.float16, 3), (5, 270000, torch.bfloat16, 64)):
        x, tokens = logits_of(g, rows, cols, dtype=dt), tokens_of(g, rows, cols=cols)
        logprob, peak, logsum, entropy, tv, ti = new(rows), new(rows), new(rows), new(rows), new(rows, k), new(rows, k, dtype=torch.int32)
        bound(ewf.token_logprobs, (logprob, peak, logsum, entropy, tv, ti), x, tokens, logprob, peak=peak, logsum=logsum, entropy=entropy, top_values=tv,
              top_indices=ti, scale=0.8)
        dx = torch.empty_like(x)
        bound(ewf.token_logprobs_grad, (dx,), x, tokens, torch.randn(rows, generator=g, device="cuda"), dx, peak=peak, logsum=logsum, entropy=entropy,
              dentropy=torch.randn(rows, generator=g, device="cuda"), scale=0.8)
        y = logits_of(g, rows, cols, dtype=dt)
        loss, p2, l2, tail, dy, dz = new(rows), new(rows), new(rows), new(rows), torch.empty_like(y), torch.empty_like(y)
        bound(ewf.distill, (loss, p2, l2, tail, dy), y, tv, ti, loss, peak=p2, logsum=l2, tail=tail, dlogits=dy)
        bound(ewf.distill_grad, (dz,), y, tv, ti, dz, peak=p2, logsum=l2, tail=tail)
        only = new(rows)
        bound(ewf.distill, (only,), y, tv, ti, only)
    return made


def clear(calls):
    for _, results in calls:
        for r in results:
            r.view(-1).view(torch.uint8).zero_()


def same(a, b):
    return torch.equal(a.view(-1).view(torch.uint8), b.view(-1).view(torch.uint8))


def test_all_in_a_captured_graph():
    calls = vocab_calls(gen(50))
    for call, _ in calls:
        call.launch(stream())
    torch.cuda.synchronize()
    eager = [[r.clone() for r in results] for _, results in calls]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            for call, _ in calls:
                call.launch(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for replay in range(4):
        clear(calls)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for (_, results), want in zip(calls, eager):
            assert all(same(r, e) for r, e in zip(results, want)), replay
        # eager work and the same operators between the replays, the workspaces left dirty
        assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())
        for call, _ in calls:
            call.launch(stream())
        torch.cuda.synchronize()


def test_calls_on_several_streams_at_once():
    sets = [vocab_calls(gen(60 + k)) for k in range(3)]
    for calls in sets:
        for call, _ in calls:
            call.launch(stream())
    torch.cuda.synchronize()
    want = [[[r.clone() for r in results] for _, results in calls] for calls in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for calls in sets:
        clear(calls)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, calls in zip(streams, sets):
            for call, _ in calls:
                call.launch(s.cuda_stream)
    torch.cuda.synchronize()
    for calls, w in zip(sets, want):
        for (_, results), e in zip(calls, w):
            assert all(same(r, x) for r, x in zip(results, e))


def test_workspaces_of_the_wrong_size_are_refused():
    x = torch.randn(1, 300000, device="cuda")
    peak = torch.empty(1, device="cuda")
    n = ewf.token_logprobs.workspace_bytes(x, peak=peak)
    assert n > 16
    with pytest.raises(ewf.EwfError) as e:
        ewf.token_logprobs(x, peak=peak, workspace=torch.empty(n - 16, dtype=torch.uint8, device="cuda"), stream=stream())
    assert e.value.status == ewf.ENOMEM


# ------------------------------------------------------------------ all together

@pytest.mark.parametrize("dtype", ("f32", "bf16"))
def test_a_student_learns_from_a_teacher(dtype):
    """A teacher's pass writes its likeliest tokens, a student's step reads them: loss and gradient in one call, through the projection to the
    hidden rows, and beside it an entropy term by the tokens' log probabilities; each step against the formulas, and the whole
    gradient against differences of the objective in 64 bits."""
    g = gen(80)
    dt, B, T, H, V, k = DT[dtype], 3, 30, 24, 501, 16
    hidden = torch.randn(B, T, H, generator=g, device="cuda")
    wt, ws = (torch.randn(H, V, generator=g, device="cuda") * s for s in (0.9, 0.7))
    teacher, student = (hidden @ wt).to(dt), (hidden @ ws).to(dt)
    tokens = tokens_of(g, B, T, cols=V)
    out = scored(teacher, tokens, 1.0, k)
    check_scored(teacher, tokens, out, 1.0, k)
    # rows of padding have no alternatives: no loss, no gradient
    dloss = torch.rand(B, T, generator=g, device="cuda")
    got, dx = distilled(student, out["top_values"], out["top_indices"], True, dloss=dloss)
    check_distilled(student, out["top_values"], out["top_indices"], True, got, dx, 1.0, 1.0, dloss)
    pad = (tokens < 0) | (tokens >= V)
    assert pad.any() and (got["loss"][pad] == 0).all() and (dx[pad] == 0).all()
    own = scored(student, tokens)
    de = torch.randn(B, T, generator=g, device="cuda")
    de_x = torch.empty_like(student)
    run(ewf.token_logprobs_grad, student, tokens, None, de_x, peak=own["peak"], logsum=own["logsum"], entropy=own["entropy"], dentropy=de)
    if dtype == "f32":
        dw = hidden.reshape(-1, H).t().double() @ (dx + de_x).reshape(-1, V).double()
        values, index = out["top_values"], out["top_indices"]

        def objective(w):
            x = (hidden.double() @ w).reshape(-1, V)
            loss = ref.distill(x, values, index, 1.0, 1.0, True)["loss"]
            return float((loss * dloss.reshape(-1)).sum() + (ref.token_logprobs(x, tokens, 1.0)["entropy"] * de.reshape(-1)).sum())

        for _ in range(4):
            step = torch.randn(H, V, generator=g, device="cuda", dtype=torch.float64)
            h = 1e-5
            slope = (objective(ws.double() + h * step) - objective(ws.double() - h * step)) / (2 * h)
            # float32 logits are half a step off, as are their gradients: about 1e-6 of the products' sum of magnitudes
            room = 1e-5 * float((dw.abs() * step.abs()).sum())
            assert abs(slope - float((dw * step).sum())) < room, (slope, float((dw * step).sum()), room)


# ------------------------------------------------------------------ beyond 2^31 elements

def test_logits_of_more_than_2_31_elements():
    rows, cols, bf = 17000, 131072, torch.bfloat16
    g = gen(90)
    x = torch.empty(rows, cols, dtype=bf, device="cuda")
    for r in range(0, rows, 1000):
        x[r:r + 1000] = torch.randn(min(1000, rows - r), cols, generator=g, device="cuda") * 3
    tokens = tokens_of(g, rows, cols=cols)
    say("more than 2^31", rows, cols)
    out = scored(x, tokens, 1.0, 20)
    parts = (slice(0, 3), slice(16383, 16387), slice(rows - 3, rows))
    for part in parts:
        check_scored(x[part], tokens[part], {n: t[part] for n, t in out.items()}, 1.0, 20)
    gp = torch.randn(rows, generator=g, device="cuda")
    dx = torch.empty_like(x)
    run(ewf.token_logprobs_grad, x, tokens, gp, dx, peak=out["peak"], logsum=out["logsum"])
    for part in parts:
        want, bound = ref.token_logprobs_grad(x[part], tokens[part], gp[part], None, out["peak"][part], out["logsum"][part], None, 1.0, bf)
        ref.close("dlogits", dx[part], want, bound)
    values, index = out["top_values"], out["top_indices"]
    got, _ = distilled(x, values, index, True, dloss=gp, into=dx)
    for part in parts:
        check_distilled(x[part], values[part], index[part], True, {n: t[part] for n, t in got.items()}, dx[part], 1.0, 1.0, gp[part])
    run(ewf.distill_grad, x, values, index, x, peak=got["peak"], logsum=got["logsum"], tail=got["tail"], dloss=gp)
    assert all(torch.equal(x[part].isnan(), dx[part].isnan()) and (x[part].double() - dx[part].double()).abs().max() < 1e-2 for part in parts)
    del x, dx
    torch.cuda.empty_cache()


def test_a_row_of_the_longest():
    cols = 1 << 24
    g = gen(91)
    x = logits_of(g, 2, cols, dtype=torch.bfloat16)
    tokens = torch.tensor([cols - 1, 5], dtype=torch.int32, device="cuda")
    out = scored(x, tokens, 1.0, 128)
    check_scored(x, tokens, out, 1.0, 128)
    got, dx = distilled(x, out["top_values"], out["top_indices"], True)
    check_distilled(x, out["top_values"], out["top_indices"], True, got, dx, 1.0, 1.0, None)
