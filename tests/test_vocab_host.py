"""The operators over a vocabulary without a GPU: their formulas against differences and torch's own gradients, and what the library refuses.
Calls that must be refused are made on made-up addresses; a workspace query makes all checks and launches nothing."""
import math

import pytest
import torch

import tests.vocab_ref as ref
from paper_1605_02688_amd import ewf
from tests.test_operators_host import T, refused, _differences

F32, F16, BF16, I32 = ewf.F32, ewf.F16, ewf.BF16, ewf.I32
INF = float("inf")


# ------------------------------------------------------------------ the formulas against differences

def _rand(*s, seed=1):
    return torch.randn(*s, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("scale", (1.0, 0.6))
def test_token_logprobs_formula_is_the_gradient(scale):
    x, g, h = _rand(5, 7), _rand(5, seed=2), _rand(5, seed=3)
    tokens = torch.tensor([0, 6, 3, -1, 2], dtype=torch.int32)
    x[4, 5] = -INF

    def value(x):
        o = ref.token_logprobs(x, tokens, scale)
        return float((o["logprob"] * g + o["entropy"] * h).sum())

    o = ref.token_logprobs(x, tokens, scale)
    got, _ = ref.token_logprobs_grad(x, tokens, g, h, o["peak"], o["logsum"], o["entropy"], scale, torch.float32)
    want = _differences(value, x)
    want[4, 5] = 0
    assert torch.allclose(got, want, rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("tail", (False, True))
@pytest.mark.parametrize("scale", (1.0, 0.6))
def test_distill_formula_is_the_gradient(tail, scale):
    x, w = _rand(4, 9), _rand(4, seed=2)
    index = torch.tensor([[0, 8, 3], [2, 2, 5], [-1, 4, 9], [-1, -1, -1]], dtype=torch.int32)
    values = torch.log_softmax(_rand(4, 3, seed=3), 1) - 0.4

    def value(x):
        return float((ref.distill(x, values, index, scale, 0.8, tail)["loss"] * w).sum())

    o = ref.distill(x, values, index, scale, 0.8, tail)
    got, _ = ref.distill_grad(x, values, index, o["peak"], o["logsum"], o.get("tail"), w, scale, 0.8, torch.float32)
    assert torch.allclose(got, _differences(value, x), rtol=1e-6, atol=1e-8)


def test_distill_is_a_divergence():
    # of the teacher's own logits: nothing, and no gradient; with a tail over all of the vocabulary's classes also
    x = _rand(3, 6)
    index = torch.arange(6, dtype=torch.int32).expand(3, 6)
    for tail in (False, True):
        values = torch.log_softmax(x, 1)
        o = ref.distill(x, values, index, 1.0, 1.0, tail)
        assert o["loss"].abs().max() < 1e-14
        got, _ = ref.distill_grad(x, values, index, o["peak"], o["logsum"], o.get("tail"), None, 1.0, 1.0, torch.float32)
        assert got.abs().max() < 1e-14
    o = ref.distill(x, torch.log_softmax(x, 1)[:, :2], index[:, :2], 1.0, 1.0, True)
    assert o["loss"].abs().max() < 1e-14


def test_alternatives_of_known_rows():
    x = torch.tensor([[1.0, 3.0, 3.0, -INF, 2.0], [-INF] * 5, [0.0, -0.0, 0.0, -0.0, 0.0]])
    assert ref.top(x, 7).tolist() == [[1, 2, 4, 0, -1, -1, -1], [-1] * 7, [0, 1, 2, 3, 4, -1, -1]]


# ------------------------------------------------------------------ refusals

def test_token_logprobs_refusals():
    x, t, lp, st = T((6, 40)), T((6,), I32), T((6,), F32), T((6,), F32)
    q = ewf.token_logprobs.workspace_bytes
    assert q(x, t, lp) == 0
    refused(ewf.EINVAL, "logits is needed", q, None, t, lp)
    refused(ewf.EINVAL, "a result is needed", q, x, t)
    refused(ewf.EINVAL, "comes with tokens", q, x, None, lp)
    refused(ewf.EINVAL, "come together", q, x, t, lp, top_values=T((6, 4), F32))
    refused(ewf.ESHAPE, "1 to 128", q, x, t, lp, top_values=T((6, 129), F32), top_indices=T((6, 129), I32))
    refused(ewf.ESHAPE, "1 to 128", q, x, t, lp, top_values=T((6, 0), F32), top_indices=T((6, 0), I32))
    refused(ewf.ESHAPE, "extent", q, x, t, lp, top_values=T((6, 4), F32), top_indices=T((6, 5), I32))
    refused(ewf.ESHAPE, "extent", q, x, t, lp, top_values=T((5, 4), F32), top_indices=T((6, 4), I32))
    refused(ewf.EUNSUPPORTED, "contiguous", q, x, t, lp, top_values=T((6, 4), F32, strides=(1, 6)), top_indices=T((6, 4), I32))
    refused(ewf.EUNSUPPORTED, "contiguous", q, T((6, 40), strides=(1, 6)), t, lp)
    refused(ewf.ESHAPE, "extent", q, x, T((7,), I32), lp)
    refused(ewf.ESHAPE, "rank", q, x, T((6, 1), I32), lp)
    refused(ewf.ETYPE, "int32", q, x, T((6,), F32), lp)
    refused(ewf.ETYPE, "float32", q, x, t, T((6,), F16))
    refused(ewf.ETYPE, "float32", q, T((6, 40), I32), t, lp)
    refused(ewf.ESHAPE, "1 to 2^24", q, T((6, 0)), t, lp)
    refused(ewf.ESHAPE, "1 to 2^24", q, T((1, (1 << 24) + 1)), T((1,), I32), T((1,), F32))
    for bad in (0.0, -1.0, float("nan"), INF, 1e-30, 1e30):
        refused(ewf.EINVAL, "scale", q, x, t, lp, scale=bad)
    refused(ewf.EALIAS, "logprob overlaps tokens", q, x, t, T((6,), F32, at=t.ptr))
    refused(ewf.EALIAS, "peak overlaps logprob", q, x, t, lp, peak=lp)
    refused(ewf.EALIAS, "share memory", q, x, t, T((6,), F32, strides=(0,)))
    refused(ewf.EALIAS, "top_indices overlaps top_values", q, x, t, lp, top_values=T((6, 4), F32, at=0x7A0000000000),
            top_indices=T((6, 4), I32, at=0x7A0000000000))
    refused(ewf.EINVAL, "null pointer", q, x, T((6,), I32, at=0), lp)
    refused(ewf.EINVAL, "aligned", q, T((6, 40), off=1), t, lp)
    a = T((3, 4, 5, 8))
    refused(ewf.EUNSUPPORTED, "merge", q, a, None, None, peak=T((3, 4, 5), F32, strides=(4000, 1, 400)))
    assert q(T((0, 40)), T((0,), I32), T((0,), F32)) == 0
    ewf.token_logprobs(T((0, 40)), T((0,), I32), T((0,), F32))
    # rows that several workgroups share
    n = q(T((1, 1 << 20)), T((1,), I32), T((1,), F32))
    assert n > 0 and q(T((1, 1 << 20)), T((1,), I32), T((1,), F32), top_values=T((1, 9), F32), top_indices=T((1, 9), I32)) > n
    refused(ewf.ENOMEM, "needed", ewf.token_logprobs, T((1, 1 << 20)), T((1,), I32), T((1,), F32))
    big = T((1, 1 << 20), F32), T((1,), I32), T((1,), F32)

    class Odd:
        def data_ptr(self): return 0x7D0000000008
        def numel(self): return 1 << 30
        def element_size(self): return 1
    refused(ewf.EINVAL, "16-byte", ewf.token_logprobs, *big, workspace=Odd())


def test_token_logprobs_grad_refusals():
    x, t, g, dx, st = T((6, 40)), T((6,), I32), T((6,), F32), T((6, 40)), T((6,), F32)
    f = ewf.token_logprobs_grad
    refused(ewf.EINVAL, "dlogprob or dentropy", f, x, t, None, dx, peak=st, logsum=st)
    refused(ewf.EINVAL, "comes with tokens", f, x, None, g, dx, peak=st, logsum=st)
    refused(ewf.EINVAL, "peak is needed", f, x, t, g, dx, peak=None, logsum=st)
    refused(ewf.EINVAL, "logsum is needed", f, x, t, g, dx, peak=st, logsum=None)
    refused(ewf.EINVAL, "entropy is needed", f, x, t, g, dx, peak=st, logsum=st, dentropy=g)
    refused(ewf.EINVAL, "dlogits is needed", f, x, t, g, None, peak=st, logsum=st)
    refused(ewf.ETYPE, "bfloat16", f, x, t, g, T((6, 40), F32), peak=st, logsum=st)
    refused(ewf.EALIAS, "dlogits overlaps logits", f, x, t, g, ewf.TensorRef(x.ptr + 2, x.shape, x.strides, BF16), peak=st, logsum=st)
    refused(ewf.EALIAS, "dlogits overlaps peak", f, x, t, g, T((6, 40), at=st.ptr), peak=st, logsum=T((6,), F32))
    refused(ewf.EINVAL, "scale", f, x, t, g, dx, peak=st, logsum=st, scale=0.0)
    f(T((0, 40)), T((0,), I32), T((0,), F32), T((0, 40)), peak=T((0,), F32), logsum=T((0,), F32))


def test_distill_refusals():
    x, v, i, loss, st, dx = T((6, 40)), T((6, 4), F32), T((6, 4), I32), T((6,), F32), T((6,), F32), T((6, 40))
    q = ewf.distill.workspace_bytes
    assert q(x, v, i, loss) == 0 and q(x, v, i, loss, dlogits=dx) == 0 and q(x, T((6, 4)), i, loss, dlogits=x) == 0
    refused(ewf.EINVAL, "teacher_values is needed", q, x, None, i, loss)
    refused(ewf.EINVAL, "teacher_indices is needed", q, x, v, None, loss)
    refused(ewf.EINVAL, "loss is needed", q, x, v, i, None)
    refused(ewf.EINVAL, "dloss comes with dlogits", q, x, v, i, loss, dloss=st)
    refused(ewf.ETYPE, "teacher", q, x, T((6, 4), F16), i, loss)
    refused(ewf.ETYPE, "int32", q, x, v, T((6, 4), F32), loss)
    refused(ewf.ESHAPE, "1 to 128", q, x, T((6, 129), F32), T((6, 129), I32), loss)
    refused(ewf.ESHAPE, "extent", q, x, v, T((6, 5), I32), loss)
    refused(ewf.ESHAPE, "rank", q, x, T((4,), F32), i, loss)
    refused(ewf.EUNSUPPORTED, "contiguous", q, x, T((6, 4), F32, strides=(1, 6)), i, loss)
    for bad in (0.0, float("nan"), -2.0, 1e30):
        refused(ewf.EINVAL, "scale", q, x, v, i, loss, scale=bad)
        refused(ewf.EINVAL, "teacher_scale", q, x, v, i, loss, teacher_scale=bad)
    refused(ewf.EALIAS, "loss overlaps teacher_values", q, x, v, i, T((6,), F32, at=v.ptr))
    refused(ewf.EALIAS, "tail overlaps loss", q, x, v, i, loss, tail=loss)
    refused(ewf.EALIAS, "dlogits overlaps teacher_indices", q, x, v, i, loss, dlogits=T((6, 40), at=i.ptr))
    refused(ewf.EALIAS, "dlogits overlaps logits", q, x, v, i, loss, dlogits=ewf.TensorRef(x.ptr + 2, x.shape, x.strides, BF16))
    # rows whose gradient is a launch of its own
    long = T((300, 400000)), T((300, 4), F32), T((300, 4), I32), T((300,), F32)
    assert q(*long) == 0 and q(*long, dlogits=T((300, 400000))) > 0
    g = ewf.distill_grad
    refused(ewf.EINVAL, "peak is needed", g, x, v, i, dx, peak=None, logsum=st)
    refused(ewf.EINVAL, "dlogits is needed", g, x, v, i, None, peak=st, logsum=st)
    refused(ewf.EALIAS, "dlogits overlaps peak", g, x, v, i, T((6, 40), at=st.ptr), peak=st, logsum=T((6,), F32))
    refused(ewf.ENOMEM, "needed", g, x, v, i, dx, peak=st, logsum=T((6,), F32))
    assert g.workspace_bytes(x, v, i, dx, peak=st, logsum=T((6,), F32)) > 0
    ewf.distill(T((0, 40)), T((0, 4), F32), T((0, 4), I32), T((0,), F32), dlogits=T((0, 40)))


def test_reserved_words_and_null_arguments():
    lib, by = ewf._lib, ewf.ctypes.byref
    f = ewf._token_logprobs(T((2, 8)), T((2,), I32), T((2,), F32))
    f.args.reserved = 1
    assert lib.ewf_token_logprobs(by(f.args), None, 0, None) == ewf.EINVAL
    f = ewf._distill(T((2, 8)), T((2, 3), F32), T((2, 3), I32), T((2,), F32))
    f.args.reserved = 1
    assert lib.ewf_distill(by(f.args), None, 0, None) == ewf.EINVAL
    f.args.reserved, f.args.dtype = 0, 77
    assert lib.ewf_distill(by(f.args), None, 0, None) == ewf.ETYPE
    for call in (lib.ewf_token_logprobs, lib.ewf_distill, lib.ewf_distill_grad):
        assert call(None, None, 0, None) == ewf.EINVAL
    assert lib.ewf_token_logprobs_grad(None, None) == ewf.EINVAL
    assert lib.ewf_distill_grad_workspace(None, None) == ewf.EINVAL
    assert lib.ewf_token_logprobs_workspace(None, None) == ewf.EINVAL and lib.ewf_distill_workspace(None, None) == ewf.EINVAL
    f = ewf._token_logprobs(T((2, 8)), T((2,), I32), T((2,), F32))
    assert lib.ewf_token_logprobs_workspace(by(f.args), None) == ewf.EINVAL
    f.args.ndim = 9
    assert lib.ewf_token_logprobs(by(f.args), None, 0, None) == ewf.EINVAL


def test_tensors_outside_device_memory_are_refused():
    x = torch.zeros(2, 8)
    refused(ewf.EINVAL, "device memory", ewf.token_logprobs, x, None, None, peak=torch.zeros(2))
    refused(ewf.EINVAL, "device memory", ewf.distill, x, torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2))
