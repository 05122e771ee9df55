"""The operators over a vocabulary on rows of which a part is masked by finite numbers (-1e9, -1e30, the type's lowest one and the like), against the formulas in
64 bits: every workgroup size and form, masks before, behind and between the ordinary logits."""
import pytest
import torch

import tests.vocab_ref as ref
from paper_1605_02688_amd import ewf
from tests.test_gpu_vocab import DT, check_distilled, check_scored, distilled, entries_of, gen, run, say, scored

pytestmark = pytest.mark.gpu
MASKS = {"f32": (-1e4, -3e6, -1e9, -3e9, -1e10, -1e12, -1e20, -1e25, -1e30, -1e37, -1.7e38, -3.4028234e38),
         "bf16": (-1e4, -3e6, -1e9, -3e9, -1e10, -1e12, -1e20, -1e25, -1e30, -1e37, -1.7e38, -3.3895313e38),
         "f16": (-3e4, -5e4, -6e4, -65504.0)}
# (float16's masks are far from its logits only at low temperatures, where the logits are small)
SCALES = {"f32": (0.1, 0.5, 0.7, 1.0, 1.25), "bf16": (0.1, 0.5, 0.7, 1.0, 1.25), "f16": (2.0 ** 17, 3e5)}
CASES = [(dtype, scale) for dtype in sorted(DT) for scale in SCALES[dtype]]


@pytest.fixture(autouse=True)
def longest_chain(monkeypatch):
    """Additions that a row's sum passes through where one wavefront may take it (up to 2048 vectors, 16384 logits): a lane's own, and the rest as
    tests/vocab_ref.py counts it."""
    monkeypatch.setattr(ref, "chain", lambda cols: 100 + (cols // 64 if cols <= 16384 else cols // 256))


def masked(g, rows, cols, dtype, scale):
    """Ordinary logits (one at least) and masks, kinds and depths in turn."""
    at = torch.arange(cols, device="cuda")
    vec = 16 // DT[dtype].itemsize
    kinds = torch.stack([at < cols - max(1, cols // 8), at >= max(1, cols // 4), at // vec % 2 == 0, at != cols // 2, at // (256 * vec) % 2 == 0,
                         at % 64 >= 3, torch.rand(cols, generator=g, device="cuda") < 0.9])
    r = torch.arange(rows, device="cuda")
    depth = torch.tensor(MASKS[dtype], dtype=torch.float32, device="cuda")[r // len(kinds) % len(MASKS[dtype])]
    gone = kinds[r % len(kinds)]
    gone[:, cols // 2] = False
    x = torch.randn(rows, cols, generator=g, device="cuda") * 3.0 / (scale if dtype == "f16" else 1.0)
    mask = depth.unsqueeze(1).expand(rows, cols)
    # in some rows of two depths
    mask = torch.where((r % 5 == 3).unsqueeze(1) & (torch.rand(rows, cols, generator=g, device="cuda") < 0.5), mask * 0.37, mask)
    return torch.where(gone, mask, x).to(DT[dtype]), gone


def cols_of(dtype, vectors):
    return vectors * 16 // DT[dtype].itemsize - 3


@pytest.mark.parametrize("dtype,scale", CASES)
@pytest.mark.parametrize("rows,vectors,k", ((84, 2, 3), (84, 40, 0), (84, 40, 20), (84, 200, 128), (84, 1000, 0), (84, 1000, 20), (1100, 1500, 0), (1100, 2048, 0), (300, 5000, 64),
                                            (84, 13000, 0), (84, 13000, 20), (2, 30000, 5), (300, 13000, 0)))
def test_log_probabilities_beside_finite_masks(dtype, scale, rows, vectors, k):
    cols = cols_of(dtype, vectors)
    say("finite masks", dtype, scale, rows, cols, k)
    g = gen(rows + cols + k)
    x, gone = masked(g, rows, cols, dtype, scale)
    tokens = torch.randint(0, cols, (rows,), generator=g, device="cuda")
    tokens = torch.where(torch.arange(rows, device="cuda") % 3 == 0, tokens, x.float().argmax(1)).to(torch.int32)
    tokens[5::11] = -1
    for entropy in (True, False):
        out = scored(x, tokens, scale, k, entropy=entropy)
        assert not any(torch.isnan(t).any() for t in out.values())
        check_scored(x, tokens, out, scale, k)
    out = scored(x, tokens, scale)
    gp, ge = torch.randn(rows, generator=g, device="cuda") / scale, torch.randn(rows, generator=g, device="cuda") / scale
    for h in (ge, None):
        dx = torch.full_like(x, 77)
        run(ewf.token_logprobs_grad, x, tokens, gp, dx, peak=out["peak"], logsum=out["logsum"], entropy=out["entropy"], dentropy=h, scale=scale)
        want, bound = ref.token_logprobs_grad(x, tokens, gp, h, out["peak"], out["logsum"], out["entropy"], scale, DT[dtype])
        ref.close("dlogits", dx, want, bound)
        # nothing goes to a masked logit but a token's own
        mine = torch.zeros_like(gone).scatter_(1, tokens.clamp_min(0).long().unsqueeze(1), True)
        assert ((dx == 0) | ~gone | mine | (x.double() * scale > -2e4)).all()


# every size that is held in registers, by one wavefront and by several, and the ones that are not
HELD = ((84, 3), (84, 60), (84, 100), (1100, 100), (1100, 250), (2100, 500), (2100, 1000), (84, 1000), (84, 2000), (84, 4000), (84, 6000), (84, 8000), (84, 12000), (84, 16000),
        (84, 17000), (260, 17000))


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows,vectors", HELD)
@pytest.mark.parametrize("tail", (False, True))
def test_distillation_beside_finite_masks(dtype, rows, vectors, tail):
    cols = cols_of(dtype, vectors)
    for scale, k in ((SCALES[dtype][0], 20), (SCALES[dtype][-1], 100), (1.0 if dtype != "f16" else SCALES[dtype][0], 5)):
        k = min(k, cols)
        say("distill, finite masks", dtype, scale, rows, cols, k, tail)
        g = gen(rows + cols + k)
        x, gone = masked(g, rows, cols, dtype, scale)
        values, index = entries_of(g, torch.where(gone, -50.0, x.float() * scale), k, tail)
        dloss = torch.randn(rows, generator=g, device="cuda") / scale
        # (an entry at a masked logit counts with its small probability and a large loss, but not where that may leave float32)
        values = torch.where(x.gather(1, index.long()) < -1e38, values - 300.0, values)
        loss, _ = distilled(x, values, index, tail, scale, gradient=False)
        check_distilled(x, values, index, tail, loss, None, scale, 1.0, None)
        both, dx = distilled(x, values, index, tail, scale, 1.0, dloss)
        assert not any(torch.isnan(t).any() for t in both.values()) and not torch.isnan(dx).any()
        check_distilled(x, values, index, tail, both, dx, scale, 1.0, dloss)
        alone = torch.full_like(x, 77)
        run(ewf.distill_grad, x, values, index, alone, peak=both["peak"], logsum=both["logsum"], tail=both.get("tail"), dloss=dloss, scale=scale)
        check_distilled(x, values, index, tail, both, alone, scale, 1.0, dloss)


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("rows,vectors", HELD)
def test_entries_that_name_all_that_is_not_masked(dtype, rows, vectors):
    # behind the entries only masks are left: the tail lies far below them, and does not count
    cols, scale = cols_of(dtype, vectors), 0.5
    say("all named", dtype, rows, cols)
    g = gen(rows + cols)
    k = min(6, cols)
    x = torch.tensor(MASKS[dtype], device="cuda")[torch.arange(rows, device="cuda") % len(MASKS[dtype])].unsqueeze(1).expand(rows, cols).to(DT[dtype]).clone()
    index = torch.rand(rows, cols, generator=g, device="cuda").topk(k, 1).indices
    x.scatter_(1, index, torch.randn(rows, k, generator=g, device="cuda").to(x.dtype) * 3)
    values = torch.log_softmax(torch.randn(rows, k, generator=g, device="cuda"), 1) - 0.1
    index = index.to(torch.int32)
    both, dx = distilled(x, values, index, True, scale, 1.0, None)
    assert not torch.isnan(dx).any() and torch.isfinite(both["loss"]).all()
    check_distilled(x, values, index, True, both, dx, scale, 1.0, None)
    alone = torch.full_like(x, 77)
    run(ewf.distill_grad, x, values, index, alone, peak=both["peak"], logsum=both["logsum"], tail=both["tail"], scale=scale)
    check_distilled(x, values, index, True, both, alone, scale, 1.0, None)


@pytest.mark.parametrize("scale", (1.0, 0.1, 2.0 ** 20))
@pytest.mark.parametrize("rows,vectors,k", ((84, 40, 5), (84, 1000, 5), (1100, 1500, 0), (84, 13000, 20)))
def test_rows_about_the_lowest_point(scale, rows, vectors, k):
    # lanes, wavefronts and parts each side of the logits from which on sums are taken about a whole number of powers of two, and rows that cross it
    cols = cols_of("f32", vectors)
    say("lowest point", scale, rows, cols, k)
    g = gen(cols)
    c = scale * 1.44269504
    step = torch.tensor([-300.0, -40.0, -9.0, -1.0, 0.0, 1.0, 9.0, 40.0, 300.0], device="cuda", dtype=torch.float64)[torch.arange(rows, device="cuda") % 9]
    for sign in (-1.0, 1.0):
        t = sign * 2.0 ** 22 + step.unsqueeze(1) + torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.float64) * 20.0
        t -= torch.rand(rows, 16, generator=g, device="cuda", dtype=torch.float64).mul_(60.0).repeat_interleave((cols + 15) // 16, 1)[:, :cols]
        x = (t / c).float()
        out = scored(x, None, scale, k)
        check_scored(x, None, out, scale, k)
        values, index = entries_of(g, x - x.amax(1, keepdim=True), 20, True)
        values = torch.log_softmax(values, 1) - 0.5
        got, dx = distilled(x, values, index, True, scale)
        check_distilled(x, values, index, True, got, dx, scale, 1.0, None)
