"""The operators over a vocabulary where a sum or an offset is longest: the longest rows that one wavefront takes, and the gradient alone beyond 2^31 logits."""
import pytest
import torch

from paper_1605_02688_amd import ewf
from tests.test_gpu_vocab import check_distilled, check_scored, distilled, gen, run, say, scored
from tests.test_gpu_vocab_masks import longest_chain  # noqa: F401

pytestmark = pytest.mark.gpu


def test_single_wavefronts_take_the_longest_rows_that_they_may():
    rows, cols = 1300, 16384
    g = gen(17)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * 3).to(torch.bfloat16)
    say("one wavefront", rows, cols)
    check_scored(x, None, scored(x, None), 1.0)


def test_the_gradient_alone_of_more_than_2_31_logits():
    rows, cols, bf, k = 17000, 131072, torch.bfloat16, 20
    g = gen(92)
    x = torch.empty(rows, cols, dtype=bf, device="cuda")
    for r in range(0, rows, 1000):
        x[r:r + 1000] = torch.randn(min(1000, rows - r), cols, generator=g, device="cuda") * 3
    values = torch.log_softmax(torch.randn(rows, k, generator=g, device="cuda"), 1) - 0.5
    index = torch.randint(0, cols, (rows, k), generator=g, device="cuda").to(torch.int32)
    dloss = torch.randn(rows, generator=g, device="cuda")
    say("gradient alone, more than 2^31", rows, cols)
    got, _ = distilled(x, values, index, True, gradient=False)
    parts = (slice(0, 3), slice(8191, 8193), slice(16383, 16387), slice(rows - 3, rows))
    before = [x[p].clone() for p in parts]
    run(ewf.distill_grad, x, values, index, x, peak=got["peak"], logsum=got["logsum"], tail=got["tail"], dloss=dloss)
    for p, y in zip(parts, before):
        check_distilled(y, values[p], index[p], True, {n: t[p] for n, t in got.items()}, x[p], 1.0, 1.0, dloss[p])
    del x
    torch.cuda.empty_cache()
