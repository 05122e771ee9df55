"""The operators of sequence models on the GPU against the formulas in 64 bits (tests/operators_ref.py, which also
derives the bounds): sizes around every row shape and tile, strides, masks of lengths, values that are not finite, calls in
place, on other streams and in captured graphs."""
import pytest
import torch

import tests.operators_ref as ref
from paper_1605_02688_amd import ewf

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def stream():
    return torch.cuda.current_stream().cuda_stream


def say(*words):
    print("[case]", *words, flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, mean=0.0, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


def work_for(op, *args, **kw):
    n = op.workspace_bytes(*args, **kw)
    return torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda") if n else None


def run(op, *args, **kw):
    op(*args, workspace=work_for(op, *args, **kw), stream=stream(), **kw)


# ------------------------------------------------------------------ layer normalisation

# each side of: one vector, the threads of a row with one, two and four vectors, whole and cut vectors
NORM_COLS = (1, 2, 3, 7, 8, 9, 31, 32, 33, 64, 100, 128, 129, 256, 257, 300, 512, 513, 600, 1000, 1024, 1025, 1152, 1300, 2048, 2049, 2304,
             4096, 4097, 4608, 6144, 8192, 8199, 10000, 12001, 16384, 16390, 32768, 32771, 40005)


def norm_case(g, rows, cols, dtype, params):
    x = randn(g, rows, cols, mean=0.3, std=1.7, dtype=dtype)
    pt = dtype if params == "own" else torch.float32
    w, b = (None, None) if params == "none" else (randn(g, cols, mean=1, std=0.3, dtype=pt), randn(g, cols, std=0.3, dtype=pt))
    return x, w, b, pt


def check_norm(x, w, b, y, mean, rstd, eps=1e-5):
    want = ref.layer_norm(x, w, b, eps, y.dtype)
    ref.close("y", y, want["y"], want["e_y"])
    if mean is not None:
        ref.close("mean", mean, want["mean"], want["e_mean"])
        ref.close("rstd", rstd, want["rstd"], want["e_rstd"])
    return want


def check_norm_grad(dy, x, w, mean, rstd, dx, dw, db, pt, n=None):
    if n is None:
        n = (x.double() - mean.double().unsqueeze(-1)) * rstd.double().unsqueeze(-1)
        e_n = 2 * ref.U * n.abs()
    else:
        e_n = 0.0
    want = ref.layer_norm_grad(dy, w, n, rstd, e_n, dx.dtype, pt)
    ref.close("dx", dx.reshape(want["dx"].shape), want["dx"], want["e_dx"])
    if dw is not None:
        ref.close("dweight", dw, want["dw"], want["e_dw"])
        ref.close("dbias", db, want["db"], want["e_db"])


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", NORM_COLS)
def test_layer_norm_and_its_gradient(dtype, cols):
    dt = DT[dtype]
    for rows, params in ((1, "own"), (5, "f32"), (67, "none") if cols < 9000 else (3, "none")):
        say("layer norm", dtype, rows, cols, params)
        g = gen(cols * 7 + rows)
        x, w, b, pt = norm_case(g, rows, cols, dt, params)
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        run(ewf.layer_norm, x, w, b, y, mean=mean, rstd=rstd)
        check_norm(x, w, b, y, mean, rstd)
        dy = randn(g, rows, cols, dtype=dt)
        dx, dw, db = torch.empty_like(x), torch.empty(cols, dtype=pt, device="cuda"), torch.empty(cols, dtype=pt, device="cuda")
        run(ewf.layer_norm_grad, dy, w, rstd, dx, x=x, mean=mean, dweight=dw, dbias=db)
        check_norm_grad(dy, x, w, mean, rstd, dx, dw, db, pt)


@pytest.mark.parametrize("dtype,rows,cols", (("bf16", 4099, 1001), ("f16", 20011, 72), ("f32", 3001, 260), ("bf16", 1500, 4096), ("f32", 66000, 8),
                                             ("f16", 700, 16392)))
def test_layer_norm_gradient_over_many_rows(dtype, rows, cols):
    say("layer norm gradient", dtype, rows, cols)
    dt, g = DT[dtype], gen(3)
    x, w, b, pt = norm_case(g, rows, cols, dt, "f32")
    dy, dx = randn(g, rows, cols, dtype=dt), torch.empty_like(x)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    run(ewf.layer_norm, x, w, b, y, mean=mean, rstd=rstd)
    check_norm(x, w, b, y, mean, rstd)
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    run(ewf.layer_norm_grad, dy, w, rstd, dx, x=x, mean=mean, dweight=dw, dbias=db)
    check_norm_grad(dy, x, w, mean, rstd, dx, dw, db, pt)
    again = [torch.empty_like(t) for t in (dx, dw, db)]
    run(ewf.layer_norm_grad, dy, w, rstd, again[0], x=x, mean=mean, dweight=again[1], dbias=again[2])
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))
    only = torch.empty(cols, device="cuda")
    run(ewf.layer_norm_grad, dy, w, rstd, dx, x=x, mean=mean, dbias=only)
    assert torch.equal(only, db)


def test_layer_norm_far_from_zero_and_without_spread():
    # a mean a thousand deviations away, one element that dwarfs its row, rows of one value
    g = gen(5)
    for cols in (33, 1000, 4096, 20000):
        x = randn(g, 6, cols, mean=1000.0)
        x[1] = 3.0
        x[2, cols // 2] = 1e6
        x[3] = 0.0
        y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
        run(ewf.layer_norm, x, None, None, y, mean=mean, rstd=rstd)
        check_norm(x, None, None, y, mean, rstd)


def test_layer_norm_of_rows_that_are_not_finite():
    x = torch.randn(4, 1000, device="cuda")
    x[1, 7] = float("nan")
    x[2, 999] = float("inf")
    y = torch.empty_like(x)
    run(ewf.layer_norm, x, None, None, y)
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 999]) and torch.isfinite(y[0]).all() and torch.isfinite(y[3]).all()


@pytest.mark.parametrize("dtype", sorted(DT))
def test_layer_norm_strides_and_in_place(dtype):
    dt, g = DT[dtype], gen(6)
    for cols in (40, 129, 1000):
        say("strides", dtype, cols)
        wide = randn(g, 5, 6, 2 * cols + 3, dtype=dt)
        x = wide[:, :, 1:cols + 1]                                   # rows that begin at odd elements
        xt = x.transpose(0, 1)                                       # [6, 5, cols]: two axes
        w, b = randn(g, cols), randn(g, cols)
        out = torch.full((6, 5, cols + 5), 7.0, dtype=dt, device="cuda")
        y = out[:, :, 2:cols + 2]
        stats = torch.full((6, 10), 7.0, device="cuda")
        mean, rstd = stats[:, :5], stats[:, 5:]
        run(ewf.layer_norm, xt, w, b, y, mean=mean, rstd=rstd)
        check_norm(xt, w, b, y, mean, rstd)
        assert (out[:, :, :2] == 7).all() and (out[:, :, cols + 2:] == 7).all()
        dy, dx = randn(g, 6, 5, cols, dtype=dt), torch.empty(6, 5, cols, dtype=dt, device="cuda")
        dw, db = torch.empty_like(w), torch.empty_like(b)
        run(ewf.layer_norm_grad, dy, w, rstd, dx, x=xt, mean=mean, dweight=dw, dbias=db)
        check_norm_grad(dy, xt, w, mean.contiguous(), rstd.contiguous(), dx, dw, db, torch.float32)
        # a gradient that is the same for every row; over dy, over x; y over x; one row alone
        same = randn(g, cols, dtype=dt).expand(6, 5, cols)
        run(ewf.layer_norm_grad, same, w, rstd, dx, x=xt, mean=mean, dweight=dw, dbias=db)
        check_norm_grad(same, xt, w, mean.contiguous(), rstd.contiguous(), dx, dw, db, torch.float32)
        for over in ("dy", "x"):
            d, xx = dy.clone(), xt.contiguous()
            run(ewf.layer_norm_grad, dy, w, rstd, dx, x=xx, mean=mean, dweight=dw, dbias=db)
            target = d if over == "dy" else xx
            ow, ob = torch.empty_like(w), torch.empty_like(b)
            run(ewf.layer_norm_grad, d, w, rstd, target, x=xx, mean=mean, dweight=ow, dbias=ob)
            assert torch.equal(target, dx) and torch.equal(ow, dw) and torch.equal(ob, db)
        xx, yy = xt.contiguous(), torch.empty(6, 5, cols, dtype=dt, device="cuda")
        run(ewf.layer_norm, xx, w, b, yy)
        run(ewf.layer_norm, xx, w, b, xx)
        assert torch.equal(xx, yy)
        one = x[0, 0]
        y1, m1, r1 = torch.empty(cols, dtype=dt, device="cuda"), torch.empty((), device="cuda"), torch.empty((), device="cuda")
        run(ewf.layer_norm, one, w, b, y1, mean=m1, rstd=r1)
        check_norm(one, w, b, y1, m1, r1)


def test_layer_norm_gradient_in_place_on_long_rows():
    g = gen(8)
    x, dy = randn(g, 3, 40005), randn(g, 3, 40005)
    mean, rstd = x.mean(1), torch.rsqrt(x.var(1, correction=0) + 1e-5)
    dx, dw, db = torch.empty_like(x), torch.empty(40005, device="cuda"), torch.empty(40005, device="cuda")
    run(ewf.layer_norm_grad, dy, None, rstd, dx, x=x, mean=mean, dweight=dw, dbias=db)
    ow, ob = torch.empty_like(dw), torch.empty_like(db)
    run(ewf.layer_norm_grad, dy, None, rstd, x, x=x, mean=mean, dweight=ow, dbias=ob)
    assert torch.equal(x, dx) and torch.equal(ow, dw) and torch.equal(ob, db)


def test_layer_norm_of_no_rows():
    x = torch.empty(0, 40, device="cuda")
    dw, db = torch.full((40,), 3.0, device="cuda"), torch.full((40,), 3.0, device="cuda")
    run(ewf.layer_norm, x, None, None, x)
    run(ewf.layer_norm_grad, x, None, torch.empty(0, device="cuda"), torch.empty_like(x), x=torch.empty_like(x),
        mean=torch.empty(0, device="cuda"), dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("cols", (1, 3, 5, 7, 8, 15, 20, 24, 41, 136, 1001, 1032, 1300, 4100, 8199, 40005))
def test_layer_norm_gradient_of_large_rows_of_one_value(dtype, cols):
    # n is 0 throughout and -mean rstd, what a zero behind the row's end would have for it, infinite
    dt, g = DT[dtype], gen(cols)
    x = torch.full((5, cols), 4e36, dtype=dt, device="cuda")
    x[1], x[3] = -4e36, 1.0
    mean, rstd = x[:, 0].float(), torch.full((5,), 1e-5 ** -0.5, device="cuda")
    dy, w = randn(g, 5, cols, dtype=dt), randn(g, cols)
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    run(ewf.layer_norm_grad, dy, w, rstd, dx, x=x, mean=mean, dweight=dw, dbias=db)
    assert torch.isfinite(dx).all() and (dw == 0).all()
    check_norm_grad(dy, x, w, mean, rstd, dx, dw, db, torch.float32)


@pytest.mark.parametrize("dtype,rows,cols", (("bf16", 300, 1024), ("f16", 300, 1001), ("bf16", 9, 14171), ("f32", 700, 20), ("f32", 3, 40005)))
def test_layer_norm_gradient_without_sums_leaves_a_workspace_alone(dtype, rows, cols):
    # dx alone needs none: one that a program hands to every call may be of any size and alignment
    say("dx alone", dtype, rows, cols)
    dt, g = DT[dtype], gen(9)
    x, dy, w = randn(g, rows, cols, dtype=dt), randn(g, rows, cols, dtype=dt), randn(g, cols)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    codes = torch.empty((rows, cols), dtype=torch.int8, device="cuda")
    scales = torch.empty((rows, (cols + 31) // 32), dtype=torch.uint8, device="cuda")
    ewf.keep8(x, codes, scales, stream=stream())
    for source in (dict(x=x, mean=mean), dict(codes=codes, scales=scales)):
        want, dx = torch.empty_like(x), torch.empty_like(x)
        assert ewf.layer_norm_grad.workspace_bytes(dy, w, rstd, want, **source) == 0
        ewf.layer_norm_grad(dy, w, rstd, want, stream=stream(), **source)
        whole = torch.full((64 << 20,), 0x5A, dtype=torch.uint8, device="cuda")
        for part in (whole[4096:4160], whole[4097:4098]):
            ewf.layer_norm_grad(dy, w, rstd, dx, workspace=part, stream=stream(), **source)
            assert torch.equal(dx, want) and (whole == 0x5A).all()


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype", sorted(DT))
def test_layer_norm_kept_in_8_bits(dtype, kind):
    dt = DT[dtype]
    for rows, cols in ((1, 1), (3, 7), (5, 33), (130, 64), (9, 1001), (6, 2048), (3, 4097), (2, 16400), (2, 40005)):
        say("kept", dtype, kind, rows, cols)
        g = gen(cols + rows)
        x, w, b, pt = norm_case(g, rows, cols, dt, "own")
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        codes = torch.empty((rows, cols), dtype=CODES[kind], device="cuda")
        scales = torch.full((rows, (cols + 31) // 32), 99, dtype=torch.uint8, device="cuda")
        run(ewf.layer_norm, x, w, b, y, mean=mean, rstd=rstd, codes=codes, scales=scales)
        want = check_norm(x, w, b, y, mean, rstd)
        n8 = torch.empty((rows, cols), device="cuda")
        run(ewf.read8, codes, scales, n8)
        # within half a step of the grid at n, and what n itself is off by.  The block's unit may be the next power where its
        # largest element is within that of the border; the grid's steps are then twice as wide
        _, byte, _, unit = ref.keep8(want["n"], kind)
        step = unit if kind == "i8" else unit * ref.e4m3_step(want["n"] / unit)
        exact_unit = (byte == scales).all()
        ref.close("n", n8, want["n"], (0.5 if exact_unit else 1.0) * step * (1 + 1e-6) + 2 * want["e_n"] + (step if kind == "e4m3" else 0) * 1e-3)
        assert ((scales.int() - byte.int()).abs() <= 1).all()
        dy, dx = randn(g, rows, cols, dtype=dt), torch.empty_like(x)
        dw, db = torch.empty(cols, dtype=pt, device="cuda"), torch.empty(cols, dtype=pt, device="cuda")
        run(ewf.layer_norm_grad, dy, w, rstd, dx, codes=codes, scales=scales, dweight=dw, dbias=db)
        check_norm_grad(dy, None, w, None, rstd, dx, dw, db, pt, n=n8)


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", (1, 8, 33, 64, 136, 300, 1000, 1001, 1400, 2048, 4097, 4608, 8192, 8199, 12000, 16384, 20000, 40005))
def test_layer_norm_kept_in_8_bits_block_by_block(cols, dtype, kind):
    # A scale is that of n's block in 64 bits, but where the block's largest n lies within its own error of a border; a code is n's, but
    # where n lies within its error of half a step
    dt, rows, g = DT[dtype], 5, gen(cols)
    x = randn(g, rows, cols, mean=0.3, std=1.7, dtype=dt)
    x[1] *= torch.exp2(torch.arange(cols, device="cuda") % 64 // 4 - 8.0).to(dt)          # blocks of different powers in a row
    y = torch.empty_like(x)
    codes = torch.empty((rows, cols), dtype=CODES[kind], device="cuda")
    scales = torch.full((rows, (cols + 31) // 32), 99, dtype=torch.uint8, device="cuda")
    run(ewf.layer_norm, x, None, None, y, codes=codes, scales=scales)
    want = ref.layer_norm(x, None, None, 1e-5, dt)
    n, e = want["n"], want["e_n"]
    lo, hi = (ref.keep8(torch.clamp_min(n.abs() + s * e, 0.0), kind)[1].int() for s in (-1, 1))
    got = scales.int()
    assert ((lo <= got) & (got <= hi)).all()
    assert float((lo == hi).double().mean()) > 0.9 or cols < 64
    unit = ref.pow2(got - 127).repeat_interleave(32, -1)[:, :cols]
    step = unit if kind == "i8" else unit * ref.e4m3_step(torch.maximum(n.abs() + e, codes.double().abs() * unit) / unit)
    ref.close("codes", codes.double() * unit, n, 0.5 * step + e)


# ------------------------------------------------------------------ activations in 8 bits

def special_values(dt):
    if dt == torch.float32:
        x = torch.tensor([0.0, -0.0, 1e-45, -1e-40, 2.0 ** -126, 3.4e38, -3.4e38, 1.0, 127.0, 127.0000076, 448.0, 449.0, 1e-30])
        return x.cuda()
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(dt).cuda()
    return x[torch.isfinite(x)]


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype", sorted(DT))
def test_codes_to_the_bit(dtype, kind):
    dt, g = DT[dtype], gen(11)
    v = special_values(dt)
    cases = {"values": v[: v.numel() // 32 * 32].reshape(-1, 32) if v.numel() >= 64 else v[None],
             # every value alone beside a magnitude that sets the block's power
             "random": randn(g, 200, 1003, std=3, dtype=dt), "wide": (randn(g, 64, 96) * torch.exp2(randn(g, 64, 96, std=12 if dtype != "f16" else 3))).to(dt),
             "one": randn(g, 3, 1, dtype=dt), "short": randn(g, 70, 31, dtype=dt), "ties": (torch.arange(-508, 509, device="cuda") / 4).to(dt)[None].repeat(3, 1),
             "grid": torch.cat((torch.arange(-1792, 1793, device="cuda") / 4, torch.arange(-64, 65, device="cuda") / 2048)).to(dt)[None]}
    for name, x in cases.items():
        say("codes", dtype, kind, name, tuple(x.shape))
        rows, cols = x.shape
        codes = torch.empty((rows, cols), dtype=CODES[kind], device="cuda")
        scales = torch.full((rows, (cols + 31) // 32), 99, dtype=torch.uint8, device="cuda")
        ewf.keep8(x, codes, scales, stream=stream())
        code, byte, value, _ = ref.keep8(x, kind)
        assert torch.equal(scales, byte)
        assert torch.equal(codes.float().double(), code)
        back = torch.empty((rows, cols), device="cuda")
        ewf.read8(codes, scales, back, stream=stream())
        assert torch.equal(back, value.float())              # (2^128, which the largest floats round to, is an infinity)
        own = torch.empty_like(x)
        ewf.read8(codes, scales, own, stream=stream())
        assert torch.equal(own, back.to(dt))


@pytest.mark.parametrize("kind", sorted(CODES))
def test_blocks_that_are_not_finite(kind):
    x = torch.randn(4, 100, device="cuda")
    x[0, 40] = float("nan")
    x[1, 0] = float("inf")
    x[3, 99] = -float("inf")
    codes = torch.empty((4, 100), dtype=CODES[kind], device="cuda")
    scales = torch.empty((4, 4), dtype=torch.uint8, device="cuda")
    ewf.keep8(x, codes, scales, stream=stream())
    code, byte, value, _ = ref.keep8(x, kind)
    assert torch.equal(scales, byte) and torch.equal(codes.float().double(), code)
    back = torch.empty_like(x)
    ewf.read8(codes, scales, back, stream=stream())
    assert torch.equal(torch.isnan(back), torch.isnan(value)) and int(torch.isnan(back).sum()) == 32 + 32 + 4
    for act in ewf.ACTIVATIONS:
        dx = torch.empty_like(x)
        ewf.activation_grad(act, torch.ones_like(x), dx, codes=codes, scales=scales, stream=stream())
        assert torch.equal(torch.isnan(dx), torch.isnan(value)), act


@pytest.mark.parametrize("act", sorted(ewf.ACTIVATIONS))
@pytest.mark.parametrize("dtype", sorted(DT))
def test_activation_and_its_gradient(dtype, act):
    dt, g = DT[dtype], gen(13)
    value, slope = ref.ACTS[act]
    for kind, rows, cols in (("i8", 1, 1), ("e4m3", 1, 8), ("i8", 65, 33), ("e4m3", 7, 1000), ("i8", 129, 1003), ("e4m3", 64, 4096), ("i8", 2, 100001)):
        say("activation", act, dtype, kind, rows, cols)
        x, dy = randn(g, rows, cols, std=3, dtype=dt), randn(g, rows, cols, dtype=dt)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        codes = torch.empty((rows, cols), dtype=CODES[kind], device="cuda")
        scales = torch.empty((rows, (cols + 31) // 32), dtype=torch.uint8, device="cuda")
        ewf.activation(act, x, y, codes=codes, scales=scales, stream=stream())
        ev, _ = ref.act_bounds(act, x.double())
        want = value(x.double())
        ref.close("y", y, want, ref.stored(ev, want, dt))
        _, byte, x8, _ = ref.keep8(x, kind)
        assert torch.equal(scales, byte)
        ewf.activation_grad(act, dy, dx, codes=codes, scales=scales, stream=stream())
        _, es = ref.act_bounds(act, x8)
        want = dy.double() * slope(x8)
        ref.close("dx", dx, want, ref.stored(dy.double().abs() * es + ref.U * want.abs(), want, dt))
        only = torch.empty_like(x)
        ewf.activation(act, x, only, stream=stream())
        assert torch.equal(only, y)
        ewf.activation(act, x, x, stream=stream())                  # in place
        assert torch.equal(x, y)
        ewf.activation_grad(act, dy, dy, codes=codes, scales=scales, stream=stream())
        assert torch.equal(dy, dx)


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("act", ("relu", "tanh", "sigmoid", "silu", "gelu"))
@pytest.mark.parametrize("dtype", sorted(DT))
def test_activation_of_the_largest_numbers(dtype, act, kind):
    # far from zero the slopes are their limits (2^-100 is more than any of them is away from its own at 1000), also where
    # the code of a type's largest number stands for 2^128
    dt = DT[dtype]
    big = torch.finfo(dt).max
    x = torch.tensor([-big, big, -big / 4, big / 4] + ([-3e38, 3e38, -1e36, 1e36, -1e30, 1e30] if dtype != "f16" else []) + [-2000.0, 2000.0], device="cuda")
    x = x.to(dt)[:, None].repeat(1, 40).contiguous()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    codes = torch.empty(x.shape, dtype=CODES[kind], device="cuda")
    scales = torch.empty(x.shape[0], 2, dtype=torch.uint8, device="cuda")
    ewf.activation(act, x, y, codes=codes, scales=scales, stream=stream())
    ewf.activation_grad(act, torch.ones_like(x), dx, codes=codes, scales=scales, stream=stream())
    up = (x > 0).double()
    value = {"tanh": 2 * up - 1, "sigmoid": up}.get(act, x.double() * up)
    slope = 0 * up if act in ("tanh", "sigmoid") else up
    assert float((y.double() - value).abs().max()) <= 2.0 ** -100
    assert float((dx.double() - slope).abs().max()) <= 2.0 ** -100


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("act", ("tanh", "gelu"))
@pytest.mark.parametrize("dtype", sorted(DT))
def test_activation_far_from_zero_to_its_own_precision(dtype, act, kind):
    # the slope of tanh at 9 is 6e-8, gelu of -9 is -1e-18: relative to what 1 - tanh^2 and 1 + erf are taken from, nothing
    dt = DT[dtype]
    x = torch.linspace(-12, -2, 4001, device="cuda").to(dt)[None]
    if act == "tanh":
        x = torch.cat((x, -x))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    codes = torch.empty(x.shape, dtype=CODES[kind], device="cuda")
    scales = torch.empty(x.shape[0], 126, dtype=torch.uint8, device="cuda")
    ewf.activation(act, x, y, codes=codes, scales=scales, stream=stream())
    ewf.activation_grad(act, torch.ones_like(x), dx, codes=codes, scales=scales, stream=stream())
    x8 = ref.keep8(x, kind)[2]
    if act == "gelu":
        want = ref.ACTS[act][0](x.double())
        ref.close("y", y, want, ref.stored(ref.act_relative_bounds(act, x.double())[0], want, dt))
    want = ref.ACTS[act][1](x8)
    ref.close("dx", dx, want, ref.stored(ref.act_relative_bounds(act, x8)[1], want, dt))


def gate_arguments():
    return torch.cat((torch.linspace(-80, 80, 3001), torch.randn(1095) * 4)).cuda()


def test_float32_sigmoids_to_float32s_precision():
    x = gate_arguments()[None]
    y, dx = torch.empty_like(x), torch.empty_like(x)
    codes, scales = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(1, 128, dtype=torch.uint8, device="cuda")
    for act, rel, slope in (("sigmoid", ref.GATE, 2 * ref.GATE + ref.U), ("silu", ref.GATE + ref.U, None), ("tanh", None, 2 * ref.GATE + ref.U)):
        ewf.activation(act, x, y, codes=codes, scales=scales, stream=stream())
        if rel:
            want = ref.ACTS[act][0](x.double())
            ref.close(act, y, want, rel * want.abs() + ref.TINY[torch.float32])
        if slope:
            ewf.activation_grad(act, torch.ones_like(x), dx, codes=codes, scales=scales, stream=stream())
            x8 = ref.keep8(x, "i8")[2]
            want = ref.ACTS[act][1](x8)
            normal = want > 2.0 ** -123                              # (a factor below 2^-126 counts as 0)
            ref.close(act, dx[normal], want[normal], slope * want[normal])


@pytest.mark.parametrize("dtype", sorted(DT))
def test_activation_strides(dtype):
    dt, g = DT[dtype], gen(14)
    x = randn(g, 5, 6, 150, dtype=dt)[:, :, 3:104].transpose(0, 1)   # [6, 5, 101], rows at odd elements
    out = torch.full((6, 5, 110), 7.0, dtype=dt, device="cuda")
    box = torch.zeros((6, 5, 107), dtype=torch.int8, device="cuda")
    y, codes = out[:, :, 4:105], box[:, :, 1:102]
    scales = torch.zeros((5, 6, 4), dtype=torch.uint8, device="cuda").transpose(0, 1)
    ewf.activation("silu", x, y, codes=codes, scales=scales, stream=stream())
    code, byte, x8, _ = ref.keep8(x, "i8")
    assert torch.equal(scales, byte) and torch.equal(codes.double(), code)
    assert (out[:, :, :4] == 7).all() and (out[:, :, 105:] == 7).all() and (box[:, :, 0] == 0).all() and (box[:, :, 102:] == 0).all()
    dx = torch.empty(6, 5, 101, dtype=dt, device="cuda")
    dy = randn(g, 101, dtype=dt).expand(6, 5, 101)
    ewf.activation_grad("silu", dy, dx, codes=codes, scales=scales, stream=stream())
    _, es = ref.act_bounds("silu", x8)
    want = dy.double() * ref.ACTS["silu"][1](x8)
    ref.close("dx", dx, want, ref.stored(dy.double().abs() * es + ref.U * want.abs(), want, dt))


# ------------------------------------------------------------------ recurrence

def rec_case(g, B, T, D, dt, tied, lengths):
    c = dict(u=randn(g, B, T, D, mean=1.0, std=2.0, dtype=dt), v=randn(g, B, T, D, dtype=dt), w=None if tied else randn(g, B, T, D, dtype=dt),
             h0=randn(g, B, D), lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    return c


def rec_forward(c, h=None, last=None):
    h = torch.full_like(c["u"], 7.0) if h is None else h
    last = torch.full((c["u"].shape[0], c["u"].shape[2]), 7.0, device="cuda") if last is None else last
    run(ewf.recurrence, c["u"], c["v"], h, w=c["w"], h0=c["h0"], last=last, lengths=c["lengths"])
    return h, last


def check_rec(c, h, last):
    want = ref.recurrence(c["u"], c["v"], c["w"], c["h0"], c["lengths"], c["u"].dtype)
    on = want["valid"]
    ref.close("h", torch.where(on, h.double(), 0.0), torch.where(on, want["h"], 0.0), want["e_h"])
    ref.close("last", last, want["last"], want["e_last"])
    return on


def rec_backward(c, h, dh, dlast, dh0=None):
    d = {k: torch.full_like(c["u"], 7.0) for k in ("du", "dv", "dw")}
    if c["w"] is None:
        d["dw"] = None
    d["dh0"] = torch.full((c["u"].shape[0], c["u"].shape[2]), 7.0, device="cuda")
    run(ewf.recurrence_grad, c["u"], c["v"], h, dh, d["du"], d["dv"], w=c["w"], dw=d["dw"], h0=c["h0"], dh0=d["dh0"], dlast=dlast,
        lengths=c["lengths"])
    return d


def check_rec_grad(c, h, dh, dlast, d):
    want = ref.recurrence_grad(c["u"], c["v"], c["w"], h, c["h0"], dh, dlast, c["lengths"], c["u"].dtype)
    on = want["valid"]
    for k in ("du", "dv", "dw"):
        if d[k] is not None:
            ref.close(k, torch.where(on, d[k].double(), 0.0), torch.where(on, want[k], 0.0), want["e_" + k])
            assert (d[k][~on] == 7).all(), k
    ref.close("dh0", d["dh0"], want["dh0"], want["e_dh0"])


REC_SHAPES = ((1, 1, 1), (3, 1, 2), (2, 2, 3), (64, 1, 300), (2, 16, 65), (3, 17, 1), (2, 17, 2), (1, 63, 64), (2, 64, 63), (1, 65, 130), (3, 127, 5),
              (2, 128, 64), (1, 129, 66), (2, 200, 129), (1, 256, 7), (1, 257, 128), (5, 300, 40), (1, 1500, 67), (2, 2049, 192))


@pytest.mark.parametrize("tied", (True, False))
@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("B,T,D", REC_SHAPES)
def test_recurrence_and_its_gradient(B, T, D, dtype, tied):
    dt, g = DT[dtype], gen(B + T + D)
    lens = [None]
    if B > 1:
        lens.append([(T * k) // (B - 1) for k in range(B)])          # from none to all
    for lengths in lens:
        say("recurrence", B, T, D, dtype, "tied" if tied else "gated", lengths)
        c = rec_case(g, B, T, D, dt, tied, lengths)
        h, last = rec_forward(c)
        on = check_rec(c, h, last)
        assert (h[~on] == 7).all()
        dh, dlast = randn(g, B, T, D, dtype=dt), randn(g, B, D)
        check_rec_grad(c, h, dh, dlast, rec_backward(c, h, dh, dlast))
        # nothing given that may be absent
        c["h0"] = None
        h, last = rec_forward(c)
        check_rec(c, h, last)
        d = rec_backward(c, h, dh, None)
        check_rec_grad(c, h, dh, None, d)


@pytest.mark.parametrize("B,T,D,dtype,tied", (
    (8, 2100, 1000, "bf16", True), (8, 2100, 1000, "f16", False), (8, 2100, 500, "f32", True),      # chains of long and of wide tiles
    (8, 150, 2000, "bf16", False), (16, 300, 600, "f32", True),                                    # a workgroup for a strip
    (1, 9000, 9, "f32", True), (2, 5000, 70, "bf16", False)))                                      # few chains of many tiles
def test_recurrence_of_many_tiles(B, T, D, dtype, tied):
    say("recurrence", B, T, D, dtype, tied)
    g = gen(B + T + D)
    for lengths in (None, [T - (T * k) // (2 * B) for k in range(B)]):
        c = rec_case(g, B, T, D, DT[dtype], tied, lengths)
        h, last = rec_forward(c)
        on = check_rec(c, h, last)
        assert (h[~on] == 7).all()
        dh, dlast = randn(g, B, T, D, dtype=DT[dtype]), randn(g, B, D)
        d = rec_backward(c, h, dh, dlast)
        check_rec_grad(c, h, dh, dlast, d)
        again = rec_forward(c), rec_backward(c, h, dh, dlast)
        assert torch.equal(again[0][0], h) and torch.equal(again[0][1], last)
        assert all(torch.equal(again[1][k], d[k]) for k in d if d[k] is not None)


@pytest.mark.parametrize("B,T,D,dtype,tied", (
    (4, 3000, 1, "bf16", False), (3, 2600, 2, "f16", True), (2, 300, 3, "bf16", True), (5, 1300, 1, "f32", False),   # rows of less than a lane's
    (3, 2500, 26, "bf16", False), (40, 260, 13, "f32", True), (2, 1025, 32, "f16", False),                            # rows of a slim tile
    (200, 40, 1032, "bf16", True), (200, 20, 1030, "f16", False), (130, 33, 520, "f32", False),                       # walks of many channels
    (20, 800, 160, "bf16", False), (20, 800, 200, "bf16", True)))                                                     # strips part empty, and filled
def test_recurrence_of_few_channels_and_of_many_rows(B, T, D, dtype, tied):
    test_recurrence_of_many_tiles(B, T, D, dtype, tied)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("T", (5, 700))
@pytest.mark.parametrize("D", (1, 3, 29))
def test_recurrence_of_few_channels_in_place(T, D, dtype):
    g, dt, B = gen(24), DT[dtype], 3
    lengths = torch.tensor([T, T // 2, 0], dtype=torch.int32, device="cuda")
    both = randn(g, B, T, 3 * D + 1, dtype=dt)                        # column blocks of a projection
    u, v, dh = both[:, :, 1: D + 1], both[:, :, D + 1: 2 * D + 1], both[:, :, 2 * D + 1:]
    copies = [t.contiguous() for t in (u, v, dh)]
    h, du, dv = (torch.full((B, T, D), 7.0, dtype=dt, device="cuda") for _ in range(3))
    run(ewf.recurrence, copies[0], copies[1], h, lengths=lengths)
    run(ewf.recurrence_grad, copies[0], copies[1], h, copies[2], du, dv, lengths=lengths)
    before = both.clone()
    run(ewf.recurrence_grad, u, v, h, dh, u, dh, lengths=lengths)     # du over u, dv over dh
    on = torch.arange(T, device="cuda")[None, :] < lengths[:, None]
    assert torch.equal(u[on], du[on]) and torch.equal(dh[on], dv[on]) and torch.equal(v, before[:, :, D + 1: 2 * D + 1])
    assert torch.equal(both[~on], before[~on]) and torch.equal(both[:, :, 0], before[:, :, 0])
    both.copy_(before)
    run(ewf.recurrence, u, v, v, lengths=lengths)                     # h over v
    assert torch.equal(v[on], h[on]) and torch.equal(both[~on], before[~on])
    assert torch.equal(both[:, :, : D + 1], before[:, :, : D + 1]) and torch.equal(both[:, :, 2 * D + 1:], before[:, :, 2 * D + 1:])


@pytest.mark.parametrize("T", (3, 40, 700))
def test_recurrence_lengths_out_of_range_and_what_lies_behind(T):
    g = gen(T)
    c = rec_case(g, 5, T, 70, torch.bfloat16, False, [-3, T + 9, 0, T // 2, 1])
    clean = dict(c)
    h, last = rec_forward(c)
    on = check_rec(c, h, last)
    dh, dlast = randn(g, 5, T, 70, dtype=torch.bfloat16), randn(g, 5, 70)
    d = rec_backward(c, h, dh, dlast)
    check_rec_grad(c, h, dh, dlast, d)
    # what the inputs hold behind a sequence has no effect
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.bfloat16).min):
        for k in ("u", "v", "w"):
            clean[k] = torch.where(on, c[k], torch.full_like(c[k], bad))
        h2, last2 = rec_forward(clean)
        assert torch.equal(h2, h) and torch.equal(last2, last)
        d2 = rec_backward(clean, torch.where(on, h, bad), torch.where(on, dh, bad), dlast)
        assert all(torch.equal(d2[k], d[k]) for k in d), bad


def test_recurrence_gates_at_their_ends():
    # a shut gate forgets, an open one keeps, through hundreds of steps
    B, T, D = 1, 400, 64
    u = torch.full((B, T, D), 200.0, device="cuda")
    u[0, 100] = -200.0
    u[0, 300] = -float("inf")
    v = torch.randn(B, T, D, device="cuda")
    h, last = torch.empty_like(u), torch.empty(B, D, device="cuda")
    h0 = torch.randn(B, D, device="cuda")
    run(ewf.recurrence, u, v, h, h0=h0, last=last)
    assert torch.equal(h[0, 0:100], h0.expand(100, D))
    assert torch.equal(h[0, 100:300], v[0, 100].expand(200, D)) and torch.equal(h[0, 300:], v[0, 300].expand(100, D))
    assert torch.equal(last[0], v[0, 300])


@pytest.mark.parametrize("tied", (True, False))
@pytest.mark.parametrize("T", (1, 9, 40, 333))
def test_recurrence_shut_gates_forget_the_largest_states(T, tied):
    # e^-300 of 3e38 is nothing, of a state and of a gradient
    g, D = gen(23), 70
    u, v, dh = torch.full((2, T, D), -300.0, device="cuda"), randn(g, 2, T, D), randn(g, 2, T, D)
    w = None if tied else torch.full_like(u, 300.0)
    h0 = torch.full((2, D), 3e38, device="cuda")
    h, last = torch.empty_like(u), torch.empty_like(h0)
    run(ewf.recurrence, u, v, h, w=w, h0=h0, last=last)
    assert torch.equal(h, v) and torch.equal(last, v[:, -1])
    du, dv, dw, dh0 = torch.empty_like(u), torch.empty_like(u), None if tied else torch.empty_like(u), torch.empty_like(h0)
    run(ewf.recurrence_grad, u, v, h, dh, du, dv, w=w, dw=dw, h0=h0, dh0=dh0, dlast=torch.full_like(h0, -1e38))
    dh[:, -1] += -1e38
    assert torch.equal(dv, dh) and (du == 0).all() and (dh0 == 0).all() and (tied or (dw == 0).all())


@pytest.mark.parametrize("tied", (True, False))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("T", (1, 9, 40, 333))
def test_recurrence_gradients_of_the_largest_states(T, dtype, tied):
    # shut gates, the largest inputs in turn positive and negative: two states are further apart than float32 reaches, and each gradient
    # is finite; one gate stands half open
    dt, g, D = DT[dtype], gen(25), 70
    u, v = torch.full((2, T, D), -300.0, dtype=dt, device="cuda"), torch.full((2, T, D), 3e38, dtype=dt, device="cuda")
    v[:, ::2] = -3e38
    u[:, T // 2] = 0
    c = dict(u=u, v=v, w=None if tied else torch.full_like(u, 300.0), h0=torch.full((2, D), 3e38, device="cuda"), lengths=None)
    if not tied:
        c["w"][:, T // 2] = 0
    h, last = rec_forward(c)
    check_rec(c, h, last)
    dh, dlast = randn(g, 2, T, D, std=1e-3, dtype=dt), randn(g, 2, D, std=1e-3)
    d = rec_backward(c, h, dh, dlast)
    assert all(torch.isfinite(t).all() for t in d.values() if t is not None)
    check_rec_grad(c, h, dh, dlast, d)


@pytest.mark.parametrize("tied", (True, False))
@pytest.mark.parametrize("T", (1, 40, 300))
def test_recurrence_float32_gates_to_float32s_precision(T, tied):
    # one step with gates to be looked at, the others hold what it leaves
    x = gate_arguments()
    D = x.numel()
    u, v, w = torch.full((1, T, D), 200.0, device="cuda"), torch.zeros(1, T, D, device="cuda"), torch.full((1, T, D), -200.0, device="cuda")
    u[0, 0], w[0, 0] = x, x
    h, last, h0 = torch.empty_like(u), torch.empty(1, D, device="cuda"), torch.zeros(1, D, device="cuda")
    f, g = torch.sigmoid(x.double()), torch.sigmoid(-x.double())
    i = g if tied else f
    some = dict(w=None if tied else w, h0=h0, last=last)
    for a, b, want in ((1.0, 0.0, f), (0.0, 1.0, i)):                # from the state, from the input
        h0.fill_(a)
        v[0, 0] = b
        run(ewf.recurrence, u, v, h, **some)
        ref.close("last", last[0], want, (ref.GATE + ref.U) * want)
        assert torch.equal(h[0, -1], last[0])
    h0.fill_(1.0)
    v.zero_()
    du, dv, dw, dh0, dh = torch.empty_like(u), torch.empty_like(u), torch.empty_like(u), torch.empty_like(h0), torch.zeros_like(u)
    dh[0, 0] = 1.0
    if not tied:
        v[0, 0] = 1.0
    run(ewf.recurrence, u, v, h, **some)
    run(ewf.recurrence_grad, u, v, h, dh, du, dv, w=some["w"], dw=None if tied else dw, h0=h0, dh0=dh0)
    ref.close("dv", dv[0, 0], i, (ref.GATE + ref.U) * i)
    ref.close("dh0", dh0[0], f, (ref.GATE + ref.U) * f)
    ref.close("du", du[0, 0], f * g, (2 * ref.GATE + 3 * ref.U) * f * g)
    if not tied:
        ref.close("dw", dw[0, 0], f * g, (2 * ref.GATE + 3 * ref.U) * f * g)


@pytest.mark.parametrize("T", (5, 333))
def test_recurrence_keeps_what_is_not_finite_in_its_channel(T):
    g = gen(20 + T)
    c = rec_case(g, 2, T, 66, torch.float32, True, None)
    h, last = rec_forward(c)
    c["v"][1, T // 2, 65] = float("nan")
    c["v"][0, 1, 3] = float("inf")
    h2, last2 = rec_forward(c)
    touched = torch.zeros_like(h, dtype=torch.bool)
    touched[1, T // 2:, 65] = True
    touched[0, 1:, 3] = True
    assert torch.equal(h2[~touched], h[~touched]) and not torch.isfinite(h2[touched]).any()
    assert torch.isnan(last2[1, 65]) and not torch.isfinite(last2[0, 3])


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("T", (1, 7, 150))
def test_recurrence_strides_and_in_place(dtype, T):
    dt, g = DT[dtype], gen(30 + T)
    for D in (1, 33, 64, 130):
        say("strides", dtype, T, D)
        B = 3
        # time-major column blocks of one projection, each beginning at any element
        p = randn(g, T, B, 3 * D + 1, dtype=dt)
        blocks = [p[:, :, 1 + k * D:1 + (k + 1) * D].transpose(0, 1) for k in range(3)]
        state = randn(g, B, D + 3)
        c = dict(u=blocks[0], v=blocks[1], w=blocks[2], h0=state[:, 2:D + 2], lengths=torch.tensor([[T, 9], [T // 2, 9], [T, 9]], dtype=torch.int32, device="cuda")[:, 0])
        keep = p.clone()
        out = torch.full((T, B, D + 2), 7.0, dtype=dt, device="cuda")
        h = out[:, :, 1:D + 1].transpose(0, 1)
        h, last = rec_forward(c, h=h)
        on = check_rec(c, h, last)
        assert torch.equal(p, keep) and (out[:, :, 0] == 7).all() and (out[:, :, D + 1] == 7).all() and (h[~on] == 7).all()
        dh, dlast = randn(g, B, T, D, dtype=dt), randn(g, B, D)
        d = rec_backward(c, h, dh, dlast)
        check_rec_grad(c, h, dh, dlast, d)
        # gradients as column blocks over the operands themselves
        dlast2 = dlast.clone()
        saved = [b.clone() for b in blocks]
        run(ewf.recurrence_grad, blocks[0], blocks[1], h, dh, blocks[0], blocks[1], w=blocks[2], dw=blocks[2], h0=c["h0"], dh0=dlast2, dlast=dlast2,
            lengths=c["lengths"])
        for k, b, s in zip(("du", "dv", "dw"), blocks, saved):
            assert torch.equal(b[on], d[k][on]) and torch.equal(b[~on], s[~on])
        assert torch.equal(dlast2, d["dh0"])
        # forward over each operand, the state in place
        p.copy_(keep)
        for k in ("u", "v", "w"):
            p.copy_(keep)
            s = state[:, 2:D + 2].clone()
            c2 = dict(c, h0=s)
            rec_forward(c2, h=c2[k], last=s)
            assert torch.equal(c2[k][on], h[on]) and torch.equal(s, last)
        p.copy_(keep)


def test_recurrence_step_by_step_is_the_whole():
    g = gen(41)
    c = rec_case(g, 4, 30, 100, torch.float32, False, None)
    h, last = rec_forward(c)
    s = c["h0"].clone()
    steps = torch.empty_like(h)
    for t in range(30):
        sl = lambda x: x[:, t:t + 1]
        run(ewf.recurrence, sl(c["u"]), sl(c["v"]), sl(steps), w=sl(c["w"]), h0=s, last=s)
    want = ref.recurrence(c["u"], c["v"], c["w"], c["h0"], None, torch.float32)
    ref.close("h", steps, want["h"], want["e_h"])
    ref.close("last", s, want["last"], want["e_last"])


def test_recurrence_of_no_steps():
    u = torch.empty(2, 0, 5, device="cuda")
    h0, last = torch.randn(2, 5, device="cuda"), torch.empty(2, 5, device="cuda")
    run(ewf.recurrence, u, torch.empty_like(u), torch.empty_like(u), h0=h0, last=last)
    assert torch.equal(last, h0)
    dh0 = torch.empty(2, 5, device="cuda")
    run(ewf.recurrence_grad, u, torch.empty_like(u), torch.empty_like(u), torch.empty_like(u), torch.empty_like(u), torch.empty_like(u),
        dlast=h0, dh0=dh0)
    assert torch.equal(dh0, h0)


# ------------------------------------------------------------------ streams, graphs, several calls at once

def small_calls(g):
    """One bound call of every operator on tensors of its own: [(call, results)]."""
    bf = torch.bfloat16
    made = []

    def bound(op, results, *args, **kw):
        made.append((op.bind(*args, workspace=work_for(op, *args, **kw), **kw), results))

    x, w, b = randn(g, 300, 1000, dtype=bf), randn(g, 1000), randn(g, 1000)
    y, mean, rstd = torch.empty_like(x), torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    codes, scales = torch.empty((300, 1000), dtype=torch.int8, device="cuda"), torch.empty((300, 32), dtype=torch.uint8, device="cuda")
    bound(ewf.layer_norm, (y, mean, rstd, codes, scales), x, w, b, y, mean=mean, rstd=rstd, codes=codes, scales=scales)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    bound(ewf.layer_norm_grad, (dx, dw, db), y, w, rstd, dx, dweight=dw, dbias=db, codes=codes, scales=scales)
    z, zc, zs = torch.empty_like(x), torch.empty((300, 1000), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((300, 32), dtype=torch.uint8, device="cuda")
    bound(ewf.activation, (z, zc, zs), "gelu", y, z, codes=zc, scales=zs)
    dz, back = torch.empty_like(x), torch.empty_like(x)
    bound(ewf.activation_grad, (dz,), "gelu", dx, dz, codes=zc, scales=zs)
    bound(ewf.read8, (back,), zc, zs, back)
    c = rec_case(g, 3, 700, 130, bf, False, [700, 0, 123])
    h, last, dh, dlast = torch.zeros_like(c["u"]), torch.empty(3, 130, device="cuda"), randn(g, 3, 700, 130, dtype=bf), randn(g, 3, 130)
    bound(ewf.recurrence, (h, last), c["u"], c["v"], h, w=c["w"], h0=c["h0"], last=last, lengths=c["lengths"])
    du, dv, dq = (torch.zeros_like(c["u"]) for _ in range(3))
    dh0 = torch.empty(3, 130, device="cuda")
    bound(ewf.recurrence_grad, (du, dv, dq, dh0), c["u"], c["v"], h, dh, du, dv, w=c["w"], dw=dq, h0=c["h0"], dh0=dh0, dlast=dlast, lengths=c["lengths"])
    return made


def clear(calls):
    for _, results in calls:
        for r in results:
            r.view(torch.uint8).zero_()


def test_all_operators_in_a_captured_graph():
    calls = small_calls(gen(50))
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
            for r, e in zip(results, want):
                assert torch.equal(r.view(torch.uint8), e.view(torch.uint8)), replay
        # eager work and the same operators between the replays, the workspaces left dirty
        assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())
        for call, _ in calls:
            call.launch(stream())
        torch.cuda.synchronize()


def test_calls_on_several_streams_at_once():
    sets = [small_calls(gen(60 + k)) for k in range(3)]
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
            assert all(torch.equal(r.view(torch.uint8), x.view(torch.uint8)) for r, x in zip(results, e))


def test_long_recurrences_on_two_streams_at_once():
    # chains whose tiles wait for each other, twice, side by side
    g = gen(70)
    made = []
    for k in range(2):
        c = rec_case(g, 1, 20000, 300, torch.float32, True, None)
        h, last = torch.empty_like(c["u"]), torch.empty(1, 300, device="cuda")
        args, kw = (c["u"], c["v"], h), dict(h0=c["h0"], last=last)
        made.append((ewf.recurrence.bind(*args, workspace=work_for(ewf.recurrence, *args, **kw), **kw), h, last))
    want = []
    for call, h, last in made:
        call.launch(stream())
        torch.cuda.synchronize()
        want.append((h.clone(), last.clone()))
        h.zero_()
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(6):
        for s, (call, _, _) in zip(streams, made):
            call.launch(s.cuda_stream)
    torch.cuda.synchronize()
    for (call, h, last), (wh, wl) in zip(made, want):
        assert torch.equal(h, wh) and torch.equal(last, wl)


def test_workspace_of_the_wrong_size_is_refused():
    g = gen(71)
    c = rec_case(g, 1, 5000, 64, torch.bfloat16, True, None)
    h = torch.empty_like(c["u"])
    n = ewf.recurrence.workspace_bytes(c["u"], c["v"], h)
    assert n > 16
    with pytest.raises(ewf.EwfError) as e:
        ewf.recurrence(c["u"], c["v"], h, workspace=torch.empty(n - 16, dtype=torch.uint8, device="cuda"), stream=stream())
    assert e.value.status == ewf.ENOMEM


def test_an_error_of_an_earlier_call_is_not_the_operators():
    import ctypes
    hip = ctypes.CDLL(next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line))
    calls = small_calls(gen(72))
    try:
        for call, _ in calls:
            assert hip.hipSetDevice(99) != 0                          # refused, and left unread
            call.launch(stream())
    finally:
        hip.hipGetLastError()
    torch.cuda.synchronize()


# ------------------------------------------------------------------ all together

def test_a_block_of_a_recurrent_language_model():
    """Norm, gates, recurrence, activation, projection and the loss of the expressions, forward and backward, with 8 bits
    kept of the norm's rows and of the activation's argument; each step against the formulas in 64 bits, on what the
    step before it handed over."""
    from workloads import configs as wl
    import tests.harness as hn
    g = gen(80)
    B, T, D, H, V = 3, 90, 96, 80, 200
    x = randn(g, B, T, D, mean=0.2)
    lw, lb = randn(g, D, mean=1, std=0.2), randn(g, D, std=0.2)
    wu, wv, wo = (randn(g, D, H, std=D ** -0.5), randn(g, D, H, std=D ** -0.5), randn(g, H, V, std=H ** -0.5))
    target = torch.randint(0, V, (B * T,), generator=g, device="cuda", dtype=torch.int32)
    dev = dict(device="cuda")
    n8, ns = torch.empty(B, T, D, dtype=torch.int8, **dev), torch.empty(B, T, 3, dtype=torch.uint8, **dev)
    y, rstd = torch.empty_like(x), torch.empty(B, T, **dev)
    run(ewf.layer_norm, x, lw, lb, y, rstd=rstd, codes=n8, scales=ns)
    p = torch.empty(B, T, 2 * H, **dev)                              # both gates' projections beside each other
    torch.matmul(y.view(-1, D), torch.cat((wu, wv), 1), out=p.view(-1, 2 * H))
    u, v = p[:, :, :H], p[:, :, H:]
    h, last = torch.empty(B, T, H, **dev), torch.empty(B, H, **dev)
    run(ewf.recurrence, u, v, h, last=last)
    z, zc, zs = torch.empty_like(h), torch.empty(B, T, H, dtype=torch.int8, **dev), torch.empty(B, T, 3, dtype=torch.uint8, **dev)
    run(ewf.activation, "silu", h, z, codes=zc, scales=zs)
    logits = z.view(-1, H) @ wo
    # the loss's gradient is one of the library's expressions: softmax minus one-hot, by ewf_grad
    w = wl.layout_only(wl.c3_softmax_xent_backward, rows=B * T, vocab=V)
    expr = ewf.Expression(w.spec)
    ins = [logits, target.view(-1, 1)]
    (dlogits,) = outs = hn.alloc_outputs(expr, w.spec, ins)
    expr.run(ins, outs, w.scalars, hn.make_workspace(expr, ins, outs), stream())
    dz = (dlogits @ wo.t()).view(B, T, H)
    dh = torch.empty_like(h)
    run(ewf.activation_grad, "silu", dz, dh, codes=zc, scales=zs)
    dp = torch.empty_like(p)
    run(ewf.recurrence_grad, u, v, h, dh, dp[:, :, :H], dp[:, :, H:])
    dy = (dp.view(-1, 2 * H) @ torch.cat((wu, wv), 1).t()).view(B, T, D)
    dx, dlw, dlb = torch.empty_like(x), torch.empty_like(lw), torch.empty_like(lb)
    run(ewf.layer_norm_grad, dy, lw, rstd, dx, dweight=dlw, dbias=dlb, codes=n8, scales=ns)
    # each step against the formulas on the values that the step before it handed over
    want = check_norm(x, lw, lb, y, None, None)
    check_rec(dict(u=u, v=v, w=None, h0=None, lengths=None), h, last)
    ev, _ = ref.act_bounds("silu", h.double())
    ref.close("z", z, ref.ACTS["silu"][0](h.double()), ref.stored(ev, z.double(), torch.float32))
    _, zbyte, h8, _ = ref.keep8(h, "i8")
    assert torch.equal(zs, zbyte)
    _, es = ref.act_bounds("silu", h8)
    wdh = dz.double() * ref.ACTS["silu"][1](h8)
    ref.close("dh", dh, wdh, ref.stored(dz.double().abs() * es + ref.U * wdh.abs(), wdh, torch.float32))
    check_rec_grad(dict(u=u, v=v, w=None, h0=None, lengths=None), h, dh, None,
                   dict(du=dp[:, :, :H], dv=dp[:, :, H:], dw=None, dh0=ref.recurrence_grad(u, v, None, h, None, dh, None, None, torch.float32)["dh0"]))
    n = torch.empty(B, T, D, **dev)
    run(ewf.read8, n8, ns, n)
    _, byte, _, unit = ref.keep8(want["n"], "i8")
    ref.close("n", n, want["n"], (0.5 if torch.equal(byte, ns) else 1.0) * unit * (1 + 1e-6) + 2 * want["e_n"])
    soft = torch.softmax(logits.double(), 1)
    soft[torch.arange(B * T, device="cuda"), target.long()] -= 1
    hn.compare("dlogits", dlogits.cpu().numpy(), (soft / (B * T)).float().cpu().numpy(), 1e-5, 1e-9)
    check_norm_grad(dy, None, lw, None, rstd, dx, dlw, dlb, torch.float32, n=n)


# ------------------------------------------------------------------ beyond 2^31 elements

def test_tensors_of_more_than_2_31_elements():
    bf = torch.bfloat16
    g = gen(90)
    rows, cols = 2_000_003, 1100
    say("layer norm and codes", rows, cols)
    x = torch.randn(rows, cols, dtype=bf, device="cuda", generator=g)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    codes, scales = torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, 35, dtype=torch.uint8, device="cuda")
    w, b = randn(g, cols), randn(g, cols)
    run(ewf.layer_norm, x, w, b, y, mean=mean, rstd=rstd)
    for part in (slice(0, 50), slice(rows - 50, rows)):
        check_norm(x[part], w, b, y[part], mean[part], rstd[part])
    dx = y                                                          # (dy is x: the gradient of half a square)
    run(ewf.layer_norm_grad, x, w, rstd, dx, x=x, mean=mean)
    n = (x[-50:].double() - mean[-50:].double()[:, None]) * rstd[-50:].double()[:, None]
    want = ref.layer_norm_grad(x[-50:], w, n, rstd[-50:], 2 * ref.U * n.abs(), bf, torch.float32)
    ref.close("dx", dx[-50:], want["dx"], want["e_dx"])
    ewf.keep8(x, codes, scales, stream=stream())
    for part in (slice(0, 50), slice(rows - 50, rows)):
        code, byte, _, _ = ref.keep8(x[part], "i8")
        assert torch.equal(scales[part], byte) and torch.equal(codes[part].double(), code)
    ewf.read8(codes, scales, y, stream=stream())
    assert torch.equal(y[-50:], ref.keep8(x[-50:], "i8")[2].to(bf))
    del x, y, dx, codes, scales
    B, T, D = 70_000, 33, 1000
    say("recurrence", B, T, D)
    u, v, dh = (torch.randn(B, T, D, dtype=bf, device="cuda", generator=g) for _ in range(3))
    h, du, dv, last = torch.empty_like(u), torch.empty_like(u), torch.empty_like(u), torch.empty(B, D, device="cuda")
    run(ewf.recurrence, u, v, h, last=last)
    run(ewf.recurrence_grad, u, v, h, dh, du, dv)
    for part in (slice(0, 3), slice(B - 3, B)):
        c = dict(u=u[part], v=v[part], w=None, h0=None, lengths=None)
        check_rec(c, h[part], last[part])
        want = ref.recurrence_grad(u[part], v[part], None, h[part], None, dh[part], None, None, bf)
        for k, got in (("du", du), ("dv", dv)):
            ref.close(k, got[part], want[k], want["e_" + k])


def test_recurrence_of_more_than_2_32_records():
    # 2^27 chains of two tiles, 32 records each; inputs that all sequences share, states of their own
    torch.cuda.empty_cache()
    B, T = (1 << 27) + 1000, 257
    g = gen(91)
    u, v = torch.full((1, T, 1), 8.0, dtype=torch.bfloat16, device="cuda"), randn(g, 1, T, 1, dtype=torch.bfloat16)
    h0 = torch.rand(B, 1, device="cuda", generator=g) * 20 - 10
    h, last = torch.empty(B, T, 1, dtype=torch.bfloat16, device="cuda"), torch.empty_like(h0)
    say("recurrence", B, T, 1)
    run(ewf.recurrence, u.expand(B, T, 1), v.expand(B, T, 1), h, h0=h0, last=last)
    torch.cuda.synchronize()
    # the last state is linear in the first, and its bound largest where that is
    ends = torch.tensor([[0.0], [10.0]], device="cuda")
    want = ref.recurrence(u.expand(2, T, 1), v.expand(2, T, 1), None, ends, None, torch.bfloat16)
    offset, slope, bound = want["last"][0, 0], (want["last"][1, 0] - want["last"][0, 0]) / 10, float(want["e_last"].max())
    for at in range(0, B, 1 << 24):
        part = slice(at, min(B, at + (1 << 24)))
        assert float((last[part].double() - (h0[part].double() * slope + offset)).abs().max()) <= bound, at
    for part in (slice(0, 3), slice((1 << 27) - 2, (1 << 27) + 3), slice(B - 3, B)):
        k = part.stop - part.start
        check_rec(dict(u=u.expand(k, T, 1), v=v.expand(k, T, 1), w=None, h0=h0[part], lengths=None), h[part], last[part])
    del h, last, h0
    torch.cuda.empty_cache()
