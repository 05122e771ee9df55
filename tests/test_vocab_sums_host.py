"""The sums over a row of logits (`add`, `move`, `point_of` and `settle` of the operators over a vocabulary), run on the CPU: tests/host_sums/vocab_sums.hip is
compiled with the library's own header, for the host alone."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LANES, WAVE, EACH = 16, 4, 6
U = 2.0 ** -24
# finite masks, from those that float32 can still place to the lowest numbers
MASKS = (-1e4, -3e6, -1e9, -3e9, -1e10, -1e12, -1e20, -1e25, -1e30, -1e37, -3.3895314e38, -3.4028235e38)


@pytest.fixture(scope="module")
def sums(tmp_path_factory):
    """rows [n, LANES, EACH] at a scale -> peak, whether they are summed again, sums, weighted sums"""
    program = str(tmp_path_factory.mktemp("host_sums") / "vocab_sums")
    subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-ffp-contract=off", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_1605_02688_amd", "csrc"), os.path.join(ROOT, "tests", "host_sums", "vocab_sums.hip"), "-o", program],
                   check=True, timeout=240)

    def run(rows, scale):
        text = "".join(f"{float(np.float32(scale)).hex()} {LANES} {WAVE} {EACH} " + " ".join(float(x).hex() for x in r.ravel()) + "\n" for r in rows)
        out = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=60).stdout.split("\n")[:-1]
        assert len(out) == len(rows)
        return [(float.fromhex(p) if "0x" in p else float(p), int(b), float.fromhex(s) if "0x" in s else float(s), float.fromhex(w) if "0x" in w else float(w))
                for p, b, s, w in (line.split() for line in out)]
    return run


def bf16(x):
    """to the nearest bfloat16, as float32"""
    b = np.float32(x).view(np.uint32).astype(np.uint64)
    return ((b + 0x7fff + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def check(sums, rows, scale):
    got = sums(rows, scale)
    c = np.float64(np.float32(np.float32(scale) * np.float32(1.44269504)))
    for row, (peak, again, s, w) in zip(rows, got):
        x = row.astype(np.float64).ravel()
        assert peak == x.max()
        beyond = not abs(peak * c) < 2.0 ** 22 * (1 - U)         # (half a step below it the product rounds to it)
        assert again == beyond
        if beyond:                                      # (swept again about its largest: these sums are not used)
            continue
        t = (x - peak) * c
        p = np.exp2(t)
        ps = p * np.where(p > 0, t, 0.0)
        # a term's exponent: the multiply-add's one rounding of at most |t| + 9 away from the point (half a power of two and the 2^8 that it lags); exponentials and
        # moves (of lanes, wavefronts, the row; one every eight powers of two of the way before): three roundings each; EACH additions and conversions to float32
        near = np.minimum(np.abs(t), 200.0)
        e = U * (2 * (near + 9) + 3 * (near / 8 + 4) + EACH + 4)
        lost = x.size * 2.0 ** -125
        assert abs(s - p.sum()) <= (p * e).sum() + lost, (row, s, p.sum())
        assert abs(w - ps.sum()) <= (p * (near + 9) * (e + 4 * U)).sum() + (p * (near + 9)).sum() * 4 * U + lost * 200, (row, w, ps.sum())


@pytest.mark.parametrize("half", (False, True))
@pytest.mark.parametrize("scale", (1.0, 0.5, 0.7, 0.1, 1.25))
@pytest.mark.parametrize("mask", MASKS)
def test_finite_masks_beside_ordinary_logits(sums, mask, scale, half):
    rng = np.random.default_rng(int(-np.log2(-mask) * -100) + int(scale * 100))
    store = bf16 if half else np.float32
    mask = max(mask, -3.3895314e38) if half else mask
    rows = []
    for _ in range(8):
        x = rng.standard_normal((LANES, EACH)).astype(np.float32) * np.float32(3.0)
        for gone in (x * 0 + (np.arange(EACH) < 3), x * 0 + (np.arange(EACH) >= 3), x * 0 + (np.arange(EACH) % 2), x * 0 + (np.arange(LANES)[:, None] < 9),
                     x * 0 + (np.arange(LANES)[:, None] > 0), x * 0 + (np.arange(LANES)[:, None] % 4 != 2), rng.random(x.shape) < 0.9):
            y = np.where(gone > 0, np.float32(mask), x)
            if not (y > mask).any():
                y[0, 0] = 1.0
            rows.append(store(y))
            # ... of several depths
            z = np.where((gone > 0) & (rng.random(x.shape) < 0.5), np.float32(mask) * np.float32(0.37), y)
            rows.append(store(z))
    check(sums, rows, scale)


@pytest.mark.parametrize("scale", (1.0, 0.1, 2.0 ** 20, 2.0 ** -20))
def test_rows_about_the_end_of_the_range_of_points(sums, scale):
    # lanes and wavefronts each side of -2^22 and 2^22
    rng = np.random.default_rng(7)
    c = np.float64(np.float32(np.float32(scale) * np.float32(1.44269504)))
    rows = []
    for at in (-(2.0 ** 22), 2.0 ** 22):
        for step in (-40.0, -9.0, -3.0, 0.0, 3.0, 9.0, 40.0):
            for std in (1.0, 10.0, 100.0):
                t = at + step + rng.standard_normal((LANES, EACH)) * std
                rows.append((t / c).astype(np.float32))
                t[:LANES // 2] -= rng.random() * 30
                rows.append((t / c).astype(np.float32))
                t[LANES // 2:] = -np.inf
                rows.append((t / c).astype(np.float32))
    check(sums, rows, scale)


def test_minus_infinities_and_nothing_else(sums):
    empty = np.full((LANES, EACH), -np.inf, dtype=np.float32)
    one = empty.copy()
    one[9, 4] = -7.0
    assert sums([empty], 1.0) == [(-np.inf, 0, 0.0, 0.0)]
    check(sums, [one], 1.0)
