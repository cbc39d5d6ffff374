"""The arithmetic of the KL divergence's running sums (csrc/lopt_kl_sums.h) on the CPU, in the layouts of lanes, pieces, wavefronts and segments that the kernels have, against the
definition in float64. Tolerances: those of the kernels' own test."""
import os
import subprocess

import numpy as np
import pytest

from tests.test_gpu_more_ops import kl_exact, kl_tolerance, logits_pair

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# (lanes, logits a lane, pack, wavefronts, pieces of a segment), logits of a row
FORMS = [((16, 8, 4, 1, 0), 9), ((16, 8, 8, 1, 0), 100), ((16, 16, 8, 1, 0), 200), ((16, 32, 4, 1, 0), 500), ((64, 8, 8, 1, 0), 500), ((64, 16, 4, 1, 0), 1000),
         ((64, 32, 8, 1, 0), 2000), ((64, 16, 8, 1, 0), 3000), ((64, 16, 4, 4, 0), 20000), ((64, 16, 8, 8, 0), 9000), ((64, 16, 8, 4, 4), 40000)]


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("kl") / "probe")
    # products and sums as written: the kernels' compiler may fuse them, which only takes roundings away
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-Wno-unknown-pragmas", "-I" + os.path.join(ROOT, "paper_2506_10315_amd", "csrc"),
                    os.path.join(ROOT, "tests", "kl_probe.cpp"), "-o", out], check=True, capture_output=True, text=True)

    def run(form, x, r, scale=1.0):
        x, r = np.ascontiguousarray(x, np.float32), np.ascontiguousarray(r, np.float32)
        p = subprocess.run([out, *map(str, form), repr(scale)], input=np.array(x.shape, np.int32).tobytes() + x.tobytes() + r.tobytes(), capture_output=True, check=True)
        return np.frombuffer(p.stdout, np.float32).reshape(x.shape[0], 6).astype(np.float64)
    return run


def check(run, form, x, r, scale=1.0, what=""):
    """kl, and the mean difference among the stats."""
    x, r = np.asarray(x, np.float32), np.asarray(r, np.float32)
    want = kl_exact(x.astype(np.float64), r.astype(np.float64), scale)
    tol, _ = kl_tolerance(x.astype(np.float64), r.astype(np.float64), scale, want)
    got = run(form, x, r, scale)
    for name, have, exact in (("kl", got[:, 0], want[0]), ("mean", got[:, 5], want[1][:, 4])):
        with np.errstate(invalid="ignore"):
            right = (have == exact) | (np.isnan(have) & np.isnan(exact)) | (np.abs(have - exact) <= tol + 4e-7 * np.abs(np.where(np.isfinite(exact), exact, 0.0)))
        assert right.all(), (name, what, [(i, have[i], exact[i], tol[i]) for i in np.flatnonzero(~right)])
    return got


@pytest.mark.parametrize("form,vocab", FORMS)
def test_sums(probe, form, vocab):
    for scale, masked, apart in ((1.0, 0.0, 0.3), (0.5, 0.5, 0.3), (1.25, 0.0, 5.0), (1.0, 0.2, 0.0)):
        x, y = logits_pair(8, vocab, vocab, masked, apart)
        x[1], y[1] = -np.inf, -np.inf
        y[2, vocab // 2] = -np.inf
        x[2, vocab // 2] = -3.0
        x[3, vocab // 2] = -np.inf
        x[4, 1] = np.nan
        y[5, 2] = np.inf
        got = check(probe, form, x, y, scale, (scale, masked, apart))
        assert got[1, 0] == 0 and got[2, 0] == np.inf and np.isnan(got[4:6, 0]).all()


def runs_of(vocab):
    """Runs of tokens at a row's beginning, in its middle and at its end, some of which whole lanes, pieces and wavefronts lie in."""
    for length in sorted({1, min(16, vocab // 2), min(64, vocab // 3), vocab // 3}):
        for first in sorted({0, (vocab - length) // 2, vocab - length}):
            yield slice(first, first + length)


def rows_that_x_masks(vocab, low, seed=3):
    """x masks tokens by a finite value, down to the lowest, and r some of the same by the lowest: masked tokens that are their lane's largest in x while the row has far larger ones."""
    x, y = logits_pair(1, vocab, seed)
    at, rows = np.arange(vocab), []
    kept = np.isin(at, [1, vocab // 2, vocab - 2, vocab - 1])
    for mask in (low, -1e4):
        for off in (at == 0, at % 2 == 0, at < vocab // 2, at >= vocab // 2):
            rows.append((np.where(kept, x[0], mask), np.where(off & ~kept, low, y[0])))
        for run in runs_of(vocab):
            for step in (1, 2):
                a, b = x[0].copy(), y[0].copy()
                a[run] = mask
                b[run][::step] = low
                rows.append((a, b))
    return tuple(np.stack(v) for v in zip(*rows))


@pytest.mark.parametrize("low", [-3.4028234663852886e38, -3.3895313892515355e38])
@pytest.mark.parametrize("form,vocab", FORMS)
def test_tokens_that_x_masks_by_a_finite_value_and_r_by_the_lowest(probe, form, vocab, low):
    x, y = rows_that_x_masks(vocab, low)
    for scale in (1.0, 0.5, 2.0, 70.0, 1e-3):
        check(probe, form, x, y, scale, scale)


def rows_with_unlikely_tokens_that_r_masks(vocab, low, masked=False):
    """Runs of tokens that x has at p = 1e-37, 1e-30 or 1e-4 each and r at the lowest value: KL is p times that value, 1e1 to 1e36. `masked`: x masks some others by the lowest."""
    x, y = logits_pair(1, vocab, 4)
    rows = []
    for run in runs_of(vocab):
        for under in (85.0, 69.0, 9.2):
            if under < 10 and run.stop - run.start > 64:   # KL beyond 1e38
                continue
            a, b = x[0].copy(), y[0].copy()
            a[run] = -np.inf
            a[run] = a.max() - under
            b[run] = low
            if masked:
                off = (np.arange(vocab) % 3 == 1) & (a < a.max() - 10)
                off[run] = False
                a[off] = low
            rows.append((a, b))
    return tuple(np.stack(v) for v in zip(*rows))


@pytest.mark.parametrize("low", [-3.4028234663852886e38, -3.3895313892515355e38])
@pytest.mark.parametrize("form,vocab", FORMS)
def test_unlikely_tokens_that_r_masks_by_the_lowest(probe, form, vocab, low):
    for masked in (False, True):
        x, y = rows_with_unlikely_tokens_that_r_masks(vocab, low, masked)
        for scale in (1.0, 0.5, 2.0):
            assert np.isfinite(check(probe, form, x, y, scale, (scale, masked))[:, 0]).all()


@pytest.mark.parametrize("form,vocab", FORMS)
def test_enormous_scales(probe, form, vocab):
    """Scales that make p one token's, from which the others are 1e20 and more away, masked ones beyond the type."""
    for scale in (1e20, 1e30):
        s32 = float(np.float32(scale))
        for x, y in (logits_pair(8, vocab, 1), logits_pair(8, vocab, 2, 0.3, 2.0), rows_that_x_masks(vocab, -3.4028234663852886e38), rows_that_x_masks(vocab, -65504.0)):
            check(probe, form, x, y, s32, scale)
    x, _ = logits_pair(8, vocab, 3)
    for y in (x, x + 1.0):
        assert np.isfinite(probe(form, x, y, 1e38)).all()
