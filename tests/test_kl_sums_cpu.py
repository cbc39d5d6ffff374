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
