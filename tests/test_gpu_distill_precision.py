"""w2l_distill_fwd_bwd where its results are small differences of large numbers.  Every element is held to a bound of its own, in units of
U = 2^-24 (half a step of fp32, relative)."""
import numpy as np
import pytest

import oracle
from test_gpu_scores import U, check_distill, close, distill_case, rounded, run_distill

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


def near_case(C, centre, repeat, K=16, T=6):
    """Student scores that bf16 holds, K classes with all of the mass at `centre` or up to 4 below (the others are 40 and more below), and a teacher
    that differs by about 2^-12.  repeat: three classes are named in two entries, each with half their probability."""
    rng = np.random.default_rng(C + int(centre))
    centre = float(rounded(centre, "bf16"))
    step = 2.0 ** (np.floor(np.log2(max(centre, 1))) - 7)      # of bf16 at the centre
    z = np.full((1, T, C), centre - max(40.0, 8 * step))
    ids = np.stack([rng.permutation(C)[:K] for _ in range(T)])[None]
    at = -rng.integers(0, 2, ids.shape) * (step if step <= 4 else 0.0)
    np.put_along_axis(z, ids, centre + at, 2)
    sc = at + 2.0 ** -12 * rng.standard_normal(ids.shape)
    if repeat:
        sc[..., :3] -= np.log(2.0)
        ids, sc = np.concatenate([ids, ids[..., :3]], 2), np.concatenate([sc, sc[..., :3]], 2)
    assert np.array_equal(z, rounded(z, "bf16"))
    return z, ids, sc.astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("repeat", [False, True], ids=["once", "repeated"])
@pytest.mark.parametrize("centre", [0.0, 100.0, 300.0, 650.0, 5e3, 3e7])
@pytest.mark.parametrize("C,T", [(29, 6), (300, 6), (4096, 2048), (4096, 6), (20000, 6), (40001, 130), (140001, 6)])
def test_gradient_where_student_and_teacher_agree(P, C, T, centre, repeat):
    """dz = ws (p - q) with |p - q| about 2^-12 p.  Of p and of q, fp32 leaves:
      p   k = log2 e, its product with x - m and their rounding: 3 |d| U, |d| <= 4 (or 40 and more, where p < 2^-57);  the power of two 2 U, its
          correction 2 U, s 15 additions of the K classes and these errors of each term, the division and the products 4 U:  2 (3 |d| + 2) + 23
      q   the same, |d| <= 4 + ln 2, and at most 19 additions
    and their difference and its product 3 U.  In all 2 (12 + 2) + 23 + 2 (15 + 2) + 27 + 3 = 115 U of p.  bf16 rounds the difference by 2^-8 of it."""
    z, ids, sc = near_case(C, centre, repeat)
    live = z.shape[1]
    pad = lambda a, v: np.concatenate([a, np.full((1, T - live) + a.shape[2:], v, a.dtype)], 1)      # more frames: another launch form
    zp, ip, sp = pad(z, 0.), pad(ids, -1), pad(sc, 0.)
    for gs in (1.0, -0.75):
        ref = oracle.distill(z, ids, sc, 1.0, None, None, gs)[2]
        p = np.exp(oracle._log_probs(z)[0])
        for dz_dtype in ("fp32", "bf16"):
            got = run_distill(P, zp, ip, sp, 1.0, None, [live], gs, "bf16", dz_dtype)[2][:, :live]
            bound = abs(gs) * 115 * U * p + 2.0 ** -126
            if dz_dtype == "bf16":
                bound = bound * 1.01 + 2.0 ** -8 * np.abs(ref)
            close(got, ref, bound, "dz " + dz_dtype)


@pytest.mark.parametrize("K", [1, 30, 60, 64])
@pytest.mark.parametrize("C", [200, 1000, 4096, 20000, 70000])
def test_loss_at_the_largest_temperatures(P, C, K):
    """p and q are even and the loss is weight tau^2 log(C / K), which fp32 holds where tau log C, tau log K or both are beyond it."""
    z, ids, sc, _, _ = distill_case(2, 3, C, K, "fp32", 5)
    for tau in (2.0 ** 124, 2.0 ** 125, 2.0 ** 126):
        w = np.full((2, 3), 2.0 ** -126)
        check_distill(run_distill(P, z, ids, sc, tau, w), z, ids, sc, tau, w)


@pytest.mark.parametrize("C", [29, 300, 20000, 70000])
def test_scores_whose_difference_is_beyond_fp32(P, C):
    """Losses that fp32 holds, of scores that are up to 6e38 apart."""
    rng = np.random.default_rng(C)
    z, ids, sc, _, _ = distill_case(2, 3, C, 5, "fp32", 6)
    z = np.where(rng.random(z.shape) < 0.5, 2e38, -3e38) + 1e37 * z
    z[..., 0] = 3e38
    z[1, :, 1] = -3e38
    z = np.clip(z, -3.4e38, 3.4e38).astype(np.float32).astype(np.float64)
    ids[0, 0], ids[1] = 0, 1
    sc[1] = np.where(rng.random(sc[1].shape) < 0.5, 3e38, -3e38)
    sc[1, :, 0] = 3e38
    sc = sc.astype(np.float32).astype(np.float64)
    for tau, w in ((2.0 ** -10, 2.0 ** -4), (2.0 ** 10, 2.0 ** -14), (2.0 ** 100, 2.0 ** -104), (2.0 ** 126, 2.0 ** -126)):
        w = np.full((2, 3), w)
        got = run_distill(P, z, ids, sc, tau, w)
        check_distill(got, z, ids, sc, tau, w)
        assert tau > 2.0 ** 120 or (np.all(np.isfinite(got[0])) and np.all(got[0][1] > 0))


@pytest.mark.parametrize("C", [29, 300, 6000, 40001])
def test_factors_whose_product_alone_is_in_range(P, C):
    """weight, grad_scale and temperature, of which two have a product beyond fp32 or below its normal numbers, and all three do not."""
    z, ids, sc, w, in_len = distill_case(2, 5, C, 6, "fp32", 12)
    for tau, weight, gs in ((1e-30, 1e30, 1e30), (1e30, 1e-30, 1e-30), (1e25, 1e-25, 1e25), (1e-25, 1e10, 1e30), (2.0 ** -126, 2.0 ** 100, 2.0 ** 27)):
        tau, weight, gs = (float(np.float32(v)) for v in (tau, weight, gs))
        size = np.float32(tau if tau > 1 else 2.0 ** -20)
        zt, st = ((a * size).astype(np.float32).astype(np.float64) for a in (z, sc))
        wt = (w * weight).astype(np.float32).astype(np.float64)
        got = run_distill(P, zt, ids, st, tau, wt, in_len, gs)
        check_distill(got, zt, ids, st, tau, wt, in_len, gs)
        assert np.all(np.isfinite(got[2])) and np.abs(got[2]).max() > 0
