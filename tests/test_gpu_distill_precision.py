"""w2l_distill_fwd_bwd where its results are small differences of large numbers.  Every element is held to a bound of its own, in units of
U = 2^-24 (half a step of fp32, relative)."""
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

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


# ------------------------------------------------------------------------------------ temperatures whose square multiplies a rounding
def exact_frame(x, ids, t, tau):
    """From the definition, in 130 digits (at tau = 2^126 the loss is tau^2 times 1e-76): tau^2 sum q (log q - log p); tau (p - sum q) and p of the
    classes that the row holds; q at them; tau |y|, the size of the terms that the loss is made of, that over tau, and tau E|y| (y, I and L as in the
    kernel's comment)."""
    with localcontext() as ctx:
        ctx.prec = 130
        D, tau = Decimal, Decimal(float(tau))
        xs = {int(c): D(float(x[c])) - D(float(x.max())) for c in np.nonzero(x > -np.inf)[0]}
        on = [(int(c), D(float(v)) - D(float(t.max()))) for c, v in zip(ids, t) if c >= 0 and v > -np.inf]
        e = {c: (v / tau).exp() for c, v in xs.items()}
        S = sum(e.values())
        w = [(v / tau).exp() for _, v in on]
        Q = sum(w)
        q = [v / Q for v in w]
        d = [xs[c] - v for c, v in on]
        mean = sum(a * b for a, b in zip(q, d))
        entries = (sum(e[c] for c, _ in on) / Q).ln() - mean / tau
        I = sum(e[c] for c, _ in on)
        others = (S / I).ln()
        again = (I - sum(e[c] for c in {c for c, _ in on})) / I
        loss = tau * tau * (entries + others)
        p = {c: v / S for c, v in e.items()}
        dz, qs, ys = ({c: v for c, v in p.items()}, {c: D(0) for c in p}, {c: D(0) for c in p})
        for (c, _), a, b in zip(on, q, d):
            dz[c] -= a
            qs[c] += a
            ys[c] = max(ys[c], abs(b - mean) / tau)
        mean_y = sum(a * abs(b - mean) for a, b in zip(q, d)) / tau
        out = [np.zeros(len(x)) for _ in range(4)]
        for o, src in zip(out, ({c: tau * v for c, v in dz.items()}, p, qs, {c: tau * v for c, v in ys.items()})):
            for c, v in src.items():
                o[c] = float(v)
        terms = [tau * tau * v for v in (abs(entries), abs(others), 2 * again)]
        return (float(loss), *out, float(sum(terms)), float(sum(terms) / tau), float(tau * mean_y))


def warm_case(C, K, dtype, seed):
    """Six frames: a teacher that is the student, one that differs by 1 and one by 2^-10, one that leaves four of the classes out that the student gives weight
    to, one that names some classes twice, one of few entries.  All other classes are -inf."""
    rng = np.random.default_rng(seed + C)
    n = min(C, 64)
    z = np.full((1, 6, C), -np.inf)
    ids, sc = np.full((1, 6, K), -1), np.full((1, 6, K), -np.inf)
    for r in range(6):
        names = rng.permutation(C)[:n]
        z[0, r, names] = rounded(rng.standard_normal(n) * 2, dtype)
        k = min(K, n)
        if r == 3:
            k = max(k - 4, 1)
        if r == 5:
            k = max(k // 8, 1)
        ids[0, r, :k] = names[:k]
        if r < 3 and k < n:
            z[0, r, names[k:]] = -np.inf
        if r == 5:
            z[0, r, names[k:]] = rounded(-8 - rng.random(n - k), dtype)
        sc[0, r, :k] = z[0, r, ids[0, r, :k]] + (0.0, 1.0, 2.0 ** -10, 1.0, 0.5, 0.25)[r] * rng.standard_normal(k)
        if r == 4 and k > 4:
            ids[0, r, k // 2:k // 2 + 2] = ids[0, r, 0]
            ids[0, r, -1] = ids[0, r, 1]
    return z, ids, sc.astype(np.float32).astype(np.float64)


WARM = [(7, 7, 6, "fp32"), (12, 16, 6, "fp32"), (29, 29, 6, "fp32"), (29, 29, 100, "bf16"), (60, 64, 6, "fp32"), (200, 60, 6, "bf16"), (256, 16, 90, "fp32"), (400, 64, 6, "bf16"),
        (1000, 64, 6, "fp32"), (1000, 64, 2100, "bf16"), (4096, 40, 2048, "fp32"), (6000, 64, 6, "fp32"), (20000, 64, 6, "bf16"), (40001, 64, 130, "fp32"),
        (70001, 64, 6, "fp32"), (140001, 50, 6, "bf16"), (262144, 64, 3, "fp32")]


@pytest.mark.parametrize("tau", [4.0, 4.5, 20.0, 100.0, 1e3, 1e5, 1e12, 1e25, 2.0 ** 126])
@pytest.mark.parametrize("C,K,T,dtype", WARM, ids=lambda v: str(v))
def test_ordinary_scores_at_high_temperatures(P, C, K, T, dtype, tau):
    """The loss of ordinary scores tends to half the variance of their differences, and so does its gradient to a limit: nothing of them grows with tau, and
    no error may.  What fp32 leaves, relative:
      q, e      of an exponential of |a| <= 20 / 4: 3 |a| + 2 = 17 U; q's sum and division 6 + 17 U more, so 40 U
      entries   q 40 U, y 4 U, f(y) 30 U (e^y - 1 - y where y = 1/2, 1.65 of the roundings of 0.15; the series 8), log 4 U: 80 U
      others    a quotient of two sums of up to 70 terms: 2 (17 + 70) + 4 U: 180 U; where classes are named again, of the difference of two sums, which are
                no larger than I times |others| + twice the share named again (both logarithms are of numbers next to 1)
      p - q     q (e^(y - L) - 1): q and e^v - 1 48 U;  y, whose mean moves by q's errors, 80 U E|y| + 4 U |y|;  L as above
      p         where the teacher says nothing: 17 + 70 + 17 U and two products
    Up to tau = 4, and of a loss above tau^2 / 4: the logarithms 87 U each, the differences of scores and their sum 8 U of up to 5 tau, in all 250 U (tau^2
    + the loss), and of the gradient 200 U (p + q) tau."""
    T0 = min(T, 6)
    tau = float(np.float32(tau))
    z, ids, sc = (a[:, :T0] for a in warm_case(C, min(K, 64, C), dtype, 3))
    pad = lambda a, v: np.concatenate([a, np.full((1, T - T0) + a.shape[2:], v, a.dtype)], 1)
    w = 0.5 + np.arange(T0)[None] / 8
    held = run_distill(P, pad(z, 0.), pad(ids, -1), pad(sc, 0.), tau, pad(w, 0.), [T0], 0.75, dtype)
    for r in range(T0):
        loss, dz, p, q, y, terms, Lt, mean_y = exact_frame(z[0, r], ids[0, r], sc[0, r], tau)
        near = tau > 4 and loss < 0.25 * tau * tau
        bound = 256 * U * terms if near else 250 * U * (tau * tau + abs(loss))
        close(held[0][0, r], w[0, r] * loss, w[0, r] * (bound + U * abs(loss)) + 2.0 ** -149, "frame_loss of frame %d" % r)
        gs = 0.75 * w[0, r]
        if w[0, r] * loss > np.finfo(np.float32).max:
            assert not held[2][0, r].any()      # a loss beyond fp32 has no gradient
            continue
        if near:
            bound = np.where(q > 0, 48 * U * np.abs(dz) + q * (80 * U * mean_y + 4 * U * y + 256 * U * Lt), 120 * U * p * tau)
        else:
            bound = 200 * U * (p + q) * tau
        close(held[2][0, r], gs * dz, gs * (bound + U * np.abs(dz)) + 2.0 ** -126, "dz of frame %d" % r)
        if r == 0 and near:      # the teacher is the student
            assert held[0][0, r] == 0 and not held[2][0, r].any()
    total = held[0][0, :T0].astype(np.float64).sum()
    close(held[1][0], total, 2 * U * abs(total), "loss")


@pytest.mark.parametrize("dz_dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C,K,T", [(29, 29, 7), (200, 64, 80), (4096, 64, 7), (40001, 64, 7)])
def test_high_temperatures_beside_other_frames(P, C, K, T, dz_dtype):
    """Frames below tau^2 / 4 between frames above it, of weight 0, without entries, with NaN, infinities and classes of probability zero, of repeated
    classes and behind the utterance; their gradients written, added, and left out."""
    rng = np.random.default_rng(C)
    tau = 20.0
    z = rounded(rng.standard_normal((2, T, C)) * 2 - 400 * (np.arange(C) >= K), "bf16")      # the others: e^-20 and less
    ids = np.broadcast_to(np.arange(K), (2, T, K)).copy()
    sc = z[..., :K] + rng.standard_normal((2, T, K))
    w = 0.5 + rng.random((2, T))
    w[0, 1] = 0.0
    ids[0, 2] = -1
    z[0, 3, 5], z[0, 4, 6] = np.nan, np.inf
    z[0, 5, 7] = -np.inf
    sc[0, 6, K // 2:] -= 400.0                     # half of the entries have next to nothing: above tau^2 / 4
    ids[1, 0, 3:6], sc[1, 1, 2], ids[1, 2, 1] = 2, np.nan, C
    w[1, 3] = -w[1, 3]
    w, sc = (a.astype(np.float32).astype(np.float64) for a in (w, sc))
    il = [T, T - 2]
    held = torch.randn(z.shape, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(5)).to(torch.bfloat16 if dz_dtype == "bf16" else torch.float32)
    for acc in (None, held):
        got = run_distill(P, z, ids, sc, tau, w, il, -0.5, "bf16", dz_dtype, acc)
        check_distill(got, z, ids, sc, tau, w, il, -0.5, dz_dtype, acc)
    alone = run_distill(P, z, ids, sc, tau, w, il, -0.5, "bf16", dz_dtype, want=(False, False))
    assert np.array_equal(alone[0], got[0], equal_nan=True) and np.all(alone[2] == -77)
    for b, r in ((0, 0), (1, 3), (1, 4)):
        loss, dz = exact_frame(z[b, r], ids[b, r], sc[b, r], tau)[:2]
        assert 0 < loss < 1 and abs(got[0][b, r] - w[b, r] * loss) <= 2.0 ** -14 * loss


@pytest.mark.parametrize("offset", [2.0 ** 12, -2.0 ** 20, 2.0 ** 30])
@pytest.mark.parametrize("C,K", [(29, 29), (300, 64), (40001, 64)])
def test_large_scores_at_high_temperatures(P, C, K, offset):
    """Ordinary differences of large scores, whose exponents fp32 has to take from differences; weights that are NaN, one of them of any bits."""
    rng = np.random.default_rng(C)
    n = min(C, K)
    z = np.full((1, 6, C), -np.inf)
    z[..., :n] = offset + np.round(rng.standard_normal((1, 6, n)) * 64) / 32
    z = rounded(z, "fp32")
    ids = np.broadcast_to(np.arange(n), (1, 6, n)).copy()
    sc = (z[..., :n] - offset + rng.standard_normal((1, 6, n))).astype(np.float32).astype(np.float64)
    w = np.ones((1, 6), np.float32)
    w[0, 4:] = np.array([0x7fc00001, 0xffc00001], np.uint32).view(np.float32)
    for tau in (5.0, 100.0):
        frame, _, dz = run_distill(P, z, ids, sc, tau, w)
        for r in range(4):
            loss, grad, p, q, y, terms, Lt, mean_y = exact_frame(z[0, r], ids[0, r], sc[0, r], tau)
            assert loss < tau * tau / 4
            close(frame[0, r], loss, 257 * U * terms, "frame_loss")
            close(dz[0, r], grad, 49 * U * np.abs(grad) + q * (80 * U * mean_y + 4 * U * y + 256 * U * Lt), "dz")
        assert np.all(np.isnan(frame[0, 4:])) and not dz[0, 4:].any()


@pytest.mark.parametrize("C,K,T", [(29, 29, 40), (3000, 64, 40), (40001, 64, 3)])
def test_high_temperatures_captured_and_replayed(P, C, K, T):
    g = torch.Generator("cuda:0").manual_seed(C)
    z = torch.empty((2, T, C), device="cuda:0")
    ids = torch.arange(K, dtype=torch.int32, device="cuda:0").expand(2, T, K).contiguous()
    sc = torch.empty((2, T, K), device="cuda:0")

    def fill():
        z.normal_(generator=g)
        z[..., K:] -= 400.0
        sc.copy_(z[..., :K] + torch.randn(sc.shape, device="cuda:0", generator=g))

    def buffers():
        return dict(fl=torch.empty((2, T), device="cuda:0"), ls=torch.empty(2, device="cuda:0"), dz=torch.empty_like(z),
                    ws=P.workspace(P.w2l_distill_workspace_bytes(2, T, C, K, 0)))

    def work(o):
        P.w2l_distill_fwd_bwd(z, ids, sc, o["fl"], o["ls"], o["dz"], temperature=20.0, workspace=o["ws"])

    eager, captured = buffers(), buffers()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    fill()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        work(captured)
    for _ in range(3):
        fill()
        for k in ("fl", "ls", "dz"):
            captured[k].fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        work(eager)
        torch.cuda.synchronize()
        for k in ("fl", "ls", "dz"):
            assert torch.equal(eager[k], captured[k]), k
        assert bool((eager["fl"] > 0).all()) and bool((eager["fl"] < 2).all())
