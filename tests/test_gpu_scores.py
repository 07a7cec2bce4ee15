"""w2l_token_logprob_fwd / _bwd and w2l_distill_fwd_bwd against the fp64 oracles, through the C ABI.

Bounds, in units of U = 2^-24 (half a step of fp32, relative):
  exp(d)          within (2 |d| + 6) U of itself: d is rounded once, its product with log2 e once, the instruction is good to an ulp
  s, u            sums of such terms, at most 160 additions deep: (166 + 2 E|d|) U of s, (166 + 2 E|d|) E|d| U of u / s at most
                  (E|d| = sum p |x - m|, taken from the oracle); log s the same in absolute terms, and rounded once
  log-probability x - m and its difference with log s rounded once each: 2 U |lp| beside the error of log s
  entropy         the errors of log s and u / s, and a rounding
  gradient        p (1 + error of lp) times the row's factor, plus a rounding for each term added; bf16 is rounded by 2^-8 more
Every element is held to its own bound.  Classes are whole numbers and have to be equal."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import DEV, empty, to_dev, to_host
from score_cases import CASES, distill_cases

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


def guarded(shape, dtype=torch.float32, fill=-77):
    """A tensor of `shape` between two bands that nothing may write to, and the check of the bands."""
    n = int(np.prod(shape))
    pad = 1024
    whole = torch.full((n + 2 * pad,), fill, dtype=dtype, device=DEV)

    def untouched():
        assert bool((whole[:pad] == fill).all()) and bool((whole[pad + n:] == fill).all()), "written outside the tensor"
    return whole[pad:pad + n].view(shape), untouched


def rounded(z, dtype):
    """fp64 values as the type holds them."""
    t = torch.from_numpy(np.asarray(z, dtype=np.float32))
    return (t.bfloat16() if dtype == "bf16" else t).double().numpy()


def dev(z, dtype):
    t = torch.from_numpy(np.asarray(z, dtype=np.float32)).to(DEV)
    return t.bfloat16() if dtype == "bf16" else t


def spread(z):
    """E|d| of every row: sum p |x - m| (0 where a row has no distribution)."""
    with np.errstate(invalid="ignore"):
        lp, odd = oracle._log_probs(z)
        p = np.exp(lp)
        m = np.where(np.isfinite(z.max(-1, keepdims=True)), z.max(-1, keepdims=True), 0)
        return np.where(odd, 0.0, (p * np.where(p > 0, np.abs(np.where(odd[..., None], 0, z) - np.where(odd[..., None], 0, m)), 0)).sum(-1))


def close(got, ref, bound, what):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    most = float(np.finfo(np.float32).max) * (1 + 2.0 ** -25)      # what lies beyond is an infinity when rounded to fp32 (IEEE 754, 7.4)
    ref = np.where(np.abs(ref) >= most, np.copysign(np.inf, ref), ref)
    fin = np.isfinite(ref)
    same = np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[~fin & ~np.isnan(ref)], ref[~fin & ~np.isnan(ref)])
    assert same, "%s: other infinities or NaN than the oracle's" % what
    err, bound = np.abs(np.where(fin, got, 0) - np.where(fin, ref, 0)), np.broadcast_to(bound, ref.shape)
    bad = fin & ~(err <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, err / bound, 0)), ref.shape)
        raise AssertionError("%s: %d of %d out of bound; worst at %r: got %r ref %r bound %.3g" % (what, bad.sum(), bad.size, i, got[i], ref[i], bound[i]))


def run_tokens(P, z, tokens, K, in_len=None, dtype="fp32", grads=None, dz_dtype=None, accumulate=None, ws=True):
    """Forward and, given grads (dlogprob, dentropy, dtop), backward call; host copies of all outputs."""
    B, T, C = z.shape
    S = tokens.shape[2]
    zd = dev(z, dtype)
    il = None if in_len is None else to_dev(np.asarray(in_len, np.int32))
    tk = to_dev(tokens) if S else None
    lp, ok1 = guarded((B, T, S))
    H, ok2 = guarded((B, T))
    ids, ok3 = guarded((B, T, K), torch.int32)
    top, ok4 = guarded((B, T, K))
    stats, ok5 = guarded((B, T, 4))
    code = P.W2L_BF16 if dtype == "bf16" else P.W2L_F32
    P.w2l_token_logprob_fwd(zd, tk, lp if S else None, H, ids if K else None, top if K else None, stats, in_len=il,
                            workspace=P.workspace(P.w2l_token_logprob_workspace_bytes(B, T, C, K, code)))
    torch.cuda.synchronize()
    for ok in (ok1, ok2, ok3, ok4, ok5):
        ok()
    out = dict(logprob=to_host(lp), entropy=to_host(H), top_ids=ids.cpu().numpy(), top_logprob=to_host(top), stats=to_host(stats))
    if grads is not None:
        dz, ok6 = guarded((B, T, C), torch.bfloat16 if dz_dtype == "bf16" else torch.float32)
        if accumulate is not None:
            dz.copy_(accumulate)
        gl, gh, gt = (None if g is None else to_dev(g) for g in grads)
        P.w2l_token_logprob_bwd(zd, stats, dz, tk, gl if S else None, gh, ids if K else None, gt if K else None, in_len=il,
                                accumulate=accumulate is not None)
        torch.cuda.synchronize()
        ok6()
        assert torch.equal(zd.nan_to_num(7.), dev(z, dtype).nan_to_num(7.))
        out["dz"] = to_host(dz)
    return out


def check_tokens(got, z, tokens, K, in_len=None, grads=None, dz_dtype="fp32", accumulate=None):
    f = oracle.token_logprob(z, tokens, K, in_len)
    D = spread(z)
    logs = (168 + 2 * D) * U                                       # of log s
    close(got["logprob"], f["logprob"], logs[..., None] + 2 * U * np.abs(np.nan_to_num(f["logprob"], neginf=0)), "logprob")
    ent = logs + (170 + 2 * D) * D * U + 2 * U * np.abs(np.nan_to_num(f["entropy"]))
    close(got["entropy"], f["entropy"], ent, "entropy")
    assert np.array_equal(got["top_ids"], f["top_ids"])
    close(got["top_logprob"], f["top_logprob"], logs[..., None] + 2 * U * np.abs(np.nan_to_num(f["top_logprob"], neginf=0)), "top_logprob")
    if grads is not None:
        gl, gh, gt = grads
        ref = oracle.token_logprob_bwd(z, tokens, gl, gh, f["top_ids"] if gt is not None else None, gt, in_len)
        n = (0 if gl is None else gl.shape[2]) + (0 if gt is None else gt.shape[2])
        mag = sum(np.abs(g).sum(-1) for g in (gl, gt) if g is not None) + np.zeros(D.shape)
        h = np.abs(gh) if gh is not None else np.zeros(D.shape)
        lp = np.where(np.isfinite(f["lp"]), f["lp"], 0)
        p = np.exp(f["lp"])
        factor = mag[..., None] + h[..., None] * np.abs(lp + np.nan_to_num(f["entropy"])[..., None])
        off = logs[..., None] + (2 * np.abs(lp) + 12 + n) * U      # of p, relative, and of lp, absolute
        bound = p * (off * factor + h[..., None] * (off + ent[..., None]))
        direct = np.zeros(z.shape)
        for ids, g in ((tokens, gl), (f["top_ids"], gt)):
            if g is not None:
                ok = (ids >= 0) & (ids < z.shape[2])
                b, t = (np.broadcast_to(i[..., None], ids.shape) for i in np.indices(ids.shape[:2]))
                np.add.at(direct, (b[ok], t[ok], ids[ok]), np.abs(g[ok]))
        # a probability below 2^-126, the least normal fp32, may come out as 0 (the exponential's instruction gives no subnormals):
        # |p - 0| < 2^-126, times the row's factor
        bound = bound + (n + 3) * U * (direct + p * factor) + 2.0 ** -126 * (1 + factor + h[..., None])
        if accumulate is not None:
            before = accumulate.double().cpu().numpy()
            ref = ref + before
            bound = bound + U * np.abs(ref)
        if dz_dtype == "bf16":
            bound = bound * 1.01 + 2.0 ** -8 * np.abs(ref)
        close(got["dz"], ref, bound, "dz")


SIZES = [  # B, T, C, K, S, dtype
    (1, 1, 1, 1, 1, "fp32"), (1, 1, 29, 4, 1, "fp32"), (3, 50, 29, 8, 1, "fp32"), (2, 41, 29, 29, 3, "bf16"), (5, 7, 2, 2, 0, "bf16"),
    (2, 30, 16, 5, 2, "fp32"), (2, 30, 17, 0, 1, "bf16"), (2, 21, 32, 32, 1, "fp32"), (2, 21, 33, 3, 1, "bf16"), (1, 37, 64, 64, 64, "fp32"),
    (3, 11, 65, 64, 1, "bf16"), (2, 9, 127, 1, 2, "fp32"), (2, 33, 256, 16, 1, "bf16"), (2, 13, 257, 64, 1, "fp32"), (1, 19, 511, 10, 1, "bf16"),
    (2, 17, 1000, 64, 5, "fp32"), (2, 9, 1024, 64, 1, "bf16"), (2, 5, 1025, 7, 1, "bf16"), (1, 9, 2049, 40, 1, "fp32"), (3, 5, 4096, 64, 1, "fp32"),
    (2, 6, 4097, 12, 1, "bf16"), (2, 3, 8192, 64, 2, "bf16"), (1, 5, 9997, 16, 1, "bf16"), (2, 3, 16385, 33, 1, "fp32"), (1, 3, 32767, 64, 1, "bf16"),
    (1, 2, 65537, 9, 1, "fp32"), (1, 2, 100003, 40, 1, "bf16"), (1, 1, 131073, 64, 1, "fp32"), (1, 2, 262144, 64, 3, "bf16"), (40, 3, 5003, 2, 1, "fp32"),
]


def token_case(B, T, C, K, S, dtype, seed=0):
    rng = np.random.default_rng(seed + C * 131 + T)
    z = rounded(rng.standard_normal((B, T, C)) * 2.5 + (rng.random((B, T, C)) < 1.5 / C) * 6, dtype)
    tokens = rng.integers(0, C, (B, T, S))
    tokens[rng.random(tokens.shape) < 0.1] = -1
    in_len = rng.integers((T + 1) // 2, T + 1, B)
    grads = (rng.standard_normal((B, T, S)).astype(np.float32).astype(np.float64) if S else None,
             rng.standard_normal((B, T)).astype(np.float32).astype(np.float64),
             rng.standard_normal((B, T, K)).astype(np.float32).astype(np.float64) if K else None)
    return z, tokens, in_len, grads


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_tokens(P, size):
    B, T, C, K, S, dtype = size
    z, tokens, in_len, grads = token_case(*size)
    for dz_dtype in (("fp32", "bf16") if dtype == "bf16" else ("fp32",)):
        check_tokens(run_tokens(P, z, tokens, K, in_len, dtype, grads, dz_dtype), z, tokens, K, in_len, grads, dz_dtype)
    none = np.zeros((B, T, 0), int)
    check_tokens(run_tokens(P, z, none, 0, None, dtype, (None, grads[1], None)), z, none, 0, None, (None, grads[1], None))


@pytest.mark.parametrize("case", CASES, ids=lambda c: "C%d-K%d-%s" % c)
def test_tokens_in_every_form(P, case):
    C, K, dtype = case
    size = (2, 3, C, K, 2, dtype)
    z, tokens, in_len, grads = token_case(*size, seed=7)
    z[:, 1] = rounded(np.sort(z[:, 1], -1)[..., ::-1], dtype)        # classes by their scores, as inventories sorted by frequency are
    dz_dtype = dtype
    check_tokens(run_tokens(P, z, tokens, K, in_len, dtype, grads, dz_dtype), z, tokens, K, in_len, grads, dz_dtype)


def hard_rows(C, dtype):
    """Rows where a statistic or the order can go wrong, as the type holds them."""
    rng = np.random.default_rng(C)
    big = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).max)
    r = [np.full(C, -np.inf), np.full(C, -big), np.full(C, big), np.full(C, 0.0), np.full(C, 1e4)]
    r += [np.where(np.arange(C) == C - 1, 3.0, -np.inf), np.where(np.arange(C) % 7 == 3, rng.standard_normal(C), -np.inf),
          np.where(np.arange(C) < C // 2, -big, rng.standard_normal(C)), np.where(np.arange(C) == 0, big, -big)]
    r += [np.arange(C) * 1.0, -np.arange(C) * 1.0, np.sort(rng.standard_normal(C)), -np.sort(rng.standard_normal(C))]
    r += [rng.integers(0, 3, C) * 1.0, rng.integers(-1, 1, C) * 1e-3 + 2e4, np.where(rng.random(C) < 0.5, 0.0, -0.0)]
    r += [1.2e7 + rng.integers(0, 4, C), -3e8 + 65536. * rng.integers(0, 3, C)]       # differences that k x - M would not keep
    r += [rng.standard_normal(C) * 1e-30, rng.standard_normal(C) * 300, np.where(np.arange(C) // 64 == (C - 1) // 64, 5.0, rng.standard_normal(C))]
    for at in (0, C // 2, C - 1):
        for v in (np.nan, np.inf):
            x = rng.standard_normal(C)
            x[at] = v
            r.append(x)
    both = np.full(C, -np.inf)
    both[0] = np.inf
    r += [both, np.full(C, np.nan), np.full(C, np.inf)]
    return rounded(np.stack(r)[None], dtype)


HARD = [(1, 1), (5, 5), (29, 29), (29, 3), (64, 64), (70, 64), (500, 20), (1024, 64), (3000, 64), (4097, 1), (10001, 64), (50000, 64), (140001, 33)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C,K", HARD)
def test_tokens_of_hard_rows(P, C, K, dtype):
    z = hard_rows(C, dtype)
    T = z.shape[1]
    rng = np.random.default_rng(C + 1)
    tokens = np.stack([rng.integers(0, C, T), np.full(T, C - 1), np.zeros(T, int)], -1)[None]
    gl, gh, gt = (rng.standard_normal(s).astype(np.float32).astype(np.float64) for s in ((1, T, 3), (1, T), (1, T, K)))
    check_tokens(run_tokens(P, z, tokens, K, None, dtype, (gl, gh, gt)), z, tokens, K, None, (gl, gh, gt))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [300, 512, 1000, 9001, 60001])
def test_rows_without_a_distribution_beside_full_lists(P, C, dtype):
    """Rows of equal scores and one NaN or +inf, which leave more candidates than a list holds, between rows whose candidates nearly fill
    theirs: the second kind's classes and log-probabilities are as they would be alone."""
    rng = np.random.default_rng(C)
    rows = []
    for k in range(24):
        x = np.full(C, 1.0)
        if k % 2 == 0:
            x[rng.integers(0, C)] = (np.nan, np.inf)[k // 2 % 2]
        else:
            x[rng.permutation(C)[120 + k // 4:]] = -1.0 - rng.random(C - 120 - k // 4)     # 120 to 125 equal scores, the largest
        rows.append(x)
    z = rounded(np.stack(rows)[None], dtype)
    tokens = rng.integers(0, C, (1, 24, 2))
    check_tokens(run_tokens(P, z, tokens, 64, None, dtype), z, tokens, 64)


def test_tokens_that_are_not_there_and_lengths(P):
    C, K = 37, 5
    rng = np.random.default_rng(8)
    z = rng.standard_normal((6, 9, C)).astype(np.float32).astype(np.float64)
    z[:, -1] = np.nan                                     # padding is not read
    z[4:] = np.nan
    tokens = rng.integers(0, C, (6, 9, 8))
    tokens[0, 0] = [-1, C, -2, 2 ** 31 - 1, -2 ** 31, 3, 3, 3]   # and the same token three times
    in_len = [8, 1, 0, 5, 10, -1]
    grads = tuple(rng.standard_normal(s).astype(np.float32).astype(np.float64) for s in ((6, 9, 8), (6, 9), (6, 9, K)))
    got = run_tokens(P, z, tokens, K, in_len, "fp32", grads)
    check_tokens(got, z, tokens, K, in_len, grads)
    assert np.all(got["dz"][2] == 0) and np.all(got["dz"][4:] == 0) and np.all(np.isnan(got["entropy"][4:])) and np.all(got["stats"][2] == 0)
    held = torch.from_numpy(rng.standard_normal(z.shape).astype(np.float32)).to(DEV)
    got = run_tokens(P, z, tokens, K, in_len, "fp32", grads, accumulate=held)
    check_tokens(got, z, tokens, K, in_len, grads, accumulate=held)
    assert np.array_equal(got["dz"][2], to_host(held)[2])


@pytest.mark.parametrize("C", [29, 700, 6000, 40001])
@pytest.mark.parametrize("dz_dtype", ["fp32", "bf16"])
def test_token_gradient_is_added(P, C, dz_dtype):
    z, tokens, in_len, grads = token_case(2, 5, C, 6, 2, "bf16", 3)
    held = torch.randn((2, 5, C), device=DEV, generator=torch.Generator(DEV).manual_seed(5)).to(torch.bfloat16 if dz_dtype == "bf16" else torch.float32)
    got = run_tokens(P, z, tokens, 6, in_len, "bf16", grads, dz_dtype, held)
    check_tokens(got, z, tokens, 6, in_len, grads, dz_dtype, held)


# ------------------------------------------------------------------------------------ distillation
def run_distill(P, z, ids, sc, tau=1.0, weight=None, in_len=None, gs=1.0, dtype="fp32", dz_dtype="fp32", accumulate=None, want=(True, True)):
    B, T, C = z.shape
    K = ids.shape[2]
    frame, ok1 = guarded((B, T))
    loss, ok2 = guarded((B,))
    dz, ok3 = guarded((B, T, C), torch.bfloat16 if dz_dtype == "bf16" else torch.float32)
    if accumulate is not None:
        dz.copy_(accumulate)
    code = P.W2L_BF16 if dtype == "bf16" else P.W2L_F32
    P.w2l_distill_fwd_bwd(dev(z, dtype), to_dev(ids), to_dev(sc), frame, loss if want[0] else None, dz if want[1] else None,
                          in_len=None if in_len is None else to_dev(np.asarray(in_len, np.int32)), weight=None if weight is None else to_dev(weight),
                          temperature=tau, grad_scale=gs, accumulate=accumulate is not None,
                          workspace=P.workspace(P.w2l_distill_workspace_bytes(B, T, C, K, code)))
    torch.cuda.synchronize()
    for ok in (ok1, ok2, ok3):
        ok()
    return to_host(frame), to_host(loss), to_host(dz)


def check_distill(got, z, ids, sc, tau=1.0, weight=None, in_len=None, gs=1.0, dz_dtype="fp32", accumulate=None):
    frame, loss, dz = oracle.distill(z, ids, sc, tau, weight, in_len, gs)
    lp, odd = oracle._log_probs(z / tau)
    D = spread(z / tau)
    logs = (170 + 2 * D) * U                       # of log s; the scores' product with 1 / tau is one more rounding of d
    w = np.ones(frame.shape) if weight is None else np.where(np.isfinite(weight), np.abs(weight), 0)    # others: no finite loss, no gradient
    here = (ids >= 0) & (ids < z.shape[2])
    with np.errstate(invalid="ignore"):
        at = np.abs(np.where(here, np.take_along_axis(lp, np.where(here, ids, 0), 2), 0))
        t = np.where(here & np.isfinite(sc), sc / tau, -np.inf)
        tm = np.where(np.isfinite(t.max(-1, keepdims=True)), t.max(-1, keepdims=True), 0)
        q = np.where(np.isfinite(t), np.exp(t - tm), 0)
        q = q / np.maximum(q.sum(-1, keepdims=True), 1e-300)
        dt = np.where(np.isfinite(t), np.abs(t - tm), 0)
        span = (q * np.where(np.isfinite(at) & (q > 0), at + dt, 0)).sum(-1)     # size of the logarithms that are subtracted
        Dt = (q * dt).sum(-1)
    bound = w * tau ** 2 * (logs + (80 + 4 * Dt) * U * (1 + span) + 6 * U * span) + 8 * U * np.abs(np.nan_to_num(frame, posinf=0))
    close(got[0], frame, bound, "frame_loss")
    with np.errstate(invalid="ignore"):
        close(got[1], loss, bound.sum(1) + 2 * U * np.abs(np.nan_to_num(loss, posinf=0)), "loss")
    p = np.exp(lp)
    size = p.copy()
    b, r = (np.broadcast_to(i[..., None], ids.shape) for i in np.indices(ids.shape[:2]))
    qs = np.zeros(z.shape)
    np.add.at(qs, (b[here], r[here], ids[here]), np.broadcast_to(q, ids.shape)[here])
    qerr = np.zeros(z.shape)
    np.add.at(qerr, (b[here], r[here], ids[here]), (q * (90 + 4 * Dt[..., None] + 4 * dt) * U)[here])
    lpf = np.where(np.isfinite(lp), lp, 0)
    bound = abs(gs) * tau * w[..., None] * (p * (logs[..., None] + (4 * np.abs(lpf) + 12) * U) + qerr + (ids.shape[2] + 4) * U * (size + qs))
    bound = bound + 2.0 ** -126 * (1 + abs(gs) * tau * w[..., None])         # as above
    if accumulate is not None:
        dz = dz + accumulate.double().cpu().numpy()
        bound = bound + U * np.abs(dz)
    if dz_dtype == "bf16":
        bound = bound * 1.01 + 2.0 ** -8 * np.abs(dz)
    close(got[2], dz, bound, "dz")


def distill_case(B, T, C, K, dtype, seed=0):
    rng = np.random.default_rng(seed + C * 17 + K)
    z = rounded(rng.standard_normal((B, T, C)) * 2, dtype)
    teacher = z + rng.standard_normal(z.shape)
    ids = np.argsort(-teacher, axis=-1)[..., :K]
    sc = np.take_along_axis(teacher, ids, 2).astype(np.float32).astype(np.float64)
    ids = np.where(rng.random(ids.shape) < 0.1, -1, ids)
    w = rng.random((B, T)).astype(np.float32).astype(np.float64)
    return z, ids, sc, w, rng.integers((T + 1) // 2, T + 1, B)


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_distill(P, size):
    B, T, C, K, S, dtype = size
    z, ids, sc, w, in_len = distill_case(B, T, C, max(K, 1), dtype)
    tau = (1.0, 2.0, 0.7, 3.0)[C % 4]
    for dz_dtype in (("fp32", "bf16") if dtype == "bf16" else ("fp32",)):
        got = run_distill(P, z, ids, sc, tau, w, in_len, 0.5, dtype, dz_dtype)
        check_distill(got, z, ids, sc, tau, w, in_len, 0.5, dz_dtype)
    alone = run_distill(P, z, ids, sc, tau, None, None, 1.0, dtype, want=(False, False))
    check = run_distill(P, z, ids, sc, tau, None, None, 1.0, dtype)
    assert np.array_equal(alone[0], check[0]) and np.all(alone[1] == -77) and np.all(alone[2] == -77)
    check_distill(check, z, ids, sc, tau)


@pytest.mark.parametrize("tau", [2.0 ** -126, 1e-30, 1e-12, 1e-3, 1e3, 1e12, 1e25])
@pytest.mark.parametrize("C", [29, 1000, 20000])
def test_distill_at_the_ends_of_the_temperature(P, C, tau):
    """Scores of the temperature's size, so that the distributions are ordinary ones; at the smallest, differences of many temperatures, one class
    with all the weight.  Weights that keep losses and gradients within fp32's normal numbers."""
    z, ids, sc, w, in_len = distill_case(2, 3, C, 5, "fp32")
    tau = float(np.float32(tau))
    size = tau if tau > 1e-6 else 2.0 ** -20
    z, sc = (np.asarray(a * size, np.float32).astype(np.float64) for a in (z, sc))
    w = w / tau if not 1e-6 < tau < 1e10 else w
    w = w.astype(np.float32).astype(np.float64)
    check_distill(run_distill(P, z, ids, sc, tau, w, in_len), z, ids, sc, tau, w, in_len)


def test_distill_of_more_utterances_than_a_launch_has_workgroups(P):
    """2^24 + 5 utterances of one frame of two classes, one of them the teacher's: the frame's loss is -log p of it, the utterance's is the frame's."""
    B = 2 ** 24 + 5
    z = torch.randn((B, 1, 2), device=DEV, generator=torch.Generator(DEV).manual_seed(4))
    ids = torch.ones((B, 1, 1), dtype=torch.int32, device=DEV)
    frame, loss, dz = empty((B, 1)), empty((B,)), torch.empty_like(z)
    P.w2l_distill_fwd_bwd(z, ids, torch.zeros((B, 1, 1), device=DEV), frame, loss, dz)
    torch.cuda.synchronize()
    assert torch.equal(frame[:, 0], loss)
    d = (z[:, 0, 0] - z[:, 0, 1]).double()
    # |d| < 12: d and the loss are rounded once each (12 U), exp(d) by (2 |d| + 6) U of itself (at most 8 U), log s and p follow it (10 U)
    assert float((loss - torch.nn.functional.softplus(d)).abs().max()) <= 64 * U
    assert float((dz[:, 0, 0] - torch.sigmoid(d)).abs().max()) <= 64 * U
    assert float((dz[:, 0, 1] + torch.sigmoid(d)).abs().max()) <= 64 * U


@pytest.mark.parametrize("C", [200, 1000, 20000, 140001])
def test_large_scores(P, C):
    """Rows of one large score, of either sign, and of two neighbouring ones, up to the largest whose products with log2 e fp32 still separates, and
    beyond: what the rounding of such a product moves must not reach a result."""
    rng = np.random.default_rng(C)
    rows = []
    for k in range(8, 27):
        for sign in (1.0, -1.0):
            x = np.full(C, sign * 2.0 ** k * (1 + 0.78125 * rng.random()))
            x[rng.random(C) < 0.5] -= min(2.0 ** (k - 8), 8.0)
            rows.append(x)
    z = rounded(np.stack(rows)[None], "bf16")
    T = z.shape[1]
    ids = rng.integers(0, C, (1, T, 4))
    sc = rng.standard_normal((1, T, 4)).astype(np.float32).astype(np.float64)
    for dz_dtype in ("bf16", "fp32"):
        for gs, tau in ((0.7, 1.0), (-1.5, 2.5)):
            check_distill(run_distill(P, z, ids, sc, tau, None, None, gs, "bf16", dz_dtype), z, ids, sc, tau, None, None, gs, dz_dtype)
        grads = tuple(rng.standard_normal(s).astype(np.float32).astype(np.float64) for s in ((1, T, 4), (1, T), (1, T, 3)))
        check_tokens(run_tokens(P, z, ids, 3, None, "bf16", grads, dz_dtype), z, ids, 3, None, grads, dz_dtype)


def _distill_case_ids():
    import paper_1812_07625_amd as Pm
    return distill_cases(Pm)


@pytest.mark.parametrize("case", _distill_case_ids(), ids=lambda c: "rows%d-C%d-K%d-%s" % c)
def test_distill_in_every_form(P, case):
    rows, C, K, dtype = case
    live = min(rows, 20)
    z, ids, sc, w, _ = distill_case(1, live, C, K, dtype, 11)
    pad = lambda a, v: np.concatenate([a, np.full((1, rows - live) + a.shape[2:], v, a.dtype)], 1)    # what is behind the utterance is not read
    w = np.where(np.arange(live) % 7 == 3, -w, w)
    z, ids, sc, w = pad(z, np.nan), pad(ids, -7), pad(sc, np.nan), pad(w, np.nan)
    for gs in (0.5, -2.0):
        check_distill(run_distill(P, z, ids, sc, 2.0, w, [live], gs, dtype, dtype), z, ids, sc, 2.0, w, [live], gs, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C,K", HARD)
def test_distill_of_hard_rows(P, C, K, dtype):
    z = hard_rows(C, dtype)
    T = z.shape[1]
    rng = np.random.default_rng(C + 2)
    ids = rng.integers(0, C, (1, T, K))
    sc = rng.standard_normal((1, T, K)).astype(np.float32).astype(np.float64)
    check_distill(run_distill(P, z, ids, sc, 2.0, dtype=dtype), z, ids, sc, 2.0)


def test_distill_entries_weights_and_lengths(P):
    C, K = 37, 5
    rng = np.random.default_rng(18)
    z = rng.standard_normal((7, 9, C)).astype(np.float32).astype(np.float64)
    ids, sc = rng.integers(0, C, (7, 9, K)), rng.standard_normal((7, 9, K)).astype(np.float32).astype(np.float64)
    w = rng.random((7, 9)).astype(np.float32).astype(np.float64)
    z[5:] = np.nan
    in_len = [9, 1, 0, 5, 9, 10, -1]
    ids[0, 0] = -1                                        # no entry
    sc[0, 1] = -np.inf
    ids[0, 2] = [4, 4, 4, -1, 9]                          # the same class three times
    ids[0, 3, 2], ids[0, 4, 2], ids[0, 5, 2] = C, -2, 2 ** 31 - 1
    sc[0, 6, 1], sc[0, 7, 1] = np.nan, np.inf
    ids[0, 8, 3], sc[0, 8, 3] = -1, np.nan                # the score of an entry that is not there
    z[4, 0, ids[4, 0, 0]] = -np.inf                       # weight on a class of probability zero
    z[4, 1, 3], z[4, 2, 3] = np.nan, np.inf
    w[4, 3], z[4, 3], sc[4, 3] = 0.0, np.nan, np.nan      # weight 0: not read
    w[4, 4], w[4, 5], w[4, 6] = np.nan, -1.5, np.inf
    for acc in (None, torch.from_numpy(rng.standard_normal(z.shape).astype(np.float32)).to(DEV)):
        got = run_distill(P, z, ids, sc, 1.5, w, in_len, accumulate=acc)
        check_distill(got, z, ids, sc, 1.5, w, in_len, accumulate=acc)
        assert got[1][2] == 0 and np.isnan(got[1][5]) and np.isnan(got[1][6]) and np.isnan(got[1][0])
    assert got[0][4, 0] == np.inf


@pytest.mark.parametrize("C", [29, 700, 6000, 40001])
@pytest.mark.parametrize("dz_dtype", ["fp32", "bf16"])
def test_distill_gradient_is_added(P, C, dz_dtype):
    z, ids, sc, w, in_len = distill_case(2, 5, C, 6, "bf16", 3)
    held = torch.randn((2, 5, C), device=DEV, generator=torch.Generator(DEV).manual_seed(5)).to(torch.bfloat16 if dz_dtype == "bf16" else torch.float32)
    got = run_distill(P, z, ids, sc, 2.0, w, in_len, 1.0, "bf16", dz_dtype, held)
    check_distill(got, z, ids, sc, 2.0, w, in_len, 1.0, dz_dtype, held)


@pytest.mark.parametrize("B,T", [(1, 1), (64, 1), (1, 64), (5, 12), (1, 65), (9, 8)])
def test_distill_losses_of_few_frames(P, B, T):
    """Up to 64 frames of a short row are one workgroup's, utterance losses included."""
    z, ids, sc, w, in_len = distill_case(B, T, 29, 8, "fp32", 5)
    check_distill(run_distill(P, z, ids, sc, 2.0, w, in_len), z, ids, sc, 2.0, w, in_len)


@pytest.mark.parametrize("C,T,dtype", [(40001, 230, "fp32"), (9000, 2100, "bf16")])
def test_large_gradients(P, C, T, dtype):
    """Gradients of more than 32 MB, which are stored past the caches: written, added, and zeros behind the utterance."""
    live = 12
    z, tokens, _, grads = token_case(1, live, C, 4, 1, dtype, 9)
    pad = lambda a, v: np.concatenate([a, np.full((1, T - live) + a.shape[2:], v, a.dtype)], 1)
    z, tokens, grads = pad(z, np.nan), pad(tokens, -1), tuple(pad(g, 0.) for g in grads)
    ids, sc = pad(np.argsort(-z[:, :live], -1)[..., :5], -1), pad(-np.sort(-z[:, :live], -1)[..., :5], 0.)
    held = torch.full((1, T, C), 0.5, device=DEV).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    for acc in (None, held):
        check_tokens(run_tokens(P, z, tokens, 4, [live], dtype, grads, dtype, acc), z, tokens, 4, [live], grads, dtype, acc)
        check_distill(run_distill(P, z, ids, sc, 1.0, None, [live], 1.0, dtype, dtype, acc), z, ids, sc, 1.0, None, [live], 1.0, dtype, acc)


def test_offsets_beyond_32_bits(P):
    """Frames at the end of a tensor of more than 2^31 scores give what they give alone."""
    C, B, K = 70000, 31000, 5
    g = torch.Generator(DEV).manual_seed(3)
    z = torch.empty((B, 1, C), dtype=torch.bfloat16, device=DEV)
    assert z.numel() > 2 ** 31
    z[-2:] = torch.randn((2, 1, C), generator=g, device=DEV)
    il = torch.zeros(B, dtype=torch.int32, device=DEV)
    il[-2:] = 1
    tok = torch.randint(0, C, (B, 1, 1), generator=g, device=DEV, dtype=torch.int32)
    gl, gh = torch.ones((B, 1, 1), device=DEV), torch.ones((B, 1), device=DEV)

    def run(z, tok, gl, gh, il):
        n = z.shape[0]
        o = dict(lp=empty((n, 1, 1)), H=empty((n, 1)), ids=torch.zeros((n, 1, K), dtype=torch.int32, device=DEV), top=empty((n, 1, K)), st=empty((n, 1, 4)))
        P.w2l_token_logprob_fwd(z, tok, o["lp"], o["H"], o["ids"], o["top"], o["st"], in_len=il,
                                workspace=P.workspace(P.w2l_token_logprob_workspace_bytes(n, 1, C, K, P.W2L_BF16)))
        dz = torch.zeros_like(z)
        P.w2l_token_logprob_bwd(z, o["st"], dz, tok, gl, gh, in_len=il, accumulate=True)
        o["dz"] = dz[-2:].clone()
        dz.zero_()
        o["fl"] = empty((n, 1))
        P.w2l_distill_fwd_bwd(z, o["ids"], o["top"], o["fl"], None, dz, in_len=il, temperature=2.0, accumulate=True,
                              workspace=P.workspace(P.w2l_distill_workspace_bytes(n, 1, C, K, P.W2L_BF16)))
        o["dk"] = dz[-2:].clone()
        torch.cuda.synchronize()
        return {k: v[-2:].clone() for k, v in o.items()}

    far = run(z, tok, gl, gh, il)
    near = run(z[-2:].clone(), tok[-2:].clone(), gl[-2:].clone(), gh[-2:].clone(), il[-2:].clone())
    for k in near:
        if k in ("dk", "fl"):       # by other numbers of workgroups a row: other roundings of the sums
            assert torch.allclose(far[k].float(), near[k].float(), rtol=2 ** -7, atol=1e-6), k
        else:
            assert torch.equal(far[k], near[k]), k


def test_same_results_twice_and_on_two_streams(P):
    """Bit-reproducible, whatever runs beside: two streams with workspaces of their own."""
    C, K, T = 50001, 64, 40
    zd = torch.randn((1, T, C), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).bfloat16()
    def call():
        o = [torch.zeros((1, T, K), dtype=torch.int32, device=DEV), empty((1, T, K)), empty((1, T)), empty((1, T)), empty((1, T, C))]
        P.w2l_token_logprob_fwd(zd, entropy=o[2], top_ids=o[0], top_logprob=o[1], workspace=P.workspace(P.w2l_token_logprob_workspace_bytes(1, T, C, K, 1)))
        P.w2l_distill_fwd_bwd(zd, o[0], o[1], o[3], None, o[4], workspace=P.workspace(P.w2l_distill_workspace_bytes(1, T, C, K, 1)))
        return o
    first = call()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    out = []
    for st in (a, b, a, b):
        with torch.cuda.stream(st):
            out.append(call())
    torch.cuda.synchronize()
    for o in out:
        assert all(torch.equal(x, y) for x, y in zip(first, o))


# ------------------------------------------------------------------------------------ together
def test_teacher_to_student_with_ctc(P):
    """As a training program uses them: the teacher's best classes from its scores, then the student's CTC loss and gradient, to which
    the distillation's gradient is added."""
    B, T, C, K, L = 3, 60, 29, 6, 9
    rng = np.random.default_rng(21)
    teacher = (rng.standard_normal((B, T, C)) * 3).astype(np.float32)
    student = (rng.standard_normal((B, T, C)) * 2).astype(np.float32)
    targets, il, tl = rng.integers(1, C, (B, L)).astype(np.int32), np.array([60, 47, 33], np.int32), np.array([9, 5, 7], np.int32)
    ild = to_dev(il)
    ids, top = torch.empty((B, T, K), dtype=torch.int32, device=DEV), empty((B, T, K))
    P.w2l_token_logprob_fwd(to_dev(teacher), top_ids=ids, top_logprob=top, in_len=ild,
                            workspace=P.workspace(P.w2l_token_logprob_workspace_bytes(B, T, C, K, 0)))
    zs, loss, grad = to_dev(student), empty((B,)), empty((B, T, C))
    P.w2l_ctc_fwd_bwd(zs, 1, to_dev(targets), ild, to_dev(tl), loss, grad, 0, 1.0, P.workspace(P.w2l_ctc_workspace_bytes(B, T, C, L)))
    before = grad.clone()
    frame, kd = empty((B, T)), empty((B,))
    P.w2l_distill_fwd_bwd(zs, ids, top, frame, kd, grad, in_len=ild, temperature=2.0, grad_scale=0.3, accumulate=True,
                          workspace=P.workspace(P.w2l_distill_workspace_bytes(B, T, C, K, 0)))
    torch.cuda.synchronize()
    f = oracle.token_logprob(teacher, np.zeros((B, T, 0), int), K, il)
    assert np.array_equal(ids.cpu().numpy(), f["top_ids"])
    check_distill((to_host(frame), to_host(kd), to_host(grad)), student.astype(np.float64), ids.cpu().numpy(), to_host(top), 2.0, None, il, 0.3,
                  accumulate=before)
    _, _, kd_o = oracle.distill(student, f["top_ids"], f["top_logprob"], 2.0, None, il, 0.3)
    loss_o, _, dz_o = oracle.ctc_from_logits(student.astype(np.float64), targets, il, tl)
    assert np.all(np.abs(to_host(loss) - loss_o) <= 1e-4 * np.abs(loss_o))
    assert np.linalg.norm(to_host(grad) - dz_o - kd_o) <= 1e-4 * np.linalg.norm(dz_o + kd_o)


@pytest.mark.parametrize("B,T,C,K,dtype", [(4, 20, 29, 8, "fp32"), (2, 6, 5000, 16, "bf16"), (1, 2, 100003, 40, "bf16")])
def test_captured_and_replayed_on_another_stream(P, B, T, C, K, dtype):
    """Forward, backward and distillation captured into a graph on a stream of its own; replays, on new inputs and with eager calls in
    between, give the eager results bit for bit."""
    code = P.W2L_BF16 if dtype == "bf16" else P.W2L_F32
    rng = np.random.default_rng(31)
    zd = torch.empty((B, T, C), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=DEV)
    tok, il = torch.zeros((B, T, 1), dtype=torch.int32, device=DEV), to_dev(np.full(B, T, np.int32))
    gl, gh = empty((B, T, 1)), empty((B, T))

    def buffers():
        return dict(lp=empty((B, T, 1)), H=empty((B, T)), ids=torch.zeros((B, T, K), dtype=torch.int32, device=DEV), top=empty((B, T, K)),
                    st=empty((B, T, 4)), dz=empty((B, T, C)), fl=empty((B, T)), ls=empty((B,)), dk=empty((B, T, C), dtype),
                    w1=P.workspace(P.w2l_token_logprob_workspace_bytes(B, T, C, K, code)), w2=P.workspace(P.w2l_distill_workspace_bytes(B, T, C, K, code)))

    def work(o):
        P.w2l_token_logprob_fwd(zd, tok, o["lp"], o["H"], o["ids"], o["top"], o["st"], in_len=il, workspace=o["w1"])
        P.w2l_token_logprob_bwd(zd, o["st"], o["dz"], tok, gl, gh, in_len=il)
        P.w2l_distill_fwd_bwd(zd, o["ids"], o["top"], o["fl"], o["ls"], o["dk"], in_len=il, temperature=2.0, workspace=o["w2"])

    def fill(seed):
        r = np.random.default_rng(seed)
        zd.copy_(dev(r.standard_normal((B, T, C)) * 2, dtype))
        tok.copy_(to_dev(r.integers(0, C, (B, T, 1))))
        gl.copy_(to_dev(r.standard_normal((B, T, 1))))
        gh.copy_(to_dev(r.standard_normal((B, T))))

    eager, captured = buffers(), buffers()
    side = torch.cuda.Stream()
    fill(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        work(captured)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            work(captured)
    torch.cuda.synchronize()
    for seed in (1, 2, 3):
        fill(seed)
        for k in ("lp", "H", "top", "st", "dz", "fl", "ls", "dk"):
            captured[k].fill_(float("nan"))
        captured["ids"].fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        work(eager)
        torch.cuda.synchronize()
        for k in eager:
            if k not in ("w1", "w2"):
                assert torch.equal(eager[k], captured[k]), (seed, k)


def test_binding_refuses_what_does_not_fit(P):
    z = torch.zeros((2, 3, 5), device=DEV)
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    f = lambda *s: torch.zeros(s, device=DEV)
    for bad in (dict(tokens=i(2, 3, 1), logprob=f(2, 3, 2)), dict(tokens=i(2, 4, 1), logprob=f(2, 3, 1)), dict(entropy=f(3, 2)),
                dict(stats=f(2, 3, 3)), dict(top_ids=i(2, 3, 2), top_logprob=f(2, 3, 1)), dict(in_len=i(3)), dict(entropy=torch.zeros(2, 3))):
        with pytest.raises(ValueError):
            P.w2l_token_logprob_fwd(z, **bad)
    for bad in (dict(tokens=i(2, 3, 1).long(), logprob=f(2, 3, 1)), dict(entropy=f(2, 3).double())):
        with pytest.raises(TypeError):
            P.w2l_token_logprob_fwd(z, **bad)
    with pytest.raises(TypeError):
        P.w2l_token_logprob_fwd(z.half(), entropy=f(2, 3))
    with pytest.raises(ValueError):
        P.w2l_token_logprob_fwd(z.transpose(0, 1), entropy=f(3, 2))
    with pytest.raises(P.W2LError):
        P.w2l_token_logprob_fwd(f(31)[1:].view(2, 3, 5), entropy=f(2, 3))          # not 16-byte aligned
    with pytest.raises(P.W2LError):
        P.w2l_token_logprob_fwd(z, top_ids=i(2, 3, 6), top_logprob=f(2, 3, 6))    # more alternatives than classes
    with pytest.raises(P.W2LError):
        P.w2l_token_logprob_bwd(z, f(2, 3, 4), torch.zeros((2, 3, 5), dtype=torch.bfloat16, device=DEV), i(2, 3, 1), f(2, 3, 1))
    with pytest.raises(ValueError):
        P.w2l_distill_fwd_bwd(z, i(2, 3, 2), f(2, 3, 3), f(2, 3))
    with pytest.raises(ValueError):
        P.w2l_distill_fwd_bwd(z, i(2, 3, 2), f(2, 3, 2), f(2, 3), dz=f(2, 3, 4))
    with pytest.raises(P.W2LError):
        P.w2l_distill_fwd_bwd(z, i(2, 3, 2), f(2, 3, 2), f(2, 3), temperature=0.0)
    torch.cuda.synchronize()
