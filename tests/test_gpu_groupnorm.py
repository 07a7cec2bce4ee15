"""w2l_groupnorm_fwd / _bwd against the fp64 oracle, through the C ABI.

Bounds, in units of U = 2^-24 (half a step of fp32, relative); for a group, R is the span of its values, M the largest magnitude, sd = 1 / rstd:
  mean      a thread sums up to 64 deviations from one of its values: 64 U R; its mean rounded: U M; the rest in 64 bits; rounded: 2 U M
  rstd      squares of those deviations, each at most R^2: 68 U R^2 / sd^2 of the variance (66 additions and roundings, and the mean's rounding squared); half
            of that, and 6 U for division, root and reciprocal
  xhat      (64 U R + 3 U M) / sd from the mean, its own share of rstd's error, 3 U
  u         gamma times that, and 3 U (|gamma xhat| + |beta|)
  sigmoid   within 10 U of itself (exponential, sum, reciprocal: the argument's rounding is u's)
  y         the activation's slope (at most 1.1 for SiLU, 1 and |a| / 4 for GLU) times u's error, and 12 U |y|
  du        the slope's own slope (1/2 for SiLU; GLU 1/4 for the value, 1/4 and |a| / 10 for the gate) times u's error, 16 U |du|.  ReLU: where |u| is
            below its error either slope is right
  sums      of n values by threads of up to 128, then lanes, then runs of frames: (128 + 16 + 2 log2 n) U of the sum of magnitudes
bf16 outputs add 2^-8 of the value.  Every element is held to its own bound, and whole tensors to the relative L2 of 1e-5 (bf16 3e-3) that the repository's single
kernels have."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import BF16_L2, DEV, to_dev, to_host
from norm_cases import ACTS, SHAPES, code, fits

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


def guarded(shape, dtype):
    """A tensor of `shape` between two bands that nothing may write to, and the check of the bands."""
    n, pad = int(np.prod(shape)), 1024
    whole = torch.full((n + 2 * pad,), -77, dtype=dtype, device=DEV)

    def untouched():
        assert bool((whole[:pad] == -77).all()) and bool((whole[pad + n:] == -77).all()), "written outside the tensor"
    return whole[pad:pad + n].view(shape), untouched


def held(x, dtype):
    """fp64 values as the type holds them."""
    t = torch.from_numpy(np.asarray(x, dtype=np.float32))
    return (t.bfloat16() if dtype == "bf16" else t).double().numpy()


def on_gpu(x, dtype):
    t = torch.from_numpy(np.asarray(x, dtype=np.float32)).to(DEV)
    return t.bfloat16() if dtype == "bf16" else t


def run(P, x, G, gamma, beta, n, act, dtype, dy=None, eps=1e-5, accumulate=None, stream=None):
    B, T, C = x.shape
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    Cy = C // 2 if act == "glu" else C
    xd, gd, bd = on_gpu(x, dtype), None if gamma is None else to_dev(gamma), None if beta is None else to_dev(beta)
    nd = None if n is None else to_dev(np.asarray(n, np.int32))
    y, ok1 = guarded((B, T, Cy), td)
    mean, ok2 = guarded((B, G), torch.float32)
    rstd, ok3 = guarded((B, G), torch.float32)
    ws = P.workspace(P.w2l_groupnorm_workspace_bytes(B, T, C, G, code(P, act), P.W2L_BF16 if dtype == "bf16" else P.W2L_F32))
    P.w2l_groupnorm_fwd(xd, y, mean, rstd, gd, bd, in_len=nd, eps=eps, act=code(P, act), workspace=ws)
    out = dict(y=y, mean=mean, rstd=rstd)
    checks = [ok1, ok2, ok3]
    if dy is not None:
        out["dx"], ok = guarded((B, T, C), td)
        checks.append(ok)
        for k in ("dgamma", "dbeta"):
            out[k], ok = guarded((C,), torch.float32)
            checks.append(ok)
            if accumulate is not None:
                out[k].copy_(to_dev(accumulate))
        ws.random_(0, 255)                                                 # nothing is kept there between the calls
        P.w2l_groupnorm_bwd(xd, on_gpu(dy, dtype), mean, rstd, out["dx"], gd, bd, out["dgamma"], out["dbeta"], in_len=nd, act=code(P, act),
                            accumulate=accumulate is not None, workspace=ws)
    torch.cuda.synchronize()
    for ok in checks:
        ok()
    return {k: to_host(v) for k, v in out.items()}


def close(got, ref, bound, what):
    assert got.shape == ref.shape and np.array_equal(np.isnan(got), np.isnan(ref)), what
    err = np.where(np.isnan(ref), 0, np.abs(got - np.where(np.isnan(ref), got, ref)))
    bad = err > bound
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, err / np.maximum(bound, 1e-300), 0)), ref.shape)
        raise AssertionError("%s: %d of %d out of bound; worst at %r: got %r ref %r bound %.3g" % (what, bad.sum(), bad.size, i, got[i], ref[i], np.broadcast_to(bound, ref.shape)[i]))


def near(got, ref, dtype, what):
    d, n = np.linalg.norm(np.nan_to_num(got - ref)), np.linalg.norm(np.nan_to_num(ref))
    assert d <= (BF16_L2 if dtype == "bf16" else 1e-5) * n + 1e-30, "%s: relative L2 %.3g" % (what, d / n)


def check(got, x, G, gamma, beta, n, act, dtype, dy=None, eps=1e-5, accumulate=None, l2=True):
    o = oracle.groupnorm(x, G, gamma, beta, n, eps, act, dy)
    B, T, C = x.shape
    live = np.arange(T)[None] < (np.full(B, T) if n is None else np.asarray(n))[:, None]
    xz = np.where(live[..., None], x, 0)
    g = lambda a: a.reshape(B, T, G, C // G)
    count = np.maximum(live.sum(1) * (C // G), 1)[:, None]
    lo = np.where(live[..., None], x, np.inf).reshape(B, T, G, -1).min((1, 3))
    hi = np.where(live[..., None], x, -np.inf).reshape(B, T, G, -1).max((1, 3))
    R = np.where(np.isfinite(hi - lo), hi - lo, 0)
    M = np.abs(g(xz)).max((1, 3))
    rs = np.nan_to_num(o["rstd"])
    e_mean = 64 * U * R + 3 * U * M
    e_rstd = 34 * U * R ** 2 * rs ** 2 + (e_mean * rs) ** 2 + 6 * U        # relative
    close(got["mean"], o["mean"], e_mean, "mean")
    close(got["rstd"], o["rstd"], e_rstd * rs, "rstd")
    wide = lambda a: np.repeat(a, C // G, 1)[:, None]
    hat, u = o["hat"], o["u"]
    gm = np.ones(C) if gamma is None else np.asarray(gamma, np.float64)
    bt = np.zeros(C) if beta is None else np.asarray(beta, np.float64)
    e_hat = wide(e_mean * rs) + np.abs(hat) * (wide(e_rstd) + 3 * U)
    e_u = np.abs(gm) * e_hat + 3 * U * (np.abs(gm * hat) + np.abs(bt))
    low = 2.0 ** -8 if dtype == "bf16" else 0.0
    h = C // 2
    if act == "glu":
        a = np.abs(u[..., :h])
        e_y = e_u[..., :h] + a / 4 * e_u[..., h:]
    else:
        e_y = e_u * (1.1 if act == "silu" else 1)
    y = np.nan_to_num(o["y"])
    close(got["y"], o["y"], np.where(live[..., None], e_y, 0) + (12 * U + low) * np.abs(y), "y")
    if l2:
        near(got["y"], o["y"], dtype, "y")
    if dy is None:
        return
    d = np.abs(np.where(live[..., None], dy, 0))
    du = o["du"]
    if act == "glu":
        e_du = np.concatenate((d / 4 * e_u[..., h:], d * (e_u[..., :h] / 4 + a / 10 * e_u[..., h:])), -1)
    elif act == "silu":
        e_du = d * e_u / 2
    elif act == "relu":
        e_du = d * (np.abs(u) <= e_u)
    else:
        e_du = np.zeros(u.shape)
    e_du = np.where(live[..., None], e_du + 16 * U * np.abs(du), 0)
    k = lambda m: 144 + 2 * np.log2(m + 1)
    s1, s2 = np.abs(du), np.abs(du * hat)
    e1, e2 = e_du, e_du * np.abs(hat) + s1 * e_hat
    total = live.sum()
    extra = 0 if accumulate is None else np.asarray(accumulate, np.float64)
    for name, mag, e in (("dbeta", s1, e1), ("dgamma", s2, e2)):
        ref = o[name] + extra
        close(got[name], ref, k(total) * U * mag.sum((0, 1)) + e.sum((0, 1)) + U * np.abs(ref) + 2.0 ** -149, name)
    mean_of = lambda v: g(v).sum((1, 3)) / count
    m1, m2 = mean_of(gm * du), mean_of(gm * du * hat)
    e_m1 = k(count) * U * mean_of(np.abs(gm) * s1) + mean_of(np.abs(gm) * e1)
    e_m2 = k(count) * U * mean_of(np.abs(gm) * s2) + mean_of(np.abs(gm) * e2)
    e_dx = np.abs(gm) * e_du + wide(e_m1) + np.abs(hat) * wide(e_m2) + wide(np.abs(m2)) * e_hat + 4 * U * (np.abs(gm * du) + wide(np.abs(m1)) + np.abs(hat) * wide(np.abs(m2)))
    e_dx = np.where(live[..., None], e_dx * wide(rs), 0) + np.abs(o["dx"]) * (wide(e_rstd) + 2 * U + low)
    close(got["dx"], o["dx"], e_dx, "dx")
    if l2:
        near(got["dx"], o["dx"], dtype, "dx")


def case(seed, B, T, C, act, dtype, level=1.0):
    rng = np.random.default_rng(seed)
    x = held(rng.standard_normal((B, T, C)) * (0.5 + rng.random(C)) + level * rng.standard_normal(C), dtype)
    dy = held(rng.standard_normal((B, T, C // 2 if act == "glu" else C)), dtype)
    f = lambda a: a.astype(np.float32).astype(np.float64)
    return x, f(1 + 0.3 * rng.standard_normal(C)), f(0.3 * rng.standard_normal(C)), dy


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_directions(P, shape, dtype, act):
    B, T, C, G = shape
    if not fits(shape, act):
        pytest.skip("GLU halves the channels")
    x, gamma, beta, dy = case(C + T, B, T, C, act, dtype)
    few = T * C // G < 64                                                 # groups of few values: their gradients cancel, and have their own bounds alone
    n = np.maximum(T - 7 * np.arange(B), 1)
    check(run(P, x, G, gamma, beta, n, act, dtype, dy), x, G, gamma, beta, n, act, dtype, dy, l2=not few)


# utterances whose sums are joined a few channels at a time; runs so many that a lane joins batches of them; groups of rows wider than a workgroup's vectors
@pytest.mark.parametrize("shape,group", [((600, 9, 24, 3), 1), ((1, 3000, 2048, 64), 0), ((1, 300, 8192, 64), 1)], ids=str)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_long_joins(P, shape, group, dtype):
    B, T, C, G = shape
    assert P.w2l_groupnorm_launch_config(*shape, P.W2L_ACT_SILU, P.W2L_BF16 if dtype == "bf16" else P.W2L_F32)[0] == group
    x, gamma, beta, dy = case(C + B, B, T, C, "silu", dtype)
    check(run(P, x, G, gamma, beta, None, "silu", dtype, dy), x, G, gamma, beta, None, "silu", dtype, dy)


@pytest.mark.parametrize("C", [7, 9, 31, 255])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_odd_channels(P, C, dtype):
    x, gamma, beta, dy = case(C, 2, 37, C, "silu", dtype)
    for G in (1, C):
        check(run(P, x, G, gamma, beta, None, "silu", dtype, dy), x, G, gamma, beta, None, "silu", dtype, dy)


@pytest.mark.parametrize("act", ["none", "glu"])
def test_without_gamma_or_beta(P, act):
    x, gamma, beta, dy = case(3, 2, 50, 64, act, "fp32")
    for gm, bt in ((None, None), (gamma, None), (None, beta)):
        check(run(P, x, 8, gm, bt, None, act, "fp32", dy), x, 8, gm, bt, None, act, "fp32", dy)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_frames_that_are_not_there_are_not_read(P, dtype):
    B, T, C, G = 7, 130, 64, 4
    n = [130, 129, 64, 1, 0, -1, 131]
    for act in ACTS:
        x, gamma, beta, dy = case(11, B, T, C, act, dtype)
        for b, k in enumerate(n):
            x[b, max(k, 0):] = [np.nan, np.inf, -np.inf, 3e38][b % 4] if k < T else 0
            dy[b, max(k, 0):] = np.nan
        if dtype == "bf16":
            x = held(x, dtype)
        got = run(P, x, G, gamma, beta, n, act, dtype, dy)
        clean = [k if 0 <= k <= T else 0 for k in n]
        xc = np.where(np.arange(T)[None, :, None] < np.array(clean)[:, None, None], x, 0)
        dc = np.where(np.arange(T)[None, :, None] < np.array(clean)[:, None, None], dy, 0)
        for name in ("y", "mean", "rstd"):
            assert np.isnan(got[name][5:]).all(), name
            got[name][5:] = 0
        assert not got["dx"][5:].any()
        check(got, xc, G, gamma, beta, clean, act, dtype, dc)
        for b, k in enumerate(clean):
            assert not got["y"][b, k:].any() and not got["dx"][b, k:].any()
        assert not got["mean"][4].any() and not got["rstd"][4].any()


def test_a_group_with_nan_is_nan_and_the_others_are_not(P):
    x, gamma, beta, dy = case(12, 2, 40, 32, "none", "fp32")
    x[1, 3, 9] = np.nan
    x[0, 5, 30] = np.inf
    got = run(P, x, 4, gamma, beta, None, "none", "fp32", dy)
    bad = np.zeros((2, 4), bool)
    bad[1, 1] = bad[0, 3] = True
    assert np.array_equal(np.isnan(got["y"]).reshape(2, 40, 4, 8).all((1, 3)), bad) and np.array_equal(np.isnan(got["y"]).reshape(2, 40, 4, 8).any((1, 3)), bad)
    assert np.array_equal(np.isnan(got["dx"]).reshape(2, 40, 4, 8).any((1, 3)), bad)


@pytest.mark.parametrize("level", [100.0, 3000.0])
def test_levels_far_above_the_deviation(P, level):
    """Channels of one level, thousands of deviations from 0: what mean(x^2) - mean(x)^2 would lose."""
    rng = np.random.default_rng(13)
    x = held(level + rng.standard_normal((2, 300, 64)), "fp32")
    dy = held(rng.standard_normal(x.shape), "fp32")
    check(run(P, x, 4, None, None, None, "silu", "fp32", dy), x, 4, None, None, None, "silu", "fp32", dy, l2=False)


def test_values_without_deviation(P):
    x = np.full((1, 50, 16), 3.0)
    dy = np.ones(x.shape)
    got = run(P, x, 2, None, np.full(16, 0.5), None, "none", "fp32", dy, eps=1e-3)
    assert np.array_equal(got["y"], np.full(x.shape, 0.5)) and np.allclose(got["rstd"], 1e-3 ** -0.5, rtol=1e-6) and np.abs(got["dx"]).max() < 1e-4


@pytest.mark.parametrize("T,C,G,lengths", [(90, 48, 6, [90, 10, 55]), (90, 48, 6, [71]), (2500, 58, 1, [2500, 800]), (2500, 58, 1, [2000])], ids=str)
def test_gradients_are_added(P, T, C, G, lengths):
    x, gamma, beta, dy = case(14, len(lengths), T, C, "glu", "bf16")
    before = np.random.default_rng(15).standard_normal(C).astype(np.float32).astype(np.float64)
    check(run(P, x, G, gamma, beta, lengths, "glu", "bf16", dy, accumulate=before), x, G, gamma, beta, lengths, "glu", "bf16", dy, accumulate=before)


@pytest.mark.parametrize("B,T,G", [(2, 30, 3), (1, 30, 3), (2, 3000, 1)])
def test_one_gradient_alone(P, B, T, G):
    x, gamma, beta, dy = case(16, B, T, 24, "silu", "fp32")
    full = run(P, x, G, gamma, beta, None, "silu", "fp32", dy)
    xd, dyd, gd, bd = to_dev(x), to_dev(dy), to_dev(gamma), to_dev(beta)
    y, mean, rstd = torch.empty_like(xd), torch.empty(B, G, device=DEV), torch.empty(B, G, device=DEV)
    ws = P.workspace(P.w2l_groupnorm_workspace_bytes(B, T, 24, G, P.W2L_ACT_SILU, P.W2L_F32))
    P.w2l_groupnorm_fwd(xd, y, mean, rstd, gd, bd, act=P.W2L_ACT_SILU, workspace=ws)
    for which in ("dgamma", "dbeta", None):
        out = torch.empty(24, device=DEV)
        dx = torch.empty_like(xd)
        P.w2l_groupnorm_bwd(xd, dyd, mean, rstd, dx, gd, bd, act=P.W2L_ACT_SILU, workspace=ws, **({which: out} if which else {}))
        torch.cuda.synchronize()
        assert np.array_equal(to_host(dx), full["dx"]) and (which is None or np.array_equal(to_host(out), full[which]))


def test_utterances_do_not_depend_on_the_batch_and_bits_are_reproducible(P):
    x, gamma, beta, dy = case(17, 4, 200, 96, "glu", "bf16")
    n = [200, 150, 90, 3]
    a, b = (run(P, x, 12, gamma, beta, n, "glu", "bf16", dy) for _ in range(2))
    for k in a:
        assert np.array_equal(a[k], b[k]), k
    for i in range(4):
        one = run(P, x[i:i + 1], 12, gamma, beta, n[i:i + 1], "glu", "bf16", dy[i:i + 1])
        np.testing.assert_allclose(one["mean"][0], a["mean"][i], rtol=0, atol=1e-6)


def test_captured_and_replayed_with_new_values(P):
    B, T, C, G = 2, 150, 64, 4
    x, gamma, beta, dy = case(18, B, T, C, "glu", "bf16")
    xd, dyd, gd, bd = on_gpu(x, "bf16"), on_gpu(dy, "bf16"), to_dev(gamma), to_dev(beta)
    n = to_dev(np.array([150, 77], np.int32))
    o = dict(y=torch.empty(B, T, C // 2, dtype=torch.bfloat16, device=DEV), mean=torch.empty(B, G, device=DEV), rstd=torch.empty(B, G, device=DEV))
    g = dict(dx=torch.empty_like(xd), dgamma=torch.empty(C, device=DEV), dbeta=torch.empty(C, device=DEV))
    ws = P.workspace(P.w2l_groupnorm_workspace_bytes(B, T, C, G, P.W2L_ACT_GLU, P.W2L_BF16))

    def step():
        P.w2l_groupnorm_fwd(xd, o["y"], o["mean"], o["rstd"], gd, bd, in_len=n, act=P.W2L_ACT_GLU, workspace=ws)
        P.w2l_groupnorm_bwd(xd, dyd, o["mean"], o["rstd"], g["dx"], gd, bd, g["dgamma"], g["dbeta"], in_len=n, act=P.W2L_ACT_GLU, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        xd.copy_(on_gpu(case(20 + k, B, T, C, "glu", "bf16")[0], "bf16"))
        n.copy_(to_dev(np.array([150 - k, 20 * k], np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        got = {a: to_host(b) for a, b in {**o, **g}.items()}
        step()
        torch.cuda.synchronize()
        for a, b in {**o, **g}.items():
            assert np.array_equal(got[a], to_host(b)), (k, a)


def test_runs_of_frames_captured_and_replayed(P):
    B, T, C, G = 2, 1300, 58, 2
    assert P.w2l_groupnorm_launch_config(B, T, C, G, P.W2L_ACT_GLU, P.W2L_BF16)[0] == 0
    x, gamma, beta, dy = case(38, B, T, C, "glu", "bf16")
    xd, dyd, gd, bd = on_gpu(x, "bf16"), on_gpu(dy, "bf16"), to_dev(gamma), to_dev(beta)
    n = to_dev(np.array([1300, 77], np.int32))
    o = dict(y=torch.empty(B, T, C // 2, dtype=torch.bfloat16, device=DEV), mean=torch.empty(B, G, device=DEV), rstd=torch.empty(B, G, device=DEV))
    g = dict(dx=torch.empty_like(xd), dgamma=torch.empty(C, device=DEV), dbeta=torch.empty(C, device=DEV))
    ws = P.workspace(P.w2l_groupnorm_workspace_bytes(B, T, C, G, P.W2L_ACT_GLU, P.W2L_BF16))

    def step():
        P.w2l_groupnorm_fwd(xd, o["y"], o["mean"], o["rstd"], gd, bd, in_len=n, act=P.W2L_ACT_GLU, workspace=ws)
        P.w2l_groupnorm_bwd(xd, dyd, o["mean"], o["rstd"], g["dx"], gd, bd, g["dgamma"], g["dbeta"], in_len=n, act=P.W2L_ACT_GLU, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        xd.copy_(on_gpu(case(40 + k, B, T, C, "glu", "bf16")[0], "bf16"))
        n.copy_(to_dev(np.array([1300 - k, 300 * k], np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        got = {a: to_host(b) for a, b in {**o, **g}.items()}
        step()
        torch.cuda.synchronize()
        for a, b in {**o, **g}.items():
            assert np.array_equal(got[a], to_host(b)), (k, a)


def test_on_another_stream(P):
    x, gamma, beta, dy = case(19, 2, 100, 32, "silu", "fp32")
    want = run(P, x, 4, gamma, beta, None, "silu", "fp32")
    xd, gd, bd = to_dev(x), to_dev(gamma), to_dev(beta)
    y, mean, rstd = torch.zeros_like(xd), torch.zeros(2, 4, device=DEV), torch.zeros(2, 4, device=DEV)
    ws = P.workspace(P.w2l_groupnorm_workspace_bytes(2, 100, 32, 4, P.W2L_ACT_SILU, P.W2L_F32))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    P.w2l_groupnorm_fwd(xd, y, mean, rstd, gd, bd, act=P.W2L_ACT_SILU, workspace=ws, stream=side)
    side.synchronize()
    assert np.array_equal(to_host(y), want["y"])


def test_a_tensor_beyond_2_31_values(P):
    """Offsets within the tensor pass 32 bits: the last utterances are as they are alone."""
    B, T, C, G = 9, 60000, 4096, 8
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GiB")
    x = torch.zeros((B, T, C), dtype=torch.bfloat16, device=DEV)
    y = torch.empty((B, T, C // 2), dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    tail = torch.randn((2, T, C), generator=gen, device=DEV).bfloat16()
    x[-2:] = tail
    mean, rstd = torch.empty(B, G, device=DEV), torch.empty(B, G, device=DEV)
    ws = P.workspace(P.w2l_groupnorm_workspace_bytes(B, T, C, G, P.W2L_ACT_GLU, P.W2L_BF16))
    P.w2l_groupnorm_fwd(x, y, mean, rstd, act=P.W2L_ACT_GLU, workspace=ws)
    y2, m2, r2 = torch.empty((2, T, C // 2), dtype=torch.bfloat16, device=DEV), torch.empty(2, G, device=DEV), torch.empty(2, G, device=DEV)
    P.w2l_groupnorm_fwd(tail, y2, m2, r2, act=P.W2L_ACT_GLU, workspace=ws)
    torch.cuda.synchronize()
    assert float((mean[-2:] - m2).abs().max()) < 1e-6 and float((rstd[-2:] - r2).abs().max()) < 1e-5
    assert float((y[-2:].float() - y2.float()).abs().max()) < 0.05 and not bool(y[:-2].any())
    dx = torch.empty_like(x)
    dg, db = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    P.w2l_groupnorm_bwd(x, y, mean, rstd, dx, dgamma=dg, dbeta=db, act=P.W2L_ACT_GLU, workspace=ws)
    dx2, dg2, db2 = torch.empty_like(tail), torch.empty_like(dg), torch.empty_like(db)
    P.w2l_groupnorm_bwd(tail, y2, m2, r2, dx2, dgamma=dg2, dbeta=db2, act=P.W2L_ACT_GLU, workspace=ws)
    torch.cuda.synchronize()
    assert float((dx[-2:].float() - dx2.float()).abs().max()) < 0.05 and not bool(dx[:-2].any())
    assert float((db - db2).norm() / db2.norm()) < 1e-3 and float((dg - dg2).norm() / dg2.norm()) < 1e-3


def test_tensors_of_another_shape_or_place(P):
    x, s = torch.zeros(2, 5, 8, device=DEV), torch.zeros(2, 2, device=DEV)
    y, ws = torch.zeros_like(x), P.workspace(1 << 20)
    with pytest.raises(ValueError, match="y must have shape"):
        P.w2l_groupnorm_fwd(x, y, s, s.clone(), act=P.W2L_ACT_GLU, workspace=ws)
    with pytest.raises(TypeError, match="y must be"):
        P.w2l_groupnorm_fwd(x, y.bfloat16(), s, s.clone(), workspace=ws)
    with pytest.raises(TypeError, match="unsupported"):
        P.w2l_groupnorm_fwd(x.half(), y.half(), s, s.clone(), workspace=ws)
    with pytest.raises(ValueError, match="rstd must have shape"):
        P.w2l_groupnorm_fwd(x, y, s, torch.zeros(2, 4, device=DEV), workspace=ws)
    with pytest.raises(ValueError, match="gamma must have shape"):
        P.w2l_groupnorm_fwd(x, y, s, s.clone(), torch.zeros(7, device=DEV), workspace=ws)
    with pytest.raises(ValueError, match="x must be contiguous"):
        P.w2l_groupnorm_fwd(x.transpose(1, 2).contiguous().transpose(1, 2), y, s, s.clone(), workspace=ws)
    with pytest.raises(ValueError, match="in_len is on cpu"):
        P.w2l_groupnorm_fwd(x, y, s, s.clone(), in_len=torch.zeros(2, dtype=torch.int32), workspace=ws)
    with pytest.raises(P.W2LError, match="-5"):
        P.w2l_groupnorm_fwd(x, y, s, s.clone())
    with pytest.raises(P.W2LError, match="-8"):
        P.w2l_groupnorm_fwd(x, x, s, s.clone(), workspace=ws)
    with pytest.raises(P.W2LError, match="-8"):
        P.w2l_groupnorm_fwd(x, y, s, s, workspace=ws)
    with pytest.raises(ValueError, match="dgamma must have shape"):
        P.w2l_groupnorm_bwd(x, y, s, s.clone(), torch.zeros_like(x), dgamma=s, workspace=ws)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_by_differences(P, act):
    """The kernel's gradients against central differences of its own forward pass in fp32: a step of 2^-7 leaves 2^-14 / 6 of the third derivative (a few units here) and
    the forward pass's own rounding over the step, 2^7 * 50 U * sum |dy|, a quarter of a percent of a gradient of one."""
    rng = np.random.default_rng(40)
    B, T, C, G = 1, 6, 8, 2
    x = held(rng.standard_normal((B, T, C)), "fp32")
    gamma, beta = held(1 + 0.3 * rng.standard_normal(C), "fp32"), held(0.5 + 0.3 * rng.standard_normal(C), "fp32")
    dy = held(rng.standard_normal((B, T, C // 2 if act == "glu" else C)), "fp32")
    got = run(P, x, G, gamma, beta, None, act, "fp32", dy, eps=0.1)
    near_kink = (np.abs(oracle.groupnorm(x, G, gamma, beta, None, 0.1, act)["u"]) < 0.1).any() if act == "relu" else False
    h = 2.0 ** -7
    loss = lambda a: (run(P, a, G, gamma, beta, None, act, "fp32", eps=0.1)["y"] * dy).sum()  # noqa: E731
    for i in [(0, 0, 0), (0, 3, 5), (0, 5, 7), (0, 2, 2)]:
        up, dn = x.copy(), x.copy()
        up[i] += h
        dn[i] -= h
        num = (loss(held(up, "fp32")) - loss(held(dn, "fp32"))) / (held(up, "fp32") - held(dn, "fp32"))[i]
        most = h * h * 8 + 50 * U * np.abs(dy).sum() / h
        # a rectifier's kink within the step is worth up to the step times the slope's jump
        assert abs(num - got["dx"][i]) <= most + (2 * h * np.abs(dy).max() * 4 if near_kink else 0), (i, num, got["dx"][i])
