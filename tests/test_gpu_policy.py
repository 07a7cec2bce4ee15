"""w2l_policy_fwd_bwd against the fp64 oracle, through the C ABI.

Bounds, in units of U = 2^-24 (half a step of fp32, relative):
  exp(d)     within (2 |d| + 6) U of itself: d is rounded once, its product with log2 e once, the instruction is good to an ulp
  s          sums of such terms, at most 160 additions deep: (166 + 2 E|d|) U of s with E|d| = sum p |x - m|; log s the same in absolute terms, rounded once
  lp         x - m and its difference with log s rounded once each: e_lp = (168 + 2 E|d|) U + 2 U |lp|
  r          its exponent has the errors of lp and of old, and a rounding of each difference: e_lp + U (|lp| + |old|) + 8 U, relative
  excess     exp(e) - 1 - e: derivative exp(e) - 1, so |exp(e) - 1| (e_lp + U (|ref| + |lp|)), and 12 U (|e|^2 exp(|e|) / 2 for the series below 1/4, the terms' sizes
             exp(e) + 1 + |e| beyond)
  loss       weight times (r |A| its error, kl_coef times excess's), 4 U of the terms
  f          the same with kl_coef |exp(e)| (...) and 4 U of the terms
  gradient   f p (errors of f, of lp in p, 12 U); in the token's column f (1 - p) with the error of lp times p; bf16 adds 2^-8 of the value
A ratio within its error of a border of the clip may be taken on either side: the cases keep away from borders by 1e-4.  Every element has its own bound."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import DEV, to_dev, to_host
from score_cases import CASES, distill_cases
from test_gpu_scores import close, dev, guarded, rounded, spread

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LOW, HIGH = 0.2, 0.3
F32 = np.float32


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


def f32(a):
    return np.asarray(a, np.float32).astype(np.float64)


def case(seed, B, T, C, dtype, scale=2.0, peak=6.0):
    """Scores, and what a slightly different network said of sampled tokens; ratios that keep away from the clip's borders."""
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((B, T, C)) * scale
    top = rng.integers(0, C, (B, T))
    np.put_along_axis(z, top[..., None], np.take_along_axis(z, top[..., None], 2) + peak * rng.random((B, T, 1)), 2)
    z = rounded(z, dtype)
    tok = np.where(rng.random((B, T)) < 0.7, top, rng.integers(0, C, (B, T))).astype(np.int32)
    lp = np.take_along_axis(oracle._log_probs(z)[0], tok[..., None], 2)[..., 0]
    gap = 0.3 * rng.standard_normal((B, T))
    for border in (np.log(1 - LOW), np.log(1 + HIGH)):
        gap = np.where(np.abs(gap - border) < 1e-3, border + 2e-3, gap)
    return dict(z=z, tokens=tok, old=f32(lp - gap), ref=f32(lp + rng.standard_normal((B, T)) * rng.choice([0.05, 1.0], (B, T))), A=f32(rng.standard_normal((B, T))),
                w=f32(rng.random((B, T)) + 0.25))


def run(P, c, dtype="fp32", in_len=None, kl=0.1, gs=0.5, gtype=None, accumulate=None, want=("loss", "logprob", "dz"), low=LOW, high=HIGH):
    z = dev(c["z"], dtype)
    B, T, C = z.shape
    gtype = gtype or dtype
    o, checks = {}, []
    for k, shape, dt in (("frame", (B, T), torch.float32), ("loss", (B,), torch.float32), ("logprob", (B, T), torch.float32),
                         ("dz", (B, T, C), torch.bfloat16 if gtype == "bf16" else torch.float32)):
        if k == "frame" or k in want:
            o[k], ok = guarded(shape, dt)
            checks.append(ok)
    if accumulate is not None:
        o["dz"].copy_(accumulate)
    opt = lambda k: None if c.get(k) is None else to_dev(c[k])  # noqa: E731
    n = None if in_len is None else to_dev(np.asarray(in_len, np.int32))
    ws = P.workspace(P.w2l_policy_workspace_bytes(B, T, C, P.W2L_BF16 if dtype == "bf16" else P.W2L_F32))
    P.w2l_policy_fwd_bwd(z, to_dev(c["tokens"]), to_dev(c["old"]), to_dev(c["A"]), o["frame"], o.get("loss"), o.get("dz"), o.get("logprob"), ref_logprob=opt("ref"),
                         weight=opt("w"), in_len=n, clip_low=low, clip_high=high, kl_coef=kl, grad_scale=gs, accumulate=accumulate is not None, workspace=ws)
    torch.cuda.synchronize()
    for ok in checks:
        ok()
    assert torch.equal(z.nan_to_num(7.), dev(c["z"], dtype).nan_to_num(7.))
    return {k: to_host(v) for k, v in o.items()}


def check(got, c, in_len=None, kl=0.1, gs=0.5, gtype="fp32", accumulate=None, low=LOW, high=HIGH):
    f_ = lambda k: None if c.get(k) is None else c[k]  # noqa: E731
    frame, loss, lp, dz, f = oracle.policy(c["z"], c["tokens"], c["old"], c["A"], f_("ref"), f_("w"), in_len, low, high, kl, gs)
    D = spread(c["z"])
    fin = lambda a: np.where(np.isfinite(a), a, 0.0)  # noqa: E731
    l0 = fin(lp)
    e_lp = (168 + 2 * D) * U + 2 * U * np.abs(l0)
    if "logprob" in got:
        close(got["logprob"], lp, e_lp, "logprob")
    w = np.ones(lp.shape) if c.get("w") is None else np.abs(c["w"])
    A = np.abs(np.broadcast_to(np.asarray(c["A"]).reshape(lp.shape[0], -1), lp.shape))
    with np.errstate(over="ignore", invalid="ignore"):
        r = fin(np.exp(l0 - c["old"]))
        e_r = e_lp + U * (np.abs(l0) + np.abs(fin(c["old"]))) + 8 * U
        e_loss = r * A * (e_r + 4 * U) + (1 + (high if high < 1e9 else 0)) * A * 4 * U
        e_f = r * A * (e_r + 4 * U)
        if kl:
            e = fin(c["ref"] - l0)
            q = fin(np.exp(e))
            e_e = e_lp + U * (np.abs(fin(c["ref"])) + np.abs(l0))
            size = np.where(np.abs(e) < 0.25, e * e * np.exp(np.abs(e)) / 2, q + 1 + np.abs(e))
            e_loss = e_loss + kl * (np.abs(q - 1) * e_e + q * e_e ** 2 + 12 * U * size)
            e_f = e_f + kl * (q * e_e + 8 * U * np.abs(q - 1) + 4 * U * q)
    e_loss = fin(w * e_loss)
    close(got["frame"], frame, e_loss + 2 * U * np.abs(fin(frame)), "frame_loss")
    if "loss" in got:
        close(got["loss"], loss, (e_loss + 2 * U * np.abs(fin(frame))).sum(1) + U * np.abs(fin(loss)), "loss")
    if "dz" not in got:
        return
    e_f = fin(abs(gs) * w * e_f) + 4 * U * np.abs(f)
    lps = oracle._log_probs(c["z"])[0]
    p = np.exp(lps)
    off = e_lp[..., None] + 2 * U * np.abs(fin(lps)) + 12 * U               # of p, relative
    bound = p * (e_f[..., None] + np.abs(f)[..., None] * off)
    # the token's column: 1 - p is off by p times the error of lp
    tk = np.clip(c["tokens"], 0, dz.shape[2] - 1)[..., None]
    pt = np.take_along_axis(p, tk, 2)[..., 0]
    np.put_along_axis(bound, tk, ((1 - pt) * e_f + np.abs(f) * (pt * e_lp + 4 * U * (1 - pt) + U * pt))[..., None], 2)
    bound = bound * (f != 0)[..., None] + 2.0 ** -126 * (1 + np.abs(f))[..., None]
    ref = dz
    if accumulate is not None:
        ref = dz + accumulate.double().cpu().numpy()
        bound = bound + U * np.abs(ref)
    if gtype == "bf16":
        bound = bound + 2.0 ** -8 * np.abs(ref)
    close(got["dz"], ref, bound, "dz")


@pytest.mark.parametrize("C,K,dtype", CASES, ids=str)
def test_every_width(P, C, K, dtype):
    c = case(C, 2, 4 if C > 20000 else 9, C, dtype)
    n = [c["z"].shape[1], 2]
    check(run(P, c, dtype, n), c, n, gtype=dtype)


def test_every_form(P):
    """The forms that a row's width and the number of frames choose (those of the distillation)."""
    for rows, C, K, dtype in distill_cases(P):
        c = case(rows + C, 1, min(rows, 2048), C, dtype) if rows * C < 1 << 22 else None
        if c is None:  # large: the frames are eight different ones in turn, and the oracle sees these
            small = case(rows + C, 1, 8, C, dtype)
            many = {k: np.concatenate([v] * (rows // 8 + 1), 1)[:, :rows] for k, v in small.items()}
            got = run(P, many, dtype)
            for k in ("frame", "logprob", "dz"):
                for i in range(0, rows - 8, 8):
                    assert np.array_equal(got[k][:, i:i + 8], got[k][:, :8]), (rows, C, dtype, k, i)
            got = {k: v[:, :8] for k, v in got.items() if k != "loss"}
            check(got, small, gtype=dtype)
        else:
            check(run(P, c, dtype), c, gtype=dtype)


# six, seven and fourteen slots a wavefront, two to seven wavefronts; seven and ten with a row in sixteen workgroups
@pytest.mark.parametrize("rows,C,dtype", [(1100, 2801, "fp32"), (1100, 5631, "bf16"), (2056, 4500, "fp32"), (2056, 8999, "bf16"), (2056, 5101, "fp32"), (2056, 10001, "bf16"),
                                          (416, 8500, "fp32"), (416, 17001, "bf16"), (136, 16601, "fp32"), (136, 33203, "bf16"), (8, 200001, "fp32"), (8, 262143, "fp32")],
                         ids=str)
def test_wavefronts_that_fit_the_row(P, rows, C, dtype):
    c = case(rows + C, 1, 8, C, dtype)  # eight frames in turn: they begin alike within a vector
    got = run(P, {k: np.concatenate([v] * (rows // 8), 1) for k, v in c.items()} if rows > 8 else c, dtype)
    for k in ("frame", "logprob", "dz"):
        for i in range(0, rows // 8 * 8, 8):
            assert np.array_equal(got[k][:, i:i + 8], got[k][:, :8]), (k, i)
    check({k: v[:, :8] for k, v in got.items() if k != "loss"}, c, gtype=dtype)


@pytest.mark.parametrize("C,dtype,gtype", [(29, "fp32", "fp32"), (29, "bf16", "bf16"), (29, "bf16", "fp32"), (1000, "bf16", "fp32"), (20001, "bf16", "fp32")])
def test_types_and_added_gradients(P, C, dtype, gtype):
    c = case(3, 3, 21, C, dtype)
    n = [21, 0, 13]
    check(run(P, c, dtype, n, gtype=gtype), c, n, gtype=gtype)
    before = torch.from_numpy(np.random.default_rng(4).standard_normal((3, 21, C)).astype(np.float32)).to(DEV).to(torch.bfloat16 if gtype == "bf16" else torch.float32)
    check(run(P, c, dtype, n, gtype=gtype, accumulate=before), c, n, gtype=gtype, accumulate=before)


@pytest.mark.parametrize("C", [29, 300, 5000])
def test_what_is_optional(P, C):
    c = case(5, 2, 70, C, "fp32")
    check(run(P, {**c, "ref": None, "w": None}, kl=0.0), {**c, "w": None}, kl=0.0)
    check(run(P, c, want=()), c)
    full = run(P, c)
    for k in ("loss", "logprob", "dz"):
        assert np.array_equal(run(P, c, want=(k,))[k], full[k])
    u = {**c, "A": f32([0.7, -1.3])}                                       # of the utterances
    check(run(P, u), u)
    check(run(P, c, low=1.0, high=float("inf")), c, low=1.0, high=float("inf"))
    hard = dict(c, old=f32(c["old"] + np.where(np.abs(c["A"]) > 0, np.where(np.random.default_rng(6).random(c["A"].shape) < .5, 1e-2, -1e-2), 0)))
    check(run(P, hard, low=0.0, high=0.0), hard, low=0.0, high=0.0)


@pytest.mark.parametrize("C", [5, 29, 700, 5000, 40000])
def test_frames_that_say_nothing(P, C):
    T = 12
    c = case(7, 3, T, C, "fp32")
    z, tok, old, A, w, ref = (c[k] for k in ("z", "tokens", "old", "A", "w", "ref"))
    z[0, 0, C - 1] = np.nan
    z[0, 1, 0] = np.inf
    tok[0, 2] = -1
    z[0, 2] = np.nan
    w[0, 3] = 0
    z[0, 3] = np.nan
    tok[0, 4], tok[0, 5] = C, -2
    z[0, 6, tok[0, 6]] = -np.inf                                           # probability zero
    z[0, 7] = -np.inf
    A[0, 8] = 0
    old[0, 9] = np.nan
    ref[0, 10] = -np.inf
    w[0, 11] = np.inf
    z[1, 4:] = np.nan                                                      # beyond the utterance
    n = [T, 4, -1]
    for kl in (0.1, 0.0):
        got = run(P, c, in_len=n, kl=kl)
        check(got, c, n, kl=kl)
        assert not got["dz"][1, 4:].any() and not got["dz"][2].any() and not got["dz"][0, [0, 1, 2, 3, 4, 5, 7, 9, 11]].any()
        before = torch.ones(3, T, C, device=DEV)
        check(run(P, c, in_len=n, kl=kl, accumulate=before), c, n, kl=kl, accumulate=before)


@pytest.mark.parametrize("C", [29, 2000])
def test_large_scores_and_masked_classes(P, C):
    """Scores of thousands and millions keep the bits of their differences; classes masked by -inf or by the type's lowest value have no part."""
    for level in (1e4, 3e7):
        c = case(8, 2, 20, C, "fp32")
        c["z"] = f32(np.round(c["z"]) * 4 + level)
        lp = np.take_along_axis(oracle._log_probs(c["z"])[0], c["tokens"][..., None], 2)[..., 0]
        c["old"], c["ref"] = f32(np.maximum(lp, -50) - 0.05), f32(np.maximum(lp, -50) + 0.1)
        check(run(P, c), c)
    c = case(9, 2, 20, C, "fp32")
    c["z"][:, :, ::3] = np.where(np.arange(20)[None, :, None] % 2, -np.inf, float(np.finfo(np.float32).min))
    c["tokens"] = (c["tokens"] // 3 * 3 + 1).clip(max=C - 2).astype(np.int32)
    c["tokens"][c["tokens"] % 3 == 0] = 1
    lp = np.take_along_axis(oracle._log_probs(c["z"])[0], c["tokens"][..., None], 2)[..., 0]
    c["old"], c["ref"] = f32(lp - 0.05), f32(lp + 0.1)
    check(run(P, c), c)


def test_one_class(P):
    z = np.zeros((1, 3, 1))
    c = dict(z=z, tokens=np.zeros((1, 3), np.int32), old=np.zeros((1, 3)), ref=np.zeros((1, 3)), A=np.ones((1, 3)), w=np.ones((1, 3)))
    got = run(P, c)
    assert np.array_equal(got["frame"], -np.ones((1, 3))) and not got["dz"].any() and not got["logprob"].any() and got["loss"][0] == -3


def test_gradient_by_differences(P):
    """d loss / dz of the kernel's own losses, by central differences in fp32: a step of 2^-6 leaves 2^-12 / 6 of the third derivative and 2 U |loss| / 2^-5."""
    c = case(10, 1, 6, 8, "fp32", scale=1.0, peak=1.0)
    got = run(P, c, gs=1.0)
    h = 2.0 ** -6
    base = np.exp(np.take_along_axis(oracle._log_probs(c["z"])[0], c["tokens"][..., None], 2)[..., 0] - c["old"])
    safe = (np.abs(base - 0.8) > 0.05) & (np.abs(base - 1.3) > 0.05)       # frames that stay on their side of the clip over the step
    assert safe.sum() >= 3
    for k in range(8):
        up, dn = (dict(c, z=f32(c["z"] + s * h * (np.arange(8) == k))) for s in (1, -1))
        num = (run(P, up)["frame"] - run(P, dn)["frame"]) / (up["z"] - dn["z"])[..., k]
        size = c["w"] * (np.abs(c["A"]) * base + 0.1 * np.exp(np.abs(c["ref"] - np.log(base) - c["old"])))
        assert (np.abs(num - got["dz"][..., k])[safe] <= (size * 16 * h * h + 16 * U * size / h)[safe]).all()


def test_captured_and_replayed(P):
    for B, T, C, dtype in ((2, 20, 29, "fp32"), (2, 40, 3000, "bf16"), (1, 3, 100003, "bf16")):
        cs = [case(20 + i, B, T, C, dtype) for i in range(3)]
        d = {k: (dev(v, dtype) if k == "z" else to_dev(v)) for k, v in cs[0].items()}
        frame, loss, dz = torch.empty(B, T, device=DEV), torch.empty(B, device=DEV), torch.empty_like(d["z"])
        ws = P.workspace(P.w2l_policy_workspace_bytes(B, T, C, P.W2L_BF16 if dtype == "bf16" else P.W2L_F32))
        call = lambda: P.w2l_policy_fwd_bwd(d["z"], d["tokens"], d["old"], d["A"], frame, loss, dz, ref_logprob=d["ref"], weight=d["w"], kl_coef=0.1, workspace=ws)  # noqa: E731
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for c in cs[1:] + cs:
            for k, v in c.items():
                d[k].copy_(dev(v, dtype) if k == "z" else to_dev(v))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (frame, loss, dz)]
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (frame, loss, dz)))


def test_tensors_of_another_shape_or_place(P):
    c = case(11, 2, 5, 29, "fp32")
    z, tok, old, A = dev(c["z"], "fp32"), to_dev(c["tokens"]), to_dev(c["old"]), to_dev(c["A"])
    frame = torch.empty(2, 5, device=DEV)
    with pytest.raises(ValueError, match="tokens must have shape"):
        P.w2l_policy_fwd_bwd(z, tok[:, :4].contiguous(), old, A, frame)
    with pytest.raises(TypeError, match="tokens must be"):
        P.w2l_policy_fwd_bwd(z, tok.long(), old, A, frame)
    with pytest.raises(ValueError, match="contiguous"):
        P.w2l_policy_fwd_bwd(z, tok, old.t().contiguous().t(), A, frame)
    with pytest.raises(ValueError, match="advantage must have shape"):
        P.w2l_policy_fwd_bwd(z, tok, old, A[0], frame)
    with pytest.raises(ValueError, match="is on cpu"):
        P.w2l_policy_fwd_bwd(z, tok, old, A.cpu(), frame)
    with pytest.raises(P.W2LError):
        P.w2l_policy_fwd_bwd(z, tok, old, A, frame, kl_coef=0.1)          # a KL term without a reference


def test_scores_beyond_2_31(P):
    """Offsets that pass 32 bits: the last frames are as they are alone."""
    T, C = 8400, 262144                                                    # 2.2e9 scores
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GiB")
    c = case(12, 1, 3, C, "bf16")
    z = torch.zeros((1, T, C), dtype=torch.bfloat16, device=DEV)
    z[:, -3:] = dev(c["z"], "bf16")
    far = lambda k: torch.cat((torch.zeros((1, T - 3), dtype=torch.from_numpy(c[k]).dtype), torch.from_numpy(c[k])), 1).to(torch.int32 if k == "tokens" else torch.float32).to(DEV)  # noqa: E731
    frame, dz = torch.empty(1, T, device=DEV), torch.empty_like(z)
    ws = P.workspace(P.w2l_policy_workspace_bytes(1, T, C, P.W2L_BF16))
    P.w2l_policy_fwd_bwd(z, far("tokens"), far("old"), far("A"), frame, dz=dz, ref_logprob=far("ref"), weight=far("w"), clip_low=LOW, clip_high=HIGH, kl_coef=0.1, grad_scale=0.5,
                         workspace=ws)
    torch.cuda.synchronize()
    check({"frame": to_host(frame[:, -3:]), "dz": to_host(dz[:, -3:])}, c, gtype="bf16")
    assert not bool(dz[:, :-3].any()) and not bool(frame[:, :-3].any())    # weights of 0


@pytest.mark.parametrize("C", [29, 700])
def test_ratios_beyond_fp32(P, C):
    c = case(31, 2, 40, C, "fp32")
    c["old"] = c["old"] - 200                                              # the ratio is +inf in fp32
    c["A"] = np.abs(c["A"])
    got = run(P, c, kl=0.0)                                                # bounded: (1 + clip_high) A, and no gradient
    assert np.array_equal(got["frame"], (-(F32(1) + F32(HIGH)) * c["A"].astype(F32) * c["w"].astype(F32)).astype(np.float64)) and not got["dz"].any()
    got = run(P, {**c, "A": -c["A"]}, kl=0.0)                              # not bounded from above: no finite number, and no gradient
    assert np.all(got["frame"] == np.inf) and np.all(got["loss"] == np.inf) and not got["dz"].any()


def test_on_another_stream(P):
    c = case(32, 2, 60, 700, "fp32")
    want = run(P, c)
    z, tok, old, A, w, ref = (dev(c["z"], "fp32"), *(to_dev(c[k]) for k in ("tokens", "old", "A", "w", "ref")))
    frame, loss, dz = torch.zeros(2, 60, device=DEV), torch.zeros(2, device=DEV), torch.zeros_like(z)
    ws = P.workspace(P.w2l_policy_workspace_bytes(2, 60, 700, P.W2L_F32))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    P.w2l_policy_fwd_bwd(z, tok, old, A, frame, loss, dz, ref_logprob=ref, weight=w, clip_low=LOW, clip_high=HIGH, kl_coef=0.1, grad_scale=0.5, workspace=ws, stream=side)
    side.synchronize()
    for k, t in (("frame", frame), ("loss", loss), ("dz", dz)):
        assert np.array_equal(to_host(t), want[k]), k
