"""Pins of the oracles for group norm, the clipped policy loss and AdamW: torch's own operators in 64 bits, closed forms, central differences, and the rules
for what is not there."""
import numpy as np
import pytest
import torch

import oracle

ACTS = ("none", "relu", "silu", "glu")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("G", [1, 3, 12])
def test_group_norm_is_torchs(act, G):
    rng = np.random.default_rng(1)
    x, gamma, beta = rng.standard_normal((2, 7, 12)) * 3 + 1, rng.standard_normal(12), rng.standard_normal(12)
    o = oracle.groupnorm(x, G, gamma, beta, None, 1e-3, act)
    t = lambda a: torch.from_numpy(a)
    u = torch.nn.functional.group_norm(t(x).permute(0, 2, 1), G, t(gamma), t(beta), 1e-3).permute(0, 2, 1)
    y = {"none": u, "relu": u.relu(), "silu": torch.nn.functional.silu(u), "glu": torch.nn.functional.glu(u, -1)}[act]
    np.testing.assert_allclose(o["y"], y.numpy(), atol=1e-12)


@pytest.mark.parametrize("act", ACTS)
def test_group_norm_gradients_by_differences(act):
    rng = np.random.default_rng(2)
    x, gamma, beta, n = rng.standard_normal((3, 5, 8)), rng.standard_normal(8), rng.standard_normal(8), np.array([5, 2, 0])
    dy = rng.standard_normal((3, 5, 4 if act == "glu" else 8))
    loss = lambda x, g, b: (oracle.groupnorm(x, 2, g, b, n, 1e-2, act)["y"] * dy).sum()
    o = oracle.groupnorm(x, 2, gamma, beta, n, 1e-2, act, dy)
    h = 1e-6
    for name, a, grad in (("x", x, o["dx"]), ("gamma", gamma, o["dgamma"]), ("beta", beta, o["dbeta"])):
        num = np.zeros(a.shape)
        for i in np.ndindex(a.shape):
            p = a.copy()
            p[i] += h
            m = a.copy()
            m[i] -= h
            args = dict(x=x, gamma=gamma, beta=beta)
            num[i] = (loss(*dict(args, **{name: p}).values()) - loss(*dict(args, **{name: m}).values())) / (2 * h)
        np.testing.assert_allclose(grad, num, atol=2e-8, err_msg=name)


def test_group_norm_of_frames_that_are_not_there():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 6, 4))
    n = np.array([6, 3, 0, 7])
    x[1, 3:] = np.nan
    o = oracle.groupnorm(x, 2, in_len=n, act="silu", dy=np.ones((4, 6, 4)))
    alone = oracle.groupnorm(x[1:2, :3], 2, act="silu")
    np.testing.assert_allclose(o["y"][1, :3], alone["y"][0])
    assert not o["y"][1, 3:].any() and not o["dx"][1, 3:].any() and not o["y"][2].any() and not o["rstd"][2].any()
    assert np.isnan(o["y"][3]).all() and np.isnan(o["mean"][3]).all() and not o["dx"][3].any() and np.isfinite(o["dgamma"]).all()


def policy_case(seed=4, B=2, T=5, C=6):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((B, T, C)) * 2
    tok = rng.integers(0, C, (B, T))
    lp = np.take_along_axis(z - np.log(np.exp(z).sum(-1, keepdims=True)), tok[..., None], 2)[..., 0]
    return z, tok, lp - 0.4 * rng.standard_normal((B, T)), lp + 0.5 * rng.standard_normal((B, T)), rng.standard_normal((B, T)), rng.random((B, T)) + 0.1


def test_policy_loss_is_the_formula_and_its_gradient_by_differences():
    z, tok, old, ref, A, w = policy_case()
    args = (tok, old, A, ref, w, None, 0.1, 0.3, 0.2, 0.7)
    frame, loss, lp, dz, f = oracle.policy(z, *args)
    t = torch.from_numpy
    q = torch.log_softmax(t(z).requires_grad_(), -1)
    l = q.gather(2, t(tok)[..., None])[..., 0]
    r = (l - t(old)).exp()
    want = t(w) * (-torch.minimum(r * t(A), r.clamp(0.9, 1.3) * t(A)) + 0.2 * ((t(ref) - l).exp() - (t(ref) - l) - 1))
    np.testing.assert_allclose(frame, want.detach().numpy(), atol=1e-13)
    np.testing.assert_allclose(loss, frame.sum(1))
    assert (np.abs(f) < np.abs(0.7 * w * A * np.exp(lp - old))).any()       # some are held
    h, num = 1e-6, np.zeros(z.shape)
    for i in np.ndindex(z.shape):
        p, m = z.copy(), z.copy()
        p[i] += h
        m[i] -= h
        num[i] = 0.7 * (oracle.policy(p, *args)[1].sum() - oracle.policy(m, *args)[1].sum()) / (2 * h)
    np.testing.assert_allclose(dz, num, atol=1e-8)


def test_policy_of_frames_that_say_nothing():
    z, tok, old, ref, A, w = policy_case(B=2, T=8)
    z[0, 0, 3] = np.nan
    tok[0, 1] = -1
    w[0, 2] = 0
    tok[0, 3] = 6
    z[0, 4, tok[0, 4]] = -np.inf
    z[0, 5] = -np.inf
    A[0, 6] = 0
    old[0, 7] = np.nan
    frame, loss, lp, dz, f = oracle.policy(z, tok, old, A, ref, w, [8, 9], kl_coef=0.1)
    assert np.isnan(frame[0, [0, 3, 7]]).all() and not frame[0, 1:3].any() and np.isinf(frame[0, [4, 5]]).all() and np.isfinite(frame[0, 6]) and f[0, 6] != 0
    assert not dz[0, [0, 1, 2, 3, 4, 5, 7]].any() and np.isnan(frame[1]).all() and not dz[1].any()
    assert lp[0, 4] == -np.inf and lp[0, 5] == -np.inf
    one = oracle.policy(z, tok, old, A, None, w, [8, 0])[0]                # without the KL term a probability of zero is a ratio of zero
    assert np.isfinite(one[0, 4]) and not one[1].any()


def test_adamw_is_torchs():
    rng = np.random.default_rng(5)
    w, m, v = rng.standard_normal(50), np.zeros(50), np.zeros(50)
    p = torch.from_numpy(w.copy()).requires_grad_()
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.8, 0.95), eps=1e-3, weight_decay=0.1)
    for step in range(1, 5):
        g = rng.standard_normal(50)
        p.grad = torch.from_numpy(g.copy())
        norm = torch.nn.utils.clip_grad_norm_([p], 2.0)
        assert abs(float(norm) - oracle.adamw_norm([g])) < 1e-12
        opt.step()
        f = oracle.adamw_factor([g], 1.0, 2.0)
        w, m, v = oracle.adamw(w, g, m, v, f, step, 0.01, 0.8, 0.95, 1e-3, 0.1)
        np.testing.assert_allclose(w, p.detach().numpy(), rtol=1e-12)


def test_numbers_of_eight_bits_are_torchs():
    all_ = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mine = oracle.from_e4m3(np.arange(256), [0])
    assert np.array_equal(all_, mine, equal_nan=True) and oracle.E4M3[126] == 448


def test_rounding_at_random():
    rng = np.random.default_rng(6)
    x = (rng.standard_normal(1024) * np.exp(3 * rng.standard_normal(1024))).astype(np.float32).astype(np.float64)
    r = rng.integers(0, 65536, 1024) / 65536
    lo, E = oracle.to_e4m3(x, np.zeros(1024))
    hi, _ = oracle.to_e4m3(x, np.full(1024, 65535 / 65536))
    got, _ = oracle.to_e4m3(x, r)
    a, b, c = (np.abs(oracle.from_e4m3(k, E)) for k in (lo, got, hi))
    assert (a <= np.abs(x)).all() and (c >= np.minimum(np.abs(x), a.max())).all() and ((b == a) | (b == c)).all()
    for k in range(4):
        most = np.abs(x[256 * k:256 * k + 256]).max()
        assert most <= 448 * 2.0 ** E[k] and most > 448 * 2.0 ** (E[k] - 1)
    # the expectation over all 2^16 random numbers is the value, to the 2^-16 of a spacing that they resolve
    y = np.array([0.3, 5.3, 100.0, 447.0] + [448.0] + [2.0 ** -9 * 0.4] * 3)
    mean = np.mean([oracle.from_e4m3(*oracle.to_e4m3(y, np.full(8, k / 65536))) for k in range(0, 65536, 64)], 0)
    np.testing.assert_allclose(mean, y, atol=32 / 1000, rtol=0)
    zero, E = oracle.to_e4m3(np.zeros(3), np.ones(3) * 0.9, keep=True)
    assert not zero.any() and not E.any()
    kept, _ = oracle.to_e4m3(np.array([1.0, 1e-30, 0.0]), np.zeros(3), keep=True)
    assert kept[1] == 1 and kept[2] == 0
    odd, _ = oracle.to_e4m3(np.array([np.nan, np.inf, -np.inf, 2.0]), np.zeros(4))
    assert list(odd[:3] & 127) == [127] * 3 and odd[3] & 127 != 127


def test_random_bits_are_even():
    r = np.concatenate([oracle.adamw_dither(s, t, i, 4096) for s in (0, 1, 12345) for t in (1, 2, 1000) for i in (0, 5)])
    n = len(r)
    assert abs(r.mean() - 0.5) < 4 / np.sqrt(12 * n)                       # four deviations of a mean of n
    counts = np.bincount((r * 64).astype(int), minlength=64)
    chi = ((counts - n / 64) ** 2 / (n / 64)).sum()
    assert chi < 63 + 5 * np.sqrt(2 * 63)                                  # 63 degrees of freedom, five deviations
    a, b = oracle.adamw_dither(7, 3, 0, 4096), oracle.adamw_dither(7, 4, 0, 4096)
    assert abs(np.corrcoef(a, b)[0, 1]) < 5 / 64 and abs(np.corrcoef(a[:-1], a[1:])[0, 1]) < 5 / 64
