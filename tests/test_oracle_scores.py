"""Pins of the fp64 oracles for reading a frame's scores and for distillation: closed forms, torch's own 64-bit log-softmax,
central differences of both gradients, and the rules for frames and entries that are not there."""
import numpy as np
import pytest
import torch

import oracle


def _case(seed, B=2, T=5, C=7, S=2, K=3):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((B, T, C)) * 2
    return rng, z, rng.integers(0, C, (B, T, S))


def test_log_probs_entropy_and_best_classes_are_torchs():
    rng, z, tok = _case(1, C=11)
    f = oracle.token_logprob(z, tok, 4)
    lp = torch.log_softmax(torch.from_numpy(z), -1)
    np.testing.assert_allclose(f["logprob"], lp.gather(2, torch.from_numpy(tok)).numpy(), atol=1e-13)
    np.testing.assert_allclose(f["entropy"], -(lp.exp() * lp).sum(-1).numpy(), atol=1e-13)
    v, i = lp.topk(4, -1)
    assert np.array_equal(f["top_ids"], i.numpy())
    np.testing.assert_allclose(f["top_logprob"], v.numpy(), atol=1e-13)


def test_closed_forms():
    C = 8
    f = oracle.token_logprob(np.full((1, 1, C), 3e5), np.zeros((1, 1, 1), int), 3)
    assert abs(f["entropy"][0, 0] - np.log(C)) < 1e-12 and list(f["top_ids"][0, 0]) == [0, 1, 2]   # equal scores by class
    one = oracle.token_logprob(np.zeros((1, 2, 1)), np.zeros((1, 2, 1), int), 1)
    assert np.all(one["entropy"] == 0) and np.all(one["logprob"] == 0) and np.all(one["top_ids"] == 0)
    z = np.full((1, 1, 4), -np.inf)
    z[0, 0, 2] = -5.0
    f = oracle.token_logprob(z, np.array([[[2, 0]]]), 4)
    assert f["logprob"][0, 0, 0] == 0 and f["logprob"][0, 0, 1] == -np.inf and f["entropy"][0, 0] == 0
    assert list(f["top_ids"][0, 0]) == [2, 0, 1, 3]


def test_rows_and_tokens_that_are_not_there():
    z = np.zeros((3, 4, 5))
    z[0, 0] = -np.inf
    z[0, 1, 3] = np.nan
    z[0, 2, 3] = np.inf
    tok = np.zeros((3, 4, 1), int)
    tok[1, 0], tok[1, 1] = -1, 5
    f = oracle.token_logprob(z, tok, 2, in_len=[4, 2, 5])
    assert f["entropy"][0, 0] == 0 and f["logprob"][0, 0, 0] == -np.inf and list(f["top_ids"][0, 0]) == [0, 1]
    for t in (1, 2):
        assert np.isnan(f["entropy"][0, t]) and np.isnan(f["logprob"][0, t, 0]) and np.all(f["top_ids"][0, t] == -1)
        assert np.all(np.isnan(f["top_logprob"][0, t]))
    assert f["logprob"][1, 0, 0] == 0 and np.isnan(f["logprob"][1, 1, 0])
    assert np.all(f["logprob"][1, 2:] == 0) and np.all(f["top_ids"][1, 2:] == -1) and np.all(f["top_logprob"][1, 2:] == -np.inf)
    assert np.all(np.isnan(f["entropy"][2])) and np.all(f["top_ids"][2] == -1)          # length out of range
    g = oracle.token_logprob_bwd(z, tok, np.ones(tok.shape), np.ones((3, 4)), in_len=[4, 2, 5])
    assert np.all(np.isfinite(g)) and np.all(g[0, :3] == 0) and np.all(g[1, 2:] == 0) and np.all(g[2] == 0)
    assert np.all(np.abs(g[1, :2]) <= 1e-15)       # equal scores: lp + H is 0 up to a few roundings of 64 bits, 1.6 * 2^-53 each


def test_token_gradient_by_differences():
    rng, z, tok = _case(2, B=1, T=2, C=6, S=3)
    tok[0, 0] = [1, 1, -1]
    K = 2
    gl, gh, gt = rng.standard_normal(tok.shape), rng.standard_normal((1, 2)), rng.standard_normal((1, 2, K))
    top = oracle.token_logprob(z, tok, K)["top_ids"]

    def value(z):
        f = oracle.token_logprob(z, tok, 0)
        return (gl * f["logprob"]).sum() + (gh * f["entropy"]).sum() + (gt * np.take_along_axis(f["lp"], top, 2)).sum()

    dz = oracle.token_logprob_bwd(z, tok, gl, gh, top, gt)
    h = 1e-5
    for i in np.ndindex(z.shape):
        e = np.zeros_like(z)
        e[i] = h
        assert abs((value(z + e) - value(z - e)) / (2 * h) - dz[i]) < 1e-8
    assert np.all(np.abs(dz.sum(-1)) < 1e-12)      # a shift of all scores changes nothing


@pytest.mark.parametrize("tau", [1.0, 0.5, 3.0])
def test_distillation_gradient_by_differences(tau):
    rng, z, ids = _case(3, B=2, T=3, C=6, S=4)
    ids[0, 0] = [2, 2, 5, -1]
    sc, w = rng.standard_normal(ids.shape), rng.random((2, 3))
    frame, loss, dz = oracle.distill(z, ids, sc, tau, w, [3, 2], 0.7)
    np.testing.assert_allclose(loss, frame.sum(1))
    assert np.all(frame[1, 2:] == 0) and np.all(dz[1, 2:] == 0)
    h = 1e-5
    for i in np.ndindex(z.shape):
        e = np.zeros_like(z)
        e[i] = h
        up, down = (oracle.distill(z + s * e, ids, sc, tau, w, [3, 2])[1].sum() for s in (1, -1))
        assert abs(0.7 * (up - down) / (2 * h) - dz[i]) < 1e-8


def test_distillation_closed_forms():
    rng, z, _ = _case(4, B=1, T=2, C=5)
    every = np.broadcast_to(np.arange(5), (1, 2, 5))
    frame, _, dz = oracle.distill(z, every, z + 7.0, 2.0)       # the teacher's own scores, shifted: nothing to learn
    assert np.all(np.abs(frame) < 1e-12) and np.all(np.abs(dz) < 1e-12)
    f, _, dz = oracle.distill(z, np.full((1, 2, 1), 3), np.full((1, 2, 1), -9.0))   # one entry: cross entropy of that class
    lp = oracle.logsoftmax_fwd(z)
    np.testing.assert_allclose(f, -lp[..., 3], atol=1e-12)
    np.testing.assert_allclose(dz, np.exp(lp) - (np.arange(5) == 3), atol=1e-12)


def test_distillation_frames_that_are_not_there():
    z = np.zeros((6, 1, 4))
    ids, sc = np.tile(np.array([0, 1]), (6, 1, 1)), np.zeros((6, 1, 2))
    z[0, 0, 0] = -np.inf                         # the teacher gives weight to it
    z[1, 0, 2] = np.nan
    ids[2] = -1
    ids[3, 0, 1] = 4
    sc[4] = -np.inf
    sc[5, 0, 0] = np.inf
    frame, _, dz = oracle.distill(z, ids, sc)
    assert frame[0, 0] == np.inf and np.isnan(frame[1, 0]) and frame[2, 0] == 0 and np.isnan(frame[3, 0])
    assert frame[4, 0] == 0 and np.isnan(frame[5, 0]) and np.all(dz == 0)
    frame, _, dz = oracle.distill(z, ids, sc, weight=np.zeros((6, 1)))
    assert np.all(frame == 0) and np.all(dz == 0)
