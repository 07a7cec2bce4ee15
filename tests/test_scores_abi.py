"""Host-only: what w2l_token_logprob_fwd / _bwd, w2l_distill_fwd_bwd and w2l_frame_ids_check_host refuse, before anything is
launched, and what the binding refuses before the library is called."""
import numpy as np
import pytest
import torch

import paper_1812_07625_amd as P

A = 0x1000   # never dereferenced: the checks fail before any launch
N = None
WS = 0x1100


def fwd(z=A, tokens=A, in_len=A, logprob=A, entropy=A, ids=A, top=A, stats=A, B=2, T=3, C=9, S=1, K=2, dt=0, ws=WS, n=1 << 30):
    return P.raw.w2l_token_logprob_fwd(z, tokens, in_len, logprob, entropy, ids, top, stats, B, T, C, S, K, dt, ws, n, N)


def bwd(z=A, stats=A, tokens=A, dl=A, dh=A, ids=A, dtop=A, in_len=A, dz=A, B=2, T=3, C=9, S=1, K=2, dt=0, gt=0, acc=0):
    return P.raw.w2l_token_logprob_bwd(z, stats, tokens, dl, dh, ids, dtop, in_len, dz, B, T, C, S, K, dt, gt, acc, N)


def distill(z=A, ids=A, sc=A, in_len=A, w=A, frame=A, loss=A, dz=A, B=2, T=3, C=9, K=2, tau=1.0, gs=1.0, dt=0, gt=0, acc=0, ws=WS, n=1 << 30):
    return P.raw.w2l_distill_fwd_bwd(z, ids, sc, in_len, w, frame, loss, dz, B, T, C, K, tau, gs, dt, gt, acc, ws, n, N)


SIZES = [dict(B=0), dict(T=0), dict(C=0), dict(C=262145), dict(K=10), dict(K=65, C=100), dict(K=-1), dict(B=65536, T=32768)]


@pytest.mark.parametrize("kw", SIZES, ids=str)
def test_sizes(kw):
    assert fwd(**kw) == -2 and bwd(**kw) == -2 and distill(**kw) == -2


def test_forward_call():
    for kw in (dict(z=N), dict(tokens=N), dict(logprob=N), dict(ids=N), dict(top=N)):
        assert fwd(**kw) == -1, kw
    assert fwd(S=65) == -2 and fwd(S=-1, tokens=N, logprob=N) == -2
    assert fwd(dt=2) == -3
    for k in ("z", "tokens", "in_len", "logprob", "entropy", "ids", "top", "stats"):
        assert fwd(**{k: A + 4}) == -4, k


def test_backward_call():
    for kw in (dict(z=N), dict(stats=N), dict(dz=N), dict(tokens=N), dict(dl=N), dict(ids=N), dict(dtop=N)):
        assert bwd(**kw) == -1, kw
    assert bwd(dt=2) == -3 and bwd(gt=2) == -3 and bwd(dt=0, gt=1) == -3    # fp32 scores, bf16 gradient
    for k in ("z", "stats", "tokens", "dl", "dh", "ids", "dtop", "in_len", "dz"):
        assert bwd(**{k: A + 4}) == -4, k


def test_distillation_call():
    for kw in (dict(z=N), dict(ids=N), dict(sc=N), dict(frame=N)):
        assert distill(**kw) == -1, kw
    assert distill(K=0) == -2
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-45, 3e-39, 1e38, 3e38):
        assert distill(tau=tau) == -2, tau
    for gs in (float("nan"), float("inf")):
        assert distill(gs=gs) == -2
    assert distill(dt=2) == -3 and distill(gt=2) == -3 and distill(dt=0, gt=1) == -3
    for k in ("z", "ids", "sc", "in_len", "w", "frame", "loss", "dz"):
        assert distill(**{k: A + 4}) == -4, k


def test_workspace():
    big = dict(C=100000, K=9)
    need = P.w2l_token_logprob_workspace_bytes(2, 3, 100000, 9, 0)
    assert need > 0
    assert fwd(ws=N, n=0, **big) == -5 and fwd(n=need - 1, **big) == -5 and fwd(ws=WS + 16, n=need, **big) == -5
    need = P.w2l_distill_workspace_bytes(2, 3, 100000, 9, 0)
    assert need > 0
    assert distill(ws=N, n=0, **big) == -5 and distill(n=need - 1, **big) == -5 and distill(ws=WS + 16, n=need, **big) == -5
    assert fwd(C=262144, B=8192, T=600) == -2 and bwd(C=262144, B=8192, T=600) == -2 and distill(C=262144, B=8192, T=600) == -2   # over 2^40 scores


def test_host_check_of_ids():
    ids = np.array([[[0, 4], [-1, 3]], [[2, 2], [7, -9]]], np.int32)      # [2,2,2]; the last frame is out of range
    assert P.w2l_frame_ids_check_host(ids, [2, 1], 5) == 0
    assert P.w2l_frame_ids_check_host(ids, [2, 2], 5) == -6
    assert P.w2l_frame_ids_check_host(ids, None, 5) == -6
    assert P.w2l_frame_ids_check_host(ids, [2, 1], 4) == -6
    assert P.w2l_frame_ids_check_host(ids, [3, 1], 5) == -6 and P.w2l_frame_ids_check_host(ids, [-1, 1], 5) == -6
    assert P.raw.w2l_frame_ids_check_host(N, N, 1, 1, 5, 1) == -1


def test_binding_takes_no_host_tensors():
    z, one = torch.zeros(1, 2, 5), torch.zeros(1, 2)
    ids, sc = torch.zeros(1, 2, 1, dtype=torch.int32), torch.zeros(1, 2, 1)
    with pytest.raises(ValueError, match="GPU"):
        P.w2l_token_logprob_fwd(z, ids, sc)
    with pytest.raises(ValueError, match="GPU"):
        P.w2l_token_logprob_bwd(z, torch.zeros(1, 2, 4), z)
    with pytest.raises(ValueError, match="GPU"):
        P.w2l_distill_fwd_bwd(z, ids, sc, one)
    with pytest.raises(ValueError, match=r"\[B, T, C\]"):
        P.w2l_distill_fwd_bwd(z[0], ids, sc, one)
