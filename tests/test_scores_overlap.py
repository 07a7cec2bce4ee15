"""Host-only: w2l_token_logprob_fwd / _bwd and w2l_distill_fwd_bwd refuse outputs that lie on an input, before anything is launched."""
import pytest

import paper_1812_07625_amd as P

B, T, C, S, K = 2, 3, 100000, 2, 5      # many classes: with a workspace
N = None
F32, BF16 = 0, 1


def places(names):
    """An address of its own for every operand, far from the others; never dereferenced: the calls are refused before any launch."""
    return {n: 0x100000000 * (i + 1) for i, n in enumerate(names)}


FWD = ("z", "tokens", "in_len", "logprob", "entropy", "ids", "top", "stats", "ws")
BWD = ("z", "stats", "tokens", "dl", "dh", "ids", "dtop", "in_len", "dz")
DISTILL = ("z", "ids", "sc", "in_len", "w", "frame", "loss", "dz", "ws")
BYTES = dict(z=B * T * C * 2, tokens=B * T * S * 4, in_len=B * 4, logprob=B * T * S * 4, entropy=B * T * 4, ids=B * T * K * 4, top=B * T * K * 4, stats=B * T * 16,
             dl=B * T * S * 4, dh=B * T * 4, dtop=B * T * K * 4, sc=B * T * K * 4, w=B * T * 4, frame=B * T * 4, loss=B * 4, dz=B * T * C * 2)


def fwd(a, n):
    return P.raw.w2l_token_logprob_fwd(*[a[k] for k in FWD[:-1]], B, T, C, S, K, BF16, a["ws"], n, N)


def bwd(a, n):
    return P.raw.w2l_token_logprob_bwd(*[a[k] for k in BWD], B, T, C, S, K, BF16, BF16, 1, N)


def distill(a, n):
    return P.raw.w2l_distill_fwd_bwd(*[a[k] for k in DISTILL[:-1]], B, T, C, K, 1.0, 1.0, BF16, BF16, 1, a["ws"], n, N)


CALLS = [(fwd, FWD, ("z", "tokens", "in_len"), P.w2l_token_logprob_workspace_bytes(B, T, C, K, BF16)), (bwd, BWD, BWD[:-1], 0),
         (distill, DISTILL, ("z", "ids", "sc", "in_len", "w"), P.w2l_distill_workspace_bytes(B, T, C, K, BF16))]


@pytest.mark.parametrize("call,names,inputs,ws", CALLS, ids=["forward", "backward", "distillation"])
def test_outputs_on_inputs(call, names, inputs, ws):
    size = dict(BYTES, ws=ws)
    assert call is bwd or ws >= 256
    for o in names:
        if o in inputs:
            continue
        for i in inputs:
            a = places(names)
            a[o] = a[i]
            assert call(a, ws) == -8, (o, i)
            a = places(names)                                          # the output's end on the input's beginning, and the other way round
            a[o] = a[i] + 256 - (size[o] + 255) // 256 * 256
            if a[o] + size[o] > a[i]:
                assert call(a, ws) == -8, (o, i)
            a[o] = a[i] + (size[i] - 1) // 256 * 256
            assert call(a, ws) == -8, (o, i)


def test_the_gradient_may_not_be_the_scores():
    for gt in (F32, BF16):                      # fp32 on bf16 scores: twice as long
        a = places(DISTILL)
        a["dz"] = a["z"] - (BYTES["z"] if gt == F32 else 0)
        assert P.raw.w2l_distill_fwd_bwd(*[a[k] for k in DISTILL[:-1]], B, T, C, K, 1.0, 1.0, BF16, gt, 0, a["ws"], CALLS[2][3], N) == -8
    assert P.w2l_status_str(-8) == "output overlaps an input"
