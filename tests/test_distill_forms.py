"""Forms of w2l_distill_fwd_bwd that the type, the number of workgroups and the slots of a row do not tell apart (tests/score_cases.py has those): rows of
up to 256 classes with up to 16 entries, one a lane, or more; and each with every pair of types."""
import numpy as np
import pytest

import paper_1812_07625_amd as P
from score_cases import distill_cases

TYPES = [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16")]
SHORT = [(C, K) for C, Ks in ((20, (1, 16, 17, 20)), (50, (16, 33)), (100, (7, 64)), (256, (3, 16, 17, 64)), (200, (16, 48))) for K in Ks]


def form(C, K, dtype):
    w, g, v = P.w2l_distill_launch_config(1, 5, C, K, P.W2L_BF16 if dtype == "bf16" else P.W2L_F32)
    return (v, K > 16) if w == 0 else None


def test_cases_cover_short_rows():
    for dtype in ("fp32", "bf16"):
        want = {form(C, K, dtype) for C in range(1, 400) for K in {1, min(C, 16), min(C, 17), min(C, 64)}} - {None}
        assert len(want) == 8 and want == {form(C, K, dtype) for C, K in SHORT}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dz_dtype", TYPES, ids=lambda v: v)
@pytest.mark.parametrize("C,K", SHORT)
def test_short_rows(C, K, dtype, dz_dtype):
    from test_gpu_scores import check_distill, distill_case, run_distill
    for B, T in ((2, 7), (3, 41)):              # one workgroup for all, and several
        z, ids, sc, w, in_len = distill_case(B, T, C, K, dtype, 23)
        for tau in (1.0, 3.0):
            check_distill(run_distill(P, z, ids, sc, tau, w, in_len, 0.5, dtype, dz_dtype), z, ids, sc, tau, w, in_len, 0.5, dz_dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c in distill_cases(P) if c[3] == "bf16"], ids=lambda c: "rows%d-C%d-K%d" % c[:3])
def test_fp32_gradients_of_bf16_scores(case):
    from test_gpu_scores import check_distill, distill_case, run_distill
    rows, C, K, dtype = case
    live = min(rows, 7)
    z, ids, sc, w, _ = distill_case(1, live, C, K, dtype, 12)
    pad = lambda a, v: np.concatenate([a, np.full((1, rows - live) + a.shape[2:], v, a.dtype)], 1)
    z, ids, sc, w = pad(z, np.nan), pad(ids, -7), pad(sc, np.nan), pad(w, np.nan)
    check_distill(run_distill(P, z, ids, sc, 2.0, w, [live], 0.5, dtype, "fp32"), z, ids, sc, 2.0, w, [live], 0.5, "fp32")
