"""Host-only: every form of the kernels over frame scores that some size takes is the form of a GPU parity case
(tests/score_cases.py), and every size has a form that holds its rows.  And the library's host code for these calls under
AddressSanitizer + UBSan."""
import pytest

import paper_1812_07625_amd as P
from score_cases import CASES, ROWS, distill_cases, distill_form, token_form
from test_sanitizers import _run_pytest_under

CLASSES = list(range(1, 9000)) + list(range(9000, 262145, 41)) + [262140, 262141, 262142, 262143, 262144]


def _slots(C, dtype):
    n = 8 if dtype == "bf16" else 4
    most = C if C % n == 0 else C + 2 * (n - 1)
    return -(-most // (64 * n))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_size_has_a_form_that_holds_it(dtype):
    code = P.W2L_BF16 if dtype == "bf16" else P.W2L_F32
    for C in CLASSES:
        forms = [P.w2l_token_logprob_launch_config(2, 3, C, K, code) for K in {0, min(C, 24), min(C, 64)}]
        forms += [P.w2l_distill_launch_config(1, rows, C, 1, code) for rows in ROWS + (1, 127, 128, 2047, 30000)]
        for w, g, v in forms:
            if w == 0:
                assert C <= 256 and g == 1 and 16 * v >= C, (C, w, g, v)
            else:
                assert w * g * v >= _slots(C, dtype) and 1 <= w <= 16 and 1 <= g <= 16 and (w > 1 or g == 1), (C, w, g, v)


def test_cases_cover_every_form():
    tokens, distill = {}, {}
    for dtype in ("fp32", "bf16"):
        for C in CLASSES:
            for K in {0, min(C, 24), min(C, 64)}:
                tokens.setdefault(token_form(P, C, K, dtype), (C, K))
            for rows in ROWS + (1, 2047):
                distill.setdefault(distill_form(P, rows, C, dtype), (rows, C))
    missing = {f: eg for f, eg in tokens.items() if f not in {token_form(P, *c) for c in CASES}}
    assert not missing, "forms (type, wavefronts, joined, slots) with no parity case, e.g. (C, K): %r" % missing
    missing = {f: eg for f, eg in distill.items() if f not in {distill_form(P, r, C, d) for r, C, _, d in distill_cases(P)}}
    assert not missing, "forms (type, wavefronts, joined, slots) with no parity case, e.g. (rows, C): %r" % missing


def test_launch_config_refuses_what_the_calls_refuse():
    for bad in ((0, 1, 5, 1, 0), (1, 0, 5, 1, 0), (1, 1, 0, 0, 0), (1, 1, 262145, 1, 0), (1, 1, 5, 6, 0), (1, 1, 100, 65, 0), (1, 1, 5, 1, 2)):
        with pytest.raises(P.W2LError):
            P.w2l_token_logprob_launch_config(*bad)
        with pytest.raises(P.W2LError):
            P.w2l_distill_launch_config(*bad)
    with pytest.raises(P.W2LError):
        P.w2l_distill_launch_config(1, 1, 5, 0, 0)


def test_workspace_goes_with_the_form():
    for C, K, dtype in CASES:
        code = P.W2L_BF16 if dtype == "bf16" else P.W2L_F32
        _, g, _ = P.w2l_token_logprob_launch_config(3, 7, C, K, code)
        n = P.w2l_token_logprob_workspace_bytes(3, 7, C, K, code)
        assert (n > 0) == (g > 1) and (g == 1 or n >= 21 * g * (16 + 8 * K))
        _, g, _ = P.w2l_distill_launch_config(3, 7, C, K, code)
        assert (P.w2l_distill_workspace_bytes(3, 7, C, K, code) > 0) == (g > 1)
    assert P.w2l_token_logprob_workspace_bytes(0, 7, 100000, 1, 0) == 0 and P.w2l_distill_workspace_bytes(1, 7, 300000, 1, 0) == 0


def test_host_code_under_asan_ubsan():
    from paper_1812_07625_amd import build as hip_build
    lib = hip_build.build(sanitize=True)
    out = _run_pytest_under(hip_build.asan_runtime(), {"W2L_LIB": lib}, ["test_scores_abi.py"])
    assert "failed" not in out
