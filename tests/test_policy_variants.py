"""Host-only: every form of the policy loss's kernels that some size takes is the form of a GPU parity case (tests/policy_cases.py), and holds its rows."""
import pytest

import paper_1812_07625_amd as P
from policy_cases import CASES, ROWS, policy_form
from test_score_variants import CLASSES, _slots


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_cases_cover_every_form_that_holds_its_rows(dtype):
    code, seen = P.W2L_BF16 if dtype == "bf16" else P.W2L_F32, {}
    for C in CLASSES:
        for rows in ROWS:
            w, g, v = P.w2l_policy_launch_config(1, rows, C, code)
            if w == 0:
                assert C <= 256 and g == 1 and 16 * v >= C, (rows, C)
            else:
                assert w * g * v >= _slots(C, dtype) and 1 <= w <= 16 and 1 <= g <= 16 and (w > 1 or g == 1), (rows, C, w, g, v)
            seen.setdefault((dtype, min(w, 2), g > 1, v), (rows, C))
    missing = {f: eg for f, eg in seen.items() if f not in {policy_form(P, *c) for c in CASES}}
    assert not missing, "forms (type, wavefronts, joined, slots) with no parity case, e.g. (rows, C): %r" % missing


def test_the_sizes_picked_for_wavefronts_that_fit_have_these_forms():
    """Those of test_gpu_policy.py: six, seven and fourteen slots a wavefront, two to seven wavefronts; seven and ten with a row in sixteen workgroups."""
    picked = {(1100, 2801, 0): (2, 1, 6), (1100, 5631, 1): (2, 1, 6), (2056, 4500, 0): (3, 1, 6), (2056, 8999, 1): (3, 1, 6), (2056, 5101, 0): (3, 1, 7), (2056, 10001, 1): (3, 1, 7),
              (416, 8500, 0): (5, 1, 7), (416, 17001, 1): (5, 1, 7), (136, 16601, 0): (5, 1, 14), (136, 33203, 1): (5, 1, 14), (8, 200001, 0): (8, 16, 7), (8, 262143, 0): (8, 16, 10)}
    for (rows, C, code), form in picked.items():
        assert P.w2l_policy_launch_config(1, rows, C, code) == form, (rows, C, code)


def test_where_the_policy_loss_departs_from_the_distillation():
    """Rows of 17 to 24 vectors a lane have three wavefronts, however many they are."""
    for rows in (2048, 30000):
        assert P.w2l_distill_launch_config(1, rows, 10001, 1, P.W2L_BF16)[0] == 1 and P.w2l_policy_launch_config(1, rows, 10001, P.W2L_BF16) == (3, 1, 7)


def test_launch_config_refuses_what_the_call_refuses():
    for bad in ((0, 1, 5, 0), (1, 0, 5, 0), (1, 1, 0, 0), (1, 1, 262145, 0), (1, 1, 5, 2), (65536, 32768, 5, 0)):
        with pytest.raises(P.W2LError):
            P.w2l_policy_launch_config(*bad)
    assert P.raw.w2l_policy_launch_config(1, 1, 5, 0, None, None, None) == -1
    for rows, C, dtype in CASES:
        code = P.W2L_BF16 if dtype == "bf16" else P.W2L_F32
        assert (P.w2l_policy_workspace_bytes(1, rows, C, code) > 0) == (P.w2l_policy_launch_config(1, rows, C, code)[1] > 1)
