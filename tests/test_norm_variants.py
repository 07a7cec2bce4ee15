"""Host-only: every form of the group norm's kernels has a parity case."""
import pytest

import paper_1812_07625_amd as P
from norm_cases import ACTS, SHAPES, fits, form


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_every_form_has_a_case(act, dtype):
    seen = {form(P, s, act, dtype) for s in SHAPES if fits(s, act)}
    lengths = (1, 2, 4, 8) if dtype == "bf16" else (1, 2, 4)
    assert seen == {(g, n, act, dtype) for g in (0, 1) for n in lengths}


def test_what_is_asked_for():
    assert P.w2l_groupnorm_launch_config(8, 750, 1536, 32, P.W2L_ACT_GLU, P.W2L_BF16) == (1, 8)      # 128 workgroups of 144 KB
    assert P.w2l_groupnorm_launch_config(16, 1500, 2048, 1, P.W2L_ACT_SILU, P.W2L_BF16) == (0, 8)    # 16 of 6 MB
    assert P.w2l_groupnorm_launch_config(1, 100, 30, 3, P.W2L_ACT_GLU, P.W2L_F32) == (0, 1)          # values and gates of one group
    with pytest.raises(P.W2LError):
        P.w2l_groupnorm_launch_config(1, 1, 30, 4, 0, 0)
