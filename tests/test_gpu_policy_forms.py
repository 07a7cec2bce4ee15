"""w2l_policy_fwd_bwd against the fp64 oracle in every form of its kernels, bounds as in test_gpu_policy.py."""
import numpy as np
import pytest

from policy_cases import CASES
from test_gpu_policy import case, check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


@pytest.mark.parametrize("rows,C,dtype", CASES, ids=str)
def test_every_form(P, rows, C, dtype):
    """Eight different frames in turn (rows begin alike within a vector every eight): the oracle sees these, the others are theirs bit for bit."""
    few = min(rows, 8)
    c = case(rows + C, 1, few, C, dtype)
    many = {k: np.concatenate([v] * -(-rows // few), 1)[:, :rows] for k, v in c.items()}
    for gtype in (dtype, "fp32") if dtype == "bf16" else ("fp32",):
        got = run(P, many, dtype, gtype=gtype)
        for k in ("frame", "logprob", "dz"):
            for i in range(0, rows, few):
                n = min(few, rows - i)
                assert np.array_equal(got[k][:, i:i + n], got[k][:, :n]), (k, i)
        check({k: v[:, :few] for k, v in got.items() if k != "loss"}, c, gtype=gtype)
