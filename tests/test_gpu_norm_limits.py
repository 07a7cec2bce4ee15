"""w2l_groupnorm_fwd / _bwd at the ends of what they take."""
import numpy as np
import pytest

from norm_cases import ACTS, code
from test_gpu_groupnorm import case, check, held, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size", [1e20, 1e25, 1e38])
@pytest.mark.parametrize("T,C,G,form", [(40, 32, 4, 1), (2500, 32, 1, 0), (2500, 64, 2, 0)], ids=["a workgroup a group", "one group in runs", "two groups in runs"])
def test_a_variance_that_fp32_does_not_hold(P, T, C, G, form, size, dtype, act):
    """Finite values whose squares are beyond fp32: the group is NaN, not beta with gradients of 0; other groups, and the other utterance, are as they are without.
    Squares of 1e20 are beyond it by themselves, 3.4e38 is fp32's largest."""
    assert P.w2l_groupnorm_launch_config(2, T, C, G, code(P, act), P.W2L_BF16 if dtype == "bf16" else P.W2L_F32)[0] == (0 if act == "glu" and G == 1 else form)
    x, gamma, beta, dy = case(21, 2, T, C, act, dtype)
    big = x.copy()
    per = C // G
    big[1, :, :per] = held(size * np.sign(x[1, :, :per] + 1e-3) * (0.5 + 0.5 * np.abs(np.sin(np.arange(T)))[:, None]), dtype)
    got, plain = run(P, big, G, gamma, beta, None, act, dtype, dy), run(P, x, G, gamma, beta, None, act, dtype, dy)
    bad = np.zeros((2, G), bool)
    bad[1, 0] = True
    for k in ("mean", "rstd"):
        assert np.array_equal(np.isnan(got[k]), bad), k
        assert np.array_equal(got[k][~bad], plain[k][~bad]), k
    wide = np.repeat(bad, per, 1)                                          # of channels
    out = wide[:, :C // 2] | wide[:, C // 2:] if act == "glu" else wide    # a value or its gate
    assert np.array_equal(np.isnan(got["y"]).all(1), out) and np.array_equal(np.isnan(got["y"]).any(1), out)
    assert np.array_equal(got["y"].transpose(0, 2, 1)[~out], plain["y"].transpose(0, 2, 1)[~out])
    into = wide if act != "glu" else np.concatenate((out, out), 1)         # a group that any value of it or of its partner's reaches
    into = np.repeat(into.reshape(2, G, per).any(2), per, 1)
    assert np.array_equal(np.isnan(got["dx"]).any(1), into)
    assert np.array_equal(got["dx"].transpose(0, 2, 1)[~into], plain["dx"].transpose(0, 2, 1)[~into])
    assert np.isnan(got["dgamma"][wide[1]]).all()
    if act in ("relu", "silu"):                                            # (without an activation, and of a GLU's values, dbeta does not depend on u)
        assert np.isnan(got["dbeta"][wide[1]]).all()


def test_large_values_whose_variance_fp32_holds(P):
    """2^59 and its like are normalised as any others are."""
    for dtype in ("fp32", "bf16"):
        for T, C, G in ((40, 32, 4), (2500, 32, 1)):
            x, gamma, beta, dy = case(22, 2, T, C, "none", dtype)
            x = x * 2.0 ** 56
            check(run(P, x, G, gamma, beta, None, "none", dtype, dy), x, G, gamma, beta, None, "none", dtype, dy, l2=False)
