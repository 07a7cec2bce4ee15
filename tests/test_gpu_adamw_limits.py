"""w2l_adamw_step at the ends of what it takes, against numpy as in test_gpu_adamw.py."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import DEV
from test_gpu_adamw import F, Net, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


@pytest.mark.parametrize("gradient", [0.0, 1e-30, 1e-3])
def test_moments_with_every_exponent(P, gradient):
    """Exponents that int8 holds, of moments that came from elsewhere: 2^-127 and 2^-128 are denormal numbers of fp32, and 448 * 2^119 is its last with all codes finite."""
    exps = list(range(-128, 120))
    net = Net(P, [256 * len(exps) - 9], 8, seed=3)
    h, d = net.host[0], net.dev[0]
    h["grad"] = (np.sign(h["grad"]) * F(gradient)).astype(F)
    d["grad"].copy_(torch.from_numpy(h["grad"]))
    h["m_exp"] = np.array(exps, np.int8)
    h["v_exp"] = np.minimum(h["m_exp"], 50)[::-1].copy()                   # (squares of roots up to 448 * 2^50 are finite)
    for k in ("m_exp", "v_exp"):
        d[k].copy_(torch.from_numpy(h[k]).to(DEV))
    for step in (7, 8):
        net.step(step, eps=1e-3, check=False)
        net.check_guards()
        with np.errstate(over="ignore", under="ignore", invalid="ignore"):
            m0, root0 = (oracle.from_e4m3(h[k], h[k + "_exp"]).astype(F) for k in "mv")
            m, v = oracle.adamw_moments(h["grad"], m0, np.square(root0), 1.0, 0.9, 0.999)
            w64 = oracle.adamw(h["w"], h["grad"], m0, np.square(root0), 1.0, step, 1e-2, 0.9, 0.999, 1e-3, h["decay"])[0]
            # the largest moments, over the smallest roots, move weights by 448 * 2^119 * 1e-2 / 1e-3 = 3e39: beyond fp32, and infinite there
            beyond = np.abs(w64) > np.finfo(F).max
            moved = np.abs(w64 - h["w"].astype(np.float64) * (1 - 1e-2 * h["decay"]))
            bound = U * (14 * moved + 3 * np.abs(h["w"]) + np.abs(w64)) + 14 * U * 1e-2 * np.abs(m0) / (np.sqrt(v) + 1e-3)
            w = d["w"].cpu().numpy()
            assert np.array_equal(w[beyond], w64.astype(F)[beyond]) and (np.abs(w - w64) <= bound)[~beyond].all()
        r = oracle.adamw_dither(5, step, 0, len(w))
        want = dict(zip(("m", "m_exp"), oracle.to_e4m3(m, r))) | dict(zip(("v", "v_exp"), oracle.to_e4m3(np.sqrt(v), r, keep=True)))
        for k, x in want.items():
            got = d[k].cpu().numpy()
            assert np.array_equal(got & 127, x & 127) if k == "m" else np.array_equal(got, x), (step, k)
            h[k] = got
        assert np.array_equal(oracle.from_e4m3(h["m"], h["m_exp"]), oracle.from_e4m3(want["m"], h["m_exp"]))
        h["w"] = w
