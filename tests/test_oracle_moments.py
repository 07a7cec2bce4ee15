"""What moments in 8 bits cost AdamW's second moment in the long run, from the rule that the kernel's tests compare bit for bit."""
import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("beta2", [0.999, 0.98])
def test_the_second_moment_under_random_rounding(beta2):
    """Normal gradients of one deviation.  A step moves a root r by d = (1 - beta2) / 2 |g^2 - 1| r, E|g^2 - 1| = 4 exp(-1/2) / sqrt(2 pi) = 0.968; numbers are s = r/16 to
    r/8 apart, so that rounding at random has a variance of d s: relative to r^2 (1 - beta2) times 0.030 to 0.0605.  v holds the sum of the variances of 1 / (1 - beta2) steps, 3.0
    to 6.05 %; roots, which forget as v does, scatter by sqrt(0.030 / (1 + beta2)) to sqrt(0.0605 / (1 + beta2)), 12.3 to 17.4 %, and by their own sqrt((1 - beta2) / 2) / sqrt(2).
    The mean of 2048 values' v, each within 35 % of its own, is known to 0.8 %, three of which are left on either side."""
    rng = np.random.default_rng(1)
    n, tau = 2048, int(round(1 / (1 - beta2)))
    codes, exps = oracle.to_e4m3(np.ones(n), np.zeros(n))
    v32 = np.ones(n)
    above, spread = [], []
    for t in range(1, 4 * tau + 1):
        g = rng.standard_normal(n).astype(np.float32)
        root = oracle.from_e4m3(codes, exps).astype(np.float32)
        _, v = oracle.adamw_moments(g, np.zeros(n), np.square(root), 1.0, 0.9, beta2)
        codes, exps = oracle.to_e4m3(np.sqrt(v), oracle.adamw_dither(3, t, 0, n), keep=True)
        v32 = v32 * beta2 + g.astype(np.float64) ** 2 * (1 - beta2)
        if t > 3 * tau and t % (tau // 10) == 0:
            kept = oracle.from_e4m3(codes, exps)
            above.append((kept ** 2).mean() / v32.mean())
            spread.append(np.std(kept / np.sqrt(v32)))
    assert 1.030 - 0.024 < np.mean(above) < 1.0605 + 0.024, np.mean(above)
    assert 0.11 < np.mean(spread) < 0.19, np.mean(spread)


def test_roots_that_are_lifted_and_roots_that_are_lost():
    """Below the block's least number a root becomes it, and rounds up from there as any number; a root whose square is zero in fp32 is zero."""
    x = np.full(256, 1e-9)
    x[0] = 448.0
    for r in (0.0, 0.999):
        codes, exps = oracle.to_e4m3(x, np.full(256, r), keep=True)
        assert exps[0] == 0 and (codes[1:] == 1).all()
    with np.errstate(under="ignore"):
        for power, alive in ((-74, True), (-76, False)):
            _, v = oracle.adamw_moments(np.zeros(1), np.zeros(1), np.square(np.float32([2.0 ** power])), 1.0, 0.9, 0.999)
            assert (v[0] > 0) == alive
