"""w2l_groupnorm_fwd / _bwd at the ends of what they take."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
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


# (T, C, G, form, memory): 65534 utterances, most without frames, in more workgroups than one launch has; parts end at utterance 2^22 / workgroups of one
@pytest.mark.parametrize("T,C,G,form,part,need", [(8190, 4, 4, 0, 32768, 30), (1040, 520, 65, 1, 64527, 160)], ids=["runs of frames", "a workgroup a group"])
def test_more_workgroups_than_a_launch_has(P, T, C, G, form, part, need):
    """The utterances with frames are, bit for bit, what a batch of them alone is.  dgamma and dbeta are sums of the same fp32 numbers in 64 bits, rounded once, or once a part
    and added up in fp32: within 4 half steps of the parts' magnitudes."""
    B, act, U = 65534, P.W2L_ACT_SILU, 2.0 ** -24
    assert all(P.w2l_groupnorm_launch_config(b, T, C, G, act, P.W2L_BF16)[0] == form for b in (B, 600, 1200))
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < need << 30:
        pytest.skip("needs %d GiB" % need)
    rng = np.random.default_rng(41)
    live = np.sort(np.concatenate((rng.choice(part - 1, 599, False), [part - 1, part], part + 1 + rng.choice(B - part - 2, 598, False), [B - 1])))
    few = len(live)
    lengths = rng.integers(1, 200, few)
    lengths[[0, 598, 600, -1]] = T, T, T - 1, T
    n, at = torch.zeros(B, dtype=torch.int32, device=DEV), torch.from_numpy(live).to(DEV)
    n[at] = torch.from_numpy(lengths.astype(np.int32)).to(DEV)
    small = torch.randn(few, T, C, device=DEV, generator=torch.Generator(device=DEV).manual_seed(42)).bfloat16()
    gamma, beta = torch.linspace(0.5, 1.5, C, device=DEV), torch.linspace(-1, 1, C, device=DEV)
    x = torch.empty(B, T, C, dtype=torch.bfloat16, device=DEV)             # (frames behind an end are not read, whatever is there)
    for i, b in enumerate(live):
        x[b] = small[i]

    def both(x, n):
        b = len(x)
        y, mean, rstd = torch.empty_like(x), torch.empty(b, G, device=DEV), torch.empty(b, G, device=DEV)
        ws = P.workspace(P.w2l_groupnorm_workspace_bytes(b, T, C, G, act, P.W2L_BF16))
        P.w2l_groupnorm_fwd(x, y, mean, rstd, gamma, beta, in_len=n, act=act, workspace=ws)
        rows = at if b == B else torch.arange(b, device=DEV)
        o = dict(y=y[rows], mean=mean[rows], rstd=rstd[rows])
        nothing = torch.ones(b, dtype=torch.bool, device=DEV)
        nothing[rows] = False
        zero = lambda t: all(not bool(p[k].any()) for p, k in zip(t.split(4096), nothing.split(4096)))  # noqa: E731
        assert zero(y) and zero(mean) and zero(rstd)
        del y
        dx, dg, db = torch.empty_like(x), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
        P.w2l_groupnorm_bwd(x, x, mean, rstd, dx, gamma, beta, dg, db, in_len=n, act=act, workspace=ws)
        assert zero(dx)
        return {**o, "dx": dx[rows], "dgamma": dg, "dbeta": db}
    got = both(x, n)
    del x
    torch.cuda.empty_cache()
    m = torch.from_numpy(lengths.astype(np.int32)).to(DEV)
    want = both(small, m)
    for k in ("y", "mean", "rstd", "dx"):
        assert torch.equal(got[k], want[k]), k
    first, second = both(small[:600], m[:600]), both(small[600:], m[600:])
    for k in ("dgamma", "dbeta"):
        assert bool((got[k] - want[k]).abs().le(4 * U * (first[k].abs() + second[k].abs())).all()), k


# runs joined by a launch of their own, both ways: of 24, 32 and 64 groups, of one, of nine (not a whole number of workgroups), with vectors of every length
LONG = [(4, 40000, 48, 24), (3, 70000, 8, 1), (2, 40000, 36, 9), (1, 70000, 64, 64), (1, 40000, 64, 32)]


@pytest.mark.parametrize("act", ["silu", "glu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", LONG, ids=str)
def test_long_utterances_in_many_runs(P, shape, dtype, act):
    B, T, C, G = shape
    assert P.w2l_groupnorm_launch_config(*shape, code(P, act), P.W2L_BF16 if dtype == "bf16" else P.W2L_F32)[0] == 0
    x, gamma, beta, dy = case(C + B, B, T, C, act, dtype)
    n = [T, 17, 0, T + 1][:B]
    clean = [k if k <= T else 0 for k in n]
    x[np.arange(T)[None] >= np.array(n)[:, None]] = 0
    got = run(P, x, G, gamma, beta, n, act, dtype, dy)
    for k in ("y", "mean", "rstd"):
        assert np.isnan(got[k][3:]).all(), k
        got[k][3:] = 0
    assert not got["dx"][3:].any()
    check(got, x * (np.arange(B) < 3)[:, None, None], G, gamma, beta, clean, act, dtype, dy, l2=False)
    before = np.linspace(-1, 1, C).astype(np.float32).astype(np.float64)
    again, add = (run(P, x, G, gamma, beta, n, act, dtype, dy, accumulate=a) for a in (None, before))
    for k in ("y", "mean", "rstd", "dx", "dgamma", "dbeta"):
        assert np.array_equal(again[k][:3], got[k][:3]), k
    check({**add, **{k: got[k] for k in ("y", "mean", "rstd")}}, x * (np.arange(B) < 3)[:, None, None], G, gamma, beta, clean, act, dtype, dy, accumulate=before, l2=False)


def test_long_utterances_captured_and_replayed(P):
    B, T, C, G = 2, 40000, 64, 32
    x, gamma, beta, dy = (torch.from_numpy(a).float().to(DEV) for a in case(51, B, T, C, "glu", "bf16"))
    x, dy, n = x.bfloat16(), dy.bfloat16(), torch.tensor([T, 30000], dtype=torch.int32, device=DEV)
    new = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
    y, mean, rstd, dx, dg, db = new(B, T, C // 2, t=torch.bfloat16), new(B, G), new(B, G), new(B, T, C, t=torch.bfloat16), new(C), new(C)
    ws = P.workspace(P.w2l_groupnorm_workspace_bytes(B, T, C, G, P.W2L_ACT_GLU, P.W2L_BF16))

    def step():
        P.w2l_groupnorm_fwd(x, y, mean, rstd, gamma, beta, in_len=n, act=P.W2L_ACT_GLU, workspace=ws)
        P.w2l_groupnorm_bwd(x, dy, mean, rstd, dx, gamma, beta, dg, db, in_len=n, act=P.W2L_ACT_GLU, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.normal_()
        n.copy_(torch.tensor([T - k, 10000 * k], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, mean, rstd, dx, dg, db)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, mean, rstd, dx, dg, db))), k
