"""w2l_adamw_step against numpy: moments in 32 bits, codes and exponents of moments in 8 bits, and weights' bf16 copies bit for bit (the formulas say how every product
and sum is rounded).  Weights against fp64, in U = 2^-24: the moment and the root carry 3 U of their terms each, their constants, the denominator, its reciprocal (an ulp) and the
products 8 more, so that the step is off by 14 U of itself (and of its terms where they cancel); the decayed weight by 3 U, the result by its rounding."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F = np.float32


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


def values(rng, n, zeros=False):
    g = (rng.standard_normal(n) * np.exp(2 * rng.standard_normal((n + 255) // 256).repeat(256)[:n]) * 1e-3).astype(F)
    if zeros and n > 300:
        g[256:512] = 0
    return g


class Net:
    """Tensors of the given sizes on the GPU, each between guards, and their fp32 / byte copies on the host."""

    def __init__(self, P, sizes, bits, seed=0, grad="fp32", lowp=True, decay=0.01, moments="some"):
        rng = np.random.default_rng(seed)
        self.P, self.sizes, self.bits, self.lowp = P, sizes, bits, lowp
        self.host, self.dev, self.wholes, rows = [], [], [], []
        for i, n in enumerate(sizes):
            g = values(rng, n, True)
            h = dict(w=(0.1 * rng.standard_normal(n)).astype(F), grad=g)
            if grad == "bf16":
                h["grad"] = torch.from_numpy(g).bfloat16().float().numpy()
            m = values(rng, n) if moments == "some" else np.zeros(n, F)
            v = np.square(values(rng, n)) if moments == "some" else np.zeros(n, F)
            if bits == 32:
                h.update(m=m, v=v)
            else:
                h["m"], h["m_exp"] = oracle.to_e4m3(m, np.full(n, 0.5))
                h["v"], h["v_exp"] = oracle.to_e4m3(np.sqrt(v), np.full(n, 0.5))
            h["decay"] = decay if i % 2 == 0 else 0.0
            self.host.append(h)
            d = {}
            for k in ("w", "grad", "m", "v", "m_exp", "v_exp"):
                if k in h:
                    t = torch.from_numpy(h[k]).to(DEV)
                    if k == "grad" and grad == "bf16":
                        t = t.bfloat16()
                    d[k] = self.guard(t)
            if lowp:
                d["w_lowp"] = self.guard(torch.zeros(n, dtype=torch.bfloat16, device=DEV))
            self.dev.append(d)
            as_ = lambda k: d[k].view(torch.float8_e4m3fn) if bits == 8 and k in "mv" else d.get(k)  # noqa: E731
            rows.append({k: as_(k) for k in ("w", "grad", "m", "v", "m_exp", "v_exp", "w_lowp")} | {"weight_decay": h["decay"]})
        self.tensors = P.adamw_tensors(rows)
        self.ws = P.workspace(P.w2l_adamw_workspace_bytes(self.tensors))
        self.norm = torch.full((1,), -7.0, device=DEV)

    def guard(self, t):
        n = t.numel()
        whole = torch.full((n + 1024,), 77, dtype=t.dtype, device=DEV)
        whole[512:512 + n] = t
        self.wholes.append((whole, n))
        return whole[512:512 + n]

    def check_guards(self):
        for whole, n in self.wholes:
            assert bool((whole[:512] == 77).all()) and bool((whole[512 + n:] == 77).all()), "written outside the tensor"

    def step(self, step, lr=1e-2, b1=0.9, b2=0.999, eps=1e-8, clip=0.0, gs=1.0, seed=5, want_norm=False, check=True, **kw):
        self.P.w2l_adamw_step(self.tensors, step, lr, b1, b2, eps, gs, clip, seed, grad_norm=self.norm if want_norm else None, workspace=self.ws, **kw)
        torch.cuda.synchronize()
        if check:
            self.check(step, lr, b1, b2, eps, clip, gs, seed, want_norm)

    def check(self, step, lr, b1, b2, eps, clip, gs, seed, want_norm=False):
        self.check_guards()
        grads = [h["grad"] for h in self.host]
        factor = oracle.adamw_factor(grads, gs, clip)
        if want_norm:
            assert abs(float(self.norm) - oracle.adamw_norm(grads, gs)) <= U * oracle.adamw_norm(grads, gs) * 1.01
        for i, (h, d) in enumerate(zip(self.host, self.dev)):
            n = len(h["w"])
            m0 = h["m"] if self.bits == 32 else oracle.from_e4m3(h["m"], h["m_exp"]).astype(F)
            v0 = h["v"] if self.bits == 32 else np.square(oracle.from_e4m3(h["v"], h["v_exp"]).astype(F))
            m, v = oracle.adamw_moments(h["grad"], m0, v0, factor, b1, b2)
            w64, _, _ = oracle.adamw(h["w"], h["grad"], m0, v0, factor, step, lr, b1, b2, eps, h["decay"])
            w = d["w"].cpu().numpy()
            # the root and moment are those of fp32: what their own roundings move, relative to the step, is 2 U each
            moved = np.abs(w64 - h["w"].astype(np.float64) * (1 - lr * h["decay"]))
            assert (np.abs(w - w64) <= U * (14 * moved + 3 * np.abs(h["w"]) + np.abs(w64)) + 14 * U * lr * np.abs(m0) / (np.sqrt(v) + eps)).all(), i
            if self.lowp:
                assert torch.equal(d["w_lowp"].view(torch.int16), d["w"].bfloat16().view(torch.int16)), i
            if self.bits == 32:
                assert np.array_equal(d["m"].cpu().numpy(), m) and np.array_equal(d["v"].cpu().numpy(), v), i
                h.update(m=m, v=v, w=w)
            else:
                r = oracle.adamw_dither(seed, step, i, n)
                new = {}
                new["m"], new["m_exp"] = oracle.to_e4m3(m, r)
                new["v"], new["v_exp"] = oracle.to_e4m3(np.sqrt(v), r, keep=True)
                for k, want in new.items():
                    got = d[k].cpu().numpy()
                    assert np.array_equal(got & 127 if k == "m" else got, want & 127 if k == "m" else want), (i, k, np.nonzero(got != want)[0][:5])
                    if k == "m":
                        assert np.array_equal(oracle.from_e4m3(got, new["m_exp"]), oracle.from_e4m3(want, new["m_exp"])), i
                h.update(w=w, **{k: d[k].cpu().numpy() for k in new})


SIZES = [[1], [3, 255, 256, 257], [4096, 4097, 1, 8192, 12289], [100_003], [2 + 97 * i for i in range(130)], [0, 5, 0, 0, 700, 0]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%d tensors of %d" % (len(s), max(s)))
def test_steps(P, sizes, bits):
    net = Net(P, sizes, bits, seed=len(sizes))
    net.step(1)
    net.step(2, clip=0.01, want_norm=True)
    net.step(1000, clip=1e6, want_norm=True, lr=0.3, b1=0.0, b2=0.5, eps=1e-2)
    net.step(10 ** 6, want_norm=True, b1=0.99, gs=-0.5, clip=1e-3)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_of_bf16(P, bits):
    net = Net(P, [1000, 29, 5000], bits, grad="bf16", lowp=False)
    net.step(3, clip=0.1, want_norm=True)
    net.step(4)


@pytest.mark.parametrize("bits", [32, 8])
def test_from_nothing(P, bits):
    """Moments of zero (all bytes zero), and gradients of zero: a weight without gradient decays and does not move."""
    net = Net(P, [600, 4097], bits, moments="none")
    if bits == 8:
        assert not any(h["m"].any() or h["m_exp"].any() or h["v"].any() for h in net.host)
    before = net.host[0]["w"].copy()
    net.step(1)
    h = net.host[0]
    assert np.allclose(h["w"][256:512], before[256:512] * (1 - 1e-2 * 0.01), rtol=1e-7) and not h["m"][256:512].any()
    for k in range(2, 8):
        net.step(k)


@pytest.mark.parametrize("bits", [32, 8])
def test_extreme_gradients(P, bits):
    """Gradients from 1e-38 to 1e18 in one tensor, in one block and in blocks of their own."""
    net = Net(P, [2048], bits, moments="none")
    rng = np.random.default_rng(3)
    g = (rng.standard_normal(2048) * 10.0 ** np.concatenate([rng.uniform(-38, 18, 1024), np.repeat([-37, -30, 10, 18], 256)])).astype(F)
    net.host[0]["grad"] = g
    net.dev[0]["grad"].copy_(torch.from_numpy(g))
    with np.errstate(over="ignore", under="ignore"):
        net.step(1, eps=1e-8)
        net.step(2, eps=1e-8)
    if bits == 8:
        root = oracle.from_e4m3(net.host[0]["v"], net.host[0]["v_exp"])
        assert (root[np.square(g) * F(1e-3) > 0] > 0).all()               # a root above 0 stays above 0


def test_nan_stays_where_it_is_without_a_norm(P):
    for bits in (32, 8):
        net = Net(P, [600], bits)
        g = net.host[0]["grad"]
        g[[5, 300]] = np.nan, np.inf
        net.dev[0]["grad"].copy_(torch.from_numpy(g))
        P.w2l_adamw_step(net.tensors, 1, 1e-3)
        torch.cuda.synchronize()
        w, m = net.dev[0]["w"].cpu().numpy(), net.dev[0]["m"].cpu().numpy()
        bad = np.zeros(600, bool)
        bad[[5, 300]] = True
        assert np.array_equal(np.isnan(w), bad)
        assert np.array_equal(~np.isfinite(m) if bits == 32 else m & 127 == 127, bad)
        if bits == 8:                                                      # the others of the block are what they would be
            assert np.isfinite(oracle.from_e4m3(m, net.dev[0]["m_exp"].cpu().numpy())[~bad]).all() and net.dev[0]["m_exp"].abs().max() < 60


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
def test_a_norm_that_is_not_finite_changes_nothing(P, bits, odd):
    net = Net(P, [600, 5000], bits)
    net.dev[1]["grad"][4999] = odd
    before = [{k: t.clone() for k, t in d.items()} for d in net.dev]
    net.step(1, clip=1.0, want_norm=True, check=False)
    assert not math.isfinite(float(net.norm))
    net.step(1, want_norm=True, check=False)
    for b, d in zip(before, net.dev):
        for k in d:
            assert torch.equal(b[k].view(torch.uint8), d[k].view(torch.uint8)), k


def test_the_same_call_gives_the_same_bits_and_another_seed_others(P):
    a, b, c, d = (Net(P, [5000, 77], 8) for _ in range(4))
    a.step(9, clip=0.05, want_norm=True)
    b.step(9, clip=0.05, want_norm=True)
    c.step(9, clip=0.05, want_norm=True, seed=6)
    for x, y, z in zip(a.dev, b.dev, c.dev):
        for k in x:
            assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), k
        assert torch.equal(x["w"], z["w"]) and not torch.equal(x["m"], z["m"])
    assert d.norm.item() == -7.0


def test_rounding_at_random_keeps_small_changes(P):
    """A constant gradient: the root of the second moment follows its formula within what rounding at random scatters, where rounding to the nearest would
    leave it where it is.  Over 200 steps of 1 - beta2 = 0.02 each of 4096 roots sees some 200 roundings whose spacing is at most 1/8; their mean over 4096 values
    scatters by less than 1/8 sqrt(200) / sqrt(4096) = 0.03 of the value."""
    n = 4096
    net = Net(P, [n], 8, moments="none", lowp=False)
    net.dev[0]["grad"].copy_(torch.full((n,), 3e-3, device=DEV) * (1 + torch.arange(n, device=DEV) % 7))
    for k in range(1, 201):
        P.w2l_adamw_step(net.tensors, k, 0.0, beta2=0.98, seed=k)
    torch.cuda.synchronize()
    root = oracle.from_e4m3(net.dev[0]["v"].cpu().numpy(), net.dev[0]["v_exp"].cpu().numpy())
    want = 3e-3 * (1 + np.arange(n) % 7) * math.sqrt(1 - 0.98 ** 200)
    assert abs((root / want).mean() - 1) < 0.03


@pytest.mark.parametrize("bits", [32, 8])
def test_step_and_rate_from_the_device_and_a_captured_graph(P, bits):
    net, twin = Net(P, [3000, 31], bits), Net(P, [3000, 31], bits)
    lr, step = torch.zeros((), device=DEV), torch.zeros((), dtype=torch.int32, device=DEV)
    call = lambda: P.w2l_adamw_step(net.tensors, 1, 0.0, max_norm=0.05, seed=5, grad_norm=net.norm, lr_dev=lr, step_dev=step, workspace=net.ws)  # noqa: E731
    before = net.dev[0]["w"].clone()
    call()                                                                 # step 0: nothing
    torch.cuda.synchronize()
    assert torch.equal(net.dev[0]["w"], before)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(1, 6):
        lr.fill_(0.01 / k)
        step.fill_(k)
        for a, b in zip(net.dev, twin.dev):
            g = torch.randn(a["grad"].shape, device=DEV) * 0.01
            a["grad"].copy_(g)
            b["grad"].copy_(g)
        graph.replay()
        torch.cuda.synchronize()
        twin.step(k, lr=float(np.float32(0.01 / k)), clip=0.05, want_norm=True, check=False)
        for a, b in zip(net.dev, twin.dev):
            for key in a:
                assert torch.equal(a[key].view(torch.uint8), b[key].view(torch.uint8)), (k, key)
        assert torch.equal(net.norm, twin.norm)


def test_on_another_stream(P):
    a, b = Net(P, [9000], 8), Net(P, [9000], 8)
    a.step(2, clip=0.1, want_norm=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    P.w2l_adamw_step(b.tensors, 2, 1e-2, max_norm=0.1, seed=5, grad_norm=b.norm, workspace=b.ws, stream=side)
    side.synchronize()
    assert torch.equal(a.dev[0]["m"], b.dev[0]["m"]) and torch.equal(a.dev[0]["w"], b.dev[0]["w"])


def test_a_tensor_beyond_2_31_values(P):
    """Offsets that pass 32 bits: the last values are as they are in a tensor of their own, random bits (of a value's index) aside."""
    n = (1 << 31) + 4096 + 5
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GiB")
    w, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    tail = 5000
    w[-tail:], g[-tail:] = torch.linspace(-1, 1, tail, device=DEV), torch.linspace(1, 2, tail, device=DEV)
    m, v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    norm = torch.zeros(1, device=DEV)
    t = P.adamw_tensors([dict(w=w, grad=g, m=m, v=v)])
    P.w2l_adamw_step(t, 1, 1e-2, grad_norm=norm, workspace=P.workspace(P.w2l_adamw_workspace_bytes(t)))
    small = [x[-tail:].clone() for x in (g,)]
    ws, ms, vs = torch.linspace(-1, 1, tail, device=DEV), torch.zeros(tail, device=DEV), torch.zeros(tail, device=DEV)
    P.w2l_adamw_step(P.adamw_tensors([dict(w=ws, grad=small[0], m=ms, v=vs)]), 1, 1e-2)
    torch.cuda.synchronize()
    assert torch.equal(w[-tail:], ws) and torch.equal(m[-tail:], ms) and torch.equal(v[-tail:], vs) and not bool(w[:-tail].any())
    assert abs(float(norm) - float(small[0].double().square().sum().sqrt())) < 1e-4
    del m, v
    m8, v8 = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV)
    e8, f8 = (torch.zeros((n + 255) // 256, dtype=torch.int8, device=DEV) for _ in range(2))
    w[-tail:] = torch.linspace(-1, 1, tail, device=DEV)
    P.w2l_adamw_step(P.adamw_tensors([dict(w=w, grad=g, m=m8, v=v8, m_exp=e8, v_exp=f8)]), 1, 1e-2)
    torch.cuda.synchronize()
    assert torch.equal(w[-tail:], ws) and not bool(w[:-tail].any()) and not bool(m8[:-tail].any()) and bool(m8[-tail:].all())


def test_lists_that_cannot_be_stepped(P):
    z = lambda n=8, t=torch.float32: torch.zeros(n, dtype=t, device=DEV)  # noqa: E731
    with pytest.raises(TypeError, match="moments"):
        P.adamw_tensors([dict(w=z(), grad=z(), m=z(8, torch.bfloat16), v=z(8, torch.bfloat16))])
    with pytest.raises(ValueError, match="need m_exp"):
        P.adamw_tensors([dict(w=z(), grad=z(), m=z(8, torch.uint8), v=z(8, torch.uint8))])
    with pytest.raises(TypeError, match="m must be"):
        P.adamw_tensors([dict(w=z(), grad=z(), m=z(), v=z()), dict(w=z(), grad=z(), m=z(8, torch.uint8), v=z(8, torch.uint8))])
    with pytest.raises(TypeError, match="grad must be"):
        P.adamw_tensors([dict(w=z(), grad=z(), m=z(), v=z()), dict(w=z(), grad=z(8, torch.bfloat16), m=z(), v=z())])
    with pytest.raises(ValueError, match="shape"):
        P.adamw_tensors([dict(w=z(), grad=z(7), m=z(), v=z())])
    with pytest.raises(ValueError, match="none of"):
        P.adamw_tensors([dict(w=z(), grad=z(), m=z(), v=z(), decay=0.1)])
    with pytest.raises(ValueError, match="contiguous"):
        P.adamw_tensors([dict(w=z(16)[::2], grad=z(), m=z(), v=z())])
    a = dict(w=z(), grad=z(), m=z(), v=z())
    with pytest.raises(P.W2LError, match="overlap"):
        P.w2l_adamw_step(P.adamw_tensors([a, a]), 1, 1e-3)
    with pytest.raises(ValueError, match="one value"):
        P.w2l_adamw_step(P.adamw_tensors([a]), 1, 1e-3, lr_dev=z(2))
    with pytest.raises(P.W2LError, match="-5"):
        P.w2l_adamw_step(P.adamw_tensors([a]), 1, 1e-3, max_norm=1.0)
