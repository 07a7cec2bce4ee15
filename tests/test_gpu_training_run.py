"""The operators of a training step together, as a program runs them: convolution, group norm with GLU, a class layer, the clipped policy loss, the backward passes, and an
AdamW step over all tensors with their norm clipped -- against the same chain of fp64 oracles, and captured into a graph.

Every tensor is held to the relative L2 of the repository's whole train steps (fp32 1e-4, bf16 2e-2, the weights' change in bf16 5e-2: an early Adam step divides
each gradient by its own size, so that a change carries the relative error of the single gradients)."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from gpu_util import DEV, to_dev, to_host

pytestmark = pytest.mark.gpu
B, T, FEAT, H, C, K, G = 3, 90, 40, 64, 29, 5, 8
LENGTHS = np.array([90, 61, 17], np.int32)
LR, B1, B2, EPS, CLIP, DECAY = 1e-2, 0.9, 0.99, 1e-3, 0.3, 0.01


@pytest.fixture(scope="module")
def P():
    import paper_1812_07625_amd as P
    return P


def inputs(bf16):
    rng = np.random.default_rng(31)
    low = W.round_to_bf16 if bf16 else lambda a: a
    f = lambda a: a.astype(np.float32)  # noqa: E731
    p = dict(w1=low(f(rng.standard_normal((2 * H, K, FEAT)) / np.sqrt(K * FEAT))), b1=f(0.1 * rng.standard_normal(2 * H)), gamma=f(1 + 0.1 * rng.standard_normal(2 * H)),
             beta=f(0.1 * rng.standard_normal(2 * H)), w2=low(f(rng.standard_normal((C, 1, H)) / np.sqrt(H))), b2=f(0.1 * rng.standard_normal(C)))
    x = low(f(rng.standard_normal((B, T, FEAT))))
    x[np.arange(T)[None] >= LENGTHS[:, None]] = 0
    return p, x, rng.integers(0, C, (B, T)).astype(np.int32), f(rng.standard_normal(B)), rng


class Program:
    """One training step on the GPU: what a program keeps, and the calls."""

    def __init__(self, P, p, x, tokens, A, old, ref, bf16, bits):
        self.P, td = P, torch.bfloat16 if bf16 else torch.float32
        self.code = P.W2L_BF16 if bf16 else P.W2L_F32
        e = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device=DEV)  # noqa: E731
        self.master = {k: to_dev(v) for k, v in p.items()}
        self.low = {k: self.master[k].to(td) for k in ("w1", "w2")} if bf16 else self.master
        self.x, self.tokens, self.A, self.old, self.ref, self.n = to_dev(x).to(td), to_dev(tokens), to_dev(A), to_dev(old), to_dev(ref), to_dev(LENGTHS)
        self.y, self.h, self.z = e(B, T, 2 * H, dtype=td), e(B, T, H, dtype=td), e(B, T, C)
        self.mean, self.rstd = e(B, G), e(B, G)
        self.frame, self.loss, self.dz = e(B, T), e(B), e(B, T, C)
        self.dh, self.dy = e(B, T, H, dtype=td), e(B, T, 2 * H, dtype=td)
        self.grads = {k: e(*v.shape) for k, v in self.master.items()}
        self.norm, self.lr, self.step = e(1), torch.full((1,), LR, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        rows = []
        for k, w in self.master.items():
            n = w.numel()
            m = {a: e(*w.shape) if bits == 32 else e(*w.shape, dtype=torch.uint8) for a in "mv"}
            if bits == 8:
                m |= {a: e((n + 255) // 256, dtype=torch.int8) for a in ("m_exp", "v_exp")}
            rows.append(dict(w=w, grad=self.grads[k], w_lowp=self.low[k] if bf16 and k in self.low else None, weight_decay=DECAY if k[0] == "w" else 0.0, **m))
        self.tensors = P.adamw_tensors(rows)
        sizes = [P.w2l_groupnorm_workspace_bytes(B, T, 2 * H, G, P.W2L_ACT_GLU, self.code), P.w2l_policy_workspace_bytes(B, T, C, P.W2L_F32),
                 P.w2l_adamw_workspace_bytes(self.tensors), P.w2l_conv1d_fwd_workspace_bytes(B, T, FEAT, 2 * H, K, 1, self.code),
                 P.w2l_conv1d_fwd_workspace_bytes(B, T, H, C, 1, 1, self.code), P.w2l_conv1d_bwd_data_workspace_bytes(B, T, H, C, 1, 1, self.code),
                 P.w2l_conv1d_bwd_weight_workspace_bytes(B, T, H, C, 1, 1, self.code), P.w2l_conv1d_bwd_weight_workspace_bytes(B, T, FEAT, 2 * H, K, 1, self.code)]
        self.ws = P.workspace(max(sizes))                                  # one for all: the calls follow one another on a stream

    def __call__(self):
        P, m, low, ws, g = self.P, self.master, self.low, self.ws, self.grads
        act = P.W2L_ACT_GLU
        P.w2l_conv1d_fwd(self.x, low["w1"], m["b1"], self.y, workspace=ws)
        P.w2l_groupnorm_fwd(self.y, self.h, self.mean, self.rstd, m["gamma"], m["beta"], in_len=self.n, act=act, workspace=ws)
        P.w2l_conv1d_fwd(self.h, low["w2"], m["b2"], self.z, workspace=ws)
        P.w2l_policy_fwd_bwd(self.z, self.tokens, self.old, self.A, self.frame, self.loss, self.dz, ref_logprob=self.ref, in_len=self.n, kl_coef=0.1, workspace=ws)
        P.w2l_conv1d_bwd_weight(self.h, self.dz, g["w2"], g["b2"], workspace=ws)
        P.w2l_conv1d_bwd_data(self.dz, low["w2"], self.dh, workspace=ws)
        P.w2l_groupnorm_bwd(self.y, self.dh, self.mean, self.rstd, self.dy, m["gamma"], m["beta"], g["gamma"], g["beta"], in_len=self.n, act=act, workspace=ws)
        P.w2l_conv1d_bwd_weight(self.x, self.dy, g["w1"], g["b1"], workspace=ws)
        self.step.add_(1)
        P.w2l_adamw_step(self.tensors, 1, LR, B1, B2, EPS, max_norm=CLIP, grad_norm=self.norm, lr_dev=self.lr, step_dev=self.step, seed=3, workspace=ws)


def scores(p, x):
    d = {k: v.astype(np.float64) for k, v in p.items()}
    y = oracle.conv1d_fwd(x.astype(np.float64), d["w1"], d["b1"])
    h = oracle.groupnorm(y, G, d["gamma"], d["beta"], LENGTHS, 1e-5, "glu")["y"]
    return y, h, oracle.conv1d_fwd(h, d["w2"], d["b2"])


def by_oracle(p, x, tokens, A, old, ref):
    d = {k: v.astype(np.float64) for k, v in p.items()}
    y, h, z = scores(p, x)
    frame, loss, _, dz, _ = oracle.policy(z, tokens, old, A, ref, None, LENGTHS, 0.2, 0.2, 0.1, 1.0)
    g = {}
    g["w2"], g["b2"] = oracle.conv1d_bwd_weight(h, dz, 1)
    dh = oracle.conv1d_bwd_data(dz, d["w2"], T)
    o = oracle.groupnorm(y, G, d["gamma"], d["beta"], LENGTHS, 1e-5, "glu", dh)
    g["gamma"], g["beta"] = o["dgamma"], o["dbeta"]
    g["w1"], g["b1"] = oracle.conv1d_bwd_weight(x.astype(np.float64), o["dx"], K)
    f = oracle.adamw_factor(g.values(), 1.0, CLIP)
    new = {k: oracle.adamw(d[k], g[k], 0 * d[k], 0 * d[k], f, 1, LR, B1, B2, EPS, DECAY if k[0] == "w" else 0.0)[0] for k in d}
    return loss, g, oracle.adamw_norm(g.values()), new


def rel(a, b):
    return np.linalg.norm((a - b).ravel()) / np.linalg.norm(np.asarray(b).ravel())


def problem(bf16):
    p, x, tokens, A, rng = inputs(bf16)
    lp = np.take_along_axis(oracle._log_probs(scores(p, x)[2])[0], tokens[..., None], 2)[..., 0]
    gap = 0.1 * rng.standard_normal((B, T)).clip(-1.4, 1.4)                # ratios well inside the clip, or well outside it
    gap[:, ::5] = np.where(rng.random((B, T)) < 0.5, 0.5, -0.5)[:, ::5]
    return p, x, tokens, A, (lp - gap).astype(np.float32), (lp + 0.2 * rng.standard_normal((B, T))).astype(np.float32)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
def test_a_training_step(P, bf16, bits):
    args = problem(bf16)
    prog = Program(P, *args, bf16, bits)
    start = {k: to_host(v) for k, v in prog.master.items()}
    prog()
    torch.cuda.synchronize()
    loss, g, norm, new = by_oracle(*args)
    most = 2e-2 if bf16 else 1e-4
    assert norm > CLIP                                                     # the clip does something
    assert abs(float(prog.norm) - norm) <= most * norm and rel(to_host(prog.loss), loss) <= most
    for k in g:
        assert rel(to_host(prog.grads[k]), g[k]) <= most, k
        assert rel(to_host(prog.master[k]) - start[k], new[k] - start[k]) <= (5e-2 if bf16 else 1e-3), k
        if bf16 and k in prog.low:
            assert torch.equal(prog.low[k], prog.master[k].bfloat16())


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_of_a_captured_graph(P, bits):
    args = problem(False)
    a, b = Program(P, *args, False, bits), Program(P, *args, False, bits)
    a()
    b()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a()
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        b()
        torch.cuda.synchronize()
        assert int(a.step) == int(b.step) == k + 2
        for key in a.master:
            assert torch.equal(a.master[key], b.master[key]), (k, key)
        assert torch.equal(a.loss, b.loss) and torch.equal(a.norm, b.norm)
    assert float(a.loss.sum()) == float(a.loss.sum()) and not torch.equal(a.master["w1"], to_dev(args[0]["w1"]))
