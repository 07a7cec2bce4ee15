"""Host-only: what w2l_groupnorm_fwd / _bwd, w2l_policy_fwd_bwd and w2l_adamw_step refuse, before anything is launched, and what the binding refuses before
the library is called."""
import ctypes
import itertools

import pytest
import torch

import paper_1812_07625_amd as P

N = None
NAN, INF = float("nan"), float("inf")
BIG = 1 << 40


def places(names):
    """An address of its own for every operand, far from the others; never dereferenced."""
    return {n: 0x10000000000 * (i + 1) for i, n in enumerate(names)}


# ---- group norm
FWD = ("x", "gamma", "beta", "in_len", "y", "mean", "rstd", "ws")
BWD = ("x", "dy", "mean", "rstd", "gamma", "beta", "in_len", "dx", "dgamma", "dbeta", "ws")


def norm_fwd(B=2, T=40, C=24, G=4, eps=1e-5, act=3, dt=1, n=BIG, **kw):
    a = {**places(FWD), **kw}
    return P.raw.w2l_groupnorm_fwd(*[a[k] for k in FWD[:-1]], B, T, C, G, eps, act, dt, a["ws"], n, N)


def norm_bwd(B=2, T=40, C=24, G=4, act=3, dt=1, acc=0, n=BIG, **kw):
    a = {**places(BWD), **kw}
    return P.raw.w2l_groupnorm_bwd(*[a[k] for k in BWD[:-1]], B, T, C, G, act, dt, acc, a["ws"], n, N)


@pytest.mark.parametrize("kw", [dict(B=0), dict(T=0), dict(C=0), dict(G=0), dict(G=5), dict(G=-4), dict(C=8193, G=1, act=0), dict(C=27, G=27), dict(act=4), dict(act=-1),
                                dict(B=65535, T=1), dict(T=(1 << 24) + 1), dict(B=60000, T=60000), dict(B=1000, T=1 << 20, C=4096)], ids=str)
def test_norm_sizes(kw):
    assert norm_fwd(**kw) == -2 and norm_bwd(**kw) == -2
    shape = {**dict(B=2, T=40, C=24, G=4, act=3), **kw}
    assert P.w2l_groupnorm_workspace_bytes(shape["B"], shape["T"], shape["C"], shape["G"], shape["act"], 0) == 0


def test_norm_operands():
    for eps in (0.0, -1.0, NAN, INF):
        assert norm_fwd(eps=eps) == -2
    assert norm_fwd(dt=2) == -3 and norm_bwd(dt=2) == -3
    for k in ("x", "y", "mean", "rstd"):
        assert norm_fwd(**{k: N}) == -1, k
    for k in ("x", "dy", "mean", "rstd", "dx"):
        assert norm_bwd(**{k: N}) == -1, k
    for call, names in ((norm_fwd, FWD), (norm_bwd, BWD)):
        for k in names[:-1]:
            assert call(**{k: places(names)[k] + 4}) == -4, k
        need = P.w2l_groupnorm_workspace_bytes(2, 40, 24, 4, 3, 1)
        assert need > 0
        assert call(ws=N) == -5 and call(n=need - 1) == -5 and call(ws=places(names)["ws"] + 16) == -5


@pytest.mark.parametrize("call,names,inputs", [(norm_fwd, FWD, FWD[:4]), (norm_bwd, BWD, BWD[:7])], ids=["forward", "backward"])
def test_norm_outputs_on_other_operands(call, names, inputs):
    at = places(names)
    for o in names:
        if o not in inputs:
            for other in names:
                if other != o:
                    assert call(**{o: at[other]}) == -8, (o, other)


def test_norm_gradient_on_the_last_values_of_dy():
    assert norm_bwd(dx=places(BWD)["dy"] + 2 * 40 * 12 * 2 - 16) == -8


# ---- policy
POLICY = ("z", "tokens", "old", "ref", "adv", "w", "in_len", "frame", "loss", "lp", "dz", "ws")


def policy(B=2, T=3, C=100000, per=1, low=0.2, high=0.2, kl=0.1, gs=1.0, dt=1, gt=1, acc=0, n=BIG, **kw):
    a = {**places(POLICY), **kw}
    return P.raw.w2l_policy_fwd_bwd(a["z"], a["tokens"], a["old"], a["ref"], a["adv"], per, a["w"], a["in_len"], a["frame"], a["loss"], a["lp"], a["dz"], B, T, C, low,
                                    high, kl, gs, dt, gt, acc, a["ws"], n, N)


def test_policy_arguments():
    for kw in (dict(B=0), dict(T=0), dict(C=0), dict(C=262145), dict(B=65536, T=32768), dict(C=262144, B=8192, T=600), dict(low=-0.1), dict(low=1.1), dict(low=NAN),
               dict(high=-0.1), dict(high=NAN), dict(kl=-0.1), dict(kl=NAN), dict(kl=INF), dict(gs=NAN), dict(gs=INF)):
        assert policy(**kw) == -2, kw
    for k in ("z", "tokens", "old", "ref", "adv", "frame"):
        assert policy(**{k: N}) == -1, k
    assert policy(dt=2) == -3 and policy(gt=2) == -3 and policy(dt=0, gt=1) == -3
    for k in POLICY[:-1]:
        assert policy(**{k: places(POLICY)[k] + 4}) == -4, k
    need = P.w2l_policy_workspace_bytes(2, 3, 100000, 1)
    assert need > 0
    assert policy(ws=N) == -5 and policy(n=need - 1) == -5 and policy(ws=places(POLICY)["ws"] + 16) == -5


def test_policy_outputs_on_inputs():
    at = places(POLICY)
    for o, i in itertools.product(POLICY[7:], POLICY):
        if o != i:
            assert policy(**{o: at[i]}) == -8, (o, i)


# ---- AdamW
KEYS = ("w", "grad", "m", "v", "m_exp", "v_exp", "w_lowp")


def adamw(sizes=(100, 7), bits=8, gt=0, step=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, gs=1.0, clip=1.0, seed=1, lr_dev=N, step_dev=N, norm=N, ws=0x100, n=BIG, decay=0.0,
          count=None, change=lambda a: None):
    a = (P.w2l_adamw_tensor * max(1, len(sizes)))()
    for i, size in enumerate(sizes):
        for j, k in enumerate(KEYS):
            setattr(a[i], k, 0x10000000000 * (i * 8 + j + 1))
        a[i].n, a[i].weight_decay = size, decay
    change(a)
    return P.raw.w2l_adamw_step(a, len(sizes) if count is None else count, gt, bits, step, lr, b1, b2, eps, gs, clip, seed, lr_dev, step_dev, norm, ws, n, N)


def test_adamw_numbers():
    for kw in (dict(count=0), dict(count=-1), dict(count=65537), dict(sizes=(100, -1)), dict(sizes=((1 << 33) + 1,)), dict(step=0), dict(step=-5), dict(lr=-1.0), dict(lr=NAN),
               dict(lr=INF), dict(b1=-0.1), dict(b1=1.0), dict(b1=NAN), dict(b2=1.0), dict(b2=-1.0), dict(eps=0.0), dict(eps=1e-45), dict(eps=NAN), dict(gs=INF), dict(gs=NAN),
               dict(clip=-1.0), dict(clip=NAN), dict(clip=INF), dict(decay=-0.1), dict(decay=NAN), dict(decay=INF)):
        assert adamw(**kw) == -2, kw
    assert adamw(bits=16) == -3 and adamw(bits=0) == -3 and adamw(gt=2) == -3
    assert P.raw.w2l_adamw_step(N, 1, 0, 32, 1, 1e-3, 0.9, 0.999, 1e-8, 1.0, 0.0, 1, N, N, N, N, 0, N) == -1


def test_adamw_pointers():
    for k in ("w", "grad", "m", "v", "m_exp", "v_exp"):
        assert adamw(change=lambda a: setattr(a[1], k, N)) == -1, k
    for k in ("w", "grad", "m", "v", "w_lowp"):
        assert adamw(change=lambda a: setattr(a[1], k, getattr(a[1], k) + 4)) == -4, k
    assert adamw(lr_dev=0x302) == -4 and adamw(norm=0x301) == -4 and adamw(step_dev=0x303) == -4
    need = 256 + 256                                                       # scalars, and the sums of two workgroups
    assert adamw(ws=N) == -5 and adamw(n=need - 1) == -5 and adamw(ws=0x110) == -5
    assert adamw(clip=0.0, norm=0x9000, ws=N) == -5 and adamw(clip=0.0, lr_dev=0x9000, ws=N) == -5 and adamw(clip=0.0, step_dev=0x9000, ws=N) == -5


def test_adamw_tensors_on_one_another():
    for bits in (32, 8):
        for k, o in itertools.product(KEYS, KEYS):
            if bits == 32 and ("exp" in k or "exp" in o):
                continue
            if not k == o == "grad":                                       # gradients may be shared: they are read alone
                assert adamw(bits=bits, change=lambda a: setattr(a[1], k, getattr(a[0], o))) == -8, (bits, k, o)
            if k != o:
                assert adamw(bits=bits, change=lambda a: setattr(a[1], k, getattr(a[1], o))) == -8, (bits, k, o)
    assert adamw(change=lambda a: setattr(a[1], "grad", a[0].w + 384)) == -8     # its last values
    assert adamw(norm=0x10000000000) == -8 and adamw(lr_dev=0x10000000000) == -8 and adamw(ws=0x10000000000) == -8 and adamw(norm=0x100) == -8


def test_workspace_queries():
    a = (P.w2l_adamw_tensor * 2)()
    a[0].n, a[1].n = 0, 1 << 30
    assert P.raw.w2l_adamw_workspace_bytes(a, 2) == 256 + (257 * 8 + 255) // 256 * 256
    assert P.raw.w2l_adamw_workspace_bytes(a, 0) == 0 and P.raw.w2l_adamw_workspace_bytes(N, 1) == 0
    a[0].n = -1
    assert P.raw.w2l_adamw_workspace_bytes(a, 2) == 0
    assert P.w2l_policy_workspace_bytes(2, 3, 29, 0) == 0 and P.w2l_groupnorm_workspace_bytes(2, 3, 29, 1, 0, 2) == 0


def test_binding_takes_no_host_tensors():
    x, s, f = torch.zeros(1, 2, 4), torch.zeros(1, 2), torch.zeros(1, 2)
    with pytest.raises(ValueError, match="GPU"):
        P.w2l_groupnorm_fwd(x, x, s, s)
    with pytest.raises(ValueError, match="GPU"):
        P.w2l_groupnorm_bwd(x, x, s, s, x)
    with pytest.raises(ValueError, match=r"\[B, T, C\]"):
        P.w2l_groupnorm_fwd(x[0], x, s, s)
    with pytest.raises(ValueError, match="GPU"):
        P.w2l_policy_fwd_bwd(x, f.int(), f, f, f)
    with pytest.raises(ValueError, match="no tensors"):
        P.adamw_tensors([])
    with pytest.raises(ValueError, match="GPU"):
        P.adamw_tensors([dict(w=s, grad=s, m=s, v=s)])


def test_the_structure_is_the_headers():
    assert ctypes.sizeof(P.w2l_adamw_tensor) == 72
