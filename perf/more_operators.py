"""What a deeper network is trained with besides convolutions and their criteria, as cases that can be timed and compared.

Three operators, in the order in which a training step reaches them:

  norm     group norm over a channels-last tensor x [B,T,C] of which utterance b has in_len[b] frames, and the activation
           after it: none, ReLU, SiLU or GLU (w2l_groupnorm_fwd);  "norm train": its gradient as well
           (w2l_groupnorm_fwd, then w2l_groupnorm_bwd).
  policy   clipped policy loss of sampled tokens with a KL term against a reference network, from per-frame scores
           z [B,T,C] to their gradient (w2l_policy_fwd_bwd): a network that is rewarded for what it transcribes.
  adamw    AdamW over all of a network's tensors at once, with clipping by their gradients' norm; moments in 32 bits, or in 8 bits
           with an exponent for every 256 of them, rounded at random (w2l_adamw_step).

Moments in 8 bits are e4m3 values; they are returned as these, beside their blocks' exponents.
"""
import math

import torch

DEV = "cuda:0"
own = False


# ------------------------------------------------------------------------------------ the cases
def _norm(name, B, T, lo, C, G, act, dtype, train):
    return dict(name=name, kind="norm", B=B, T=T, lo=lo, C=C, G=G, act=act, dtype=dtype, train=train)


def _policy(name, B, T, lo, C, dtype, kl):
    return dict(name=name, kind="policy", B=B, T=T, lo=lo, C=C, dtype=dtype, kl=kl)


def _adamw(name, feat, half, k, body, top, bits, clip):
    return dict(name=name, kind="adamw", feat=feat, half=half, k=k, body=body, top=top, bits=bits, clip=clip)


def listed():
    return [
        # a few frames of the tiny network's layers, fp32: latency alone
        _norm("norm 1x16x128 fp32 relu", 1, 16, 16, 128, 8, "relu", "fp32", False),
        # between the body layers of the 105M-parameter network: its gated linear unit behind a norm
        _norm("norm 8x750x1536 bf16 glu", 8, 750, 500, 1536, 32, "glu", "bf16", False),
        # the same in training
        _norm("norm train 8x750x1536 bf16 glu", 8, 750, 500, 1536, 32, "glu", "bf16", True),
        # a width and groups that no vector divides, a ragged batch
        _norm("norm train 5x333x500 fp32 silu", 5, 333, 20, 500, 20, "silu", "fp32", True),
        # the widest layers before the first stride, one group: statistics over whole utterances
        _norm("norm train 16x1500x2048 bf16 silu", 16, 1500, 1000, 2048, 1, "silu", "bf16", True),
        # one short utterance of a grapheme network: latency
        _policy("policy 1x40, 29 fp32", 1, 40, 40, 29, "fp32", 0.0),
        # the criterion's batch of this repository's benchmark
        _policy("policy 32x750, 29 fp32", 32, 750, 600, 29, "fp32", 0.05),
        # word pieces, rows that are never 16-byte aligned
        _policy("policy 8x375, 10001 bf16", 8, 375, 300, 10001, "bf16", 0.05),
        # a large inventory
        _policy("policy 4x750, 32000 bf16", 4, 750, 700, 32000, "bf16", 0.1),
        # the tiny network's six tensors: latency of a step
        _adamw("adamw tiny, 32 bits", 40, 64, 5, 1, 0, 32, 0.0),
        # the 105M-parameter network, clipped, with moments of either kind
        _adamw("adamw 105M, 32 bits", 80, 768, 11, 8, 1024, 32, 1.0),
        _adamw("adamw 105M, 8 bits", 80, 768, 11, 8, 1024, 8, 1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "policy", "adamw"))
    if kind == "norm":
        train = rng.random() < 0.6
        # (a rectifier's gradient jumps at 0, and of millions of values some are within fp32's reach of it: forward alone)
        act = rng.choice(("none", "silu", "glu") if train else ("none", "relu", "silu", "glu"))
        G = rng.choice((1, 2, 4, 7, 16, 32))
        C = 2 * G * max(1, _log(rng, 16, 2048) // (2 * G))
        rows = _log(rng, 1, min(24000, (1 << 25) // C))
        least = -(-64 * G // C)             # frames: a group of a few values is its own mean and deviation, and its gradient nothing but roundings
        B = min(max(1, rows // least), _log(rng, 1, 64))
        T = max(least, rows // B)
        return dict(kind=kind, B=B, T=T, lo=rng.randint(max(least, T // 3), T), C=C, G=G, act=act, dtype=rng.choice(("fp32", "bf16")), train=train)
    if kind == "policy":
        C = _log(rng, 2, 130000)
        rows = _log(rng, 1, min(24000, (1 << 26) // C))
        B = min(rows, _log(rng, 1, 64))
        T = max(1, rows // B)
        return dict(kind=kind, B=B, T=T, lo=rng.randint(max(1, T // 2), T), C=C, dtype=rng.choice(("fp32", "bf16")), kl=rng.choice((0.0, 0.02, 0.1)))
    half = _log(rng, 4, 700)
    return dict(kind=kind, feat=rng.choice((1, 39, 40, 80)), half=half, k=rng.choice((1, 3, 5, 11)), body=rng.randint(0, 8), top=rng.choice((0, 1)) * _log(rng, 8, 1024),
                bits=rng.choice((32, 8)), clip=rng.choice((0.0, 1.0, 100.0)))


def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def _lengths(c):
    """in_len of the batch: sorted by length, from T down to lo."""
    return [c["T"] - (c["T"] - c["lo"]) * b // max(1, c["B"] - 1) for b in range(c["B"])]


def _tensors(c):
    """Values of every tensor of a gated network, weights and bias in turn: a first layer over features, body layers, a wide 1x1 layer, classes."""
    half, k = c["half"], c["k"]
    layers = [((k + 2 if c["top"] else k) * c["feat"], 2 * half)] + [(k * half, 2 * half)] * c["body"]
    if c["top"]:
        layers += [(half, 2 * c["top"])]
    layers += [(c["top"] or half, 29)]
    return [n for fan, out in layers for n in (fan * out, out)]


def work(case):
    if case["kind"] == "norm":
        values, e = sum(_lengths(case)) * case["C"], _size(case)
        out = values // 2 if case["act"] == "glu" else values
        if case["train"]:                # x in, y out; dy in, dx out
            return {"bytes": e * 2 * (values + out), "flops": 30.0 * values}
        return {"bytes": e * (values + out), "flops": 10.0 * values}
    if case["kind"] == "policy":         # scores in, their gradient out
        rows, C = sum(_lengths(case)), case["C"]
        return {"bytes": rows * (2 * C * _size(case) + 24), "flops": 8.0 * rows * C}
    n = sum(_tensors(case))              # gradients in, weights and both moments in and out, a bf16 copy of the weights out
    return {"bytes": n * (4 + 8 + (16 if case["bits"] == 32 else 4) + 2), "flops": 20.0 * n}


# ------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"norm": _norm_inputs, "policy": _policy_inputs, "adamw": _adamw_inputs}[case["kind"]](case, g)
    s["kind"], s["case"] = case["kind"], case
    return s


def _norm_inputs(c, g):
    B, T, C = c["B"], c["T"], c["C"]
    td = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    # a convolution's output: channels of different levels and sizes; frames beyond an utterance hold what its kernel reaches there
    s = {"x": (randn(B, T, C) * (0.5 + randn(C).abs()) + randn(C)).to(td), "gamma": 1 + 0.2 * randn(C), "beta": 0.2 * randn(C)}
    s["in_len"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    if c["train"]:
        s["dy"] = randn(B, T, C // 2 if c["act"] == "glu" else C).to(td)
    return s


def _policy_inputs(c, g):
    B, T, C = c["B"], c["T"], c["C"]
    td = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    rand = lambda *shape: torch.rand(shape, generator=g, device=DEV)  # noqa: E731
    # scores as trained networks give them: one class well above the others in most frames
    z = randn(B, T, C) * 2.0
    peak = torch.randint(0, C, (B, T, 1), generator=g, device=DEV)
    z.scatter_add_(2, peak, rand(B, T, 1) * 8.0)
    s = {"z": z.to(td)}
    # sampled labels: mostly the likely class; frames that the sample leaves out have none
    tokens = torch.where(rand(B, T, 1) < 0.8, peak, torch.randint(0, C, (B, T, 1), generator=g, device=DEV))
    x = s["z"].double()
    lp = (x.gather(2, tokens) - torch.logsumexp(x, 2, True))[..., 0]
    del x
    s["tokens"] = torch.where(rand(B, T) < 0.05, -1, tokens[..., 0]).int()
    # the network that sampled, some steps ago, and the one that training started from
    old = (lp - 0.15 * randn(B, T)).float()
    ratio = (lp - old.double()).exp()
    # which side of a border fp32 puts a frame on is chance within a few 1e-7 of it: none of them is that close
    near = ((ratio - 1.3).abs() < 1e-4) | ((ratio - 0.8).abs() < 1e-4)
    s["old"] = torch.where(near, old + 1e-3, old)
    s["ref"] = (lp - 0.5 * randn(B, T)).float() if c["kl"] else None
    s["advantage"] = randn(B)                # of an utterance's sample over others of the same utterance
    s["weight"] = rand(B, T) * 0.5 + 0.5
    s["in_len"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    return s


_LOW, _HIGH, _SCALE = 0.2, 0.3, 0.25         # the clip's range below and above 1; grad_scale
_LR, _B1, _B2, _EPS, _DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def _adamw_inputs(c, g):
    sizes = _tensors(c)
    room = [(n + 255) // 256 * 256 for n in sizes]     # all tensors in one buffer, each from a multiple of 256 on
    total = sum(room)
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    which = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), torch.tensor(room, device=DEV))
    start = torch.tensor([sum(room[:i]) for i in range(len(room))], device=DEV)
    place = torch.arange(total, device=DEV) - start[which]
    live = place < torch.tensor(sizes, device=DEV)[which]
    # gradients and moments in the middle of training: sizes that differ from filter to filter and tensor to tensor
    level = (1e-3 * randn(total // 256).mul(1.5).exp()).repeat_interleave(256)
    s = {"w": 0.05 * randn(total), "grad": level * randn(total), "sizes": sizes, "room": room, "step": 1000, "seed": 12345}
    m, v = 0.3 * level * randn(total), (level * (0.5 + randn(total).abs())).square()
    s["decay"] = [_DECAY, 0.0] * (len(sizes) // 2)     # weights decay, biases do not
    for k in ("w", "grad"):
        s[k].mul_(live)
    m.mul_(live)
    v.mul_(live)
    s["lowp"] = s["w"].bfloat16()
    if c["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_exp"] = _to_e4m3(m)
        s["v"], s["v_exp"] = _to_e4m3(v.sqrt(), keep=True)
    s["which"], s["place"] = which.int(), place.int()
    return s


# ------------------------------------------------------------------------------------ moments in 8 bits
# A block of 256 values has an exponent E, the least (but at least -100) with which the block's largest magnitude is at most 448 * 2^E, and
# a value is an e4m3 number times 2^E.  e4m3 numbers are multiples of 2^-9: below 2^-6 all of them, above those of four significant bits.
def _two_to(e):
    return ((e.int() + 127) << 23).view(torch.float32)


def _to_e4m3(x, dither=None, keep=False):
    """x [n * 256] rounded at random (dither: a whole number below 2^16 for every value; None: to the nearest) -> e4m3 values, exponents.
    keep: what is no zero does not become one."""
    a = x.abs().view(-1, 256)
    most = a.amax(1, keepdim=True).view(torch.int32)
    E = ((most >> 23) - 135 + ((most & 0x7FFFFF) > 0x600000)).clamp(min=-100)      # 448 = 1.75 * 2^8
    E = torch.where(most > 0, E, 0)
    u = (a * _two_to(9 - E)).view(-1)                     # in units of 2^-9: up to 14 * 2^14
    r = torch.full_like(u, 32768, dtype=torch.int32) if dither is None else dither
    small = (u + r.float() / 65536).int()
    large = ((u.view(torch.int32) + (r << 4)) >> 20) - 1032
    code = torch.where(u < 8, small, large).clamp(max=126)
    if keep:
        code = torch.where(u > 0, code.clamp(min=1), code)
    code = torch.where(x < 0, code | 128, code)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), E.view(-1).to(torch.int8)


def _from_e4m3(q, E):
    return (q.float().view(-1, 256) * _two_to(E)[:, None]).view(-1)


def _mix(x):
    """A whole number below 2^32 to another: the finaliser of MurmurHash3 (Appleby 2008)."""
    x = x ^ (x >> 16)
    x = x * 0x85EBCA6B & 0xFFFFFFFF
    x = x ^ (x >> 13)
    x = x * 0xC2B2AE35 & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(seed, step, tensor):
    """What a tensor's random bits of a step come from."""
    return _mix(_mix(_mix(seed & 0xFFFFFFFF) ^ (step & 0xFFFFFFFF)) ^ tensor)


# ------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return {"norm": _own_norm, "policy": _own_policy, "adamw": _own_adamw}[state["kind"]](state)
    return {"norm": _plain_norm, "policy": _plain_policy, "adamw": _plain_adamw}[state["kind"]](state)


def _plain_norm(s):
    c = s["case"]
    B, T, C, G, act = c["B"], c["T"], c["C"], c["G"], c["act"]
    live = (torch.arange(T, device=DEV) < s["in_len"][:, None])[..., None]
    there = live[..., None]
    x = torch.where(live, s["x"].float(), 0.0).view(B, T, G, C // G)
    n = (s["in_len"] * (C // G)).float()[:, None]
    mean = x.sum((1, 3)) / n
    d = torch.where(there, x - mean[:, None, :, None], 0.0)
    rstd = (d.square().sum((1, 3)) / n + 1e-5).rsqrt()
    hat = (d * rstd[:, None, :, None]).view(B, T, C)
    u = hat * s["gamma"] + s["beta"]
    if act == "glu":
        a, gate = u[..., :C // 2], torch.sigmoid(u[..., C // 2:])
        y = a * gate
    elif act == "silu":
        gate = torch.sigmoid(u)
        y = u * gate
    else:
        y = u.clamp(min=0) if act == "relu" else u
    out = {"y": torch.where(live, y, 0.0).to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if c["train"]:
        dy = torch.where(live, s["dy"].float(), 0.0)
        if act == "glu":
            du = torch.cat((dy * gate, dy * a * gate * (1 - gate)), 2)
        elif act == "silu":
            du = dy * gate * (1 + u * (1 - gate))
        else:
            du = torch.where(u > 0, dy, 0.0) if act == "relu" else dy
        out["dbeta"], out["dgamma"] = du.sum((0, 1)), (du * hat).sum((0, 1))
        dh, hat = (du * s["gamma"]).view(B, T, G, C // G), hat.view(B, T, G, C // G)
        m1, m2 = dh.sum((1, 3)) / n, (dh * hat).sum((1, 3)) / n
        dx = (dh - m1[:, None, :, None] - hat * m2[:, None, :, None]) * rstd[:, None, :, None]
        out["dx"] = torch.where(there, dx, 0.0).view(B, T, C).to(s["x"].dtype)
    return out


def _plain_policy(s):
    c = s["case"]
    live = torch.arange(c["T"], device=DEV) < s["in_len"][:, None]
    tokens = s["tokens"].long()
    there = live & (tokens >= 0)
    ids = tokens.clamp(min=0)[..., None]
    x = s["z"].float()
    d = x - x.amax(-1, keepdim=True)
    e = d.exp()
    total = e.sum(-1, keepdim=True)
    lp = (d.gather(2, ids) - total.log())[..., 0]
    A = s["advantage"][:, None]
    ratio = (lp - s["old"]).exp()
    clipped = ratio.clamp(1 - _LOW, 1 + _HIGH)
    loss = -torch.minimum(ratio * A, clipped * A)
    dlp = torch.where(ratio * A <= clipped * A, -A * ratio, 0.0)
    if c["kl"]:
        gap = (s["ref"] - lp).double()                    # exp(gap) - gap - 1 vanishes with its square
        loss = loss + c["kl"] * (torch.expm1(gap) - gap).float()
        dlp = dlp - c["kl"] * torch.expm1(gap).float()
    frame = torch.where(there, s["weight"] * loss, 0.0)
    f = torch.where(there, s["weight"] * dlp * _SCALE, 0.0)[..., None]
    dz = (-f * (e / total)).scatter_add_(2, ids, f)
    return {"frame_loss": frame, "loss": frame.double().sum(1).float(), "logprob": torch.where(there, lp, 0.0), "dz": dz.to(s["z"].dtype)}


def _plain_adamw(s):
    c, step = s["case"], s["step"]
    s["step"] = step + 1
    grad = s["grad"]
    if c["clip"]:
        norm = grad.double().square().sum().sqrt()
        grad = grad * (c["clip"] / (norm + 1e-6)).clamp(max=1.0).float()
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, v = _from_e4m3(s["m"], s["m_exp"]), _from_e4m3(s["v"], s["v_exp"]).square()
    m = m * _B1 + grad * (1 - _B1)
    v = v * _B2 + (grad * grad) * (1 - _B2)
    root = v.sqrt()
    decay = torch.tensor([1 - _LR * d for d in s["decay"]], device=DEV)[s["which"]]
    w = s["w"] * decay - (_LR / (1 - _B1 ** step)) * m / (root / math.sqrt(1 - _B2 ** step) + _EPS)
    s["w"], s["lowp"] = w, w.bfloat16()
    out = {"w": w, "lowp": s["lowp"]}
    if c["clip"]:
        out["norm"] = norm.float()
    if c["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        keys = torch.tensor([_key(s["seed"], step, t) for t in range(len(s["sizes"]))], device=DEV)[s["which"]]
        h = _mix(((s["place"].long() >> 1) * 0x9E3779B1 + keys) & 0xFFFFFFFF)
        dither = torch.where(s["place"] % 2 == 0, h & 0xFFFF, h >> 16).int()
        s["m"], s["m_exp"] = _to_e4m3(m, dither)
        s["v"], s["v_exp"] = _to_e4m3(root, dither, keep=True)   # the root is what is kept, and stays above 0
        out |= {"m_exp": s["m_exp"], "v_exp": s["v_exp"]}
    return out | {"m": s["m"], "v": s["v"]}


def _own_norm(s):
    import paper_1812_07625_amd as P

    x, c = s["x"], s["case"]
    B, T, C = x.shape
    o = s.get("out")
    if o is None:  # outputs and workspace, which a program keeps from call to call
        f = lambda *shape: torch.empty(shape, device=DEV)  # noqa: E731
        s["act"] = {"none": P.W2L_ACT_NONE, "relu": P.W2L_ACT_RELU, "silu": P.W2L_ACT_SILU, "glu": P.W2L_ACT_GLU}[c["act"]]
        code = P.W2L_BF16 if x.dtype == torch.bfloat16 else P.W2L_F32
        o = {"y": torch.empty((B, T, C // 2 if c["act"] == "glu" else C), dtype=x.dtype, device=DEV), "mean": f(B, c["G"]), "rstd": f(B, c["G"])}
        s["ws"] = P.workspace(P.w2l_groupnorm_workspace_bytes(B, T, C, c["G"], s["act"], code))
        if c["train"]:
            o |= {"dx": torch.empty_like(x), "dgamma": f(C), "dbeta": f(C)}
        s["out"] = o
    P.w2l_groupnorm_fwd(x, o["y"], o["mean"], o["rstd"], s["gamma"], s["beta"], in_len=s["in_len"], eps=1e-5, act=s["act"], workspace=s["ws"])
    if c["train"]:
        P.w2l_groupnorm_bwd(x, s["dy"], o["mean"], o["rstd"], o["dx"], s["gamma"], s["beta"], o["dgamma"], o["dbeta"], in_len=s["in_len"], act=s["act"],
                            workspace=s["ws"])
    return o


def _own_policy(s):
    import paper_1812_07625_amd as P

    z, c = s["z"], s["case"]
    B, T, C = z.shape
    o = s.get("out")
    if o is None:
        f = lambda *shape: torch.empty(shape, device=DEV)  # noqa: E731
        o = s["out"] = {"frame_loss": f(B, T), "loss": f(B), "logprob": f(B, T), "dz": torch.empty_like(z)}
        s["ws"] = P.workspace(P.w2l_policy_workspace_bytes(B, T, C, P.W2L_BF16 if z.dtype == torch.bfloat16 else P.W2L_F32))
    P.w2l_policy_fwd_bwd(z, s["tokens"], s["old"], s["advantage"], o["frame_loss"], o["loss"], o["dz"], o["logprob"], ref_logprob=s["ref"], weight=s["weight"],
                         in_len=s["in_len"], clip_low=_LOW, clip_high=_HIGH, kl_coef=c["kl"], grad_scale=_SCALE, workspace=s["ws"])
    return o


def _own_adamw(s):
    import paper_1812_07625_amd as P

    c = s["case"]
    if "tensors" not in s:
        at, rows = 0, []
        for n, room, decay in zip(s["sizes"], s["room"], s["decay"]):
            part = lambda k: s[k][at:at + n]  # noqa: E731
            exps = lambda k: s[k][at // 256:(at + room) // 256] if c["bits"] == 8 else None  # noqa: E731
            rows.append(dict(w=part("w"), grad=part("grad"), m=part("m"), v=part("v"), m_exp=exps("m_exp"), v_exp=exps("v_exp"), w_lowp=part("lowp"), weight_decay=decay))
            at += room
        s["tensors"] = P.adamw_tensors(rows)
        s["norm"] = torch.empty((), device=DEV) if c["clip"] else None
        s["ws"] = P.workspace(P.w2l_adamw_workspace_bytes(s["tensors"]))
    P.w2l_adamw_step(s["tensors"], s["step"], lr=_LR, beta1=_B1, beta2=_B2, eps=_EPS, max_norm=c["clip"], seed=s["seed"], grad_norm=s["norm"], workspace=s["ws"])
    s["step"] += 1
    out = {"w": s["w"], "lowp": s["lowp"], "m": s["m"], "v": s["v"]}
    if c["clip"]:
        out["norm"] = s["norm"]
    if c["bits"] == 8:
        out |= {"m_exp": s["m_exp"], "v_exp": s["v_exp"]}
    return out


# ------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "policy": _exact_policy, "adamw": _exact_adamw}[case["kind"]](case, s)


def _exact_norm(c, s):
    B, C, G, act = c["B"], c["C"], c["G"], c["act"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    out = {"y": [], "mean": [], "rstd": []}
    if c["train"]:
        out |= {"dx": [], "dgamma": torch.zeros(C, dtype=torch.float64, device=DEV), "dbeta": torch.zeros(C, dtype=torch.float64, device=DEV)}
    for b, n in enumerate(_lengths(c)):
        pad = lambda t: torch.cat((t, t.new_zeros((c["T"] - n, t.shape[1]))))  # noqa: E731
        x = s["x"][b, :n].double().view(n, G, C // G)
        var, mean = torch.var_mean(x, (0, 2), correction=0)
        rstd = 1 / (var + 1e-5).sqrt()
        hat = ((x - mean[:, None]) * rstd[:, None]).view(n, C)
        u = gamma * hat + beta
        if act == "glu":
            a, sig = u[:, :C // 2], 1 / (1 + (-u[:, C // 2:]).exp())
            y = a * sig
        else:
            sig = 1 / (1 + (-u).exp())
            y = {"none": u, "relu": torch.where(u > 0, u, 0), "silu": u * sig}[act]
        out["y"].append(pad(y))
        out["mean"].append(mean)
        out["rstd"].append(rstd)
        if c["train"]:
            dy = s["dy"][b, :n].double()
            if act == "glu":
                du = torch.cat((dy * sig, dy * a * (sig - sig * sig)), 1)
            else:
                du = dy * {"none": 1, "relu": (u > 0).double(), "silu": sig + u * (sig - sig * sig)}[act]
            out["dgamma"] += (du * hat).sum(0)
            out["dbeta"] += du.sum(0)
            dh, h = (du * gamma).view(n, G, C // G), hat.view(n, G, C // G)
            out["dx"].append(pad(((dh - dh.mean((0, 2), True) - h * (dh * h).mean((0, 2), True)) * rstd[:, None]).reshape(n, C)))
    return {k: torch.stack(v) if isinstance(v, list) else v for k, v in out.items()}


def _exact_policy(c, s):
    none = (s["tokens"] < 0) | (torch.arange(c["T"], device=DEV) >= s["in_len"][:, None])
    tok = s["tokens"].long().masked_fill(none, 0)[..., None]
    logp = torch.log_softmax(s["z"].double(), 2)
    lp = logp.gather(2, tok)[..., 0]
    A, w = s["advantage"].double()[:, None], s["weight"].double().masked_fill(none, 0)
    r = (lp - s["old"].double()).exp()
    # min(r A, clip(r) A): for A > 0 the clip binds above, for A < 0 below
    held = torch.where(A > 0, r > 1 + _HIGH, r < 1 - _LOW)
    loss = -A * torch.where(held, torch.where(A > 0, 1 + _HIGH, 1 - _LOW), r)
    dlp = (-A * r).masked_fill(held, 0)
    if c["kl"]:
        q = (s["ref"].double() - lp).exp()
        loss = loss + c["kl"] * (q - 1 - q.log())
        dlp = dlp + c["kl"] * (1 - q)
    f = (w * dlp * _SCALE)[..., None]
    dz = logp.exp_().mul_(-f).scatter_add_(2, tok, f)
    frame = (w * loss).masked_fill(none, 0)
    return {"frame_loss": frame, "loss": frame.sum(1), "logprob": lp.masked_fill(none, 0), "dz": dz}


def _exact_adamw(c, s):
    value = lambda q, E: q.double() * torch.exp2(E.double()).repeat_interleave(256)  # noqa: E731
    grad = s["grad"].double()
    norm = torch.linalg.vector_norm(grad)
    if c["clip"]:
        grad = grad * min(1.0, c["clip"] / (float(norm) + 1e-6))
    m = s["m"].double() if c["bits"] == 32 else value(s["m"], s["m_exp"])
    v = s["v"].double() if c["bits"] == 32 else value(s["v"], s["v_exp"]) ** 2
    m = _B1 * m + (1 - _B1) * grad
    v = _B2 * v + (1 - _B2) * grad ** 2
    t = s["step"]
    rate = torch.tensor(s["decay"], dtype=torch.float64, device=DEV)[s["which"]]
    w = s["w"].double() * (1 - _LR * rate) - _LR * (m / (1 - _B1 ** t)) / ((v / (1 - _B2 ** t)).sqrt() + _EPS)
    out = {"w": w, "lowp": w}
    if c["clip"]:
        out["norm"] = norm
    if c["bits"] == 32:
        return out | {"m": m, "v": v}
    # rounded at random with the same numbers; the exponents are whole numbers
    keys = torch.tensor([_key(s["seed"], t, i) for i in range(len(s["sizes"]))], device=DEV)[s["which"]]
    h = _mix(((s["place"].long() // 2) * 0x9E3779B1 + keys) & 0xFFFFFFFF)
    r = torch.where(s["place"] % 2 == 0, h % 65536, h // 65536).double() / 65536
    del h, keys
    for name, x in (("m", m), ("v", v.sqrt())):
        blocks = x.abs().view(-1, 256)
        E = torch.ceil(torch.log2(blocks.amax(1, True) / 448)).nan_to_num(neginf=0).clamp(min=-100)
        u = (blocks / torch.exp2(E)).view(-1)
        spacing = torch.exp2(torch.floor(torch.log2(u.clamp(min=2.0 ** -6))) - 3)
        q = (torch.floor(u / spacing + r) * spacing).clamp(max=448.0)
        if name == "v":
            q = torch.where(u > 0, q.clamp(min=2.0 ** -9), q)
        out[name] = torch.copysign(q, x)
    return out | {"m_exp": None, "v_exp": None}
