"""Sizes (classes C, best classes K, frames, type) that between them make w2l_token_logprob_fwd and w2l_distill_fwd_bwd launch
every form of their kernels; which form a size takes is asked of the library's own host-side queries, the functions that the entry points
dispatch through."""

# sixteen lanes a row (2 to 16 values each), a wavefront a row (2 to 24 vectors a lane), workgroups of several, joined workgroups
F32 = [(20, 5), (50, 9), (100, 20), (100, 64), (200, 24), (200, 25), (256, 3), (300, 64), (509, 64), (900, 3), (1500, 10), (2000, 64), (2500, 2), (3000, 33), (3500, 1),
       (4096, 64), (5000, 17), (6000, 5), (7000, 40), (8000, 64), (8500, 30), (12000, 8), (16384, 64), (20001, 31), (24576, 2), (28000, 64), (32768, 5), (140000, 7), (262143, 3)]
BF16 = [(30, 30), (64, 64), (128, 7), (129, 64), (250, 12), (400, 64), (1024, 64), (1500, 8), (2500, 1), (4000, 64), (5000, 20), (6100, 3), (7000, 64), (8192, 31),
        (9997, 16), (12000, 64), (13000, 2), (16000, 48), (18001, 5), (32768, 64), (40000, 9), (45001, 16), (50000, 64), (60000, 1), (262143, 11), (262144, 20)]
CASES = [(C, K, "fp32") for C, K in F32] + [(C, K, "bf16") for C, K in BF16]
ROWS = (3, 150, 2048)     # distillation also goes by the number of frames


def token_form(P, C, K, dtype):
    w, g, v = P.w2l_token_logprob_launch_config(1, 1, C, K, P.W2L_BF16 if dtype == "bf16" else P.W2L_F32)
    return dtype, min(w, 2), g > 1, v


def distill_form(P, rows, C, dtype):
    w, g, v = P.w2l_distill_launch_config(1, rows, C, 1, P.W2L_BF16 if dtype == "bf16" else P.W2L_F32)
    return dtype, min(w, 2), g > 1, v


def distill_cases(P):
    """(rows, C, K, dtype), one for each form that CASES and ROWS reach, the fewest frames first."""
    seen = {}
    for rows in ROWS:
        for C, K, dtype in CASES:
            seen.setdefault(distill_form(P, rows, C, dtype), (rows, C, K, dtype))
    return list(seen.values())
