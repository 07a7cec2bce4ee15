"""Sizes (frames, classes, type) that between them make w2l_policy_fwd_bwd launch every form of its kernels; which form a size takes is asked of the library's own host-side query, the
function that the entry point dispatches through."""

# sixteen lanes a row; a wavefront a row; wavefronts of one workgroup, more of them where frames are few; eight wavefronts of several workgroups
NARROW = [(3, 29), (3, 50), (100, 100), (1, 128), (5, 200), (1, 256)]
F32 = NARROW + [(3, 257), (2048, 510), (2056, 1500), (2048, 2000), (2048, 2300), (2048, 3000), (2048, 3501), (2048, 4000), (1, 511), (3, 1500), (1104, 2801), (2056, 5101), (416, 9100), (136, 16601),
                (128, 20001), (3, 20001), (2, 150001), (1, 200001), (1, 240000), (1, 262143)]
BF16 = NARROW + [(3, 257), (2048, 1020), (2056, 2500), (2048, 4000), (2048, 5001), (2048, 6000), (2048, 7000), (2048, 8000), (1, 1500), (3, 3000), (1104, 5631), (2056, 10001), (416, 18001),
                 (136, 33203), (128, 40001), (3, 40001), (1, 262143)]
CASES = [(r, c, "fp32") for r, c in F32] + [(r, c, "bf16") for r, c in BF16]
ROWS = (1, 3, 8, 127, 128, 136, 416, 1100, 1104, 2047, 2048, 2056, 30000)


def policy_form(P, rows, C, dtype):
    """(type, wavefronts: none, one or more, whether several workgroups, slots)"""
    w, g, v = P.w2l_policy_launch_config(1, rows, C, P.W2L_BF16 if dtype == "bf16" else P.W2L_F32)
    return dtype, min(w, 2), g > 1, v
