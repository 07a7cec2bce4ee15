"""Sizes (B, T, C, G) that between them make w2l_groupnorm_fwd and _bwd launch every form of their kernels, with every activation; which form a size takes is asked of the
library's own host-side query, the function that the entry points dispatch through."""

ACTS = ("none", "relu", "silu", "glu")
# a workgroup a group: vectors of 16, 8, 4 and 2 bytes; groups of a vector and of many; one frame; more frames than a workgroup has lanes; an odd group for GLU;
# the widest; runs of frames: the same vectors, with and without a rest, more channels than a workgroup has vectors for
SHAPES = [(1, 1, 16, 2), (2, 5, 8, 8), (3, 17, 12, 3), (2, 33, 36, 2), (1, 70, 30, 1), (2, 100, 500, 20), (5, 64, 48, 4), (1, 333, 96, 96), (2, 129, 1536, 32), (1, 40, 2048, 1),
          (1, 20, 8192, 64), (1, 3, 8192, 8192), (1, 19, 4104, 27), (3, 1000, 64, 4), (40, 3, 130, 5), (8, 600, 256, 32), (2, 1300, 64, 1), (2, 1300, 60, 1), (2, 1300, 58, 1),
          (2, 2500, 29, 1), (2, 2500, 58, 2), (130, 700, 62, 2), (20, 50, 4096, 2), (2, 600, 60, 4)]


def code(P, act):
    return (P.W2L_ACT_NONE, P.W2L_ACT_RELU, P.W2L_ACT_SILU, P.W2L_ACT_GLU)[ACTS.index(act)]


def fits(shape, act):
    return act != "glu" or shape[2] % 2 == 0


def form(P, shape, act, dtype):
    return (*P.w2l_groupnorm_launch_config(*shape, code(P, act), P.W2L_BF16 if dtype == "bf16" else P.W2L_F32), act, dtype)
