// Reductions over the lanes of a wavefront.
#pragma once
#include "common.h"

#include <math.h>

namespace w2l {
namespace {

// ---- reductions over lanes ----------------------------------------------------------------------------
// (lanes that receive nothing combine with what changes nothing: then the move becomes an operand of the operation)
struct Max {
    static constexpr float none = -INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Min {
    static constexpr float none = INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
};
struct Sum {
    static constexpr float none = 0.f;
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float lane_of(float v, float none)
{
    if (ROWS == 0xf) return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// over the sixteen lanes of a DPP row, the same bits in each of them
template <typename F>
__device__ __forceinline__ float row16(float v, F f)
{
    v = f(v, lane_of<0xB1>(v, f.none));   // quad_perm [1,0,3,2]
    v = f(v, lane_of<0x4E>(v, f.none));   // quad_perm [2,3,0,1]
    v = f(v, lane_of<0x141>(v, f.none));  // row_half_mirror
    return f(v, lane_of<0x140>(v, f.none));  // row_mirror
}
// over the wavefront, uniform
template <typename F>
__device__ __forceinline__ float wave64(float v, F f)
{
    v = row16(v, f);
    v = f(v, lane_of<0x142, 0xa>(v, f.none));  // row_bcast:15 into rows 1 and 3
    v = f(v, lane_of<0x143, 0xc>(v, f.none));  // row_bcast:31 into rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
// LDS written by some lanes of a wavefront (MULTI: a workgroup) and read by others after this
template <bool MULTI>
__device__ __forceinline__ void exchange()
{
    if (MULTI) __syncthreads();
    else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace
}  // namespace w2l
