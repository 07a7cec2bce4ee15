// What the operators over a frame's scores share: rows of a tensor [rows][C] in registers, reductions over lanes, gradients stored by row, and
// how rows are dealt out (frame_scores.hip, policy.hip).
#pragma once
#include "lanes.h"

#include <initializer_list>
#include <type_traits>

namespace w2l {
namespace {

constexpr int MAX_CLASSES = 262144, MAX_ENTRIES = 64;
constexpr int THREADS = 256, MAX_WAVES = 16, MAX_SLOTS = 16, MAX_GROUPS = 16, NARROW = 256, FEW_ROWS = 64;
constexpr float FAR = 16777216.f;  // 2^24: k m from here on has roundings that are no small shift
constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;
enum Frame { LIVE = 0, PADDING = 1, BAD = 2 };

// Rows of utterances of Tp frames: r / Tp for r < 2^31 as a product, a fifth of the division's instructions
struct Frames {
    const int* in_len;
    unsigned rows, Tp, mul, shift;
};
Frames frames_of(const int* in_len, int B, int Tp)
{
    unsigned bits = 0;
    while ((1ull << bits) < (unsigned)Tp) ++bits;  // 2^bits >= Tp: mul = 2^(31 + bits) / Tp rounded up is exact for 31 bits, and fits 32
    return {in_len, (unsigned)B * (unsigned)Tp, (unsigned)Tp, (unsigned)(((1ull << (31 + bits)) + Tp - 1) / (unsigned)Tp), bits};
}
__device__ __forceinline__ Frame frame_of(const Frames& fr, unsigned r)
{
    if (!fr.in_len) return LIVE;
    const unsigned b = (unsigned)((unsigned long long)r * fr.mul >> 31 >> fr.shift);
    const int n = fr.in_len[b];
    return n < 0 || n > (int)fr.Tp ? BAD : (int)(r - b * fr.Tp) < n ? LIVE : PADDING;
}

// ---- rows in registers ---------------------------------------------------------------------------------
// A row lies in 16-byte vectors on the grid of the whole tensor (rows of odd length begin inside one): nv of them, `head`
// elements before the row's first.  They are dealt out in slots of 64, a vector a lane, in turn over the row's wavefronts
// (one, those of a workgroup, or those of several), so that the row is read once, with whole loads, and stays in
// registers: V slots a wavefront.  Lanes beyond the row, and elements of a vector that belong to its neighbours, are -inf.
template <typename T> constexpr int LANE_VALUES = 16 / sizeof(T);

// Registers that the compiler must not remember the unpacked values of: unpacking again costs less than holding them
template <int V>
__device__ __forceinline__ void opaque(uint4 (&q)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) asm volatile("" : "+v"(q[v].x), "+v"(q[v].y), "+v"(q[v].z), "+v"(q[v].w));
}

struct Row {
    size_t first;    // element of the tensor that vector 0 begins with
    int head, nv;
};
template <typename T>
__device__ __forceinline__ Row row_at(unsigned r, int C)
{
    constexpr int N = LANE_VALUES<T>;
    const size_t i = (size_t)r * C;
    const int head = (int)(i & (N - 1));
    return {i - head, head, (head + C + N - 1) / N};
}

__device__ __forceinline__ void unpack(uint4 q, float (&x)[4])
{
    x[0] = __uint_as_float(q.x); x[1] = __uint_as_float(q.y); x[2] = __uint_as_float(q.z); x[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(uint4 q, float (&x)[8])
{
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 pack(const float (&x)[4])
{
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8])
{
    typedef float float2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __builtin_bit_cast(unsigned, __builtin_convertvector((float2_t){x[2 * j], x[2 * j + 1]}, bf16x2_t));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Largest of a vector's elements, the instruction itself: fmaxf of loaded values costs one more each, for signalling NaN (rows with
// NaN are found by their sums, whatever their maximum)
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float largest(const float (&x)[4]) { return max3(max3(x[0], x[1], x[2]), x[3], x[3]); }
__device__ __forceinline__ float largest(const float (&x)[8])
{
    return max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), max3(x[6], x[7], x[7]));
}

// The row's elements of vector n, -inf in the places of its neighbours'
template <typename T>
__device__ __forceinline__ uint4 own_elements(uint4 q, const Row& row, int n, int C)
{
    constexpr int N = LANE_VALUES<T>, PER = N / 4;  // elements of a word
    const int c0 = n * N - row.head;
    unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        unsigned mine = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) mine |= (unsigned)(c0 + j * PER + e) < (unsigned)C ? (PER == 1 ? ~0u : 0xffffu << 16 * e) : 0u;
        w[j] = (w[j] & mine) | ((PER == 1 ? 0xff800000u : 0xff80ff80u) & ~mine);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Vectors that lie in the tensor whole are loaded whole; one that reaches past its last element (of the last row alone) is put
// together from single loads
template <typename T>
__device__ __forceinline__ int whole_vectors(size_t total, const Row& row)
{
    const size_t whole = (total - row.first) / LANE_VALUES<T>;
    return whole < (size_t)row.nv ? (int)whole : row.nv;
}
template <typename T>
__device__ __forceinline__ uint4 tail_vector(const T* __restrict__ z, size_t total, const Row& row, int whole)
{
    constexpr int N = LANE_VALUES<T>;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const size_t i = row.first + (size_t)whole * N + e;
        x[e] = i < total ? Elem<T>::load(z, i) : -INFINITY;
    }
    return pack(x);
}
// This lane's vectors n0, n0 + step, ... of a row of more than 64 elements.  Lanes beyond the row load its last whole vector again: without
// branches all loads are in flight at once.
template <typename T, int V>
__device__ __forceinline__ void load_row(uint4 (&q)[V], const T* __restrict__ z, size_t total, const Row& row, int step, int n0, int C)
{
    const int whole = whole_vectors<T>(total, row), inside = (row.head + C) / (64 * LANE_VALUES<T>);  // inside: slots that end within the row
    const char* const at = reinterpret_cast<const char*>(z + row.first);  // (a row is at most 1 MB: 32-bit offsets)
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int n = n0 + v * step;
        q[v] = *reinterpret_cast<const uint4*>(at + (unsigned)(n < whole ? n : whole - 1) * 16u);
    }
    uint4 tail = make_uint4(0, 0, 0, 0);
    if (whole < row.nv) {
        tail = tail_vector(z, total, row, whole);
        asm volatile("" : "+v"(tail.x), "+v"(tail.y), "+v"(tail.z), "+v"(tail.w));  // waited for here, not wherever its registers are used again
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int n = n0 + v * step, slot = n >> 6;
        if ((slot == 0 && row.head) || slot >= inside) q[v] = own_elements<T>(n == whole ? tail : q[v], row, n, C);
    }
}
template <typename T>
__device__ __forceinline__ uint4 load_vector(const T* __restrict__ z, size_t total, const Row& row, int n, int C)
{
    uint4 q[1];
    load_row(q, z, total, row, 64, n, C);
    return q[0];
}

// This lane's sums where k m is FAR, or m is +inf: from differences of scores, read again
template <typename T>
__device__ __forceinline__ void far_sums(const T* __restrict__ z, size_t total, const Row& row, int slots, int step, int n0, int C, float m, float kscale,
                                         float& s, float& u)
{
    s = u = 0.f;
#pragma unroll 1
    for (int v = 0; v < slots; ++v) {
        float x[LANE_VALUES<T>];
        unpack(load_vector(z, total, row, n0 + v * step, C), x);
#pragma unroll
        for (int e = 0; e < LANE_VALUES<T>; ++e) {
            const float a = (x[e] - m) * kscale, p = __builtin_amdgcn_exp2f(a);
            s += p;
            u += p * fmaxf(a, -1000.f);
        }
    }
}

// ---- gradients: p_c times a number of the row, corrected in a few columns --------------------------------------
// Adds or overwrites elements c0 .. c0 + N of a row whose vectors lie on the tensor's grid.  STREAM: a gradient beyond what the L2s hold (32 MB)
// goes past them: 2x200 frames of 65536 fp32: 60 -> 52 us with the forward call, 8x750 of 4096 bf16 distilled: 31 -> 27
enum { ADD = 1, STREAM = 2 };
template <typename G, int N>
__device__ __forceinline__ void put(G* __restrict__ dz, size_t i, int c0, int C, float (&v)[N], int how)
{
    typedef unsigned words_t __attribute__((ext_vector_type(4)));
    constexpr int PER = LANE_VALUES<G> < N ? LANE_VALUES<G> : N, STORES = N / PER;
    if (c0 >= 0 && c0 + N <= C && PER == LANE_VALUES<G>) {
#pragma unroll
        for (int j = 0; j < STORES; ++j) {
            uint4* const at = reinterpret_cast<uint4*>(dz + i + j * PER);
            float w[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) w[e] = v[j * PER + e];
            if (how & ADD) {
                float old[PER];
                unpack(*at, old);
#pragma unroll
                for (int e = 0; e < PER; ++e) w[e] += old[e];
            }
            const uint4 o = pack(w);
            if (how & STREAM) __builtin_nontemporal_store((words_t){o.x, o.y, o.z, o.w}, reinterpret_cast<words_t*>(at));
            else *at = o;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if ((unsigned)(c0 + e) < (unsigned)C) Elem<G>::store(dz, i + e, how & ADD ? Elem<G>::load(dz, i + e) + v[e] : v[e]);
}

// Zeros in place of a row's gradient
template <typename T, typename G>
__device__ __forceinline__ void clear_row(G* __restrict__ dz, const Row& row, int slots, int step, int n0, int C, int how)
{
    float zero[LANE_VALUES<T>] = {};
#pragma unroll 1
    for (int v = 0; v < slots; ++v) {
        const int n = n0 + v * step;
        if (n < row.nv) put(dz, row.first + (size_t)n * LANE_VALUES<T>, n * LANE_VALUES<T> - row.head, C, zero, how);
    }
}

// (x - m) k, k < 2^127: of halves, which fp32 holds where a difference of 6e38 and a temperature of 1e38 are no infinity
__device__ __forceinline__ float difference(float x, float m, float k) { return __builtin_fmaf(x, 0.5f, -0.5f * m) * (2.f * k); }

// loss[b] = sum of the utterance's frames, in double and in a fixed order.  8 utterances of 750: 4 us, a launch and a round trip to memory
__global__ __launch_bounds__(THREADS) void utterance_loss_k(const float* __restrict__ frame_loss, float* __restrict__ loss, unsigned utterances, unsigned Tp)
{
    __shared__ double lds[THREADS / 64];
    for (unsigned b = blockIdx.x; b < utterances; b += gridDim.x) {
        double s = 0.;
        for (unsigned t = threadIdx.x; t < Tp; t += 4 * THREADS) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = t + j * THREADS < Tp ? frame_loss[(size_t)b * Tp + t + j * THREADS] : 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) s += v[j];
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < THREADS / 64; ++w) s += lds[w];
            loss[b] = (float)s;
        }
        __syncthreads();
    }
}

bool shape_ok(int B, int Tp, int C, int S, int K)
{
    // a tensor of at most 2^40 scores: rows times workgroups (or wavefronts) a row stay below 2^32
    return B > 0 && Tp > 0 && (long long)B * Tp <= 2147483647LL && (long long)B * Tp <= (1LL << 40) / (C > 0 ? C : 1) && C > 0 && C <= MAX_CLASSES && S >= 0 && S <= MAX_ENTRIES && K >= 0 &&
           K <= MAX_ENTRIES && K <= C;
}
bool grad_dtype_ok(int z_dtype, int dz_dtype) { return valid_dtype(dz_dtype) && (dz_dtype == W2L_F32 || z_dtype == W2L_BF16); }

// How the rows are dealt out: sixteen lanes a row of up to 256 classes (W = 0), or W wavefronts of each of G workgroups, V slots of
// registers each.
struct Plan {
    int W, G, V;
};
int tight(int per, std::initializer_list<int> sizes)
{
    for (int v : sizes)
        if (per <= v) return v;
    return 0;
}
// values of a lane where sixteen lanes hold a row; 0: the row has a wavefront or more
int narrow_of(int C) { return C <= NARROW ? tight((C + 15) / 16, {2, 4, 8, 16}) : 0; }
int slots_of(int C, int dtype)
{
    const int N = dtype == W2L_BF16 ? 8 : 4, most = C % N ? C + 2 * (N - 1) : C;  // wherever in a vector a row begins
    return (most + 64 * N - 1) / (64 * N);
}

// Distillation.  The values are most of the work, and the gradient is written: a row has wavefronts enough to fill the chip (one row of 20
// slots: 8 us in five, 9.4 in three; 3000: 38 us in one, 43 in five).  More workgroups a row read it twice, so only few rows or rows beyond
// the registers of sixteen wavefronts have them (one row of 137 slots: 12 us against 17 in one workgroup; 400: 45 against 40).
Plan plan_distill(long long rows, int C, int dtype)
{
    if (const int nv = narrow_of(C)) return {0, 1, nv};
    const int slots = slots_of(C, dtype);
    if (slots <= 2 || (slots <= 24 && rows >= 2048)) return {1, 1, tight(slots, {2, 4, 6, 8, 10, 12, 14, 16, 20, 24})};
    int W, G = 1;
    if (slots <= 64) {
        W = (slots + 7) / 8;
        while (rows * W < 2048 && W * 4 <= slots && W * 2 <= MAX_WAVES) W *= 2;
        if (W < 2) W = 2;
    } else if (slots <= MAX_WAVES * MAX_SLOTS && rows >= 128)
        W = (slots + 15) / 16;
    else {
        W = 8;
        G = (slots + 31) / 32;
        if (G > MAX_GROUPS) G = MAX_GROUPS;
    }
    return {W, G, tight((slots + W * G - 1) / (W * G), {2, 4, 8, 12, 16})};
}

unsigned grid_of(long long groups) { return (unsigned)(groups < (1 << 20) ? groups : 1 << 20); }

template <typename D>
int how_of(unsigned rows, int C, int accumulate)
{
    return (accumulate ? ADD : 0) | ((size_t)rows * C * sizeof(D) > (32u << 20) ? STREAM : 0);
}
bool workspace_ok(const void* ws, size_t have, size_t need)
{
    return need == 0 || (ws && have >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0);
}

// Operands of a call (NULL: not there), of which no output may lie on an input: vectors hold elements of neighbouring rows, and some paths read a
// row again after others have been written
struct Span {
    const void* p;
    size_t bytes;
};
bool apart(std::initializer_list<Span> in, std::initializer_list<Span> out)
{
    for (const Span& o : out)
        for (const Span& i : in) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(o.p), b = reinterpret_cast<uintptr_t>(i.p);
            if (o.p && i.p && o.bytes && i.bytes && a < b + i.bytes && b < a + o.bytes) return false;
        }
    return true;
}

// f(std::integral_constant<int, V>) for the V of a plan, one of Vs; false if it is none of them
template <int... Vs, typename F>
bool with_slots(int V, F f)
{
    return ((V == Vs && (f(std::integral_constant<int, Vs>()), true)) || ...);
}

}  // namespace
}  // namespace w2l
