// Operators over a frame's scores x[0 .. C): log-probabilities of given tokens with entropy and the K best classes
// (w2l_token_logprob_fwd / _bwd), and distillation from a teacher's K best classes (w2l_distill_fwd_bwd).
// All three are one softmax statistic of the row -- m = max x, s = sum exp(x - m), u = sum exp(x - m)(x - m), from which
// lp_c = (x_c - m) - log s and H = log s - u / s -- and a few of its columns; the gradients are p_c times a number of the row,
// corrected in those columns.  Log-probabilities are formed from x - m, never from x - (m + log s): a row of large
// scores keeps the bits of its differences.  Scores are widened to fp32, all sums are fp32; a gradient is rounded once, where it is stored.
// What bounds them is memory, and close behind it the instructions: a copy moves 5.0 TB/s here (reading alone 5.9), and the vector units
// take 551 G instructions of 64 lanes a second (an exponential counts twice), which leaves a bf16 score about fourteen of them.
#include "common.h"

#include <math.h>

#include <initializer_list>
#include <type_traits>

using namespace w2l;

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

// ---- the K largest of a row --------------------------------------------------------------------------------
// Scores in the order of their bits, as unsigned integers; and a score with its class as one integer that orders by score, then by
// the lower class.  (+ 0.f: the two zeros are equal.)
__device__ __forceinline__ unsigned key_of(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(unsigned k) { return __uint_as_float(k ^ ((unsigned)((int)~k >> 31) | 0x80000000u)); }
typedef unsigned long long ranked_t;
constexpr int HELD = 128, LIST = 128;  // a wavefront's vectors and list entries (a list has room for two more)
constexpr size_t lds_of(int waves, bool multi)
{
    return waves * HELD * (sizeof(uint4) + sizeof(int)) + (multi ? waves * 64 + 2 : waves * (LIST + 2)) * sizeof(ranked_t);
}
__device__ __forceinline__ ranked_t ranked(float x, int c) { return (ranked_t)key_of(x) << 32 | ~(unsigned)c; }
__device__ __forceinline__ int class_of(ranked_t k) { return (int)~(unsigned)k; }
__device__ __forceinline__ float score_of(ranked_t k) { return of_key((unsigned)(k >> 32)); }

__device__ __forceinline__ int below(unsigned long long mask)  // bits of the mask in lanes below this one
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}

// Thresholds that at least need[j] (<= 64) values of the wavefront reach, and not many more: each lane brings the largest of up to four
// groups of its values (-inf: no group), and a threshold is bisected (over the order of the bits) until about need[j] of these 256 reach
// it.  least: the smallest of the lanes' largest, which 64 values reach; most: the largest of all.  Two thresholds are sought side by
// side: a step is a chain of dependent instructions, of which a wavefront alone leaves most cycles empty.
template <int J>
__device__ __forceinline__ void wave_thresholds(const float (&group)[4], float least, float most, const int (&need)[J], float (&t)[J])
{
    unsigned lo[J], hi[J];
#pragma unroll
    for (int j = 0; j < J; ++j) { lo[j] = key_of(least); hi[j] = key_of(most) + 1; }
    bool open = hi[0] - lo[0] > 1;
    while (open) {
        open = false;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const unsigned mid = lo[j] + (hi[j] - lo[j]) / 2;  // (lo itself once they are neighbours: nothing changes)
            const float x = of_key(mid);
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(group[i] >= x));
            if (n >= need[j]) lo[j] = mid;
            else hi[j] = mid;
            if (n >= need[j] && n <= need[j] + 4) hi[j] = mid + 1;  // near enough
            open |= hi[j] - lo[j] > 1;
        }
    }
#pragma unroll
    for (int j = 0; j < J; ++j) t[j] = of_key(lo[j]);
}

// The wavefront's K largest classes, exactly, into list[0 .. K) in any order (fewer, if it holds fewer classes); returns how many.
// For rows where thresholds leave too many: equal scores, fewer finite ones than K, or best classes that are neighbours and so few groups' largest, as in
// inventories ordered by frequency.  That costs: with scores -ln(class) + N(0,1) all rows come here at K = 64, and 24000 of 4096 fp32 take 1340 us where
// independent scores take 88 (K = 32: 80 and 76), 6000 of 9997 bf16 1470 where they take 39 (K = 32: 164 and 33, K = 16: 32 and 31).  The K-th entry in the order of scores and
// classes is bisected.  Every step reads the row's vectors again, so that the registers of the usual path carry nothing for it.
template <typename T>
__device__ __forceinline__ int exact_largest(const T* __restrict__ z, size_t total, const Row& row, int ns, int step, int n0, int C, int K, ranked_t* list)
{
    constexpr int N = LANE_VALUES<T>;
    auto entries = [&](int v, ranked_t (&a)[N]) {  // 0: not the row's
        float x[N];
        unpack(load_vector(z, total, row, n0 + v * step, C), x);
        const int c0 = (n0 + v * step) * N - row.head;
#pragma unroll
        for (int e = 0; e < N; ++e) a[e] = (unsigned)(c0 + e) < (unsigned)C ? ranked(x[e], c0 + e) : 0;
    };
    ranked_t lo = ranked(-INFINITY, MAX_CLASSES), hi = ~0ull, mid = ranked(-INFINITY, 0) + 1;  // first: are there K above -inf?
#pragma unroll 1
    while (hi - lo > 1) {
        int n = 0;
#pragma unroll 1
        for (int v = 0; v < ns; ++v) {
            ranked_t a[N];
            entries(v, a);
#pragma unroll
            for (int e = 0; e < N; ++e) n += __popcll(__ballot(a[e] >= mid));
        }
        (n >= K ? lo : hi) = mid;
        if (n == K) break;
        mid = lo + (hi - lo) / 2;
    }
    int n = 0;
#pragma unroll 1
    for (int v = 0; v < ns; ++v) {
        ranked_t a[N];
        entries(v, a);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const unsigned long long b = __ballot(a[e] >= lo);
            const int at = n + below(b);
            if (a[e] >= lo && at < K) list[at] = a[e];
            n += __popcll(b);
        }
    }
    return n < K ? n : K;
}

// list[0 .. n) of a wavefront (n <= 128) or a workgroup (MULTI: n <= its threads), all different but zeros, and list[n] = 0 (close_list):
// calls out(rank, entry) for the K first.  (A wavefront's entries beyond 64 are ranked in the same pass, two a lane: 24000 rows of 4096, K = 64: 96 -> 89 us
// against one after the other by all lanes.  Counting by the scores alone, the classes only where two are equal, was no faster.)
__device__ __forceinline__ void close_list(ranked_t* list, int n, int thread)
{
    if (thread == 0) list[n] = 0;
}
template <bool MULTI, typename F>
__device__ __forceinline__ void rank_list(const ranked_t* list, int n, int K, int thread, F out)
{
    if (MULTI && (thread & ~63) >= n) return;  // (whole wavefronts)
    const bool two = !MULTI && n > 64;  // two entries a lane
    const ranked_t a = thread < n ? list[thread] : 0, b = two && thread + 64 < n ? list[thread + 64] : 0;
    int before = 0, before_b = 0;
    if (two)
#pragma unroll 4
        for (int j = 0; j < n; j += 2) {
            const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(list + j);
            before += w.x > a;
            before_b += w.x > b;
            before += w.y > a;
            before_b += w.y > b;
        }
    else
#pragma unroll 4
        for (int j = 0; j < n; j += 2) {
            const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(list + j);
            before += w.x > a;
            before += w.y > a;
        }
    if (thread < n && before < K) out(before, a);
    if (two && thread + 64 < n && before_b < K) out(before_b, b);
}

// ---- log-probabilities, entropy, best classes --------------------------------------------------------
struct TokenOut {
    float *logprob, *entropy;
    int* top_ids;
    float *top_logprob, *stats;
    int S, K;
};
__device__ __forceinline__ void write_absent(const TokenOut& o, unsigned r, Frame f, int i, int step)
{
    const float v = f == PADDING ? 0.f : NAN;
    for (int j = i; j < o.S; j += step) o.logprob[(size_t)r * o.S + j] = v;
    for (int j = i; j < o.K; j += step) {
        o.top_ids[(size_t)r * o.K + j] = -1;
        o.top_logprob[(size_t)r * o.K + j] = f == PADDING ? -INFINITY : NAN;
    }
    if (i == 0 && o.entropy) o.entropy[r] = v;
    if (i == 0 && o.stats) reinterpret_cast<float4*>(o.stats)[r] = make_float4(v, v, v, 0.f);
}
struct Dist { float m, logs, H; };  // s = 0, nothing but -inf: m = 0, and logs is taken as 0
__device__ __forceinline__ Dist dist_of(float m, float s, float u)
{
    const bool any = s > 0.f;
    const float logs = any ? logf(s) : 0.f;
    return {m, logs, any ? logs - u / s : 0.f};
}
__device__ __forceinline__ void write_dist(const TokenOut& o, unsigned r, const Dist& d, bool any)
{
    if (o.entropy) o.entropy[r] = d.H;
    if (o.stats) reinterpret_cast<float4*>(o.stats)[r] = make_float4(d.m, any ? d.logs : -INFINITY, d.H, 0.f);
}

// Partial results of a row that several workgroups share: [rows][G] of (m or -inf, s, u, 0), then [rows][G][K] best classes, largest
// first, 0 where there are fewer
struct Parts {
    float4* sums;
    ranked_t* best;
};

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

// One row by a wavefront (!MULTI, four rows a workgroup), by a workgroup, or by G workgroups, which leave partial results (parts) for
// token_join_k.  kscale = log2 e / temperature.  The row is read once.  The first pass over its registers finds the maximum and a threshold that
// the K best reach, the second the sums; vectors with a score at the threshold go to LDS on the way, their scores to a list, and
// each entry's rank is the number of entries before it.
// 24000 rows of 4096 fp32 (393 MB): 68 us = 5.8 TB/s without best classes, 77 with 16, 82 with 48, 88 with 64 (beyond 64 candidates
// a lane has two).  5000 of 9997 bf16, K = 16: 30 us = 3.3 TB/s: 20 us of instructions beside 20 of memory.
// Loading the next row while this one's ranks are taken gained nothing (92 -> 106 us at 4096, K = 64: the loads' queue is full as it is), nor did
// one pass with a running maximum (93 us), the clamp left out of slots that hold no -inf (a branch a slot: 33 -> 35 us at 9997), the sums as
// products of the matrix pipe (33 -> 40); fewer wavefronts a SIMD, as long as nothing spills, lose nothing.
template <typename T, int V, bool MULTI>
__global__ __launch_bounds__(MULTI ? 512 : 256) __attribute__((amdgpu_waves_per_eu(V > 20 ? 2 : V > 12 ? 3 : V > 8 ? 4 : V > 4 ? 5 : 6))) void
token_rows_k(const T* __restrict__ z, const int* __restrict__ tokens, Frames fr, TokenOut o, Parts parts, int C, int groups, float kscale)
{
    const int G = MULTI ? groups : 1;
    constexpr int N = LANE_VALUES<T>;
    constexpr int ROWS = MULTI ? 1 : 4;
    extern __shared__ uint4 lds[];
    __shared__ float red[MULTI ? 3 : 1][16];
    __shared__ int count, exact;  // entries of the list; where they did not fit, those of all wavefronts' own best
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = MULTI ? blockDim.x >> 6 : 1;
    uint4* const held = lds + wave * HELD;  // the wavefront's vectors with a score at the threshold, and their numbers
    int* const held_n = reinterpret_cast<int*>(lds + (MULTI ? W : 4) * HELD) + wave * HELD;
    const int room = MULTI ? W * 64 : LIST;  // of the list: a workgroup's, or each wavefront's
    ranked_t* const list = reinterpret_cast<ranked_t*>(lds + (MULTI ? W : 4) * (HELD + HELD / 4)) + (MULTI ? 0 : wave * (LIST + 2));
    const size_t total = (size_t)fr.rows * C;
    const int thread = MULTI ? (int)threadIdx.x : lane;
    const unsigned tasks = fr.rows * G, stride = gridDim.x * ROWS;
    for (unsigned task = blockIdx.x * ROWS + (MULTI ? 0 : wave); task < tasks; task += stride) {
        const unsigned r = task / G;
        const int g = task - r * G;
        const Frame f = frame_of(fr, r);
        if (f != LIVE) {
            if (G == 1) write_absent(o, r, f, thread, MULTI ? blockDim.x : 64);
            continue;
        }
        const Row row = row_at<T>(r, C);
        const int step = W * G * 64, n0 = (g * W + (MULTI ? wave : 0)) * 64 + lane;
        uint4 q[V];
        load_row(q, z, total, row, step, n0, C);
        int token = -1;
        float xt = 0.f;
        if (G == 1 && thread < o.S) {
            token = tokens[(size_t)r * o.S + thread];
            if (token >= 0 && token < C) xt = Elem<T>::load(z, (size_t)r * C + token);
        }
        float most[V], group[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};  // largest of each vector; of up to four groups of them
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float x[N];
            unpack(q[v], x);
            most[v] = largest(x);
            if (V > 2) group[v * 4 / (V > 4 ? V : 4)] = fmaxf(group[v * 4 / (V > 4 ? V : 4)], most[v]);
            else  // one or two vectors: by element
#pragma unroll
                for (int e = 0; e < N; ++e) group[e & 3] = fmaxf(group[e & 3], x[e]);
        }
        const float lane_most = fmaxf(fmaxf(group[0], group[1]), fmaxf(group[2], group[3]));
        float m = wave64(lane_most, Max()), t = INFINITY;
        if (o.K > 0) {
            const float least = wave64(lane_most, Min());
            // W wavefronts: K scores reach the least of thresholds that K / W of each one's reach, and the largest of those that K of one's do
            if (MULTI) {
                float own[2];
                wave_thresholds<2>(group, least, m, {(o.K + W - 1) / W, o.K}, own);
                if (lane == 0) { red[1][wave] = own[0]; red[2][wave] = own[1]; }
            } else {
                float own[1] = {-INFINITY};  // a row of few more classes than are wanted is ranked whole
                if (C > LIST || o.K < C / 4) wave_thresholds<1>(group, least, m, {o.K}, own);
                t = own[0];
            }
        }
        if (MULTI) {
            if (lane == 0) red[0][wave] = m;
            if (threadIdx.x == 0) { count = 0; exact = 0; }
            __syncthreads();
            const int w = lane & 15;
            m = uniform(row16(w < W ? red[0][w] : -INFINITY, Max()));
            if (o.K > 0) t = uniform(fmaxf(row16(w < W ? red[1][w] : INFINITY, Min()), row16(w < W ? red[2][w] : -INFINITY, Max())));
        }
        // exp(x - m) as 2^(k x - M), M = k m rounded: what the rounding moves, `shift`, is taken out of the sums at the end
        const float m0 = m == -INFINITY ? 0.f : m, M = m0 * kscale, shift = __builtin_fmaf(m0, kscale, -M);
        float s = 0.f, u = 0.f;
        int n = 0, hits = 0;
        opaque(q);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float x[N];
            unpack(q[v], x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float a = __builtin_fmaf(x[e], kscale, -M), p = __builtin_amdgcn_exp2f(a);
                s += p;
                u += p * fmaxf(a, -1000.f);  // 0 * -inf is no share of the entropy
            }
            asm volatile("" : "+v"(s), "+v"(u));  // summed here: left alone, the sums sink below all slots' branches and the values stay in registers
            const unsigned long long b = __ballot(most[v] >= t);
            if (b != 0) {
                const int at = hits + below(b);
                if (most[v] >= t && at < HELD) { held[at] = q[v]; held_n[at] = n0 + v * step; }
                hits += __popcll(b);
            }
        }
        if (!(fabsf(M) < FAR)) far_sums(z, total, row, V, step, n0, C, m0, kscale, s, u);
        else {
            const float scale = __builtin_amdgcn_exp2f(-shift);
            u = (u - shift * s) * scale;
            s *= scale;
        }
        if (o.K > 0) {
            exchange<false>();
            if (hits > HELD) n = room + 1;
#pragma unroll 1
            for (int base = 0; base < hits && n <= room; base += 64) {
                float x[N];
                const int i = base + lane;
                const bool on = i < hits;
                unpack(held[on ? i : 0], x);
                const int c0 = held_n[on ? i : 0] * N - row.head;
                unsigned mine = 0;
#pragma unroll
                for (int e = 0; e < N; ++e) mine |= on && x[e] >= t && (unsigned)(c0 + e) < (unsigned)C ? 1u << e : 0u;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const bool take = mine >> e & 1;
                    const unsigned long long b = __ballot(take);
                    if (b == 0) continue;
                    int at = n;
                    if (MULTI) {
                        if (lane == 0) at = atomicAdd(&count, __popcll(b));
                        at = __builtin_amdgcn_readfirstlane(at);
                    }
                    n = at + __popcll(b);
                    at += below(b);
                    if (take && at < room) list[at] = ranked(x[e], c0 + e);
                }
            }
            if (MULTI && hits > HELD && lane == 0) atomicAdd(&count, room + 1);
        }
        s = wave64(s, Sum());
        u = wave64(u, Sum());
        if (MULTI) {
            __syncthreads();
            if (lane == 0) { red[0][wave] = s; red[1][wave] = u; }
            n = count;
            __syncthreads();
            const int w = lane & 15;
            s = uniform(row16(w < W ? red[0][w] : 0.f, Sum()));
            u = uniform(row16(w < W ? red[1][w] : 0.f, Sum()));
        }
        u *= LN2;
        if (o.K > 0 && s == s) {
            if (n > room) {
                list[wave * 64 * MULTI + lane] = 0;
                exchange<MULTI>();
                n = exact_largest(z, total, row, V, step, n0, C, o.K, list + wave * 64 * MULTI);
                if (MULTI) {
                    if (lane == 0) atomicAdd(&exact, n);
                    n = room;
                }
            }
        }
        if (o.K > 0 && s == s) close_list(list, n, thread);  // (n <= room: a row of NaN or +inf may have counted past it)
        exchange<MULTI>();
        if (MULTI && G > 1) {
            const size_t at = (size_t)r * G + g;
            if (threadIdx.x == 0) parts.sums[at] = make_float4(m, s, u, 0.f);
            if (s == s) {
                if (thread < o.K && thread >= (exact ? exact : n)) parts.best[at * o.K + thread] = 0;
                if (o.K > 0) rank_list<MULTI>(list, n, o.K, thread, [&](int k, ranked_t a) { if (a) parts.best[at * o.K + k] = a; });
            }
        } else if (!(s == s)) {
            write_absent(o, r, BAD, thread, MULTI ? blockDim.x : 64);
        } else {
            const Dist d = dist_of(m0, s, u);
            if (thread == 0) write_dist(o, r, d, s > 0.f);
            if (thread < o.S) o.logprob[(size_t)r * o.S + thread] = token == -1 ? 0.f : token < 0 || token >= C ? NAN : (xt - d.m) - d.logs;
            if (o.K > 0)
                rank_list<MULTI>(list, n, o.K, thread, [&](int k, ranked_t a) {
                    o.top_ids[(size_t)r * o.K + k] = class_of(a);
                    o.top_logprob[(size_t)r * o.K + k] = (score_of(a) - d.m) - d.logs;
                });
        }
        exchange<MULTI>();
    }
}

// The rows that G workgroups left in parts, a workgroup each.  Of the G sorted lists, entries below the largest K-th of a list or below the
// smallest ceil(K / G)-th are not among the K best; about 1.5 K pass.  4 rows, G = 4, K = 40: 4.4 us, latency.
template <typename T>
__global__ __launch_bounds__(THREADS) void token_join_k(const T* __restrict__ z, const int* __restrict__ tokens, Frames fr, TokenOut o, Parts parts,
                                                        int C, int G)
{
    __shared__ __attribute__((aligned(16))) ranked_t list[MAX_GROUPS * MAX_ENTRIES + 2];
    __shared__ int count;
    constexpr int MINE = MAX_GROUPS * MAX_ENTRIES / THREADS;
    for (unsigned r = blockIdx.x; r < fr.rows; r += gridDim.x) {
        const int tid = threadIdx.x, lane = tid & 63, need = (o.K + G - 1) / G;
        const Frame f = frame_of(fr, r);
        if (f != LIVE) {
            write_absent(o, r, f, tid, THREADS);
            continue;
        }
        // everything that is read, at once: a few rows are a chain of round trips to memory.  (A row of NaN left no lists: what is read there is not used.)
        const float4 p = lane < G ? parts.sums[(size_t)r * G + lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        const ranked_t* const best = parts.best + (size_t)r * G * o.K;
        ranked_t least = ~0ull, most = 0, mine[MINE] = {};
        if (o.K > 0 && lane < G) { least = best[lane * o.K + need - 1]; most = best[lane * o.K + o.K - 1]; }
#pragma unroll
        for (int j = 0; j < MINE; ++j)
            if (tid + j * THREADS < G * o.K) mine[j] = best[tid + j * THREADS];
        int token = -1;
        float xt = 0.f;
        if (tid < o.S) {
            token = tokens[(size_t)r * o.S + tid];
            if (token >= 0 && token < C) xt = Elem<T>::load(z, (size_t)r * C + token);
        }
        const float m = wave64(p.x, Max()), apart = p.x - m, scale = expf(apart);
        const float s = wave64(p.y != 0.f ? p.y * scale : 0.f, Sum());
        const float u = wave64(p.y != 0.f ? (p.z + p.y * fmaxf(apart, -1000.f)) * scale : 0.f, Sum());
        if (!(s == s)) {
            write_absent(o, r, BAD, tid, THREADS);
            continue;
        }
        const Dist d = dist_of(m == -INFINITY ? 0.f : m, s, u);
        if (tid == 0) write_dist(o, r, d, s > 0.f);
        if (tid < o.S) o.logprob[(size_t)r * o.S + tid] = token == -1 ? 0.f : token < 0 || token >= C ? NAN : (xt - d.m) - d.logs;
        if (o.K == 0) continue;
#pragma unroll
        for (int j = MAX_GROUPS / 2; j > 0; j >>= 1) {
            const ranked_t a = __shfl_xor(least, j, MAX_GROUPS), b = __shfl_xor(most, j, MAX_GROUPS);
            least = a < least ? a : least;
            most = b > most ? b : most;
        }
        least = __shfl(least < most ? most : least, 0, 64);
        if (tid == 0) count = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < MINE; ++j)
            if (mine[j] >= least && mine[j] != 0) list[atomicAdd(&count, 1)] = mine[j];
        __syncthreads();
        const int n = count;
        close_list(list, n, tid);
        __syncthreads();
        for (int i = tid; i < n; i += THREADS) {
            const ranked_t a = list[i];
            int before = 0;
#pragma unroll 4
            for (int j = 0; j < n; j += 2) {
                const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(list + j);
                before += w.x > a;
                before += w.y > a;
            }
            if (before < o.K) {
                o.top_ids[(size_t)r * o.K + before] = class_of(a);
                o.top_logprob[(size_t)r * o.K + before] = (score_of(a) - d.m) - d.logs;
            }
        }
        __syncthreads();
    }
}

// Rows of up to 16 * NV classes, sixteen lanes each.  The K best are taken one after the other: largest score, then lowest class.
// 24000 rows of 29: 4.1 us without best classes, 7.6 with 8 (each a round of some 25 instructions for four rows); of 200: 7, 12 with 4, 26 with 16.
template <typename T, int NV>
__global__ __launch_bounds__(THREADS) void token_narrow_k(const T* __restrict__ z, const int* __restrict__ tokens, Frames fr,
                                                          TokenOut o, int C)
{
    const int l = threadIdx.x & 15;
    const unsigned stride = gridDim.x * 16;
    for (unsigned r = blockIdx.x * 16 + (threadIdx.x >> 4); r < fr.rows; r += stride) {
        const Frame f = frame_of(fr, r);
        if (f != LIVE) {
            write_absent(o, r, f, l, 16);
            continue;
        }
        const T* const x = z + (size_t)r * C;
        float v[NV], m = -INFINITY, s = 0.f, u = 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            v[q] = l + 16 * q < C ? Elem<T>::load(x, l + 16 * q) : -INFINITY;
            m = fmaxf(m, v[q]);
        }
        m = row16(m, Max());
        const float m0 = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const float d = v[q] - m0, p = __builtin_amdgcn_exp2f(d * LOG2E);
            s += p;
            u += p * fmaxf(d, -1000.f);
        }
        s = row16(s, Sum());
        u = row16(u, Sum());
        if (!(s == s)) {
            write_absent(o, r, BAD, l, 16);
            continue;
        }
        const Dist d = dist_of(m0, s, u);
        if (l == 0) write_dist(o, r, d, s > 0.f);
        for (int j = l; j < o.S; j += 16) {
            const int c = tokens[(size_t)r * o.S + j];
            o.logprob[(size_t)r * o.S + j] = c == -1 ? 0.f : c < 0 || c >= C ? NAN : (Elem<T>::load(x, c) - d.m) - d.logs;
        }
        unsigned left = 0;  // this lane's classes that are not taken yet
#pragma unroll
        for (int q = 0; q < NV; ++q) left |= l + 16 * q < C ? 1u << q : 0u;
        float score = 0.f;
        int id = 0;
        for (int k = 0; k < o.K; ++k) {
            float w = -INFINITY;
            int c = MAX_CLASSES;
#pragma unroll
            for (int q = NV - 1; q >= 0; --q)
                if ((left >> q & 1) && v[q] >= w) { w = v[q]; c = l + 16 * q; }
            const float best = row16(w, Max());
            // the lowest class at it (whole numbers below 2^24 are exact as floats)
            const int taken = (int)row16(w == best ? (float)c : (float)MAX_CLASSES, Min());
            if (c == taken) left &= ~(1u << (c >> 4));
            if (l == (k & 15)) { score = best; id = taken; }
            if ((k & 15) == 15 || k == o.K - 1) {
                const int at = (k & ~15) + l;
                if (at <= k) {
                    o.top_ids[(size_t)r * o.K + at] = id;
                    o.top_logprob[(size_t)r * o.K + at] = (score - d.m) - d.logs;
                }
            }
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

// Columns of a row that get something of their own, an entry a lane: its column (-1: none) and the slot of the wavefront (counted in vectors of
// 64 lanes of the row) that it is in
template <int N>
__device__ __forceinline__ int slot_of(int id, const Row& row) { return id < 0 ? -1 : (id + row.head) / (64 * N); }
// Up to 128 columns, and what is added there
struct Columns {
    int id[2], slot[2];
    float add[2];
    template <int N>
    __device__ __forceinline__ void place(const Row& row)
    {
#pragma unroll
        for (int j = 0; j < 2; ++j) slot[j] = slot_of<N>(id[j], row);
    }
    // adds the entries of this slot to its lanes' values, in the order of the entries
    template <int N>
    __device__ __forceinline__ void apply(int at, const Row& row, float (&x)[N]) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            unsigned long long b = __ballot(slot[j] == at);
            while (b) {
                const int l = __ffsll((unsigned long long)b) - 1;
                b &= b - 1;
                const int c = __builtin_amdgcn_readlane(id[j], l) + row.head;
                const float a = lane == ((c / N) & 63) ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(add[j]), l)) : 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (e == (c & (N - 1))) x[e] += a;  // a uniform choice
            }
        }
    }
};
// Up to 64 columns whose values are replaced: `value`, less the `also` of every further entry of the same column
struct Replaced {
    int id, slot;
    float value, also;
    template <int N>
    __device__ __forceinline__ void apply(int at, const Row& row, float (&x)[N]) const
    {
        const int lane = threadIdx.x & 63;
        unsigned long long b = __ballot(slot == at);
        while (b) {
            const int l = __ffsll((unsigned long long)b) - 1, column = __builtin_amdgcn_readlane(id, l), c = column + row.head;
            float a = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(value), l));
            unsigned long long same = __ballot(id == column);
            b &= ~same;
            for (same &= same - 1; same; same &= same - 1)  // (its lowest lane is l)
                a -= __int_as_float(__builtin_amdgcn_readlane(__float_as_int(also), __ffsll((unsigned long long)same) - 1));
            const bool mine = lane == ((c / N) & 63);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e == (c & (N - 1))) x[e] = mine ? a : x[e];  // a uniform choice
        }
    }
};

// V slots of a row a wavefront, nothing between wavefronts.  2700 rows of 10001 bf16: 22 us = 4.9 TB/s of reading and writing; 350 of 65536
// fp32: 30 us = 6.1 TB/s.
template <typename T, typename G, int V>
__global__ __launch_bounds__(THREADS) void token_bwd_rows_k(const T* __restrict__ z, const float* __restrict__ stats, const int* __restrict__ tokens,
                                                            const float* __restrict__ dlogprob, const float* __restrict__ dentropy,
                                                            const int* __restrict__ top_ids, const float* __restrict__ dtop, Frames fr, G* __restrict__ dz, int C,
                                                            int S, int K, int P, int how)
{
    constexpr int N = LANE_VALUES<T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t total = (size_t)fr.rows * C;
    const unsigned tasks = fr.rows * P;
    for (unsigned task = blockIdx.x * 4 + wave; task < tasks; task += gridDim.x * 4) {
        const unsigned r = task / P;
        const int p = task - r * P;
        const Row row = row_at<T>(r, C);
        const int slots = (row.nv + 63) / 64, first = p * V;
        if (first >= slots) continue;
        const float4 q = reinterpret_cast<const float4*>(stats)[r];
        if (frame_of(fr, r) != LIVE || !(fabsf(q.y) < INFINITY)) {
            if (!(how & ADD)) clear_row<T>(dz, row, V, 64, first * 64 + lane, C, how);
            continue;
        }
        uint4 data[V];
        load_row(data, z, total, row, 64, first * 64 + lane, C);
        Columns cols;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = lane + 64 * j;
            int c = -1;
            float a = 0.f;
            if (i < S) { c = tokens[(size_t)r * S + i]; a = dlogprob[(size_t)r * S + i]; }
            else if (i < S + K) { c = top_ids[(size_t)r * K + i - S]; a = dtop[(size_t)r * K + i - S]; }
            const bool there = c >= 0 && c < C;
            cols.id[j] = there ? c : -1;
            cols.add[j] = there ? a : 0.f;
            if (64 * j < S + K) sum += wave64(cols.add[j], Sum());
        }
        const float h = dentropy ? dentropy[r] : 0.f;
        cols.template place<N>(row);
        const float M = q.x * LOG2E;
        if (!(fabsf(M) < FAR)) {
#pragma unroll 1
            for (int v = 0; v < V; ++v) {  // from differences
                const int n = (first + v) * 64 + lane;
                float x[N];
                unpack(load_vector(z, total, row, n, C), x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float lp = fmaxf((x[e] - q.x) - q.y, -1000.f);
                    x[e] = -__builtin_amdgcn_exp2f(lp * LOG2E) * (sum + h * (lp + q.z));
                }
                cols.apply(first + v, row, x);
                if (n < row.nv) put(dz, row.first + (size_t)n * N, n * N - row.head, C, x, how);
            }
            continue;
        }
        // with a = k x - M: lp = ln 2 (a - shift) - log s, and -p (G + h (lp + H)) = 2^a (A + B a)
        const float shift = __builtin_fmaf(q.x, LOG2E, -M), inv = -__builtin_amdgcn_exp2f(-shift) * expf(-q.y);
        const float A = inv * (sum + h * ((q.z - q.y) - LN2 * shift)), B = inv * h * LN2;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int n = (first + v) * 64 + lane;
            float x[N];
            unpack(data[v], x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float a = __builtin_fmaf(x[e], LOG2E, -M);
                x[e] = __builtin_amdgcn_exp2f(a) * __builtin_fmaf(B, fmaxf(a, -1000.f), A);
            }
            cols.apply(first + v, row, x);
            if (n < row.nv) put(dz, row.first + (size_t)n * N, n * N - row.head, C, x, how);
        }
    }
}

template <typename T, typename G, int NV>
__global__ __launch_bounds__(THREADS) void token_bwd_narrow_k(const T* __restrict__ z, const float* __restrict__ stats, const int* __restrict__ tokens,
                                                              const float* __restrict__ dlogprob, const float* __restrict__ dentropy,
                                                              const int* __restrict__ top_ids, const float* __restrict__ dtop, Frames fr, G* __restrict__ dz, int C,
                                                              int S, int K, int accumulate)
{
    const int l = threadIdx.x & 15;
    const unsigned stride = gridDim.x * 16;
    for (unsigned r = blockIdx.x * 16 + (threadIdx.x >> 4); r < fr.rows; r += stride) {
        const size_t i0 = (size_t)r * C;
        const float4 st = reinterpret_cast<const float4*>(stats)[r];
        const bool live = frame_of(fr, r) == LIVE && fabsf(st.y) < INFINITY;
        if (!live && accumulate) continue;
        float direct[NV], sum = 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q) direct[q] = 0.f;
        if (live)
            for (int j0 = 0; j0 < S + K; j0 += 16) {
                const int i = j0 + l;
                int c = -1;
                float a = 0.f;
                if (i < S) { c = tokens[(size_t)r * S + i]; a = dlogprob[(size_t)r * S + i]; }
                else if (i < S + K) { c = top_ids[(size_t)r * K + i - S]; a = dtop[(size_t)r * K + i - S]; }
                const int most = S + K - j0 < 16 ? S + K - j0 : 16;
                for (int j = 0; j < most; ++j) {
                    const int cj = __shfl(c, j, 16);
                    const float aj = __shfl(a, j, 16);
                    if (cj >= 0 && cj < C) sum += aj;
#pragma unroll
                    for (int q = 0; q < NV; ++q) direct[q] += cj == l + 16 * q ? aj : 0.f;
                }
            }
        const float h = live && dentropy ? dentropy[r] : 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q)
            if (l + 16 * q < C) {
                const size_t i = i0 + l + 16 * q;
                float v = 0.f;
                if (live) {
                    const float lp = fmaxf((Elem<T>::load(z, i) - st.x) - st.y, -1000.f);
                    v = direct[q] - __builtin_amdgcn_exp2f(lp * LOG2E) * (sum + h * (lp + st.z));
                }
                Elem<G>::store(dz, i, accumulate ? Elem<G>::load(dz, i) + v : v);
            }
    }
}

// ---- distillation --------------------------------------------------------------------------------------------
struct Teacher {
    const int* ids;
    const float *scores, *weight;
    int K;
    float tau, inv_tau, kscale, grad_scale;  // kscale = log2 e / tau
};
__device__ __forceinline__ float weight_of(const Teacher& te, unsigned r) { return te.weight ? te.weight[r] : 1.f; }

// (x - m) k, k < 2^127: of halves, which fp32 holds where a difference of 6e38 and a temperature of 1e38 are no infinity
__device__ __forceinline__ float difference(float x, float m, float k) { return __builtin_fmaf(x, 0.5f, -0.5f * m) * (2.f * k); }

// Loss of a frame from what its K <= 64 * R entries say, an entry a lane of WIDTH (16 or 64): score t of class c, student score x there; m, s of
// the student's row at the temperature.  q: the teacher's probability of the lane's entries.  Returns the loss; live: whether there is a gradient.
// The loss is off by a few tau^2 2^-24 log C.  At tau = 4 that is 4e-6 of a loss of 0.5; beyond (WARM) ordinary scores, whose loss does not grow with
// tau, would have 2e-4 at tau = 20 and all of it at 1000 (made the other way: 2e-7 at any tau).  near: a loss below tau^2 / 4 there, which distill_near_k makes, with the row's gradient.
constexpr float WARM = 4.f;
constexpr unsigned NEAR = 0x7fc00001u;  // what it finds in place of the loss: a NaN that no operation gives
template <int R, int WIDTH>
__device__ __forceinline__ float frame_loss_of(const Teacher& te, const int (&c)[R], const float (&t)[R], const float (&x)[R], float w, float m, float s,
                                               int C, float (&q)[R], bool& near, bool& live)
{
    auto all = [](float v, auto f) { return WIDTH == 16 ? row16(v, f) : wave64(v, f); };
    float odd = 0.f, tm = -INFINITY, sum = 0.f, kl = 0.f, d[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        if ((c[j] != -1 && (unsigned)c[j] >= (unsigned)C) || !(t[j] < INFINITY)) odd = 1.f;
        tm = fmaxf(tm, t[j]);
    }
    odd = all(odd, Max());
    tm = all(tm, Max());
    const bool none = tm == -INFINITY;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        d[j] = none ? -INFINITY : difference(t[j], tm, te.inv_tau);
        q[j] = none ? 0.f : expf(d[j]);
        sum += q[j];
    }
    sum = all(sum, Sum());
    const float inv = none ? 0.f : 1.f / sum;
    // tau sum q (log q - log p) = sum q ((t - tm) - (x - m)) + tau log(s / sum): differences of scores are not divided by a small tau, and tau^2 is
    // not formed.  A quarter of them, which fp32 holds whatever the scores, and the rest in 64 bits: at a large tau each logarithm's
    // product with it may be beyond fp32 where the loss is not.
#pragma unroll
    for (int j = 0; j < R; ++j) {
        q[j] *= inv;
        if (q[j] > 0.f) kl += q[j] * (__builtin_fmaf(t[j], 0.25f, -0.25f * tm) - __builtin_fmaf(x[j], 0.25f, -0.25f * m));
    }
    kl = all(kl, Sum());
    const double apart = 4. * kl + (double)te.tau * (s > 0.f ? logf(s * inv) : 0.f);
    const bool defined = odd == 0.f && s == s;
    near = te.tau > WARM && defined && !none && fabs(apart) < 0.25 * te.tau;
    const float loss = !defined ? NAN : none ? 0.f : (float)((double)w * te.tau * apart);
    live = !none && fabsf(loss) < INFINITY;
    return near ? __uint_as_float(NEAR) : loss;
}

// G > 1, where a row is too long for the registers of a workgroup, or rows are few: sums has (m or -inf, s, ., .) of each of the `parts` that
// token_rows_k read it in; else it is NULL.  The row is read once (G > 1: twice), its gradient made from the registers.
// 5400 rows of 4096 bf16: 25 us = 3.5 TB/s of reading and writing, all of them in flight at once, so that loads and stores do not overlap; 2900 of
// 32000 bf16, K = 64: 85 us = 4.4 TB/s.
template <typename T, typename D, int V, bool MULTI>
__global__ __launch_bounds__(MULTI ? 1024 : 256) void distill_rows_k(const T* __restrict__ z, Teacher te, Frames fr,
                                                                         const float4* __restrict__ sums, int parts, float* __restrict__ frame_loss,
                                                                         D* __restrict__ dz, int C, int groups, int how)
{
    const int G = MULTI ? groups : 1;
    constexpr int N = LANE_VALUES<T>;
    constexpr int ROWS = MULTI ? 1 : 4;
    __shared__ float red[2][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = MULTI ? blockDim.x >> 6 : 1;
    const size_t total = (size_t)fr.rows * C;
    const unsigned tasks = fr.rows * G, stride = gridDim.x * ROWS;
    for (unsigned task = blockIdx.x * ROWS + (MULTI ? 0 : wave); task < tasks; task += stride) {
        const unsigned r = task / G;
        const int g = task - r * G;
        const bool first = g == 0 && (MULTI ? threadIdx.x : lane) == 0;
        const Frame f = frame_of(fr, r);
        const Row row = row_at<T>(r, C);
        const int P = W * G, step = P * 64, n0 = (g * W + (MULTI ? wave : 0)) * 64 + lane;
        const float w = f != LIVE ? 0.f : weight_of(te, r);
        if (w == 0.f) {
            if (first) frame_loss[r] = f == BAD ? NAN : 0.f;
            if (dz && !(how & ADD)) clear_row<T>(dz, row, V, step, n0, C, how);
            continue;
        }
        uint4 data[V];
        load_row(data, z, total, row, step, n0, C);
        int c[1] = {-1};
        float t[1] = {-INFINITY}, x[1] = {0.f}, q[1];
        if (lane < te.K) {
            c[0] = te.ids[(size_t)r * te.K + lane];
            if (c[0] != -1) t[0] = te.scores[(size_t)r * te.K + lane];
            if ((unsigned)c[0] < (unsigned)C) x[0] = Elem<T>::load(z, (size_t)r * C + c[0]);
        }
        float m = -INFINITY, s = 0.f;
        if (MULTI && sums) {
            const float4 a = lane < parts ? sums[(size_t)r * parts + lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
            m = wave64(a.x, Max());
            s = wave64(a.y != 0.f ? a.y * expf(difference(a.x, m, te.inv_tau)) : 0.f, Sum());
            m = m == -INFINITY ? 0.f : m;
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float y[N];
                unpack(data[v], y);
                m = fmaxf(m, largest(y));
            }
            m = wave64(m, Max());
            if (MULTI) {
                if (lane == 0) red[0][wave] = m;
                __syncthreads();
                m = uniform(row16((lane & 15) < W ? red[0][lane & 15] : -INFINITY, Max()));
            }
            m = m == -INFINITY ? 0.f : m;
            opaque(data);
            const float M = m * te.kscale;
            if (!(fabsf(M) < FAR)) {
                float unused;
                far_sums(z, total, row, V, step, n0, C, m, te.kscale, s, unused);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float y[N];
                    unpack(data[v], y);
#pragma unroll
                    for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f(__builtin_fmaf(y[e], te.kscale, -M));
                }
                s *= __builtin_amdgcn_exp2f(-__builtin_fmaf(m, te.kscale, -M));
            }
            s = wave64(s, Sum());
            if (MULTI) {
                if (lane == 0) red[1][wave] = s;
                __syncthreads();
                s = uniform(row16((lane & 15) < W ? red[1][lane & 15] : 0.f, Sum()));
            }
        }
        bool near, live;
        const float loss = frame_loss_of<1, 64>(te, c, t, x, w, m, s, C, q, near, live);
        if (first) frame_loss[r] = loss;
        if (!dz || near) continue;
        if (!live) {
            if (!(how & ADD)) clear_row<T>(dz, row, V, step, n0, C, how);
            continue;
        }
        // ws (p_c - q_c): at the teacher's columns p and q may be close, so their difference is formed from fp32 values, whatever the rest of the
        // row is made from
        const float ws = (float)((double)w * te.grad_scale * te.tau), M0 = m * te.kscale;  // (a product of two of them may be beyond fp32)
        const bool far = !(fabsf(M0) < FAR);
        const float f0 = far ? ws / s : ws / s * __builtin_amdgcn_exp2f(-__builtin_fmaf(m, te.kscale, -M0));
        const float px = __builtin_amdgcn_exp2f(far ? (x[0] - m) * te.kscale : __builtin_fmaf(x[0], te.kscale, -M0)) * f0;
        const int id = q[0] > 0.f ? c[0] : -1;
        const Replaced cols{id, slot_of<N>(id, row), px - q[0] * ws, q[0] * ws};
        if (far) {
#pragma unroll 1
            for (int v = 0; v < V; ++v) {  // from differences
                const int n = n0 + v * step;
                float y[N];
                unpack(load_vector(z, total, row, n, C), y);
#pragma unroll
                for (int e = 0; e < N; ++e) y[e] = __builtin_amdgcn_exp2f((y[e] - m) * te.kscale) * f0;
                cols.apply(n >> 6, row, y);
                if (n < row.nv) put(dz, row.first + (size_t)n * N, n * N - row.head, C, y, how);
            }
            continue;
        }
        opaque(data);
        // p_c ws = 2^(k x - M) f.  Where f > 0 and the gradient is stored as bf16, f goes into M.  Below 128 the sum is rounded by 2^-18 and the
        // logarithm is off by 2^-17 at most, so that p_c ws is by less than 2^-17 of itself: where that is the result (the columns above are not
        // made this way), bf16 rounds it by up to 2^-8.
        const float folded_M = M0 - __builtin_amdgcn_logf(f0);
        const bool folded = sizeof(D) == 2 && fabsf(folded_M) < 128.f;  // (f <= 0: NaN or an infinity)
        const float M = folded ? folded_M : M0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int n = n0 + v * step;
            float y[N];
            unpack(data[v], y);
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[e], te.kscale, -M));
            if (!folded)
#pragma unroll
                for (int e = 0; e < N; ++e) y[e] *= f0;
            cols.apply(n >> 6, row, y);
            if (n < row.nv) put(dz, row.first + (size_t)n * N, n * N - row.head, C, y, how);
        }
    }
}

// Rows of up to 16 * NV classes, sixteen lanes each.  loss (nullable): one workgroup has all rows, FEW_ROWS at most, and adds the utterances' losses up as well:
// 64 rows of 29 with K = 8 in 4.6 us (65 rows, two launches: 4.8), 16 in 3.2.  Rows of many classes and entries lose by it, 64 of 64 with K = 64 11.7 (10.2),
// 64 of 256 with K = 64 24 (17.5).
template <typename T, typename D, int NV, int R>
__global__ __launch_bounds__(1024) void distill_narrow_k(const T* __restrict__ z, Teacher te, Frames fr,
                                                            float* __restrict__ frame_loss, float* __restrict__ loss, D* __restrict__ dz, int C,
                                                            int accumulate)
{
    __shared__ float few[FEW_ROWS];
    const int l = threadIdx.x & 15;
    const unsigned per = blockDim.x / 16, stride = gridDim.x * per;
    for (unsigned r = blockIdx.x * per + (threadIdx.x >> 4); r < fr.rows; r += stride) {
        const size_t i0 = (size_t)r * C;
        const Frame f = frame_of(fr, r);
        const float w = f != LIVE ? 0.f : weight_of(te, r);
        float here = f == BAD ? NAN : 0.f, g[NV];
        bool near = false, live = false;
#pragma unroll
        for (int j = 0; j < NV; ++j) g[j] = 0.f;
        if (w != 0.f) {
            float m = -INFINITY, s = 0.f, t[R], x[R], q[R];
            int c[R];
#pragma unroll
            for (int j = 0; j < R; ++j) {
                c[j] = -1;
                t[j] = -INFINITY;
                x[j] = 0.f;
                if (l + 16 * j < te.K) {
                    c[j] = te.ids[(size_t)r * te.K + l + 16 * j];
                    if (c[j] != -1) t[j] = te.scores[(size_t)r * te.K + l + 16 * j];
                    if ((unsigned)c[j] < (unsigned)C) x[j] = Elem<T>::load(z, i0 + c[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                g[j] = l + 16 * j < C ? Elem<T>::load(z, i0 + l + 16 * j) : -INFINITY;
                m = fmaxf(m, g[j]);
            }
            m = row16(m, Max());
            m = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                g[j] = __builtin_amdgcn_exp2f(difference(g[j], m, te.kscale));
                s += g[j];
            }
            s = row16(s, Sum());
            here = frame_loss_of<R, 16>(te, c, t, x, w, m, s, C, q, near, live);
            const float ws = (float)((double)w * te.grad_scale * te.tau), scale = ws / s;
#pragma unroll
            for (int j = 0; j < NV; ++j) g[j] *= scale;
#pragma unroll
            for (int k = 0; k < R; ++k)
                for (int i = 0; i < 16 && i + 16 * k < te.K; ++i) {
                    const int ci = __shfl(c[k], i, 16);
                    const float a = __shfl(q[k], i, 16) * ws;
#pragma unroll
                    for (int j = 0; j < NV; ++j) g[j] -= ci == l + 16 * j ? a : 0.f;
                }
        }
        if (l == 0) frame_loss[r] = here;
        if (l == 0 && loss) few[r] = here;
        if (!dz || near || (!live && accumulate)) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (l + 16 * j < C) {
                const size_t i = i0 + l + 16 * j;
                const float v = live ? g[j] : 0.f;
                Elem<D>::store(dz, i, accumulate ? Elem<D>::load(dz, i) + v : v);
            }
    }
    if (!loss) return;
    __syncthreads();
    for (unsigned b = threadIdx.x; b < fr.rows / fr.Tp; b += blockDim.x) {
        double sum = 0.;
        for (unsigned t = 0; t < fr.Tp; ++t) sum += few[b * fr.Tp + t];
        loss[b] = (float)sum;
    }
}

__device__ __forceinline__ double sum64(double v)  // over the wavefront, the same bits in each lane
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Loss and gradient of the frames that are NEAR, from quantities that vanish with the loss.  With d = (x - m) - (t - tm) of the entries,
// y = (d - sum q d) / tau, f(y) = e^y - 1 - y, I = sum e^((x - m) / tau) of the entries, O that of all other classes, less what classes named again
// count twice:
//   log p - log q = y - L     L = sum q (log q - log p) = log(1 + sum q f(y)) + log(1 + O / I)     p - q = q (e^(y - L) - 1)
// so that for different classes nothing cancels, whatever tau is.  (m: the largest score of an entry: below tau^2 / 4 the others' mass is no more than I's.)
// W wavefronts a row; NARROW: rows that may be shorter than a wavefront's vectors, by element.  What bounds it is the loops over entries, one after the
// other: where all rows are NEAR, 50 us for 24000 of 29 with K = 29 beside 9 of the first kernel, 123 for 6000 of 4096 bf16 with K = 64 beside 13; where none
// is, 3 to 4.
template <typename T, typename D, bool NARROW, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void distill_near_k(const T* __restrict__ z, Teacher te, Frames fr, float* __restrict__ frame_loss,
                                                                        D* __restrict__ dz, int C, int how)
{
    constexpr int N = NARROW ? 1 : LANE_VALUES<T>, ROWS = W == 1 ? 4 : 1;
    __shared__ float red[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w0 = W == 1 ? 0 : wave;
    const size_t total = (size_t)fr.rows * C;
    for (unsigned r = blockIdx.x * ROWS + (W == 1 ? wave : 0); r < fr.rows; r += gridDim.x * ROWS) {
        if (reinterpret_cast<const unsigned*>(frame_loss)[r] != NEAR) continue;
        const Row row = NARROW ? Row{(size_t)r * C, 0, C} : row_at<T>(r, C);
        auto scores = [&](int at, float (&x)[N]) {  // of slot `at`
            if constexpr (NARROW) x[0] = at * 64 + lane < C ? Elem<T>::load(z, row.first + at * 64 + lane) : -INFINITY;
            else unpack(load_vector(z, total, row, at * 64 + lane, C), x);
        };
        int c = -1;
        float t = -INFINITY, x = 0.f;
        if (lane < te.K) {
            c = te.ids[(size_t)r * te.K + lane];
            if (c != -1) t = te.scores[(size_t)r * te.K + lane];
            if ((unsigned)c < (unsigned)C) x = Elem<T>::load(z, (size_t)r * C + c);
        }
        const float tm = wave64(t, Max()), raw = expf(difference(t, tm, te.inv_tau)), q = raw * (1.f / wave64(raw, Sum()));
        const bool on = q > 0.f && x > -INFINITY;  // (the second only where q is next to nothing: the loss would be no finite number)
        const int id = on ? c : -1;
        const float m = wave64(on ? x : -INFINITY, Max()), e = on ? __builtin_amdgcn_exp2f(difference(x, m, te.kscale)) : 0.f;
        const double d = on ? ((double)x - m) - ((double)t - tm) : 0., y = (d - sum64(q * d) / sum64(q)) * te.inv_tau;
        const float yf = (float)y;
        double f = 0.;
        if (fabsf(yf) < 0.5f)  // the power series; what it leaves out is below 2^-24 of it
            f = q * (y * y) * (0.5f + yf * (1.f / 6 + yf * (1.f / 24 + yf * (1.f / 120 + yf * (1.f / 720 + yf * (1.f / 5040 + yf * (1.f / 40320)))))));
        else if (on)  // (e^60 and more of a q of 2^-87 and less: their product is of ordinary size)
            f = yf < 60.f ? q * (expf(yf) - 1.f - yf) : expf(logf(q) + yf);
        f = sum64(f);
        bool again = false;
        for (int i = 0; i < te.K; ++i) again |= on && i < lane && __builtin_amdgcn_readlane(id, i) == id;
        const float I = wave64(e, Sum()), twice = wave64(again ? e : 0.f, Sum());
        const Replaced others{id, slot_of<N>(id, row), -INFINITY, 0.f};
        float rest = 0.f;
#pragma unroll 2
        for (int at = w0; at * 64 < row.nv; at += W) {
            float v[N];
            scores(at, v);
            others.apply(at, row, v);
#pragma unroll
            for (int k = 0; k < N; ++k) rest += __builtin_amdgcn_exp2f(difference(v[k], m, te.kscale));
        }
        rest = wave64(rest, Sum());
        if (W > 1) {
            if (lane == 0) red[wave] = rest;
            __syncthreads();
            rest = uniform(row16((lane & 15) < W ? red[lane & 15] : 0.f, Sum()));
            __syncthreads();
        }
        rest -= twice;
        auto log_1p = [](double v) { return fabs(v) < 0x1p-24 ? v : (double)log1pf((float)v); };
        const double L = log_1p(f) + log_1p(rest / I), v = y - L, factor = (double)weight_of(te, r) * te.grad_scale * te.tau;
        const float loss = (float)((double)weight_of(te, r) * te.tau * (te.tau * L));
        if (w0 == 0 && lane == 0) frame_loss[r] = loss;  // (all wavefronts of the row have read it)
        if (!dz) continue;
        const bool live = fabsf(loss) < INFINITY;
        if (!live && (how & ADD)) continue;
        const float ws = live ? (float)factor : 0.f, f0 = ws / (I + rest);
        const double apart = q * (fabs(v) < 0x1p-10 ? v * (1. + 0.5 * v) : (double)expm1f((float)v));
        const Replaced cols{id, slot_of<N>(id, row), live ? (float)(factor * apart) : 0.f, q * ws};
#pragma unroll 2
        for (int at = w0; at * 64 < row.nv; at += W) {
            float v[N];
            scores(at, v);
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f(difference(v[k], m, te.kscale)) * f0;
            cols.apply(at, row, v);
            const int n = at * 64 + lane;
            if constexpr (NARROW) {
                if (n < C) Elem<D>::store(dz, row.first + n, how & ADD ? Elem<D>::load(dz, row.first + n) + v[0] : v[0]);
            } else if (n < row.nv)
                put(dz, row.first + (size_t)n * N, n * N - row.head, C, v, how);
        }
    }
}

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
// Log-probabilities, entropy, best classes.  What a row costs beside its values -- a threshold, a list, ranks: 700 instructions -- it costs every
// wavefront, so a row has few: one up to 24 slots (3000 rows of 20 slots: 22 us; two wavefronts 28, five 38; one row: 9 us either way),
// four to a workgroup beyond.  Workgroups of four that join beat one of up to sixteen that waits at its barriers (400 rows of 137
// slots: 28 us against 33; one row: 14 against 15), and one row in more of them gains little (256 slots: 13.8 us in 8, 14.9 in 4).
Plan plan_tokens(int C, int K, int dtype)
{
    if (C <= 64 || K <= 24)  // (the narrow kernel takes a round for each: 24000 rows of 200: 26 us at K = 16, 78 at 64, where a wavefront a row takes 35)
        if (const int nv = narrow_of(C)) return {0, 1, nv};
    const int slots = slots_of(C, dtype);
    if (slots <= 24) return {1, 1, tight(slots, {2, 4, 6, 8, 10, 12, 14, 16, 20, 24})};
    const int P = (slots + 15) / 16, W = P <= 4 ? P : slots <= 512 ? 4 : 8, G = (P + W - 1) / W;
    return {W, G, tight((slots + W * G - 1) / (W * G), {10, 12, 14, 16})};
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
size_t sums_bytes(long long rows, const Plan& p) { return p.G > 1 ? round_up((size_t)rows * p.G * sizeof(float4), 256) : 0; }
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
template <typename T>
bool launch_rows(const Plan& p, hipStream_t st, const void* z, const int* tokens, const Frames& fr, const TokenOut& o, const Parts& parts,
                 int C, float kscale)
{
    if (p.W > 1)
        return with_slots<10, 12, 14, 16>(p.V, [&](auto v) {
            hipLaunchKernelGGL((token_rows_k<T, decltype(v)::value, true>), dim3(grid_of((long long)fr.rows * p.G)), dim3(64 * p.W), lds_of(p.W, true), st,
                               (const T*)z, tokens, fr, o, parts, C, p.G, kscale);
        });
    return with_slots<2, 4, 6, 8, 10, 12, 14, 16, 20, 24>(p.V, [&](auto v) {
        hipLaunchKernelGGL((token_rows_k<T, decltype(v)::value, false>), dim3(grid_of(((long long)fr.rows + 3) / 4)), dim3(256), lds_of(4, false), st,
                           (const T*)z, tokens, fr, o, parts, C, 1, kscale);
    });
}
template <typename T>
int launch_tokens(const Plan& p, hipStream_t st, const void* z, const int* tokens, const Frames& fr, const TokenOut& o, void* ws, int C, float kscale, bool join)
{
    const Parts parts{(float4*)ws, (ranked_t*)((char*)ws + sums_bytes(fr.rows, p))};
    if (p.W == 0) {
        const dim3 g(grid_of(((long long)fr.rows + 15) / 16)), b(THREADS);
        if (!with_slots<2, 4, 8, 16>(p.V, [&](auto v) {
                hipLaunchKernelGGL((token_narrow_k<T, decltype(v)::value>), g, b, 0, st, (const T*)z, tokens, fr, o, C);
            }))
            return W2L_ERR_SHAPE;
    } else if (!launch_rows<T>(p, st, z, tokens, fr, o, parts, C, kscale))
        return W2L_ERR_SHAPE;
    if (int rc = launch_status()) return rc;
    if (p.G == 1 || !join) return W2L_OK;  // (the partial sums of a distillation are not joined)
    hipLaunchKernelGGL(token_join_k<T>, dim3(grid_of(fr.rows)), dim3(THREADS), 0, st, (const T*)z, tokens, fr, o, parts, C, p.G);
    return launch_status();
}

template <typename T, typename D>
void launch_bwd(hipStream_t st, const void* z, const float* stats, const int* tokens, const float* dlogprob, const float* dentropy, const int* top_ids,
                const float* dtop, const Frames& fr, void* dz, int C, int S, int K, int accumulate)
{
    constexpr int V = 4, N = 16 / sizeof(T);
    if (const int nv = narrow_of(C)) {
        with_slots<2, 4, 8, 16>(nv, [&](auto v) {
            hipLaunchKernelGGL((token_bwd_narrow_k<T, D, decltype(v)::value>), dim3(grid_of(((long long)fr.rows + 15) / 16)), dim3(THREADS), 0, st,
                               (const T*)z, stats, tokens, dlogprob, dentropy, top_ids, dtop, fr, (D*)dz, C, S, K, accumulate);
        });
        return;
    }
    const int slots = (C + 2 * (N - 1) + 64 * N - 1) / (64 * N), P = (slots + V - 1) / V;
    hipLaunchKernelGGL((token_bwd_rows_k<T, D, V>), dim3(grid_of(((long long)fr.rows * P + 3) / 4)), dim3(THREADS), 0, st, (const T*)z, stats, tokens,
                       dlogprob, dentropy, top_ids, dtop, fr, (D*)dz, C, S, K, P, how_of<D>(fr.rows, C, accumulate));
}

// the status of the launch before it, the frames that it left, and the utterances' losses if they are wanted
template <typename T, typename D>
int launch_rest(hipStream_t st, const void* z, const Teacher& te, const Frames& fr, float* frame_loss, float* loss, void* dz, int C, int accumulate)
{
    int rc = launch_status();
    if (!rc && te.tau > WARM) {
        const int how = how_of<D>(fr.rows, C, accumulate);
        if (C <= NARROW)
            hipLaunchKernelGGL((distill_near_k<T, D, true, 1>), dim3(grid_of(((long long)fr.rows + 3) / 4)), dim3(256), 0, st, (const T*)z, te, fr, frame_loss, (D*)dz, C, how);
        else if (C <= 32768)
            hipLaunchKernelGGL((distill_near_k<T, D, false, 4>), dim3(grid_of(fr.rows)), dim3(256), 0, st, (const T*)z, te, fr, frame_loss, (D*)dz, C, how);
        else
            hipLaunchKernelGGL((distill_near_k<T, D, false, 16>), dim3(grid_of(fr.rows)), dim3(1024), 0, st, (const T*)z, te, fr, frame_loss, (D*)dz, C, how);
        rc = launch_status();
    }
    if (rc || !loss) return rc;
    hipLaunchKernelGGL(utterance_loss_k, dim3(grid_of(fr.rows / fr.Tp)), dim3(THREADS), 0, st, frame_loss, loss, fr.rows / fr.Tp, fr.Tp);
    return launch_status();
}
template <typename T, typename D>
int launch_distill(const Plan& p, hipStream_t st, const void* z, const Teacher& te, const Frames& fr, float* frame_loss, float* loss, void* dz, void* ws,
                   int C, int accumulate)
{
    if (p.W == 0) {
        const bool whole = fr.rows <= FEW_ROWS && !(te.tau > WARM);  // then a launch less
        const dim3 g(whole ? 1 : grid_of(((long long)fr.rows + 15) / 16)), b(whole ? 1024 : THREADS);
        float* const sums = whole ? loss : nullptr;
        if (!with_slots<2, 4, 8, 16>(p.V, [&](auto v) {
                if (te.K <= 16)
                    hipLaunchKernelGGL((distill_narrow_k<T, D, decltype(v)::value, 1>), g, b, 0, st, (const T*)z, te, fr, frame_loss, sums, (D*)dz, C,
                                       accumulate);
                else
                    hipLaunchKernelGGL((distill_narrow_k<T, D, decltype(v)::value, 4>), g, b, 0, st, (const T*)z, te, fr, frame_loss, sums, (D*)dz, C,
                                       accumulate);
            }))
            return W2L_ERR_SHAPE;
        return whole ? launch_status() : launch_rest<T, D>(st, z, te, fr, frame_loss, loss, dz, C, accumulate);
    }
    const float4* sums = nullptr;
    int parts = 1;
    if (p.G > 1) {
        const TokenOut none{nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0};
        const Plan first = plan_tokens(C, 0, sizeof(T) == 2 ? W2L_BF16 : W2L_F32);  // (G > 1 as well: more than 64 slots)
        parts = first.G;
        if (int rc = launch_tokens<T>(first, st, z, nullptr, fr, none, ws, C, te.kscale, false)) return rc;
        sums = (const float4*)ws;
    }
    bool known;
    if (p.W > 1)
        known = with_slots<2, 4, 8, 12, 16>(p.V, [&](auto v) {
            hipLaunchKernelGGL((distill_rows_k<T, D, decltype(v)::value, true>), dim3(grid_of((long long)fr.rows * p.G)), dim3(64 * p.W), 0, st, (const T*)z, te,
                               fr, sums, parts, frame_loss, (D*)dz, C, p.G, how_of<D>(fr.rows, C, accumulate));
        });
    else
        known = with_slots<2, 4, 6, 8, 10, 12, 14, 16, 20, 24>(p.V, [&](auto v) {
            hipLaunchKernelGGL((distill_rows_k<T, D, decltype(v)::value, false>), dim3(grid_of(((long long)fr.rows + 3) / 4)), dim3(256), 0, st, (const T*)z, te,
                               fr, sums, 1, frame_loss, (D*)dz, C, 1, how_of<D>(fr.rows, C, accumulate));
        });
    if (!known) return W2L_ERR_SHAPE;
    return launch_rest<T, D>(st, z, te, fr, frame_loss, loss, dz, C, accumulate);
}

}  // namespace

extern "C" size_t w2l_token_logprob_workspace_bytes(int B, int Tp, int C, int K, int z_dtype)
{
    if (!shape_ok(B, Tp, C, 0, K) || !valid_dtype(z_dtype)) return 0;
    const long long rows = (long long)B * Tp;
    const Plan p = plan_tokens(C, K, z_dtype);
    return p.G > 1 ? sums_bytes(rows, p) + (size_t)rows * p.G * K * sizeof(ranked_t) : 0;
}

extern "C" int w2l_token_logprob_fwd(const void* z, const int* tokens, const int* in_len, float* logprob, float* entropy, int* top_ids,
                                     float* top_logprob, float* stats, int B, int Tp, int C, int S, int K, int z_dtype, void* workspace,
                                     size_t ws_bytes, void* stream)
{
    if (!z || (S > 0 && (!tokens || !logprob)) || (K > 0 && (!top_ids || !top_logprob))) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, S, K)) return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(z) || !aligned16(tokens) || !aligned16(in_len) || !aligned16(logprob) || !aligned16(entropy) || !aligned16(top_ids) ||
        !aligned16(top_logprob) || !aligned16(stats))
        return W2L_ERR_ALIGN;
    const size_t rows = (size_t)B * Tp, need = w2l_token_logprob_workspace_bytes(B, Tp, C, K, z_dtype);
    if (!workspace_ok(workspace, ws_bytes, need)) return W2L_ERR_WORKSPACE;
    if (!apart({{z, rows * C * dtype_size(z_dtype)}, {tokens, rows * S * 4}, {in_len, (size_t)B * 4}},
               {{logprob, rows * S * 4}, {entropy, rows * 4}, {top_ids, rows * K * 4}, {top_logprob, rows * K * 4}, {stats, rows * 16}, {workspace, need}}))
        return W2L_ERR_OVERLAP;
    const Frames fr = frames_of(in_len, B, Tp);
    const Plan p = plan_tokens(C, K, z_dtype);
    const TokenOut o{logprob, entropy, top_ids, top_logprob, stats, S, K};
    return z_dtype == W2L_BF16 ? launch_tokens<bf16_t>(p, (hipStream_t)stream, z, tokens, fr, o, workspace, C, LOG2E, true)
                               : launch_tokens<float>(p, (hipStream_t)stream, z, tokens, fr, o, workspace, C, LOG2E, true);
}

extern "C" int w2l_token_logprob_bwd(const void* z, const float* stats, const int* tokens, const float* dlogprob, const float* dentropy,
                                     const int* top_ids, const float* dtop, const int* in_len, void* dz, int B, int Tp, int C, int S, int K,
                                     int z_dtype, int dz_dtype, int accumulate, void* stream)
{
    if (!z || !stats || !dz || (S > 0 && (!tokens || !dlogprob)) || (K > 0 && (!top_ids || !dtop))) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, S, K)) return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype) || !grad_dtype_ok(z_dtype, dz_dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(z) || !aligned16(stats) || !aligned16(tokens) || !aligned16(dlogprob) || !aligned16(dentropy) || !aligned16(top_ids) ||
        !aligned16(dtop) || !aligned16(in_len) || !aligned16(dz))
        return W2L_ERR_ALIGN;
    const size_t rows = (size_t)B * Tp;
    if (!apart({{z, rows * C * dtype_size(z_dtype)}, {stats, rows * 16}, {tokens, rows * S * 4}, {dlogprob, rows * S * 4}, {dentropy, rows * 4},
                {top_ids, rows * K * 4}, {dtop, rows * K * 4}, {in_len, (size_t)B * 4}},
               {{dz, rows * C * dtype_size(dz_dtype)}}))
        return W2L_ERR_OVERLAP;
    const Frames fr = frames_of(in_len, B, Tp);
#define W2L_BWD(T_, G_)                                                                                                                        \
    launch_bwd<T_, G_>((hipStream_t)stream, z, stats, tokens, dlogprob, dentropy, top_ids, dtop, fr, dz, C, S, K, accumulate)
    if (z_dtype == W2L_F32) W2L_BWD(float, float);
    else if (dz_dtype == W2L_F32) W2L_BWD(bf16_t, float);
    else W2L_BWD(bf16_t, bf16_t);
#undef W2L_BWD
    return launch_status();
}

extern "C" size_t w2l_distill_workspace_bytes(int B, int Tp, int C, int K, int z_dtype)
{
    if (!shape_ok(B, Tp, C, 0, K) || !valid_dtype(z_dtype)) return 0;
    const long long rows = (long long)B * Tp;
    return plan_distill(rows, C, z_dtype).G > 1 ? sums_bytes(rows, plan_tokens(C, 0, z_dtype)) : 0;
}

extern "C" int w2l_distill_fwd_bwd(const void* z, const int* t_ids, const float* t_scores, const int* in_len, const float* weight,
                                   float* frame_loss, float* loss, void* dz, int B, int Tp, int C, int K, float temperature, float grad_scale,
                                   int z_dtype, int dz_dtype, int accumulate, void* workspace, size_t ws_bytes, void* stream)
{
    if (!z || !t_ids || !t_scores || !frame_loss) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, 0, K) || K < 1 || !(temperature > 0.f) || !isnormal(temperature) || !isnormal(1.f / temperature) || !isfinite(grad_scale))
        return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype) || !grad_dtype_ok(z_dtype, dz_dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(z) || !aligned16(t_ids) || !aligned16(t_scores) || !aligned16(in_len) || !aligned16(weight) || !aligned16(frame_loss) ||
        !aligned16(loss) || !aligned16(dz))
        return W2L_ERR_ALIGN;
    const size_t rows = (size_t)B * Tp, need = w2l_distill_workspace_bytes(B, Tp, C, K, z_dtype);
    if (!workspace_ok(workspace, ws_bytes, need)) return W2L_ERR_WORKSPACE;
    if (!apart({{z, rows * C * dtype_size(z_dtype)}, {t_ids, rows * K * 4}, {t_scores, rows * K * 4}, {in_len, (size_t)B * 4}, {weight, rows * 4}},
               {{frame_loss, rows * 4}, {loss, (size_t)B * 4}, {dz, rows * C * dtype_size(dz_dtype)}, {workspace, need}}))
        return W2L_ERR_OVERLAP;
    const Frames fr = frames_of(in_len, B, Tp);
    const Plan p = plan_distill(fr.rows, C, z_dtype);
    const Teacher te{t_ids, t_scores, weight, K, temperature, 1.f / temperature, (float)(1.4426950408889634 / temperature), grad_scale};
    int rc;
#define W2L_DISTILL(T_, G_) rc = launch_distill<T_, G_>(p, (hipStream_t)stream, z, te, fr, frame_loss, loss, dz, workspace, C, accumulate)
    if (z_dtype == W2L_F32) W2L_DISTILL(float, float);
    else if (dz_dtype == W2L_F32) W2L_DISTILL(bf16_t, float);
    else W2L_DISTILL(bf16_t, bf16_t);
#undef W2L_DISTILL
    return rc;
}

extern "C" int w2l_token_logprob_launch_config(int B, int Tp, int C, int K, int z_dtype, int* wavefronts, int* groups, int* slots)
{
    if (!wavefronts || !groups || !slots) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, 0, K)) return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype)) return W2L_ERR_DTYPE;
    const Plan p = plan_tokens(C, K, z_dtype);
    *wavefronts = p.W;
    *groups = p.G;
    *slots = p.V;
    return W2L_OK;
}

extern "C" int w2l_distill_launch_config(int B, int Tp, int C, int K, int z_dtype, int* wavefronts, int* groups, int* slots)
{
    if (!wavefronts || !groups || !slots) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, 0, K) || K < 1) return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype)) return W2L_ERR_DTYPE;
    const Plan p = plan_distill((long long)B * Tp, C, z_dtype);
    *wavefronts = p.W;
    *groups = p.G;
    *slots = p.V;
    return W2L_OK;
}

extern "C" int w2l_frame_ids_check_host(const int* ids, const int* in_len, int B, int Tp, int C, int n)
{
    if (!ids) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, n, 0)) return W2L_ERR_SHAPE;
    for (int b = 0; b < B; ++b) {
        const int len = in_len ? in_len[b] : Tp;
        if (len < 0 || len > Tp) return W2L_ERR_TARGET;
        for (size_t i = (size_t)b * Tp * n; i < ((size_t)b * Tp + len) * n; ++i)
            if (ids[i] < -1 || ids[i] >= C) return W2L_ERR_TARGET;
    }
    return W2L_OK;
}
