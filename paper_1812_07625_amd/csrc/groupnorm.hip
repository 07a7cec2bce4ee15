// Group norm over [B,T,C], channels last, and the activation behind it: w2l_groupnorm_fwd / _bwd.  Two ways:
//   runs of frames     norm_stats_k: every group's sum and sum of squares in a run of an utterance's frames;
//                      norm_apply_k: joins the runs of an utterance, normalises, applies the activation;
//                      norm_sums_k: sums over a run of du and du xhat of every channel, and of both times gamma of every group;
//                      norm_dx_k: joins them and writes dx; workgroups of its own add up dgamma and dbeta
//                      (norm_join_runs_k before norm_apply_k and norm_dx_k where an utterance has so many runs that they are joined once)
//   a workgroup a group  norm_group_k, norm_group_bwd_k (and norm_join_k for dgamma and dbeta): groups that one workgroup reads twice
// What bounds them is memory where a batch is large (16x1500x2048 bf16, one group, 20000 live frames: both calls together move 723 MB in 140 us, 5.2 TB/s), and where
// it is small the launches and a chain of loads, sums over lanes, and stores (3.6 us a launch).  The second reading finds in the caches what they hold.
// A thread has a vector of N neighbouring channels (16 bytes where groups are whole vectors, less where they are not) in some rows; what it
// knows of its channels stays in registers from row to row.
#include "lanes.h"

#include <algorithm>
#include <type_traits>

using namespace w2l;

namespace {

constexpr int MAX_CHANNELS = 8192, MAX_FRAMES = 1 << 24, MAX_THREADS = 512, BATCH = 4, JOIN_CHANNELS = 16, JOIN_GROUPS = 8, JOIN_THREADS = 256;  // (8192: a lane's pairs of floats of all channels fit 64 KB of LDS; norm_stats_k's pairs of 64-bit sums, one a vector, are 128 of its 160 where vectors are of one channel)

// A vector of N neighbouring channels as it lies in memory, and its values
template <typename T, int N> struct Vec {
    typedef unsigned raw __attribute__((ext_vector_type(N * sizeof(T) / 4)));
};
template <> struct Vec<float, 1> { typedef unsigned raw; };
template <> struct Vec<bf16_t, 2> { typedef unsigned raw; };
template <> struct Vec<bf16_t, 1> { typedef unsigned short raw; };
template <typename T, int N> using raw_t = typename Vec<T, N>::raw;

template <typename T, int N>
__device__ __forceinline__ raw_t<T, N> fetch(const T* p) { return *reinterpret_cast<const raw_t<T, N>*>(p); }
template <typename T, int N>
__device__ __forceinline__ void unpack(raw_t<T, N> q, float (&x)[N])
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (N == 1) x[0] = __uint_as_float(q);
        else
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = __uint_as_float(q[j]);
    } else if constexpr (N == 1) x[0] = bf16_to_f32(q);
    else
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            unsigned w;
            if constexpr (N == 2) w = q;
            else w = q[j];
            x[2 * j] = __uint_as_float(w << 16);
            x[2 * j + 1] = __uint_as_float(w & 0xffff0000u);
        }
}
// PAST: past the caches.  Outputs of runs of frames (16x1500x1536 bf16, SiLU: 52 -> 41 us, 77 -> 71 with a pass behind it that reads them), not of a workgroup a group,
// whose stores fill lines in parts (8x750x1536 in 32 groups: 13.6, 16.6 past them).
template <typename T, int N, bool PAST>
__device__ __forceinline__ void put(T* p, const float (&x)[N])
{
    raw_t<T, N> q;
    if constexpr (sizeof(T) == 4) {
        if constexpr (N == 1) q = __float_as_uint(x[0]);
        else
#pragma unroll
            for (int j = 0; j < N; ++j) q[j] = __float_as_uint(x[j]);
    } else if constexpr (N == 1) q = f32_to_bf16(x[0]);
    else
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            typedef float float2_t __attribute__((ext_vector_type(2)));
            typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
            const unsigned w = __builtin_bit_cast(unsigned, __builtin_convertvector((float2_t){x[2 * j], x[2 * j + 1]}, bf16x2_t));
            if constexpr (N == 2) q = w;
            else q[j] = w;
        }
    if (PAST) __builtin_nontemporal_store(q, reinterpret_cast<raw_t<T, N>*>(p));
    else *reinterpret_cast<raw_t<T, N>*>(p) = q;
}

// How a workgroup takes a run of `rows` frames: `cols` threads side by side, `lanes` rows at a time
struct Shape {
    int B, T, C, G, Cg, rows, runs, cols, lanes, split;
    const int* in_len;
    float inv_Cg, inv_cols;
    int joined = 0;  // the sums of an utterance's runs are joined already, in the place of its first run's
    __device__ __forceinline__ int runs_to_join(int len) const { return joined && len > 0 ? 1 : (len + rows - 1) / rows; }
    // column and row of a thread (a thousand of them at most: see group_of)
    __device__ __forceinline__ void place(int& col, int& lane) const
    {
        lane = (int)(((float)threadIdx.x + 0.5f) * inv_cols);
        col = (int)threadIdx.x - lane * cols;
    }
};
// Task i's utterance and run of frames.  Runs that are the same of every utterance follow one another, so that those behind short utterances' ends come last and
// take no place from others; the utterances are rotated from run to run, so that long and short ones are spread over the XCDs.
struct Task {
    int b, run;
};
__device__ __forceinline__ Task task_of(const Shape& s, unsigned i)
{
    const unsigned run = i / (unsigned)s.B, k = i - run * s.B + run % (unsigned)s.B;
    return {(int)(k < (unsigned)s.B ? k : k - s.B), (int)run};
}
// frames of utterance b; -1: its in_len is out of range
__device__ __forceinline__ int frames_of(const Shape& s, int b)
{
    if (!s.in_len) return s.T;
    const int n = s.in_len[b];
    return n < 0 || n > s.T ? -1 : n;
}

// ---- activations ---------------------------------------------------------------------------------------------
// y = act(u), du = dy act'(u).  GLU takes a value and a gate, and gives the gradient of both.
__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u * -1.44269504088896f)); }
template <int ACT>
__device__ __forceinline__ float act(float u, float gate)
{
    if (ACT == W2L_ACT_RELU) return u > 0.f ? u : u == u ? 0.f : u;
    if (ACT == W2L_ACT_SILU) return u * sigmoid(u);
    if (ACT == W2L_ACT_GLU) return u * sigmoid(gate);
    return u;
}
template <int ACT>
__device__ __forceinline__ void act_bwd(float u, float gate, float dy, float& du, float& dgate)
{
    if (ACT == W2L_ACT_RELU) du = u > 0.f ? dy : u == u ? 0.f : u;
    else if (ACT == W2L_ACT_SILU) {
        const float s = sigmoid(u);
        du = dy * s * (1.f + u * (1.f - s));
    } else if (ACT == W2L_ACT_GLU) {
        const float s = sigmoid(gate);
        du = dy * s;
        dgate = dy * u * s * (1.f - s);
    } else
        du = dy;
}

// ---- statistics ----------------------------------------------------------------------------------------------
// A thread sums its channels' deviations from the first value it reads of each, and their squares.  With n values that first one is at most
// sqrt(n) deviations off the mean of the n, so that the sums lose at most a factor of n (64 at most) of fp32's precision, whatever the
// channel's level.  From there on a group's sum and sum of squares are in 64 bits, where the difference of mean square and squared mean loses nothing that
// counts: a level of 10^5 deviations leaves 10^-6 of the variance.
template <int N>
struct Deviations {
    float base[N], sum[N], sq[N];
    int n;
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int j = 0; j < N; ++j) base[j] = sum[j] = sq[j] = 0.f;
        n = 0;
    }
    __device__ __forceinline__ void add(const float (&y)[N])
    {
        if (n == 0)
#pragma unroll
            for (int j = 0; j < N; ++j) base[j] = y[j];
        ++n;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float d = y[j] - base[j];
            sum[j] += d;
            sq[j] = __builtin_fmaf(d, d, sq[j]);
        }
    }
    // sum and sum of squares of all, where the channels are of one group
    __device__ __forceinline__ double2 group_sums() const
    {
        const float inv = n ? 1.f / (float)n : 0.f;
        float mean[N], q = 0.f, off = 0.f, about = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float m = sum[j] * inv;
            mean[j] = base[j] + m;
            q += __builtin_fmaf(-m, sum[j], sq[j]);
            off += mean[j] - mean[0];
        }
        const float m = off * (1.f / N);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float d = (mean[j] - mean[0]) - m;
            about = __builtin_fmaf(d, d, about);
        }
        const double k = (double)n * N, all = (double)mean[0] + m;
        return make_double2(k * all, k * all * all + (double)__builtin_fmaf((float)n, about, q));
    }
};
__device__ __forceinline__ double2 sum64(double2 v, int width)
{
    for (int o = width >> 1; o > 0; o >>= 1) {
        v.x += __shfl_xor(v.x, o, 64);
        v.y += __shfl_xor(v.y, o, 64);
    }
    return v;
}
// lanes that add up a group's partial results: as many as there are threads for, a power of two up to a wavefront and no more than there are results
__device__ __forceinline__ int team_of(int G, int results)
{
    int team = 64;
    while (team > 1 && (G * team > (int)blockDim.x || team >= 2 * results)) team >>= 1;
    return team;
}

__device__ __forceinline__ float2 sum64(float2 v, int width)
{
    for (int o = width >> 1; o > 0; o >>= 1) {
        v.x += __shfl_xor(v.x, o, 64);
        v.y += __shfl_xor(v.y, o, 64);
    }
    return v;
}
// out(g, sum of value(r, c) over r < rows and the group's entries c < per) for every group.  Where groups are fewer than the workgroup's teams, several teams share one
// (16x1500x2048 bf16 in one group: 34 -> 26 us for norm_stats_k).  lds: a V for every wavefront
// (only teams of a whole wavefront share a group: fewer lanes are taken where they are enough for it)
template <typename V, typename F, typename O>
__device__ __forceinline__ void sum_groups(int G, int rows, int per, V* lds, F value, O out)
{
    const int team = team_of(G, per), l = threadIdx.x & (team - 1), teams = blockDim.x / team, mine = threadIdx.x / team;
    int shares = teams / G;
    if ((shares - 1) * team >= per) shares = (per + team - 1) / team;
    if (shares <= 1) {
        for (int g0 = 0; g0 < G; g0 += teams) {
            const int g = g0 + mine;
            V k{};
            if (g < G)
                for (int r = 0; r < rows; ++r)
                    for (int c = l; c < per; c += team) {
                        const V o = value(g, r, c);
                        k.x += o.x;
                        k.y += o.y;
                    }
            k = sum64(k, team);
            if (g < G && l == 0) out(g, k);
        }
        return;
    }
    const int g = mine % G, share = mine / G;
    V k{};
    if (share < shares)
        for (int r = 0; r < rows; ++r)
            for (int c = share * team + l; c < per; c += team * shares) {
                const V o = value(g, r, c);
                k.x += o.x;
                k.y += o.y;
            }
    k = sum64(k, team);
    if (l == 0) lds[mine] = k;
    __syncthreads();
    if ((int)threadIdx.x < G) {
        V all = lds[threadIdx.x];
        for (int i = 1; i < shares; ++i) {
            all.x += lds[i * G + threadIdx.x].x;
            all.y += lds[i * G + threadIdx.x].y;
        }
        out((int)threadIdx.x, all);
    }
}

// sums [B][runs][G]: sum and sum of squares of a run
template <typename T, int N>
__global__ __launch_bounds__(MAX_THREADS) void norm_stats_k(const T* __restrict__ x, Shape s, double2* __restrict__ sums)
{
    extern __shared__ double2 lds[];  // [lanes][vectors]: a thread's sums
    __shared__ double2 part[MAX_THREADS / 64];
    constexpr int U = BATCH;
    const Task task = task_of(s, blockIdx.x);
    const int b = task.b, run = task.run, len = frames_of(s, b);
    const int t0 = run * s.rows, t1 = t0 + s.rows < len ? t0 + s.rows : len;
    if (t0 >= t1) return;  // (what reads the sums knows that there are none)
    int col, lane;
    s.place(col, lane);
    const int nv = s.C / N, here = t1 - t0;
    if (lane < s.lanes)
        for (int v = col; v < nv; v += s.cols) {
            const T* const p = x + ((size_t)b * s.T + t0) * s.C + (size_t)v * N;
            Deviations<N> d;
            d.clear();
            for (int t = lane; t < here; t += U * s.lanes) {
                raw_t<T, N> q[U];
#pragma unroll
                for (int k = 0; k < U; ++k) q[k] = fetch<T, N>(p + (size_t)(t + k * s.lanes < here ? t + k * s.lanes : t) * s.C);
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if (t + k * s.lanes >= here) break;
                    float y[N];
                    unpack<T, N>(q[k], y);
                    d.add(y);
                }
            }
            lds[lane * nv + v] = d.group_sums();
        }
    __syncthreads();
    const int live = here < s.lanes ? here : s.lanes;  // lanes that had a frame
    const int per = s.Cg / N;
    sum_groups<double2>(s.G, live, per, part, [&](int g, int r, int c) { return lds[r * nv + g * per + c]; },
                        [&](int g, double2 k) { sums[((size_t)b * s.runs + run) * s.G + g] = k; });
}

// mean and 1 / deviation from a group's sums; inv: 1 / its values (0: it has none).  A variance that fp32 does not hold (a thread's squares are fp32 too) is none: 1 / sqrt(inf)
// would be 0, every value would become beta, and every gradient 0.
__device__ __forceinline__ float2 stat_of(double2 k, double inv, float eps)
{
    const double mean = k.x * inv, var = k.y * inv - mean * mean;
    const float sum = (var < 0. ? 0.f : (float)var) + eps;
    if (!(sum < INFINITY)) return make_float2(NAN, NAN);
    return make_float2((float)mean, inv > 0. ? 1.f / sqrtf(sum) : 0.f);
}
// A lane's share of the sums of a group's runs, from p on, a row of G groups each.  Where they are many, eight loads are in flight at once (in one utterance of
// 2000x2048 with 64 groups, fp32, 39 -> 17 us for the forward call, together with the longer runs of runs_of); where they are few, the masked ones would cost 1 us.
template <typename A, typename V>
__device__ __forceinline__ A sum_runs(const V* __restrict__ p, int G, int runs, int l, int team)
{
    constexpr int U = 8;
    A k{};
    int r = l;
    for (; r + (U - 1) * team < runs; r += U * team) {
        V o[U];
#pragma unroll
        for (int i = 0; i < U; ++i) o[i] = p[(size_t)(r + i * team) * G];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            k.x += o[i].x;
            k.y += o[i].y;
        }
    }
#pragma unroll 4
    for (; r < runs; r += team) {
        const V o = p[(size_t)r * G];
        k.x += o.x;
        k.y += o.y;
    }
    return k;
}
// of every group of utterance b, into LDS
__device__ __forceinline__ void join_stats(const Shape& s, const double2* __restrict__ sums, int b, int len, float eps, float2* stat)
{
    const int runs = s.runs_to_join(len), team = team_of(s.G, runs), l = threadIdx.x & (team - 1), teams = blockDim.x / team;
    const double inv = len > 0 ? 1. / ((double)len * s.Cg) : 0.;
    for (int g0 = 0; g0 < s.G; g0 += teams) {
        const int g = g0 + threadIdx.x / team;
        double2 k = make_double2(0., 0.);
        if (g < s.G) k = sum_runs<double2>(sums + (size_t)b * s.runs * s.G + g, s.G, runs, l, team);
        k = sum64(k, team);
        if (g < s.G && l == 0) stat[g] = stat_of(k, inv, eps);
    }
    __syncthreads();
}

// The sums of groups' runs in a launch of its own, into the place of the first run's, for kernels whose workgroups would each read them all: `width` neighbouring groups
// a workgroup, whose threads take runs in turn and add up in 64 bits.
template <typename V>
__global__ __launch_bounds__(JOIN_THREADS) void norm_join_runs_k(Shape s, V* sums, int width)
{
    __shared__ double2 lds[JOIN_THREADS / 64 * JOIN_GROUPS];
    const int len = frames_of(s, blockIdx.y), l = threadIdx.x & (width - 1), g = blockIdx.x * width + l, wave = threadIdx.x / 64;
    V* const at = sums + (size_t)blockIdx.y * s.runs * s.G + g;
    double2 k = make_double2(0., 0.);
    if (g < s.G && len > 0) k = sum_runs<double2>((const V*)at, s.G, (len + s.rows - 1) / s.rows, threadIdx.x / width, JOIN_THREADS / width);
    for (int o = 32; o >= width; o >>= 1) {
        k.x += __shfl_xor(k.x, o, 64);
        k.y += __shfl_xor(k.y, o, 64);
    }
    if ((int)(threadIdx.x & 63) < width) lds[wave * width + l] = k;
    __syncthreads();  // (and all runs have been read)
    if ((int)threadIdx.x >= width || g >= s.G || len <= 0) return;
    for (int i = 1; i < JOIN_THREADS / 64; ++i) {
        k.x += lds[i * width + l].x;
        k.y += lds[i * width + l].y;
    }
    V o;
    o.x = k.x;
    o.y = k.y;
    *at = o;
}

// Values of channels c0 .. c0 + N of a vector over channels; `none` where there is none
template <int N>
__device__ __forceinline__ void channels_of(const float* __restrict__ p, int c0, float none, float (&out)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = none;
    if (!p) return;
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const float4 q = *reinterpret_cast<const float4*>(p + c0 + j);
            out[j] = q.x; out[j + 1] = q.y; out[j + 2] = q.z; out[j + 3] = q.w;
        }
    } else
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = p[c0 + j];
}
// c / Cg: (c + 1/2) / Cg is off by less than 8192 * 2^-22 / Cg, and no whole number is nearer than 1/2 / Cg
__device__ __forceinline__ int group_of(const Shape& s, int c) { return (int)(((float)c + 0.5f) * s.inv_Cg); }
// What a thread keeps of its N channels, which are all of one group: u = (x - mean) scale + shift
template <int N>
struct Affine {
    float mean, scale[N], shift[N];
    __device__ __forceinline__ void load(const float* __restrict__ gamma, const float* __restrict__ beta, int c0)
    {
        channels_of<N>(gamma, c0, 1.f, scale);
        channels_of<N>(beta, c0, 0.f, shift);
    }
    __device__ __forceinline__ void set(float2 stat)  // mean and rstd
    {
        mean = stat.x;
#pragma unroll
        for (int j = 0; j < N; ++j) scale[j] *= stat.y;
    }
    __device__ __forceinline__ float operator()(float x, int j) const { return __builtin_fmaf(x - mean, scale[j], shift[j]); }
};

template <typename T, int N, int ACT>
__global__ __launch_bounds__(MAX_THREADS) __attribute__((amdgpu_waves_per_eu(4))) void norm_apply_k(const T* __restrict__ x, Shape s, const double2* __restrict__ sums, const float* __restrict__ gamma,
                                                            const float* __restrict__ beta, float eps, T* __restrict__ y, float* __restrict__ mean,
                                                            float* __restrict__ rstd)
{
    extern __shared__ float2 stat[];
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    constexpr int U = BATCH;
    const Task task = task_of(s, blockIdx.x);
    const int b = task.b, run = task.run, len = frames_of(s, b), Cy = GLU ? s.C / 2 : s.C;
    const int t0 = run * s.rows, t1 = t0 + s.rows < s.T ? t0 + s.rows : s.T, live = t1 < len ? t1 : len;
    int col, lane;
    s.place(col, lane);
    const int nv = Cy / N;
    const T* const in = x + (size_t)b * s.T * s.C;
    // what a thread reads first is on its way while the statistics are joined
    raw_t<T, N> xv[U], xg[U];
    Affine<N> a, h;
    auto load = [&](int v, int t) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const T* const at = in + (size_t)(t + k * s.lanes < live ? t + k * s.lanes : t) * s.C + (size_t)v * N;
            xv[k] = fetch<T, N>(at);
            if (GLU) xg[k] = fetch<T, N>(at + Cy);
        }
    };
    auto load_channels = [&](int v) {
        a.load(gamma, beta, v * N);
        if (GLU) h.load(gamma, beta, Cy + v * N);
    };
    if (lane < s.lanes && t0 + lane < live) {
        load(col, t0 + lane);
        load_channels(col);
    }
    if (run == 0 || t0 < len) join_stats(s, sums, b, len < 0 ? 0 : len, eps, stat);
    if (run == 0)
        for (int g = threadIdx.x; g < s.G; g += blockDim.x) {
            mean[(size_t)b * s.G + g] = len < 0 ? NAN : stat[g].x;
            rstd[(size_t)b * s.G + g] = len < 0 ? NAN : stat[g].y;
        }
    if (lane >= s.lanes) return;
    for (int v = col; v < nv; v += s.cols) {
        T* const q = y + (size_t)b * s.T * Cy + (size_t)v * N;
        int t = t0 + lane;
        if (t < live) {
            if (v != col) {
                load(v, t);
                load_channels(v);
            }
            a.set(stat[group_of(s, v * N)]);
            if (GLU) h.set(stat[group_of(s, Cy + v * N)]);
        }
        while (t < live) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (t + k * s.lanes >= live) break;
                float u[N], w[N];
                unpack<T, N>(xv[k], u);
                if (GLU) unpack<T, N>(xg[k], w);
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] = act<ACT>(a(u[j], j), GLU ? h(w[j], j) : 0.f);
                put<T, N, true>(q + (size_t)(t + k * s.lanes) * Cy, u);
            }
            t += U * s.lanes;
            if (t < live) load(v, t);
        }
        if (t1 > live) {
            float none[N];
#pragma unroll
            for (int j = 0; j < N; ++j) none[j] = len < 0 ? NAN : 0.f;
            for (t = (live > t0 ? live : t0) + lane; t < t1; t += s.lanes) put<T, N, true>(q + (size_t)t * Cy, none);
        }
    }
}

// ---- gradients -----------------------------------------------------------------------------------------------
// chans [B][runs][2][C]: sums of du and du xhat over a run;  groups [B][runs][G][2]: both times gamma
template <typename T, int N, int ACT>
__global__ __launch_bounds__(MAX_THREADS) __attribute__((amdgpu_waves_per_eu(4))) void norm_sums_k(const T* __restrict__ x, const T* __restrict__ dy, Shape s, const float* __restrict__ mean,
                                                           const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                           float* __restrict__ chans, float2* __restrict__ groups)
{
    extern __shared__ float2 acc[];  // [lanes][C]: a lane's sums
    __shared__ float2 part[MAX_THREADS / 64];
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    constexpr int U = 2;
    const Task task = task_of(s, blockIdx.x);
    const int b = task.b, run = task.run, len = frames_of(s, b), Cy = GLU ? s.C / 2 : s.C;
    const int t0 = run * s.rows, t1 = t0 + s.rows < len ? t0 + s.rows : len;
    if (t0 >= t1) return;
    int col, lane;
    s.place(col, lane);
    const int nv = Cy / N;
    if (lane < s.lanes)
        for (int v = col; v < nv; v += s.cols) {
            Affine<N> a, h;
            auto stat_of = [&](int c) { return make_float2(mean[(size_t)b * s.G + group_of(s, c)], rstd[(size_t)b * s.G + group_of(s, c)]); };
            const float2 st = stat_of(v * N), gt = GLU ? stat_of(Cy + v * N) : st;
            a.load(gamma, beta, v * N);
            a.set(st);
            if (GLU) {
                h.load(gamma, beta, Cy + v * N);
                h.set(gt);
            }
            float s1[N], s2[N], r1[N], r2[N];
#pragma unroll
            for (int j = 0; j < N; ++j) s1[j] = s2[j] = r1[j] = r2[j] = 0.f;
            const T* const p = x + (size_t)b * s.T * s.C + (size_t)v * N;
            const T* const q = dy + (size_t)b * s.T * Cy + (size_t)v * N;
            for (int t = t0 + lane; t < t1; t += U * s.lanes) {
                raw_t<T, N> xv[U], xg[U], dv[U];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const size_t at = t + k * s.lanes < t1 ? t + k * s.lanes : t;
                    xv[k] = fetch<T, N>(p + at * s.C);
                    if (GLU) xg[k] = fetch<T, N>(p + at * s.C + Cy);
                    dv[k] = fetch<T, N>(q + at * Cy);
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if (t + k * s.lanes >= t1) break;
                    float xk[N], gk[N], d[N];
                    unpack<T, N>(xv[k], xk);
                    if (GLU) unpack<T, N>(xg[k], gk);
                    unpack<T, N>(dv[k], d);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        float du, dg = 0.f;
                        act_bwd<ACT>(a(xk[j], j), GLU ? h(gk[j], j) : 0.f, d[j], du, dg);
                        s1[j] += du;
                        s2[j] = __builtin_fmaf(du, xk[j] - a.mean, s2[j]);
                        if (GLU) {
                            r1[j] += dg;
                            r2[j] = __builtin_fmaf(dg, gk[j] - h.mean, r2[j]);
                        }
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                acc[(size_t)lane * s.C + v * N + j] = make_float2(s1[j], s2[j] * st.y);
                if (GLU) acc[(size_t)lane * s.C + Cy + v * N + j] = make_float2(r1[j], r2[j] * gt.y);
            }
        }
    __syncthreads();
    float* const out = chans + ((size_t)b * s.runs + run) * 2 * s.C;
    for (int c = threadIdx.x; c < s.C; c += blockDim.x) {
        float2 k = acc[c];
        for (int r = 1; r < s.lanes; ++r) {
            const float2 o = acc[(size_t)r * s.C + c];
            k.x += o.x;
            k.y += o.y;
        }
        out[c] = k.x;
        out[s.C + c] = k.y;
        const float gm = gamma ? gamma[c] : 1.f;
        acc[c] = make_float2(k.x * gm, k.y * gm);  // (row 0 of this channel is read by this thread alone)
    }
    __syncthreads();
    sum_groups<float2>(s.G, 1, s.Cg, part, [&](int g, int, int c) { return acc[(size_t)g * s.Cg + c]; },
                       [&](int g, float2 k) { groups[((size_t)b * s.runs + run) * s.G + g] = k; });
}

// dgamma and dbeta of `width` channels from `count` rows [2][C] of sums (dbeta's, dgamma's), those that are there(row): threads take rows in turn, and their sums are
// added up in 64 bits and a fixed order.  All loads of a batch are in flight at once.
template <typename F>
__device__ __forceinline__ void sum_channels(const float* __restrict__ chans, int count, int C, int block, int width, double2* lds, float* __restrict__ dgamma,
                                             float* __restrict__ dbeta, int accumulate, F there)
{
    constexpr int U = 8;
    const int l = threadIdx.x & (width - 1), first = threadIdx.x / width, step = blockDim.x / width, c = block * width + l;
    double2 k = make_double2(0., 0.);
    if (c < C)
        for (int i = first; i < count; i += U * step) {
            float gv[U], hv[U];
            bool on[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int r = i + j * step < count ? i + j * step : i;
                const float* const p = chans + (size_t)r * 2 * C + c;
                hv[j] = p[0];
                gv[j] = p[C];
                on[j] = i + j * step < count && there(r);
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                k.x += on[j] ? gv[j] : 0.f;
                k.y += on[j] ? hv[j] : 0.f;
            }
        }
    for (int o = 32; o >= width; o >>= 1) {
        k.x += __shfl_xor(k.x, o, 64);
        k.y += __shfl_xor(k.y, o, 64);
    }
    const int waves = blockDim.x / 64, wave = threadIdx.x / 64;
    if ((int)(threadIdx.x & 63) < width) lds[wave * width + l] = k;
    __syncthreads();
    if (first != 0 || c >= C) return;
    for (int i = 1; i < waves; ++i) {
        k.x += lds[i * width + l].x;
        k.y += lds[i * width + l].y;
    }
    if (dgamma) dgamma[c] = (float)(accumulate ? dgamma[c] + k.x : k.x);
    if (dbeta) dbeta[c] = (float)(accumulate ? dbeta[c] + k.y : k.y);
}

// Workgroups from `ahead` on: dx of a run of frames.  Those before them make dgamma and dbeta, whose longer chains of loads start first; they are a multiple of
// eight, so that a run is read on the XCD that read it in norm_sums_k (8x750x1536 bf16, GLU: 35 -> 26 us for the two kernels).
template <typename T, int N, int ACT>
__global__ __launch_bounds__(MAX_THREADS) __attribute__((amdgpu_waves_per_eu(4))) void norm_dx_k(const T* __restrict__ x, const T* __restrict__ dy, Shape s, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                         const float* __restrict__ chans, const float2* __restrict__ groups, T* __restrict__ dx,
                                                         float* __restrict__ dgamma, float* __restrict__ dbeta, int accumulate, int ahead, int width)
{
    extern __shared__ double2 lds[];  // [G] of floats: means of du gamma and du gamma xhat
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    constexpr int U = 2;
    const int Cy = GLU ? s.C / 2 : s.C;
    if ((int)blockIdx.x < ahead) {
        // (runs that are not there left nothing: what lies in their place is not added)
        sum_channels(chans, s.B * s.runs, s.C, blockIdx.x, width, lds, dgamma, dbeta, accumulate, [&](int i) {
            const int u = i / s.runs;
            return (i - u * s.runs) * s.rows < frames_of(s, u);
        });
        return;
    }
    const Task task = task_of(s, blockIdx.x - ahead);
    const int b = task.b, run = task.run, len = frames_of(s, b), t0 = run * s.rows, t1 = t0 + s.rows < s.T ? t0 + s.rows : s.T, live = t1 < len ? t1 : len;
    float2* const means = reinterpret_cast<float2*>(lds);
    int col, lane;
    s.place(col, lane);
    const int nv = Cy / N;
    const size_t row0 = (size_t)b * s.T;
    // what a thread reads first is on its way while the means are joined
    raw_t<T, N> xv[U], xg[U], dv[U];
    Affine<N> a, h;
    auto load = [&](int v, int t) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const size_t at = row0 + (t + k * s.lanes < live ? t + k * s.lanes : t);
            xv[k] = fetch<T, N>(x + at * s.C + (size_t)v * N);
            if (GLU) xg[k] = fetch<T, N>(x + at * s.C + Cy + (size_t)v * N);
            dv[k] = fetch<T, N>(dy + at * Cy + (size_t)v * N);
        }
    };
    auto load_channels = [&](int v) {
        a.load(gamma, beta, v * N);
        if (GLU) h.load(gamma, beta, Cy + v * N);
    };
    if (lane < s.lanes && t0 + lane < live) {
        load(col, t0 + lane);
        load_channels(col);
    }
    if (t0 < len) {
        const int runs = s.runs_to_join(len);
        const float inv = 1.f / ((float)len * (float)s.Cg);
        const int team = team_of(s.G, runs), l = threadIdx.x & (team - 1), teams = blockDim.x / team;
        for (int g0 = 0; g0 < s.G; g0 += teams) {
            const int g = g0 + threadIdx.x / team;
            float2 k = make_float2(0.f, 0.f);
            if (g < s.G) k = sum_runs<float2>(groups + (size_t)b * s.runs * s.G + g, s.G, runs, l, team);
            k = sum64(k, team);
            if (g < s.G && l == 0) means[g] = make_float2(k.x * inv, k.y * inv);
        }
        __syncthreads();
    }
    if (lane >= s.lanes) return;
    for (int v = col; v < nv; v += s.cols) {
        // dx = du gamma rstd + (x - mean) slope + level, slope = - rstd^2 m2, level = - rstd m1
        float2 line = make_float2(0.f, 0.f), gline = line;
        T* const o = dx + row0 * s.C + (size_t)v * N;
        int t = t0 + lane;
        if (t < live) {
            if (v != col) {
                load(v, t);
                load_channels(v);
            }
            auto set = [&](Affine<N>& f, float2& l, int c) {
                const int g = group_of(s, c);
                const float2 k = means[g];
                const float r = rstd[(size_t)b * s.G + g];
                f.set(make_float2(mean[(size_t)b * s.G + g], r));
                l = make_float2(-k.y * r * r, -k.x * r);
            };
            set(a, line, v * N);
            if (GLU) set(h, gline, Cy + v * N);
        }
        while (t < live) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (t + k * s.lanes >= live) break;
                float xk[N], gk[N], d[N];
                unpack<T, N>(xv[k], xk);
                if (GLU) unpack<T, N>(xg[k], gk);
                unpack<T, N>(dv[k], d);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float du, dg = 0.f;
                    act_bwd<ACT>(a(xk[j], j), GLU ? h(gk[j], j) : 0.f, d[j], du, dg);
                    xk[j] = __builtin_fmaf(du, a.scale[j], __builtin_fmaf(xk[j] - a.mean, line.x, line.y));
                    if (GLU) gk[j] = __builtin_fmaf(dg, h.scale[j], __builtin_fmaf(gk[j] - h.mean, gline.x, gline.y));
                }
                T* const to = o + (size_t)(t + k * s.lanes) * s.C;
                put<T, N, true>(to, xk);
                if (GLU) put<T, N, true>(to + Cy, gk);
            }
            t += U * s.lanes;
            if (t < live) load(v, t);
        }
        if (t1 > live) {
            const float none[N] = {};
            for (t = (live > t0 ? live : t0) + lane; t < t1; t += s.lanes) {
                put<T, N, true>(o + (size_t)t * s.C, none);
                if (GLU) put<T, N, true>(o + (size_t)t * s.C + Cy, none);
            }
        }
    }
}

// ---- a workgroup a group -------------------------------------------------------------------------------------
// Where groups are many or short, a workgroup has a group of an utterance (with GLU the group of the values and that of their gates) and reads it twice, the second
// time from its L2, in one launch.  Vectors and groups of one utterance that are neighbours share lines, so consecutive ones go to one XCD.
constexpr int GROUP_THREADS = 512, GROUP_BATCH = 4, FLUSH = 64;  // (512: a lane's sums of all channels fit 64 KB of LDS; batches of 4: 35.4 us, of 3 35.6, 6 37.3, 10 40.8 for 8x750x1536 with GLU and its gradient)
static_assert(FLUSH % GROUP_BATCH == 0, "sums are flushed between batches");
// Where groups are fewer than CUs, two workgroups (split) each read a whole group and write half of its frames (8x750x1536 bf16 with GLU, 128 pairs of groups, at batches of 6: 15.0 -> 14.7 us, with its
// gradient 39.5 -> 37.1; 5x333x500 fp32, SiLU, and its gradient 17.0 -> 16.5; four or eight of them gain nothing more).
struct Place {
    int b, g, part, from, to;  // frames from .. to of the utterance's are written
};
__device__ __forceinline__ Place place_of(const Shape& s, int per)  // per: groups (pairs) of an utterance
{
    const unsigned total = gridDim.x, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, q = total >> 3, r = total & 7;
    const unsigned i = xcd * q + (xcd < r ? xcd : r) + slot, j = i / s.split;
    return {(int)(j / per), (int)(j % per), (int)(i - j * s.split), 0, 0};
}
__device__ __forceinline__ void part_of(const Shape& s, Place& at, int live)
{
    at.from = (int)((long long)live * at.part / s.split);
    at.to = (int)((long long)live * (at.part + 1) / s.split);
}
// over the workgroup; lds: a value a wavefront
template <typename V>
__device__ __forceinline__ V sum_group(V v, V* lds)
{
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    V k = lds[0];
    for (int w = 1; w < waves; ++w) {
        k.x += lds[w].x;
        k.y += lds[w].y;
    }
    return k;
}

template <typename T, int N, int ACT>
__global__ __launch_bounds__(GROUP_THREADS) void norm_group_k(const T* __restrict__ x, Shape s, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                              float eps, T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd)
{
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    constexpr int U = GROUP_BATCH;
    __shared__ double2 lds[2][GROUP_THREADS / 64];
    Place at = place_of(s, GLU ? s.G / 2 : s.G);
    const int b = at.b, len = frames_of(s, b), Cy = GLU ? s.C / 2 : s.C, live = len < 0 ? 0 : len;
    part_of(s, at, live);
    int col, lane;
    s.place(col, lane);
    const int c0 = at.g * s.Cg + col * N, step = U * s.lanes;
    const bool on = lane < s.lanes;
    const T* const p = x + (size_t)b * s.T * s.C + c0;
    raw_t<T, N> xv[U], xg[U];
    auto load = [&](int t) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const T* const q = p + (size_t)(t + k * s.lanes < live ? t + k * s.lanes : t) * s.C;
            xv[k] = fetch<T, N>(q);
            if (GLU) xg[k] = fetch<T, N>(q + Cy);
        }
    };
    Affine<N> a, h;
    a.load(gamma, beta, c0);
    if (GLU) h.load(gamma, beta, Cy + c0);
    double2 k1 = make_double2(0., 0.), k2 = k1;
    int last = -1;  // the first frame of what is in registers
    {
        Deviations<N> d1, d2;
        d1.clear();
        d2.clear();
        auto flush = [&](Deviations<N>& d, double2& k) {
            const double2 o = d.group_sums();
            k.x += o.x;
            k.y += o.y;
            d.clear();
        };
        if (on)
            for (int t = lane; t < live; t += step) {
                load(t);
                last = t;
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if (t + k * s.lanes >= live) break;
                    float u[N];
                    unpack<T, N>(xv[k], u);
                    d1.add(u);
                    if (GLU) {
                        unpack<T, N>(xg[k], u);
                        d2.add(u);
                    }
                }
                if (d1.n == FLUSH) {
                    flush(d1, k1);
                    if (GLU) flush(d2, k2);
                }
            }
        if (d1.n) {
            flush(d1, k1);
            if (GLU) flush(d2, k2);
        }
    }
    k1 = sum_group(sum64(k1, 64), lds[0]);
    if (GLU) k2 = sum_group(sum64(k2, 64), lds[1]);
    const double inv = live ? 1. / ((double)live * s.Cg) : 0.;
    const float2 s1 = stat_of(k1, inv, eps), s2 = GLU ? stat_of(k2, inv, eps) : s1;
    if (threadIdx.x == 0 && at.part == 0) {
        const size_t o = (size_t)b * s.G + at.g;
        mean[o] = len < 0 ? NAN : s1.x;
        rstd[o] = len < 0 ? NAN : s1.y;
        if (GLU) {
            mean[o + s.G / 2] = len < 0 ? NAN : s2.x;
            rstd[o + s.G / 2] = len < 0 ? NAN : s2.y;
        }
    }
    if (!on) return;
    a.set(s1);
    if (GLU) h.set(s2);
    T* const q = y + (size_t)b * s.T * Cy + c0;
    const int way = s.split > 1 ? step : -step;  // a workgroup alone goes from the end, which is in registers
    int t = s.split > 1 ? at.from + lane : last;
    if (s.split > 1 && t < at.to) load(t);
    while (t >= 0 && t < at.to) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (t + k * s.lanes >= at.to) break;
            float u[N], w[N];
            unpack<T, N>(xv[k], u);
            if (GLU) unpack<T, N>(xg[k], w);
#pragma unroll
            for (int j = 0; j < N; ++j) u[j] = act<ACT>(a(u[j], j), GLU ? h(w[j], j) : 0.f);
            put<T, N, false>(q + (size_t)(t + k * s.lanes) * Cy, u);
        }
        t += way;
        if (t >= 0 && t < at.to) load(t);
    }
    float none[N];
#pragma unroll
    for (int j = 0; j < N; ++j) none[j] = len < 0 ? NAN : 0.f;
    for (t = live + at.part * s.lanes + lane; t < s.T; t += s.split * s.lanes) put<T, N, false>(q + (size_t)t * Cy, none);
}

// chans [B][2][C]: sums of du and du xhat of an utterance (NULL: not wanted).  One utterance alone has dgamma and dbeta in their place, and no launch after this.
template <typename T, int N, int ACT>
__global__ __launch_bounds__(GROUP_THREADS) void norm_group_bwd_k(const T* __restrict__ x, const T* __restrict__ dy, Shape s, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd, const float* __restrict__ gamma,
                                                                  const float* __restrict__ beta, T* __restrict__ dx, float* __restrict__ chans,
                                                                  float* __restrict__ dgamma, float* __restrict__ dbeta, int accumulate)
{
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    constexpr int U = GROUP_BATCH;
    const bool sums = chans || dgamma || dbeta;
    extern __shared__ float2 acc[];  // [GLU: 2][lanes][Cg]: a lane's sums
    __shared__ float2 lds[2][GROUP_THREADS / 64];
    Place at = place_of(s, GLU ? s.G / 2 : s.G);
    const int b = at.b, len = frames_of(s, b), Cy = GLU ? s.C / 2 : s.C, live = len < 0 ? 0 : len;
    part_of(s, at, live);
    int col, lane;
    s.place(col, lane);
    const int c0 = at.g * s.Cg + col * N, step = U * s.lanes;
    const bool on = lane < s.lanes;
    const size_t row0 = (size_t)b * s.T;
    const T* const p = x + row0 * s.C + c0;
    const T* const q = dy + row0 * Cy + c0;
    raw_t<T, N> xv[U], xg[U], dv[U];
    auto load = [&](int t) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const size_t r = t + k * s.lanes < live ? t + k * s.lanes : t;
            xv[k] = fetch<T, N>(p + r * s.C);
            if (GLU) xg[k] = fetch<T, N>(p + r * s.C + Cy);
            dv[k] = fetch<T, N>(q + r * Cy);
        }
    };
    const size_t g0 = (size_t)b * s.G + at.g;
    // (an utterance without frames, or with a length out of range, has no part in anything: its statistics may be NaN)
    const float mn = live ? mean[g0] : 0.f, rs = live ? rstd[g0] : 0.f, mg = GLU && live ? mean[g0 + s.G / 2] : 0.f, rg = GLU && live ? rstd[g0 + s.G / 2] : 0.f;
    Affine<N> a, h;
    a.load(gamma, beta, c0);
    if (GLU) h.load(gamma, beta, Cy + c0);
    a.set(make_float2(mn, rs));
    if (GLU) h.set(make_float2(mg, rg));
    int last = -1;
    float s1[N], s2[N], r1[N], r2[N];
#pragma unroll
    for (int j = 0; j < N; ++j) s1[j] = s2[j] = r1[j] = r2[j] = 0.f;
    if (on)
        for (int t = lane; t < live; t += step) {
            load(t);
            last = t;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (t + k * s.lanes >= live) break;
                float xk[N], gk[N], d[N];
                unpack<T, N>(xv[k], xk);
                if (GLU) unpack<T, N>(xg[k], gk);
                unpack<T, N>(dv[k], d);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float du, dg = 0.f;
                    act_bwd<ACT>(a(xk[j], j), GLU ? h(gk[j], j) : 0.f, d[j], du, dg);
                    s1[j] += du;
                    s2[j] = __builtin_fmaf(du, xk[j] - mn, s2[j]);
                    if (GLU) {
                        r1[j] += dg;
                        r2[j] = __builtin_fmaf(dg, gk[j] - mg, r2[j]);
                    }
                }
            }
        }
    float2 k1 = make_float2(0.f, 0.f), k2 = k1;
#pragma unroll
    for (int j = 0; j < N; ++j) {  // of du gamma rstd and du gamma rstd (x - mean)
        k1.x = __builtin_fmaf(s1[j], a.scale[j], k1.x);
        k1.y = __builtin_fmaf(s2[j], a.scale[j], k1.y);
        if (GLU) {
            k2.x = __builtin_fmaf(r1[j], h.scale[j], k2.x);
            k2.y = __builtin_fmaf(r2[j], h.scale[j], k2.y);
        }
    }
    if (sums && on && at.part == 0)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            acc[lane * s.Cg + col * N + j] = make_float2(s1[j], s2[j] * rs);
            if (GLU) acc[(s.lanes + lane) * s.Cg + col * N + j] = make_float2(r1[j], r2[j] * rg);
        }
    k1 = sum_group(make_float2(wave64(k1.x, Sum()), wave64(k1.y, Sum())), lds[0]);
    if (GLU) k2 = sum_group(make_float2(wave64(k2.x, Sum()), wave64(k2.y, Sum())), lds[1]);
    if (sums && at.part == 0) {
        if (blockDim.x == 64) __syncthreads();  // (sum_group's are the others')
        const int team = team_of(GLU ? 2 * s.Cg : s.Cg, s.lanes), l = threadIdx.x & (team - 1), teams = blockDim.x / team, count = GLU ? 2 * s.Cg : s.Cg;
        for (int i0 = 0; i0 < count; i0 += teams) {
            const int i = i0 + threadIdx.x / team, half = i >= s.Cg, c = i - half * s.Cg;
            float2 k = make_float2(0.f, 0.f);
            if (i < count)
                for (int r = l; r < s.lanes; r += team) {
                    const float2 o = acc[(half * s.lanes + r) * s.Cg + c];
                    k.x += o.x;
                    k.y += o.y;
                }
            for (int o = team >> 1; o > 0; o >>= 1) {
                k.x += __shfl_xor(k.x, o, 64);
                k.y += __shfl_xor(k.y, o, 64);
            }
            if (i < count && l == 0) {
                const int to = at.g * s.Cg + half * Cy + c;
                if (chans) {
                    float* const o = chans + (size_t)b * 2 * s.C + to;
                    o[0] = k.x;
                    o[s.C] = k.y;
                }
                if (dgamma) dgamma[to] = accumulate ? dgamma[to] + k.y : k.y;
                if (dbeta) dbeta[to] = accumulate ? dbeta[to] + k.x : k.x;
            }
        }
    }
    if (!on) return;
    const float inv = live ? 1.f / ((float)live * (float)s.Cg) : 0.f;
    // (rstd is in k1 and k2 already)
    const float slope = -k1.y * inv * rs * rs, level = -k1.x * inv, gslope = -k2.y * inv * rg * rg, glevel = -k2.x * inv;
    T* const o = dx + row0 * s.C + c0;
    const int way = s.split > 1 ? step : -step;
    int t = s.split > 1 ? at.from + lane : last;
    if (s.split > 1 && t < at.to) load(t);
    while (t >= 0 && t < at.to) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (t + k * s.lanes >= at.to) break;
            float xk[N], gk[N], d[N];
            unpack<T, N>(xv[k], xk);
            if (GLU) unpack<T, N>(xg[k], gk);
            unpack<T, N>(dv[k], d);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float du, dg = 0.f;
                act_bwd<ACT>(a(xk[j], j), GLU ? h(gk[j], j) : 0.f, d[j], du, dg);
                xk[j] = __builtin_fmaf(du, a.scale[j], __builtin_fmaf(xk[j] - mn, slope, level));
                if (GLU) gk[j] = __builtin_fmaf(dg, h.scale[j], __builtin_fmaf(gk[j] - mg, gslope, glevel));
            }
            T* const to = o + (size_t)(t + k * s.lanes) * s.C;
            put<T, N, false>(to, xk);
            if (GLU) put<T, N, false>(to + Cy, gk);
        }
        t += way;
        if (t >= 0 && t < at.to) load(t);
    }
    const float none[N] = {};
    for (t = live + at.part * s.lanes + lane; t < s.T; t += s.split * s.lanes) {
        put<T, N, false>(o + (size_t)t * s.C, none);
        if (GLU) put<T, N, false>(o + (size_t)t * s.C + Cy, none);
    }
}

// dgamma and dbeta from the utterances' sums
__global__ __launch_bounds__(JOIN_THREADS) void norm_join_k(const float* __restrict__ chans, int B, int C, float* __restrict__ dgamma, float* __restrict__ dbeta, int accumulate, int width)
{
    __shared__ double2 lds[JOIN_THREADS / 64 * JOIN_CHANNELS];
    sum_channels(chans, B, C, blockIdx.x, width, lds, dgamma, dbeta, accumulate, [](int) { return true; });
}

// ---- host ----------------------------------------------------------------------------------------------------
bool shape_ok(int B, int T, int C, int G, int act)
{
    return B > 0 && T > 0 && T <= MAX_FRAMES && C > 0 && C <= MAX_CHANNELS && G > 0 && C % G == 0 && act >= W2L_ACT_NONE && act <= W2L_ACT_GLU && (act != W2L_ACT_GLU || C % 2 == 0) &&
           B <= 65534 && (long long)B * T <= 2147483647LL && (long long)B * T <= (1LL << 40) / C;
}
// channels of a vector: as many as divide a group and a row (GLU: half a row) and make up at most 16 bytes
int vector_of(int Cg, int Cy, int dtype)
{
    int n = dtype == W2L_BF16 ? 8 : 4;
    while (Cg % n || Cy % n) n /= 2;
    return n;
}
// vectors: of a row that a thread can be given one of
Shape shape_of(int B, int T, int C, int G, const int* in_len, int vectors)
{
    Shape s{B, T, C, G, C / G, 0, 0, 0, 0, 1, in_len, 1.f / (float)(C / G), 0.f};
    const int passes = (vectors + MAX_THREADS - 1) / MAX_THREADS;
    s.cols = (vectors + passes - 1) / passes;
    s.lanes = MAX_THREADS / s.cols;
    if (s.lanes > 16) s.lanes = 16;
    s.inv_cols = 1.f / (float)s.cols;
    return s;
}
// channels whose sums a workgroup joins: fewer where rows are so many that a thread had more than four batches of them (64x2000x32 fp32, SiLU, the backward call 58 -> 26 us)
int join_width(long long rows, int threads) { return rows > 4LL * 8 * (threads / JOIN_CHANNELS) ? JOIN_CHANNELS / 4 : JOIN_CHANNELS; }
int threads_of(const Shape& s) { return (s.cols * s.lanes + 63) / 64 * 64; }
// Frames of a run, the same for all kernels of a call, so that a workgroup finds in its XCD's L2 what that of the same number read before: whole batches of loads
// (BATCH rows a thread), three runs a CU where there are so many
void runs_of(Shape& s)
{
    const int unit = BATCH * s.lanes;
    long long r = ((long long)s.B * s.T + 384) / 768 + unit / 2;
    r = r / unit * unit;
    s.rows = (int)(r < unit ? unit : r > 64 ? 64 : r);
    // (longer ones where joining an utterance's runs costs a workgroup more than its own rows)
    while (s.rows < 64 && (long long)(s.T / s.rows) * s.G * 2 > (long long)s.rows * s.C) s.rows += unit;
    s.runs = (s.T + s.rows - 1) / s.rows;
}
// Whether the sums of an utterance's runs, of `size` bytes a group, are joined by a launch of their own: where they outweigh what a run reads and writes, `tensors` times its
// frames, and all workgroups together would read 16 MB of them, which takes as long as a launch.  Each workgroup's joining them is the square of an utterance's length.  Both ways in us, forward and backward
// call: 1x131072x64 bf16 in 32 groups 239 and 244 -> 27 and 30; 1x60000x512 in 32 75 and 91 -> 38 and 59; 1x24000x512 with GLU 25 -> 18 (backward below the first limit, 33 and 28);
// below it 1x12000x1536 with GLU 30 and 45, 26 and 42 apart;  1x6000x512 12.6 and 15.6, 12.0 and 15.2;  16x1500x2048 in one group 50 and 85, 52 and 88;  below the second 32x700x80 in 80
// 11.6, 12.3 apart;  above both and slower: 1x400000x64 in one group, backward, 76 -> 80 (forward 51 -> 36).
bool joins_apart(const Shape& s, int size, int tensors, int dtype)
{
    const double sums = (double)s.runs * s.G * size;  // of an utterance
    return sums > (double)tensors * s.rows * s.C * (double)dtype_size(dtype) && sums * s.runs * s.B > (double)(16 << 20);
}
bool workspace_ok(const void* ws, size_t have, size_t need) { return ws && have >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0; }
bool meets(const void* a, size_t an, const void* b, size_t bn)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return a && b && p < q + bn && q < p + an;
}
struct Span {
    const void* p;
    size_t bytes;
};
template <int I, int O>
bool apart(const Span (&in)[I], const Span (&out)[O])
{
    for (int o = 0; o < O; ++o) {
        for (const Span& i : in)
            if (meets(out[o].p, out[o].bytes, i.p, i.bytes)) return false;
        for (int k = 0; k < o; ++k)
            if (meets(out[o].p, out[o].bytes, out[k].p, out[k].bytes)) return false;
    }
    return true;
}

struct Form {
    bool group;  // a workgroup a group, or `split` of them
    int N;       // channels of a vector
    int split;
};
// A workgroup a group saves a launch and the second reading from far away, as long as there are workgroups for the chip or what one reads is little.  Both ways
// in us, forward and backward call (SiLU unless said): 64 workgroups of 62 KB (fp32): 6.1 and 10.4 against 9.0 and 9.8; of 125 KB (bf16): 10.5 and 21 against 10.7 and 16.1; 128 of 144 KB
// (bf16, GLU): 14.0 and 24.2 against 17.3 and 25.3; 256 of 125 KB (bf16): 17.7 and 31 against 23.2 and 42; of 500 KB: 80 and 121 against 74 and 121; 1024 of 100 KB: 53 and 81 against
// 55 and 134; 16 of 500 KB: 25 and 53 against 10.9 and 16.7.  Rows of more vectors than a workgroup's threads make few and slow runs (1x500x8192 bf16, 64 of 125 KB: 10.2 and 18
// against 17.8 and 42).  Thousands of workgroups that read few bytes are slower as well (4096 of 8 KB, 16 bytes a row: 36 and 69 against 23 and 40).
Form form_of(int B, int T, int C, int G, int act, int dtype)
{
    const bool glu = act == W2L_ACT_GLU;
    const int Cg = C / G, n = vector_of(Cg, glu ? C / 2 : C, dtype);
    const long long workgroups = (long long)B * (glu ? G / 2 : G), bytes = (long long)T * Cg * (glu ? 2 : 1) * dtype_size(dtype);
    const bool wide = (glu ? C / 2 : C) / n > MAX_THREADS;
    const long long most = workgroups >= 256 ? 1 << 20 : workgroups >= 128 ? 512 << 10 : wide ? 256 << 10 : 64 << 10;
    // (a thread's sums of at most 128 rows: in fp32)
    const bool group = !(glu && G % 2) && Cg / n <= 256 && bytes <= most && !(workgroups >= 2048 && bytes < (16 << 10)) && T <= 128 * (GROUP_THREADS / (Cg / n));
    const int split = group && workgroups <= 128 && bytes >= (16 << 10) ? 2 : 1;
    return {group, n, split};
}
Shape group_shape(int B, int T, int C, int G, const int* in_len, int N, int split)
{
    Shape s{B, T, C, G, C / G, 0, 0, 0, 0, 1, in_len, 1.f / (float)(C / G), 0.f};
    s.cols = s.Cg / N;
    s.split = split;
    const int lanes = GROUP_THREADS / s.cols;
    s.lanes = lanes < T ? lanes : T;
    s.inv_cols = 1.f / (float)s.cols;
    return s;
}

// neighbouring groups of a workgroup that joins runs: their sums lie in one line
int groups_of_join(int G)
{
    int width = JOIN_GROUPS;
    while (width > 1 && width / 2 >= G) width /= 2;
    return width;
}
// Utterances of a launch, which has to stay below 2^32 threads: of 2^22 workgroups, or one (whose runs are 2^24 / (4 lanes) at most, its groups 2^14)
int utterances_of(const Shape& s, long long workgroups)
{
    const long long most = (1LL << 22) / workgroups;
    return most < 1 ? 1 : most < s.B ? (int)most : s.B;
}
// Utterances first .. first + count alone
Shape part_of(const Shape& s, int first, int count)
{
    Shape p = s;
    p.B = count;
    if (p.in_len) p.in_len += first;
    return p;
}

size_t stat_bytes(const Shape& s) { return round_up((size_t)s.B * s.runs * s.G * sizeof(double2), 256); }
size_t sum_bytes(const Shape& s) { return round_up((size_t)s.B * s.runs * s.C * 8, 256) + round_up((size_t)s.B * s.runs * s.G * 8, 256); }

template <typename T, int N>
int forward(const void* x, const Shape& st, const Shape& ap, double2* sums, const float* gamma, const float* beta, float eps, int act, void* y, float* mean,
            float* rstd, hipStream_t stream)
{
    const int most = utterances_of(st, st.runs), Cy = act == W2L_ACT_GLU ? st.C / 2 : st.C;
    for (int b = 0; b < st.B; b += most) {
        const Shape a = part_of(st, b, std::min(most, st.B - b)), p = part_of(ap, b, a.B);
        const T* const in = (const T*)x + (size_t)b * st.T * st.C;
        double2* const k = sums + (size_t)b * st.runs * st.G;
        hipLaunchKernelGGL((norm_stats_k<T, N>), dim3((unsigned)(a.runs * a.B)), dim3(threads_of(a)), (size_t)a.lanes * (a.C / N) * 16, stream, in, a, k);
        if (int rc = launch_status()) return rc;
        if (p.joined) {
            const int width = groups_of_join(p.G);
            hipLaunchKernelGGL(norm_join_runs_k<double2>, dim3((p.G + width - 1) / width, p.B), dim3(JOIN_THREADS), 0, stream, p, k, width);
            if (int rc = launch_status()) return rc;
        }
#define W2L_APPLY(A_)                                                                                                                         \
    hipLaunchKernelGGL((norm_apply_k<T, N, A_>), dim3((unsigned)(p.runs * p.B)), dim3(threads_of(p)), (size_t)p.G * 8, stream, in, p, k, gamma, beta, eps, \
                       (T*)y + (size_t)b * p.T * Cy, mean + (size_t)b * p.G, rstd + (size_t)b * p.G)
        if (act == W2L_ACT_NONE) W2L_APPLY(W2L_ACT_NONE);
        else if (act == W2L_ACT_RELU) W2L_APPLY(W2L_ACT_RELU);
        else if (act == W2L_ACT_SILU) W2L_APPLY(W2L_ACT_SILU);
        else W2L_APPLY(W2L_ACT_GLU);
#undef W2L_APPLY
        if (int rc = launch_status()) return rc;
    }
    return W2L_OK;
}
template <typename T, int N>
int forward_group(const void* x, const Shape& s, const float* gamma, const float* beta, float eps, int act, void* y, float* mean, float* rstd, hipStream_t stream)
{
    const int each = (act == W2L_ACT_GLU ? s.G / 2 : s.G) * s.split, most = utterances_of(s, each), Cy = act == W2L_ACT_GLU ? s.C / 2 : s.C;
    for (int b = 0; b < s.B; b += most) {
        const Shape p = part_of(s, b, std::min(most, s.B - b));
#define W2L_GROUP(A_)                                                                                                                              \
    hipLaunchKernelGGL((norm_group_k<T, N, A_>), dim3((unsigned)(p.B * each)), dim3(threads_of(p)), 0, stream, (const T*)x + (size_t)b * p.T * p.C, p, gamma, beta, eps, \
                       (T*)y + (size_t)b * p.T * Cy, mean + (size_t)b * p.G, rstd + (size_t)b * p.G)
        if (act == W2L_ACT_NONE) W2L_GROUP(W2L_ACT_NONE);
        else if (act == W2L_ACT_RELU) W2L_GROUP(W2L_ACT_RELU);
        else if (act == W2L_ACT_SILU) W2L_GROUP(W2L_ACT_SILU);
        else W2L_GROUP(W2L_ACT_GLU);
#undef W2L_GROUP
        if (int rc = launch_status()) return rc;
    }
    return W2L_OK;
}
template <typename T, int N, int ACT>
int backward_group(const void* x, const void* dy, const Shape& s, const float* mean, const float* rstd, const float* gamma, const float* beta, float* chans,
                   void* dx, float* dgamma, float* dbeta, int accumulate, hipStream_t stream)
{
    const bool GLU = ACT == W2L_ACT_GLU, want = dgamma || dbeta, alone = s.B == 1;
    const int each = (GLU ? s.G / 2 : s.G) * s.split, most = utterances_of(s, each), Cy = GLU ? s.C / 2 : s.C;
    for (int b = 0; b < s.B; b += most) {
        const Shape p = part_of(s, b, std::min(most, s.B - b));
        const size_t rows = (size_t)b * p.T;
        hipLaunchKernelGGL((norm_group_bwd_k<T, N, ACT>), dim3((unsigned)(p.B * each)), dim3(threads_of(p)), want ? (size_t)(GLU ? 2 : 1) * p.lanes * p.Cg * 8 : 0, stream,
                           (const T*)x + rows * p.C, (const T*)dy + rows * Cy, p, mean + (size_t)b * p.G, rstd + (size_t)b * p.G, gamma, beta, (T*)dx + rows * p.C,
                           want && !alone ? chans + (size_t)b * 2 * p.C : nullptr, alone ? dgamma : nullptr, alone ? dbeta : nullptr, accumulate);
        if (int rc = launch_status()) return rc;
    }
    if (!want || alone) return W2L_OK;
    const int width = join_width(s.B, JOIN_THREADS);
    hipLaunchKernelGGL(norm_join_k, dim3((s.C + width - 1) / width), dim3(JOIN_THREADS), 0, stream, chans, s.B, s.C, dgamma, dbeta, accumulate, width);
    return launch_status();
}
template <typename T, int N, int ACT>
int backward(const void* x, const void* dy, const Shape& s, const float* mean, const float* rstd, const float* gamma, const float* beta, float* chans,
             float2* groups, void* dx, float* dgamma, float* dbeta, int accumulate, hipStream_t stream)
{
    const int most = utterances_of(s, s.runs), Cy = ACT == W2L_ACT_GLU ? s.C / 2 : s.C;
    for (int b = 0; b < s.B; b += most) {
        const Shape p = part_of(s, b, std::min(most, s.B - b));
        const size_t rows = (size_t)b * p.T, runs = (size_t)b * p.runs;
        const T *const in = (const T*)x + rows * p.C, *const back = (const T*)dy + rows * Cy;
        const float *const mn = mean + (size_t)b * p.G, *const rs = rstd + (size_t)b * p.G;
        float* const ch = chans + runs * 2 * p.C;
        float2* const gr = groups + runs * p.G;
        hipLaunchKernelGGL((norm_sums_k<T, N, ACT>), dim3((unsigned)(p.runs * p.B)), dim3(threads_of(p)), (size_t)p.lanes * p.C * 8, stream, in, back, p, mn, rs, gamma, beta,
                           ch, gr);
        if (int rc = launch_status()) return rc;
        if (p.joined) {
            const int width = groups_of_join(p.G);
            hipLaunchKernelGGL(norm_join_runs_k<float2>, dim3((p.G + width - 1) / width, p.B), dim3(JOIN_THREADS), 0, stream, p, gr, width);
            if (int rc = launch_status()) return rc;
        }
        const int width = join_width((long long)p.runs * p.B, threads_of(p)), ahead = dgamma || dbeta ? ((p.C + width - 1) / width + 7) / 8 * 8 : 0;
        // (utterances of a launch after the first add to what those before left in dgamma and dbeta)
        hipLaunchKernelGGL((norm_dx_k<T, N, ACT>), dim3((unsigned)(ahead + (long long)p.runs * p.B)), dim3(threads_of(p)),
                           std::max((size_t)p.G * 8, (size_t)threads_of(p) / 64 * JOIN_CHANNELS * 16), stream, in, back, p, mn, rs, gamma, beta, ch, gr,
                           (T*)dx + rows * p.C, dgamma, dbeta, accumulate || b, ahead, width);
        if (int rc = launch_status()) return rc;
    }
    return W2L_OK;
}

// f(a null pointer of the type, std::integral_constant of the vector length)
template <typename F>
int with_vector(int dtype, int n, F f)
{
    if (dtype == W2L_BF16) {
        bf16_t* const t = nullptr;
        if (n == 8) return f(t, std::integral_constant<int, 8>());
        if (n == 4) return f(t, std::integral_constant<int, 4>());
        if (n == 2) return f(t, std::integral_constant<int, 2>());
        return f(t, std::integral_constant<int, 1>());
    }
    float* const t = nullptr;
    if (n == 4) return f(t, std::integral_constant<int, 4>());
    if (n == 2) return f(t, std::integral_constant<int, 2>());
    return f(t, std::integral_constant<int, 1>());
}

}  // namespace

extern "C" size_t w2l_groupnorm_workspace_bytes(int B, int T, int C, int G, int act, int dtype)
{
    if (!shape_ok(B, T, C, G, act) || !valid_dtype(dtype)) return 0;
    const Form form = form_of(B, T, C, G, act, dtype);
    if (form.group) return round_up((size_t)B * C * 8, 256);
    Shape s = shape_of(B, T, C, G, nullptr, (act == W2L_ACT_GLU ? C / 2 : C) / form.N);
    runs_of(s);
    const size_t a = stat_bytes(s), b = sum_bytes(s);
    return a > b ? a : b;
}

extern "C" int w2l_groupnorm_fwd(const void* x, const float* gamma, const float* beta, const int* in_len, void* y, float* mean, float* rstd, int B, int T,
                                 int C, int G, float eps, int act, int dtype, void* workspace, size_t ws_bytes, void* stream)
{
    if (!x || !y || !mean || !rstd) return W2L_ERR_NULL;
    if (!shape_ok(B, T, C, G, act) || !(eps > 0.f) || !(eps < INFINITY)) return W2L_ERR_SHAPE;
    if (!valid_dtype(dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(x) || !aligned16(gamma) || !aligned16(beta) || !aligned16(in_len) || !aligned16(y) || !aligned16(mean) || !aligned16(rstd)) return W2L_ERR_ALIGN;
    const size_t need = w2l_groupnorm_workspace_bytes(B, T, C, G, act, dtype), values = (size_t)B * T * C, e = dtype_size(dtype);
    if (!workspace_ok(workspace, ws_bytes, need)) return W2L_ERR_WORKSPACE;
    const int Cy = act == W2L_ACT_GLU ? C / 2 : C;
    const Span in[] = {{x, values * e}, {gamma, (size_t)C * 4}, {beta, (size_t)C * 4}, {in_len, (size_t)B * 4}};
    const Span out[] = {{y, (size_t)B * T * Cy * e}, {mean, (size_t)B * G * 4}, {rstd, (size_t)B * G * 4}, {workspace, need}};
    if (!apart(in, out)) return W2L_ERR_OVERLAP;
    const Form form = form_of(B, T, C, G, act, dtype);
    const int n = form.N;
    if (form.group)
        return with_vector(dtype, n, [&](auto* t, auto n) {
            using T_ = std::remove_pointer_t<decltype(t)>;
            return forward_group<T_, decltype(n)::value>(x, group_shape(B, T, C, G, in_len, decltype(n)::value, form.split), gamma, beta, eps, act, y, mean, rstd, (hipStream_t)stream);
        });
    Shape ap = shape_of(B, T, C, G, in_len, Cy / n), st = shape_of(B, T, C, G, in_len, C / n);
    runs_of(ap);
    ap.joined = joins_apart(ap, sizeof(double2), 2, dtype);
    st.rows = ap.rows;
    st.runs = ap.runs;
    return with_vector(dtype, n, [&](auto* t, auto n) {
        using T_ = std::remove_pointer_t<decltype(t)>;
        return forward<T_, decltype(n)::value>(x, st, ap, (double2*)workspace, gamma, beta, eps, act, y, mean, rstd, (hipStream_t)stream);
    });
}

extern "C" int w2l_groupnorm_bwd(const void* x, const void* dy, const float* mean, const float* rstd, const float* gamma, const float* beta, const int* in_len,
                                 void* dx, float* dgamma, float* dbeta, int B, int T, int C, int G, int act, int dtype, int accumulate, void* workspace,
                                 size_t ws_bytes, void* stream)
{
    if (!x || !dy || !mean || !rstd || !dx) return W2L_ERR_NULL;
    if (!shape_ok(B, T, C, G, act)) return W2L_ERR_SHAPE;
    if (!valid_dtype(dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(x) || !aligned16(dy) || !aligned16(mean) || !aligned16(rstd) || !aligned16(gamma) || !aligned16(beta) || !aligned16(in_len) || !aligned16(dx) ||
        !aligned16(dgamma) || !aligned16(dbeta))
        return W2L_ERR_ALIGN;
    const size_t need = w2l_groupnorm_workspace_bytes(B, T, C, G, act, dtype), values = (size_t)B * T * C, e = dtype_size(dtype);
    if (!workspace_ok(workspace, ws_bytes, need)) return W2L_ERR_WORKSPACE;
    const int Cy = act == W2L_ACT_GLU ? C / 2 : C;
    const Span in[] = {{x, values * e}, {dy, (size_t)B * T * Cy * e}, {mean, (size_t)B * G * 4}, {rstd, (size_t)B * G * 4}, {gamma, (size_t)C * 4}, {beta, (size_t)C * 4},
                       {in_len, (size_t)B * 4}};
    const Span out[] = {{dx, values * e}, {dgamma, (size_t)C * 4}, {dbeta, (size_t)C * 4}, {workspace, need}};
    if (!apart(in, out)) return W2L_ERR_OVERLAP;
    const Form form = form_of(B, T, C, G, act, dtype);
    const int n = form.N;
    Shape s = form.group ? group_shape(B, T, C, G, in_len, n, form.split) : shape_of(B, T, C, G, in_len, Cy / n);
    if (!form.group) {
        runs_of(s);
        s.joined = joins_apart(s, sizeof(float2), 3, dtype);
    }
    float* const chans = (float*)workspace;
    float2* const groups = (float2*)((char*)workspace + round_up((size_t)B * s.runs * C * 8, 256));
    return with_vector(dtype, n, [&](auto* t, auto n) {
        using T_ = std::remove_pointer_t<decltype(t)>;
        constexpr int N = decltype(n)::value;
#define W2L_BACKWARD(A_)                                                                                                                        \
    return form.group ? backward_group<T_, N, A_>(x, dy, s, mean, rstd, gamma, beta, chans, dx, dgamma, dbeta, accumulate, (hipStream_t)stream) : \
    backward<T_, N, A_>(x, dy, s, mean, rstd, gamma, beta, chans, groups, dx, dgamma, dbeta, accumulate, (hipStream_t)stream)
        if (act == W2L_ACT_NONE) W2L_BACKWARD(W2L_ACT_NONE);
        if (act == W2L_ACT_RELU) W2L_BACKWARD(W2L_ACT_RELU);
        if (act == W2L_ACT_SILU) W2L_BACKWARD(W2L_ACT_SILU);
        W2L_BACKWARD(W2L_ACT_GLU);
#undef W2L_BACKWARD
    });
}

extern "C" int w2l_groupnorm_launch_config(int B, int T, int C, int G, int act, int dtype, int* group, int* vector)
{
    if (!group || !vector) return W2L_ERR_NULL;
    if (!shape_ok(B, T, C, G, act)) return W2L_ERR_SHAPE;
    if (!valid_dtype(dtype)) return W2L_ERR_DTYPE;
    const Form f = form_of(B, T, C, G, act, dtype);
    *group = f.group;
    *vector = f.N;
    return W2L_OK;
}
