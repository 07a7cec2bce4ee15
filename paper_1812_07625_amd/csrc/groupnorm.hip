// Group norm over [B,T,C], channels last, and the activation behind it: w2l_groupnorm_fwd / _bwd.
//   forward   norm_stats_k: count, mean and sum of squared deviations of every group in a run of an utterance's frames;
//             norm_apply_k: joins the runs of an utterance, normalises, applies the activation
//   backward  norm_sums_k: sums over a run of frames of du and du xhat of every channel, and of both times gamma of every group;
//             norm_dx_k: joins them and writes dx; workgroups of its own add up dgamma and dbeta
// Memory bounds all four: a pass moves 2 or 4 bytes a value and takes some ten instructions.  The second pass of either call reads what the first did
// and finds it in the caches where they hold it.
// A thread has a vector of N neighbouring channels (16 bytes where rows are whole vectors, less where they are not) in some rows of the run; what it
// knows of its channels stays in registers from row to row.
#include "lanes.h"

using namespace w2l;

namespace {

constexpr int MAX_CHANNELS = 8192, MAX_FRAMES = 1 << 24, MAX_THREADS = 512;  // (8192: a pair of floats a channel fits 64 KB of LDS)

// N values of one channel vector
template <typename T, int N> struct Pack;
template <int N> struct Pack<float, N> {
    typedef float raw __attribute__((ext_vector_type(N)));
    static __device__ __forceinline__ void load(const float* p, float (&x)[N])
    {
        const raw q = *reinterpret_cast<const raw*>(p);
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = q[j];
    }
    static __device__ __forceinline__ void store(float* p, const float (&x)[N])
    {
        raw q;
#pragma unroll
        for (int j = 0; j < N; ++j) q[j] = x[j];
        *reinterpret_cast<raw*>(p) = q;
    }
};
template <> struct Pack<float, 1> {
    static __device__ __forceinline__ void load(const float* p, float (&x)[1]) { x[0] = *p; }
    static __device__ __forceinline__ void store(float* p, const float (&x)[1]) { *p = x[0]; }
};
template <int N> struct Pack<bf16_t, N> {
    typedef unsigned raw __attribute__((ext_vector_type(N / 2)));
    static __device__ __forceinline__ void load(const bf16_t* p, float (&x)[N])
    {
        const raw q = *reinterpret_cast<const raw*>(p);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) { x[2 * j] = __uint_as_float(q[j] << 16); x[2 * j + 1] = __uint_as_float(q[j] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&x)[N])
    {
        raw q;
#pragma unroll
        for (int j = 0; j < N / 2; ++j) q[j] = (unsigned)f32_to_bf16(x[2 * j]) | (unsigned)f32_to_bf16(x[2 * j + 1]) << 16;
        *reinterpret_cast<raw*>(p) = q;
    }
};
template <> struct Pack<bf16_t, 2> {
    static __device__ __forceinline__ void load(const bf16_t* p, float (&x)[2])
    {
        const unsigned q = *reinterpret_cast<const unsigned*>(p);
        x[0] = __uint_as_float(q << 16);
        x[1] = __uint_as_float(q & 0xffff0000u);
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&x)[2])
    {
        *reinterpret_cast<unsigned*>(p) = (unsigned)f32_to_bf16(x[0]) | (unsigned)f32_to_bf16(x[1]) << 16;
    }
};
template <> struct Pack<bf16_t, 1> {
    static __device__ __forceinline__ void load(const bf16_t* p, float (&x)[1]) { x[0] = bf16_to_f32(*p); }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&x)[1]) { *p = f32_to_bf16(x[0]); }
};

// How a workgroup takes a run of `rows` frames: `cols` threads side by side, `lanes` rows at a time
struct Shape {
    int B, T, C, G, Cg, rows, runs, cols, lanes, subs;  // subs: partial results of a group that a run leaves
    const int* in_len;
};
// frames of utterance b; -1: its in_len is out of range
__device__ __forceinline__ int frames_of(const Shape& s, int b)
{
    if (!s.in_len) return s.T;
    const int n = s.in_len[b];
    return n < 0 || n > s.T ? -1 : n;
}

// ---- activations ---------------------------------------------------------------------------------------------
// y = act(u), du = dy act'(u).  GLU takes a value and a gate, and gives the gradient of both.
__device__ __forceinline__ float sigmoid(float u) { return 1.f / (1.f + expf(-u)); }
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
// channel's level; partial results are then joined as count, mean, and squared deviations about the mean, where nothing cancels.
struct Part {
    double mean;  // (means are joined in 64 bits: a group's may be small beside its channels')
    float n, m2;
};
__device__ __forceinline__ double sum64(double v, int width = 64)
{
    for (int o = width >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <typename T, int N>
__global__ __launch_bounds__(MAX_THREADS) void norm_stats_k(const T* __restrict__ x, Shape s, Part* __restrict__ parts)
{
    extern __shared__ float2 chan[];  // [lanes][C]: mean and squared deviations of a channel in the rows of one lane
    const int b = blockIdx.y, run = blockIdx.x, len = frames_of(s, b);
    const int t0 = run * s.rows, t1 = t0 + s.rows < len ? t0 + s.rows : len;
    if (t0 >= t1) return;  // (norm_apply_k knows that there is nothing)
    const int col = threadIdx.x % s.cols, lane = threadIdx.x / s.cols, nv = s.C / N, here = t1 - t0;
    if (lane < s.lanes)
        for (int v = col; v < nv; v += s.cols) {
            const T* const p = x + ((size_t)b * s.T + t0) * s.C + (size_t)v * N;
            float base[N], sum[N], sq[N];
#pragma unroll
            for (int j = 0; j < N; ++j) base[j] = sum[j] = sq[j] = 0.f;
            int n = 0;
            if (lane < here) {
                Pack<T, N>::load(p + (size_t)lane * s.C, base);
                n = 1;
            }
#pragma unroll 4
            for (int t = lane + s.lanes; t < here; t += s.lanes, ++n) {
                float y[N];
                Pack<T, N>::load(p + (size_t)t * s.C, y);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float d = y[j] - base[j];
                    sum[j] += d;
                    sq[j] = __builtin_fmaf(d, d, sq[j]);
                }
            }
            const float inv = n ? 1.f / (float)n : 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float m = sum[j] * inv;
                chan[(size_t)lane * s.C + v * N + j] = make_float2(base[j] + m, fmaxf(__builtin_fmaf(-m, sum[j], sq[j]), 0.f));
            }
        }
    __syncthreads();
    // a wavefront takes a share of a group, `subs` of them each group
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int live = here < s.lanes ? here : s.lanes, entries = live * s.Cg, share = (entries + s.subs - 1) / s.subs;
    for (int q = wave; q < s.G * s.subs; q += waves) {
        const int g = q / s.subs, e0 = (q % s.subs) * share, e1 = e0 + share < entries ? e0 + share : entries;
        float n = 0.f;
        double sum = 0.;
        for (int e = e0 + l; e < e1; e += 64) {
            const int r = e / s.Cg, c = g * s.Cg + (e - r * s.Cg);
            const float nr = (float)((here - r + s.lanes - 1) / s.lanes);
            n += nr;
            sum = __builtin_fma((double)nr, (double)chan[(size_t)r * s.C + c].x, sum);
        }
        n = wave64(n, Sum());
        const double mean = n > 0.f ? sum64(sum) / n : 0.;
        float m2 = 0.f;
        for (int e = e0 + l; e < e1; e += 64) {
            const int r = e / s.Cg, c = g * s.Cg + (e - r * s.Cg);
            const float nr = (float)((here - r + s.lanes - 1) / s.lanes);
            const float2 k = chan[(size_t)r * s.C + c];
            const float d = (float)(k.x - mean);
            m2 += __builtin_fmaf(nr * d, d, k.y);
        }
        m2 = wave64(m2, Sum());
        if (l == 0) parts[((size_t)b * s.runs + run) * s.G * s.subs + q] = {mean, n, m2};
    }
}

// mean and 1 / deviation of every group of utterance b, into LDS
__device__ __forceinline__ void join_stats(const Shape& s, const Part* __restrict__ parts, int b, int len, float eps, float2* stat)
{
    const int runs = (len + s.rows - 1) / s.rows, count = runs * s.subs, per = s.G * s.subs;
    const double n = (double)len * s.Cg;
    // a team of lanes a group: as many as there are threads for, a power of two up to a wavefront
    int team = 64;
    while (team > 1 && s.G * team > (int)blockDim.x) team >>= 1;
    const int l = threadIdx.x & (team - 1), teams = blockDim.x / team;
    for (int g0 = 0; g0 < s.G; g0 += teams) {
        const int g = g0 + threadIdx.x / team;
        const bool on = g < s.G;
        double sum = 0., m2 = 0.;
        const Part* const p = parts + (size_t)b * s.runs * per;
        auto at = [&](int i) { return p[(size_t)(i / s.subs) * per + (size_t)g * s.subs + i % s.subs]; };
        if (on)
            for (int i = l; i < count; i += team) {
                const Part q = at(i);
                sum = __builtin_fma((double)q.n, q.mean, sum);
            }
        sum = sum64(sum, team);
        const double mean = len > 0 ? sum / n : 0.;
        if (on)
            for (int i = l; i < count; i += team) {
                const Part q = at(i);
                const double d = q.mean - mean;
                m2 += __builtin_fma(q.n * d, d, (double)q.m2);
            }
        m2 = sum64(m2, team);
        if (on && l == 0) stat[g] = make_float2((float)mean, len > 0 ? 1.f / sqrtf((float)(m2 / n) + eps) : 0.f);
    }
    __syncthreads();
}

// What a thread keeps of its N channels: u = (x - mean) scale + shift
template <int N>
struct Affine {
    float mean[N], scale[N], shift[N];
    __device__ __forceinline__ void set(const Shape& s, const float2* stat, const float* __restrict__ gamma, const float* __restrict__ beta, int c0)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float2 k = stat[(c0 + j) / s.Cg];
            mean[j] = k.x;
            scale[j] = gamma ? k.y * gamma[c0 + j] : k.y;
            shift[j] = beta ? beta[c0 + j] : 0.f;
        }
    }
    __device__ __forceinline__ float operator()(float x, int j) const { return __builtin_fmaf(x - mean[j], scale[j], shift[j]); }
};

template <typename T, int N, int ACT>
__global__ __launch_bounds__(MAX_THREADS) void norm_apply_k(const T* __restrict__ x, Shape s, const Part* __restrict__ parts, const float* __restrict__ gamma,
                                                            const float* __restrict__ beta, float eps, T* __restrict__ y, float* __restrict__ mean,
                                                            float* __restrict__ rstd)
{
    extern __shared__ float2 stat[];
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    const int b = blockIdx.y, run = blockIdx.x, len = frames_of(s, b), Cy = GLU ? s.C / 2 : s.C;
    join_stats(s, parts, b, len < 0 ? 0 : len, eps, stat);
    if (run == 0)
        for (int g = threadIdx.x; g < s.G; g += blockDim.x) {
            mean[(size_t)b * s.G + g] = len < 0 ? NAN : stat[g].x;
            rstd[(size_t)b * s.G + g] = len < 0 ? NAN : stat[g].y;
        }
    const int t0 = run * s.rows, t1 = t0 + s.rows < s.T ? t0 + s.rows : s.T;
    const int col = threadIdx.x % s.cols, lane = threadIdx.x / s.cols, nv = Cy / N;
    if (lane >= s.lanes) return;
    for (int v = col; v < nv; v += s.cols) {
        Affine<N> a, h;
        a.set(s, stat, gamma, beta, v * N);
        if (GLU) h.set(s, stat, gamma, beta, Cy + v * N);
        const T* const p = x + (size_t)b * s.T * s.C + (size_t)v * N;
        T* const q = y + (size_t)b * s.T * Cy + (size_t)v * N;
#pragma unroll 4
        for (int t = t0 + lane; t < t1; t += s.lanes) {
            float u[N], w[N];
            if (t < len) {
                Pack<T, N>::load(p + (size_t)t * s.C, u);
                if (GLU) Pack<T, N>::load(p + (size_t)t * s.C + Cy, w);
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] = act<ACT>(a(u[j], j), GLU ? h(w[j], j) : 0.f);
            } else
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] = len < 0 ? NAN : 0.f;
            Pack<T, N>::store(q + (size_t)t * Cy, u);
        }
    }
}

// ---- gradients -----------------------------------------------------------------------------------------------
// xhat and du of N channels (and of their gates)
template <int N>
struct Channels {
    float mean[N], rstd[N], gamma[N], beta[N];
    __device__ __forceinline__ void set(const Shape& s, int b, const float* __restrict__ mn, const float* __restrict__ rs, const float* __restrict__ gm,
                                        const float* __restrict__ bt, int c0)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const size_t g = (size_t)b * s.G + (c0 + j) / s.Cg;
            mean[j] = mn[g];
            rstd[j] = rs[g];
            gamma[j] = gm ? gm[c0 + j] : 1.f;
            beta[j] = bt ? bt[c0 + j] : 0.f;
        }
    }
    __device__ __forceinline__ float hat(float x, int j) const { return (x - mean[j]) * rstd[j]; }
    __device__ __forceinline__ float u(float x, int j) const { return __builtin_fmaf(x - mean[j], rstd[j] * gamma[j], beta[j]); }  // (as the forward call rounds it)
};

// chans [B][runs][2][C]: sums of du and du xhat over a run;  groups [B][runs][G][2]: both times gamma
template <typename T, int N, int ACT>
__global__ __launch_bounds__(MAX_THREADS) void norm_sums_k(const T* __restrict__ x, const T* __restrict__ dy, Shape s, const float* __restrict__ mean,
                                                           const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                           float* __restrict__ chans, float2* __restrict__ groups)
{
    extern __shared__ float2 acc[];  // [lanes][C]: a lane's sums
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    const int b = blockIdx.y, run = blockIdx.x, len = frames_of(s, b), Cy = GLU ? s.C / 2 : s.C;
    const int t0 = run * s.rows, t1 = t0 + s.rows < len ? t0 + s.rows : len;
    if (t0 >= t1) return;
    const int col = threadIdx.x % s.cols, lane = threadIdx.x / s.cols, nv = Cy / N;
    if (lane < s.lanes)
        for (int v = col; v < nv; v += s.cols) {
            Channels<N> a, h;
            a.set(s, b, mean, rstd, gamma, beta, v * N);
            if (GLU) h.set(s, b, mean, rstd, gamma, beta, Cy + v * N);
            float s1[N], s2[N], r1[N], r2[N];
#pragma unroll
            for (int j = 0; j < N; ++j) s1[j] = s2[j] = r1[j] = r2[j] = 0.f;
            const T* const p = x + (size_t)b * s.T * s.C + (size_t)v * N;
            const T* const q = dy + (size_t)b * s.T * Cy + (size_t)v * N;
#pragma unroll 2
            for (int t = t0 + lane; t < t1; t += s.lanes) {
                float xv[N], xg[N], d[N];
                Pack<T, N>::load(p + (size_t)t * s.C, xv);
                if (GLU) Pack<T, N>::load(p + (size_t)t * s.C + Cy, xg);
                Pack<T, N>::load(q + (size_t)t * Cy, d);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float du, dg = 0.f;
                    act_bwd<ACT>(a.u(xv[j], j), GLU ? h.u(xg[j], j) : 0.f, d[j], du, dg);
                    s1[j] += du;
                    s2[j] = __builtin_fmaf(du, a.hat(xv[j], j), s2[j]);
                    if (GLU) {
                        r1[j] += dg;
                        r2[j] = __builtin_fmaf(dg, h.hat(xg[j], j), r2[j]);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                acc[(size_t)lane * s.C + v * N + j] = make_float2(s1[j], s2[j]);
                if (GLU) acc[(size_t)lane * s.C + Cy + v * N + j] = make_float2(r1[j], r2[j]);
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
    int team = 64;
    while (team > 1 && s.G * team > (int)blockDim.x) team >>= 1;
    const int l = threadIdx.x & (team - 1), teams = blockDim.x / team;
    for (int g0 = 0; g0 < s.G; g0 += teams) {
        const int g = g0 + threadIdx.x / team;
        float2 k = make_float2(0.f, 0.f);
        if (g < s.G)
            for (int c = l; c < s.Cg; c += team) {
                k.x += acc[(size_t)g * s.Cg + c].x;
                k.y += acc[(size_t)g * s.Cg + c].y;
            }
        for (int o = team >> 1; o > 0; o >>= 1) {
            k.x += __shfl_xor(k.x, o, 64);
            k.y += __shfl_xor(k.y, o, 64);
        }
        if (g < s.G && l == 0) groups[((size_t)b * s.runs + run) * s.G + g] = k;
    }
}

// blockIdx.y < B: dx of a run of frames; = B: dgamma and dbeta of blockDim.x channels
template <typename T, int N, int ACT>
__global__ __launch_bounds__(MAX_THREADS) void norm_dx_k(const T* __restrict__ x, const T* __restrict__ dy, Shape s, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                         const float* __restrict__ chans, const float2* __restrict__ groups, T* __restrict__ dx,
                                                         float* __restrict__ dgamma, float* __restrict__ dbeta, int accumulate)
{
    extern __shared__ double2 lds[];  // [G] of floats: means of du gamma and du gamma xhat
    constexpr bool GLU = ACT == W2L_ACT_GLU;
    const int b = blockIdx.y, Cy = GLU ? s.C / 2 : s.C;
    if (b == s.B) {
        // 64 channels a workgroup at a time, the runs dealt out over its wavefronts and added up in a fixed order
        const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, l = threadIdx.x & 63;
        for (int c0 = blockIdx.x * 64; c0 < s.C; c0 += gridDim.x * 64) {
            const int c = c0 + l;
            double g = 0., h = 0.;
            if (c < s.C)
                for (int i = 0; i < s.B; ++i) {
                    const int len = frames_of(s, i), runs = len > 0 ? (len + s.rows - 1) / s.rows : 0;
                    const float* const p = chans + (size_t)i * s.runs * 2 * s.C + c;
#pragma unroll 4
                    for (int r = (wave + i) % waves; r < runs; r += waves) {
                        h += p[(size_t)r * 2 * s.C];
                        g += p[(size_t)r * 2 * s.C + s.C];
                    }
                }
            lds[threadIdx.x] = make_double2(g, h);
            __syncthreads();
            if (wave == 0 && c < s.C) {
                for (int w = 1; w < waves; ++w) {
                    g += lds[64 * w + l].x;
                    h += lds[64 * w + l].y;
                }
                if (dgamma) dgamma[c] = (float)(accumulate ? dgamma[c] + g : g);
                if (dbeta) dbeta[c] = (float)(accumulate ? dbeta[c] + h : h);
            }
            __syncthreads();
        }
        return;
    }
    const int len = frames_of(s, b), run = blockIdx.x, t0 = run * s.rows, t1 = t0 + s.rows < s.T ? t0 + s.rows : s.T;
    float2* const means = reinterpret_cast<float2*>(lds);
    if (t0 < len) {
        const int runs = (len + s.rows - 1) / s.rows;
        const float inv = 1.f / ((float)len * (float)s.Cg);
        int team = 64;
        while (team > 1 && s.G * team > (int)blockDim.x) team >>= 1;
        const int l = threadIdx.x & (team - 1), teams = blockDim.x / team;
        for (int g0 = 0; g0 < s.G; g0 += teams) {
            const int g = g0 + threadIdx.x / team;
            float2 k = make_float2(0.f, 0.f);
            if (g < s.G)
                for (int r = l; r < runs; r += team) {
                    const float2 o = groups[((size_t)b * s.runs + r) * s.G + g];
                    k.x += o.x;
                    k.y += o.y;
                }
            for (int o = team >> 1; o > 0; o >>= 1) {
                k.x += __shfl_xor(k.x, o, 64);
                k.y += __shfl_xor(k.y, o, 64);
            }
            if (g < s.G && l == 0) means[g] = make_float2(k.x * inv, k.y * inv);
        }
        __syncthreads();
    }
    const int col = threadIdx.x % s.cols, lane = threadIdx.x / s.cols, nv = Cy / N;
    if (lane >= s.lanes) return;
    for (int v = col; v < nv; v += s.cols) {
        Channels<N> a, h;
        float m1[N], m2[N], k1[N], k2[N];
        if (t0 < len) {
            a.set(s, b, mean, rstd, gamma, beta, v * N);
            if (GLU) h.set(s, b, mean, rstd, gamma, beta, Cy + v * N);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float2 o = means[(v * N + j) / s.Cg];
                m1[j] = o.x;
                m2[j] = o.y;
                if (GLU) {
                    const float2 k = means[(Cy + v * N + j) / s.Cg];
                    k1[j] = k.x;
                    k2[j] = k.y;
                }
            }
        }
        const size_t row0 = (size_t)b * s.T;
        const T* const p = x + row0 * s.C + (size_t)v * N;
        const T* const q = dy + row0 * Cy + (size_t)v * N;
        T* const o = dx + row0 * s.C + (size_t)v * N;
#pragma unroll 2
        for (int t = t0 + lane; t < t1; t += s.lanes) {
            float xv[N], xg[N], d[N];
            if (t < len) {
                Pack<T, N>::load(p + (size_t)t * s.C, xv);
                if (GLU) Pack<T, N>::load(p + (size_t)t * s.C + Cy, xg);
                Pack<T, N>::load(q + (size_t)t * Cy, d);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float du, dg = 0.f;
                    act_bwd<ACT>(a.u(xv[j], j), GLU ? h.u(xg[j], j) : 0.f, d[j], du, dg);
                    xv[j] = (__builtin_fmaf(du, a.gamma[j], -m1[j]) - a.hat(xv[j], j) * m2[j]) * a.rstd[j];
                    if (GLU) xg[j] = (__builtin_fmaf(dg, h.gamma[j], -k1[j]) - h.hat(xg[j], j) * k2[j]) * h.rstd[j];
                }
            } else
#pragma unroll
                for (int j = 0; j < N; ++j) xv[j] = xg[j] = 0.f;
            Pack<T, N>::store(o + (size_t)t * s.C, xv);
            if (GLU) Pack<T, N>::store(o + (size_t)t * s.C + Cy, xg);
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------
bool shape_ok(int B, int T, int C, int G, int act)
{
    return B > 0 && T > 0 && T <= MAX_FRAMES && C > 0 && C <= MAX_CHANNELS && G > 0 && C % G == 0 && act >= W2L_ACT_NONE && act <= W2L_ACT_GLU && (act != W2L_ACT_GLU || C % 2 == 0) &&
           B <= 65534 && (long long)B * T <= 2147483647LL && (long long)B * T <= (1LL << 40) / C;
}
// channels of a vector: as many as divide a row (GLU: half a row) and make up at most 16 bytes
int vector_of(int Cy, int dtype)
{
    int n = dtype == W2L_BF16 ? 8 : 4;
    while (Cy % n) n /= 2;
    return n;
}
// vectors: of a row that a thread can be given one of
Shape shape_of(int B, int T, int C, int G, const int* in_len, int vectors)
{
    Shape s{B, T, C, G, C / G, 0, 0, 0, 0, 1, in_len};
    const int passes = (vectors + MAX_THREADS - 1) / MAX_THREADS;
    s.cols = (vectors + passes - 1) / passes;
    s.lanes = MAX_THREADS / s.cols;
    if (s.lanes > 16) s.lanes = 16;
    return s;
}
int threads_of(const Shape& s) { return (s.cols * s.lanes + 63) / 64 * 64; }
// frames of a run: the same for all kernels of a call, so that a workgroup finds in its L2 what that of the same number read before
int rows_of(int B, int T, int C, int dtype)
{
    const long long rows = (long long)B * T;
    long long r = (rows + 767) / 768;
    if (r < 16) r = 16;
    if (r > 64) r = 64;
    return (int)(r < T ? r : T);
}
void runs_of(Shape& s, int dtype)
{
    s.rows = rows_of(s.B, s.T, s.C, dtype);
    s.runs = (s.T + s.rows - 1) / s.rows;
}
int subs_of(const Shape& s) { return s.G >= 8 ? 1 : 8 / s.G; }
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

size_t stat_bytes(const Shape& s) { return round_up((size_t)s.B * s.runs * s.G * subs_of(s) * sizeof(Part), 256); }
size_t sum_bytes(const Shape& s) { return round_up((size_t)s.B * s.runs * s.C * 8, 256) + round_up((size_t)s.B * s.runs * s.G * 8, 256); }

template <typename T, int N>
int forward(const void* x, const Shape& st, const Shape& ap, Part* parts, const float* gamma, const float* beta, float eps, int act, void* y, float* mean,
            float* rstd, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_stats_k<T, N>), dim3(st.runs, st.B), dim3(threads_of(st)), (size_t)st.lanes * st.C * 8, stream, (const T*)x, st, parts);
    if (int rc = launch_status()) return rc;
#define W2L_APPLY(A_)                                                                                                                         \
    hipLaunchKernelGGL((norm_apply_k<T, N, A_>), dim3(ap.runs, ap.B), dim3(threads_of(ap)), (size_t)ap.G * 8, stream, (const T*)x, ap, parts, gamma, beta, \
                       eps, (T*)y, mean, rstd)
    if (act == W2L_ACT_NONE) W2L_APPLY(W2L_ACT_NONE);
    else if (act == W2L_ACT_RELU) W2L_APPLY(W2L_ACT_RELU);
    else if (act == W2L_ACT_SILU) W2L_APPLY(W2L_ACT_SILU);
    else W2L_APPLY(W2L_ACT_GLU);
#undef W2L_APPLY
    return launch_status();
}
template <typename T, int N, int ACT>
int backward(const void* x, const void* dy, const Shape& s, const float* mean, const float* rstd, const float* gamma, const float* beta, float* chans,
             float2* groups, void* dx, float* dgamma, float* dbeta, int accumulate, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_sums_k<T, N, ACT>), dim3(s.runs, s.B), dim3(threads_of(s)), (size_t)s.lanes * s.C * 8, stream, (const T*)x, (const T*)dy, s,
                       mean, rstd, gamma, beta, chans, groups);
    if (int rc = launch_status()) return rc;
    hipLaunchKernelGGL((norm_dx_k<T, N, ACT>), dim3(s.runs, s.B + (dgamma || dbeta ? 1 : 0)), dim3(threads_of(s)),
                       (size_t)(s.G > 2 * threads_of(s) ? s.G : 2 * threads_of(s)) * 8, stream, (const T*)x,
                       (const T*)dy, s, mean, rstd, gamma, beta, chans, groups, (T*)dx, dgamma, dbeta, accumulate);
    return launch_status();
}

// f(type, std::integral_constant of N) for the vector length n
template <typename F>
int with_vector(int dtype, int n, F f)
{
    if (dtype == W2L_BF16) {
        if (n == 8) return f((bf16_t*)nullptr, Pack<bf16_t, 8>());
        if (n == 4) return f((bf16_t*)nullptr, Pack<bf16_t, 4>());
        if (n == 2) return f((bf16_t*)nullptr, Pack<bf16_t, 2>());
        return f((bf16_t*)nullptr, Pack<bf16_t, 1>());
    }
    if (n == 4) return f((float*)nullptr, Pack<float, 4>());
    if (n == 2) return f((float*)nullptr, Pack<float, 2>());
    return f((float*)nullptr, Pack<float, 1>());
}
template <typename P> struct Length;
template <typename T, int N> struct Length<Pack<T, N>> { static constexpr int value = N; };

}  // namespace

extern "C" size_t w2l_groupnorm_workspace_bytes(int B, int T, int C, int G, int act, int dtype)
{
    if (!shape_ok(B, T, C, G, act) || !valid_dtype(dtype)) return 0;
    const int Cy = act == W2L_ACT_GLU ? C / 2 : C;
    Shape s = shape_of(B, T, C, G, nullptr, Cy / vector_of(Cy, dtype));
    runs_of(s, dtype);
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
    const int n = vector_of(Cy, dtype);
    Shape ap = shape_of(B, T, C, G, in_len, Cy / n), st = shape_of(B, T, C, G, in_len, C / n);
    runs_of(ap, dtype);
    runs_of(st, dtype);
    ap.subs = st.subs = subs_of(st);
    return with_vector(dtype, n, [&](auto* t, auto pack) {
        using T_ = std::remove_pointer_t<decltype(t)>;
        return forward<T_, Length<decltype(pack)>::value>(x, st, ap, (Part*)workspace, gamma, beta, eps, act, y, mean, rstd, (hipStream_t)stream);
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
    const int n = vector_of(Cy, dtype);
    Shape s = shape_of(B, T, C, G, in_len, Cy / n);
    runs_of(s, dtype);
    float* const chans = (float*)workspace;
    float2* const groups = (float2*)((char*)workspace + round_up((size_t)B * s.runs * C * 8, 256));
    return with_vector(dtype, n, [&](auto* t, auto pack) {
        using T_ = std::remove_pointer_t<decltype(t)>;
        constexpr int N = Length<decltype(pack)>::value;
#define W2L_BACKWARD(A_) \
    return backward<T_, N, A_>(x, dy, s, mean, rstd, gamma, beta, chans, groups, dx, dgamma, dbeta, accumulate, (hipStream_t)stream)
        if (act == W2L_ACT_NONE) W2L_BACKWARD(W2L_ACT_NONE);
        if (act == W2L_ACT_RELU) W2L_BACKWARD(W2L_ACT_RELU);
        if (act == W2L_ACT_SILU) W2L_BACKWARD(W2L_ACT_SILU);
        W2L_BACKWARD(W2L_ACT_GLU);
#undef W2L_BACKWARD
    });
}
