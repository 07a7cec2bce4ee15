// Operators over a frame's scores x[0 .. C): log-probabilities of given tokens with entropy and the K best classes
// (w2l_token_logprob_fwd / _bwd), and distillation from a teacher's K best classes (w2l_distill_fwd_bwd).
// All three are one softmax statistic of the row -- m = max x, s = sum exp(x - m), u = sum exp(x - m)(x - m), from which
// lp_c = (x_c - m) - log s and H = log s - u / s -- and a few of its columns; the gradients are p_c times a number of the row,
// corrected in those columns.  Log-probabilities are formed from x - m, never from x - (m + log s): a row of large
// scores keeps the bits of its differences.
#include "common.h"

#include <math.h>

using namespace w2l;

namespace {

constexpr int MAX_CLASSES = 262144, MAX_ENTRIES = 64;
constexpr int THREADS = 256;
enum Frame { LIVE = 0, PADDING = 1, BAD = 2 };

__device__ __forceinline__ Frame frame_of(const int* __restrict__ in_len, unsigned r, unsigned Tp)
{
    if (!in_len) return LIVE;
    const unsigned b = r / Tp;
    const int n = in_len[b];
    return n < 0 || n > (int)Tp ? BAD : (int)(r - b * Tp) < n ? LIVE : PADDING;
}

// reductions over the workgroup, the same value in every thread
template <typename F>
__device__ __forceinline__ float block_reduce(float v, F f, float* lds)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < THREADS / 64; ++w) v = f(v, lds[w]);
    __syncthreads();
    return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }

// class `c` at score `v` comes before class `d` at score `w`
__device__ __forceinline__ bool before(float v, int c, float w, int d) { return v > w || (v == w && c < d); }

struct RowStats { float m, s, u; bool ok; };  // ok: no NaN and no +inf; m is finite (0 where every score is -inf, and then s = 0)
template <typename T>
__device__ RowStats row_stats(const T* __restrict__ x, int C, float inv_tau, float* lds)
{
    RowStats q;
    float m = -INFINITY, bad = 0.f;
    for (int c = threadIdx.x; c < C; c += THREADS) {
        const float v = Elem<T>::load(x, c);
        if (!(v < INFINITY)) bad = 1.f;
        m = fmaxf(m, v);
    }
    q.ok = block_reduce(bad, larger, lds) == 0.f;
    m = block_reduce(m, larger, lds);
    q.m = m == -INFINITY ? 0.f : m;
    float s = 0.f, u = 0.f;
    for (int c = threadIdx.x; c < C; c += THREADS) {
        const float d = (Elem<T>::load(x, c) - q.m) * inv_tau, e = expf(d);
        s += e;
        u += e * fmaxf(d, -1000.f);  // 0 * -inf is no share of the entropy
    }
    q.s = block_reduce(s, add, lds);
    q.u = block_reduce(u, add, lds);
    return q;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void token_fwd_k(const T* __restrict__ z, const int* __restrict__ tokens, const int* __restrict__ in_len,
                                                       float* __restrict__ logprob, float* __restrict__ entropy, int* __restrict__ top_ids,
                                                       float* __restrict__ top_logprob, float* __restrict__ stats, unsigned rows, unsigned Tp, int C,
                                                       int S, int K)
{
    __shared__ float lds[THREADS / 64];
    __shared__ int lds_c[THREADS / 64];
    for (unsigned r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* x = z + (size_t)r * C;
        const int tid = threadIdx.x;
        const Frame f = frame_of(in_len, r, Tp);
        RowStats q{0.f, 0.f, 0.f, false};
        if (f == LIVE) q = row_stats(x, C, 1.f, lds);
        if (f != LIVE || !q.ok) {
            const float v = f == PADDING ? 0.f : NAN;
            if (tid < S) logprob[(size_t)r * S + tid] = v;
            if (tid < K) {
                top_ids[(size_t)r * K + tid] = -1;
                top_logprob[(size_t)r * K + tid] = f == PADDING ? -INFINITY : NAN;
            }
            if (tid == 0 && entropy) entropy[r] = v;
            if (tid == 0 && stats) reinterpret_cast<float4*>(stats)[r] = make_float4(v, v, v, 0.f);
            continue;
        }
        const float logs = q.s > 0.f ? logf(q.s) : 0.f, H = q.s > 0.f ? logs - q.u / q.s : 0.f;
        if (tid == 0 && entropy) entropy[r] = H;
        if (tid == 0 && stats) reinterpret_cast<float4*>(stats)[r] = make_float4(q.m, q.s > 0.f ? logs : -INFINITY, H, 0.f);
        if (tid < S) {
            const int c = tokens[(size_t)r * S + tid];
            logprob[(size_t)r * S + tid] = c == -1 ? 0.f : c < 0 || c >= C ? NAN : (Elem<T>::load(x, c) - q.m) - logs;
        }
        float pv = INFINITY;
        int pc = -1;
        for (int k = 0; k < K; ++k) {
            float v = -INFINITY;
            int c = MAX_CLASSES;
            for (int j = tid; j < C; j += THREADS) {
                const float w = Elem<T>::load(x, j);
                if (before(pv, pc, w, j) && before(w, j, v, c)) { v = w; c = j; }
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                const float w = __shfl_xor(v, o, 64);
                const int d = __shfl_xor(c, o, 64);
                if (before(w, d, v, c)) { v = w; c = d; }
            }
            if ((tid & 63) == 0) { lds[tid >> 6] = v; lds_c[tid >> 6] = c; }
            __syncthreads();
            for (int w = 0; w < THREADS / 64; ++w)
                if (before(lds[w], lds_c[w], v, c)) { v = lds[w]; c = lds_c[w]; }
            __syncthreads();
            pv = v;
            pc = c;
            if (tid == 0) {
                top_ids[(size_t)r * K + k] = c;
                top_logprob[(size_t)r * K + k] = (v - q.m) - logs;
            }
        }
    }
}

// A gradient's element: overwritten, or added to what is there and rounded once
template <typename G>
__device__ __forceinline__ void put(G* dz, size_t i, float v, int accumulate)
{
    Elem<G>::store(dz, i, accumulate ? Elem<G>::load(dz, i) + v : v);
}

template <typename T, typename G>
__global__ __launch_bounds__(THREADS) void token_bwd_k(const T* __restrict__ z, const float* __restrict__ stats, const int* __restrict__ tokens,
                                                       const float* __restrict__ dlogprob, const float* __restrict__ dentropy,
                                                       const int* __restrict__ top_ids, const float* __restrict__ dtop, const int* __restrict__ in_len,
                                                       G* __restrict__ dz, unsigned rows, unsigned Tp, int C, int S, int K, int accumulate)
{
    __shared__ int id[2 * MAX_ENTRIES];
    __shared__ float g[2 * MAX_ENTRIES];
    for (unsigned r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* x = z + (size_t)r * C;
        G* y = dz + (size_t)r * C;
        const int tid = threadIdx.x;
        const float4 q = reinterpret_cast<const float4*>(stats)[r];
        if (frame_of(in_len, r, Tp) != LIVE || !(fabsf(q.y) < INFINITY)) {
            if (!accumulate)
                for (int c = tid; c < C; c += THREADS) Elem<G>::store(y, c, 0.f);
            continue;
        }
        if (tid < S + K) {
            const int c = tid < S ? tokens[(size_t)r * S + tid] : top_ids[(size_t)r * K + tid - S];
            const bool there = c >= 0 && c < C;
            id[tid] = there ? c : -1;
            g[tid] = there ? tid < S ? dlogprob[(size_t)r * S + tid] : dtop[(size_t)r * K + tid - S] : 0.f;
        }
        __syncthreads();
        float sum = 0.f;
        for (int j = 0; j < S + K; ++j) sum += g[j];
        const float h = dentropy ? dentropy[r] : 0.f;
        for (int c = tid; c < C; c += THREADS) {
            const float lp = fmaxf((Elem<T>::load(x, c) - q.x) - q.y, -1000.f);
            float v = -expf(lp) * (sum + h * (lp + q.z));
            for (int j = 0; j < S + K; ++j) v += id[j] == c ? g[j] : 0.f;
            put(y, c, v, accumulate);
        }
        __syncthreads();
    }
}

template <typename T, typename G>
__global__ __launch_bounds__(THREADS) void distill_k(const T* __restrict__ z, const int* __restrict__ t_ids, const float* __restrict__ t_scores,
                                                     const int* __restrict__ in_len, const float* __restrict__ weight, float* __restrict__ frame_loss,
                                                     G* __restrict__ dz, unsigned rows, unsigned Tp, int C, int K, float tau, float inv_tau,
                                                     float grad_scale, int accumulate)
{
    __shared__ float lds[THREADS / 64];
    __shared__ int id[MAX_ENTRIES];
    __shared__ float q[MAX_ENTRIES];
    for (unsigned r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* x = z + (size_t)r * C;
        G* y = dz + (size_t)r * C;
        const int tid = threadIdx.x;
        const Frame f = frame_of(in_len, r, Tp);
        float loss = f == BAD ? NAN : 0.f, w = f != LIVE ? 0.f : weight ? weight[r] : 1.f, inv_s = 0.f;
        RowStats st{0.f, 0.f, 0.f, false};
        if (w != 0.f) {
            st = row_stats(x, C, inv_tau, lds);
            inv_s = 1.f / st.s;
            const float logs = st.s > 0.f ? logf(st.s) : 0.f;
            int c = -1;
            float t = -INFINITY;
            if (tid < K) {
                c = t_ids[(size_t)r * K + tid];
                t = c == -1 ? -INFINITY : t_scores[(size_t)r * K + tid];
            }
            const bool odd = (c != -1 && (c < 0 || c >= C)) || !(t < INFINITY);
            const bool bad = block_reduce(odd ? 1.f : 0.f, larger, lds) != 0.f;
            const float tm = block_reduce(t, larger, lds);
            const bool none = tm == -INFINITY;
            const float d = none ? -INFINITY : (t - tm) * inv_tau, e = none ? 0.f : expf(d), sum = block_reduce(e, add, lds);
            const bool there = e > 0.f && !odd;
            float kl = 0.f;
            if (there) kl = e / sum * ((d - logf(sum)) - ((Elem<T>::load(x, c) - st.m) * inv_tau - logs));
            kl = block_reduce(kl, add, lds);
            if (tid < K) {
                id[tid] = there ? c : -1;
                q[tid] = there ? e / sum : 0.f;
            }
            loss = bad || !st.ok ? NAN : none ? 0.f : w * (tau * tau) * kl;
            if (none || !(fabsf(loss) < INFINITY)) w = 0.f;
            __syncthreads();
        }
        if (tid == 0) frame_loss[r] = loss;
        if (!dz) continue;
        if (w == 0.f) {
            if (!accumulate)
                for (int c = tid; c < C; c += THREADS) Elem<G>::store(y, c, 0.f);
        } else {
            const float scale = w * grad_scale * tau;
            for (int c = tid; c < C; c += THREADS) {
                float v = expf((Elem<T>::load(x, c) - st.m) * inv_tau) * inv_s;
                for (int j = 0; j < K; ++j) v -= id[j] == c ? q[j] : 0.f;
                put(y, c, scale * v, accumulate);
            }
        }
        __syncthreads();
    }
}

// loss[b] = sum of the utterance's frames, in double and in a fixed order
__global__ __launch_bounds__(THREADS) void utterance_loss_k(const float* __restrict__ frame_loss, float* __restrict__ loss, unsigned Tp)
{
    __shared__ double lds[THREADS / 64];
    double s = 0.;
    for (unsigned t = threadIdx.x; t < Tp; t += THREADS) s += frame_loss[(size_t)blockIdx.x * Tp + t];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < THREADS / 64; ++w) s += lds[w];
        loss[blockIdx.x] = (float)s;
    }
}

bool shape_ok(int B, int Tp, int C, int S, int K)
{
    return B > 0 && Tp > 0 && (long long)B * Tp <= 2147483647LL && C > 0 && C <= MAX_CLASSES && S >= 0 && S <= MAX_ENTRIES && K >= 0 &&
           K <= MAX_ENTRIES && K <= C;
}
bool grad_dtype_ok(int z_dtype, int dz_dtype) { return valid_dtype(dz_dtype) && (dz_dtype == W2L_F32 || z_dtype == W2L_BF16); }
unsigned grid_of(unsigned rows) { return rows < (1u << 20) ? rows : 1u << 20; }

}  // namespace

extern "C" size_t w2l_token_logprob_workspace_bytes(int, int, int, int, int) { return 0; }

extern "C" int w2l_token_logprob_fwd(const void* z, const int* tokens, const int* in_len, float* logprob, float* entropy, int* top_ids,
                                     float* top_logprob, float* stats, int B, int Tp, int C, int S, int K, int z_dtype, void*, size_t, void* stream)
{
    if (!z || (S > 0 && (!tokens || !logprob)) || (K > 0 && (!top_ids || !top_logprob))) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, S, K)) return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(z) || !aligned16(tokens) || !aligned16(in_len) || !aligned16(logprob) || !aligned16(entropy) || !aligned16(top_ids) ||
        !aligned16(top_logprob) || !aligned16(stats))
        return W2L_ERR_ALIGN;
    const unsigned rows = (unsigned)B * (unsigned)Tp;
    const dim3 g(grid_of(rows)), b(THREADS);
    if (z_dtype == W2L_BF16)
        hipLaunchKernelGGL(token_fwd_k<bf16_t>, g, b, 0, (hipStream_t)stream, (const bf16_t*)z, tokens, in_len, logprob, entropy, top_ids,
                           top_logprob, stats, rows, (unsigned)Tp, C, S, K);
    else
        hipLaunchKernelGGL(token_fwd_k<float>, g, b, 0, (hipStream_t)stream, (const float*)z, tokens, in_len, logprob, entropy, top_ids, top_logprob,
                           stats, rows, (unsigned)Tp, C, S, K);
    return launch_status();
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
    const unsigned rows = (unsigned)B * (unsigned)Tp;
    const dim3 g(grid_of(rows)), b(THREADS);
#define W2L_BWD(T_, G_)                                                                                                                      \
    hipLaunchKernelGGL((token_bwd_k<T_, G_>), g, b, 0, (hipStream_t)stream, (const T_*)z, stats, tokens, dlogprob, dentropy, top_ids, dtop, \
                       in_len, (G_*)dz, rows, (unsigned)Tp, C, S, K, accumulate)
    if (z_dtype == W2L_F32) W2L_BWD(float, float);
    else if (dz_dtype == W2L_F32) W2L_BWD(bf16_t, float);
    else W2L_BWD(bf16_t, bf16_t);
#undef W2L_BWD
    return launch_status();
}

extern "C" size_t w2l_distill_workspace_bytes(int, int, int, int, int) { return 0; }

extern "C" int w2l_distill_fwd_bwd(const void* z, const int* t_ids, const float* t_scores, const int* in_len, const float* weight,
                                   float* frame_loss, float* loss, void* dz, int B, int Tp, int C, int K, float temperature, float grad_scale,
                                   int z_dtype, int dz_dtype, int accumulate, void*, size_t, void* stream)
{
    if (!z || !t_ids || !t_scores || !frame_loss) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, 0, K) || K < 1 || !(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature) || !isfinite(grad_scale))
        return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype) || !grad_dtype_ok(z_dtype, dz_dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(z) || !aligned16(t_ids) || !aligned16(t_scores) || !aligned16(in_len) || !aligned16(weight) || !aligned16(frame_loss) ||
        !aligned16(loss) || !aligned16(dz))
        return W2L_ERR_ALIGN;
    const unsigned rows = (unsigned)B * (unsigned)Tp;
    const dim3 g(grid_of(rows)), b(THREADS);
#define W2L_DISTILL(T_, G_)                                                                                                                     \
    hipLaunchKernelGGL((distill_k<T_, G_>), g, b, 0, (hipStream_t)stream, (const T_*)z, t_ids, t_scores, in_len, weight, frame_loss, (G_*)dz, \
                       rows, (unsigned)Tp, C, K, temperature, 1.f / temperature, grad_scale, accumulate)
    if (z_dtype == W2L_F32) W2L_DISTILL(float, float);
    else if (dz_dtype == W2L_F32) W2L_DISTILL(bf16_t, float);
    else W2L_DISTILL(bf16_t, bf16_t);
#undef W2L_DISTILL
    if (int rc = launch_status()) return rc;
    if (!loss) return W2L_OK;
    hipLaunchKernelGGL(utterance_loss_k, dim3(B), b, 0, (hipStream_t)stream, frame_loss, loss, (unsigned)Tp);
    return launch_status();
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
