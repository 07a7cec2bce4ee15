// Clipped policy loss of sampled tokens with a KL term, from a network's scores to their gradient (w2l_policy_fwd_bwd).
// A frame's loss is a function of one number of its row, the sampled token's log-probability, so that its gradient is p_c times a number of the
// row, corrected in one column: the row is read once, stays in registers (frame_rows.h), and its gradient is made from there.
// What bounds it is memory: a row is read and written, with two exponentials a score between.
#include "frame_rows.h"

using namespace w2l;

namespace {

struct Policy {
    const int* tokens;
    const float *old_lp, *ref_lp, *advantage, *weight;
    float *frame_loss, *logprob;
    float low, high, kl, grad_scale;  // low = 1 - clip_low, high = 1 + clip_high
    int per_frame;                    // advantage: of a frame, or of its utterance
};
// What a frame says beside its scores
struct Sample {
    int token;
    float w, old_lp, ref_lp, A;
};
__device__ __forceinline__ Sample sample_of(const Policy& po, const Frames& fr, unsigned r, Frame f)
{
    Sample a{-1, 0.f, 0.f, 0.f, 0.f};
    if (f != LIVE) return a;
    a.token = po.tokens[r];
    a.w = a.token == -1 ? 0.f : po.weight ? po.weight[r] : 1.f;
    if (a.w == 0.f) return a;
    const unsigned b = (unsigned)((unsigned long long)r * fr.mul >> 31 >> fr.shift);
    a.old_lp = po.old_lp[r];
    a.ref_lp = po.kl != 0.f ? po.ref_lp[r] : 0.f;
    a.A = po.advantage[po.per_frame ? r : b];
    return a;
}
// exp(e) - 1 - e, which vanishes with e^2 / 2: below 1/4 its series, whose first term left out is 2e-9 of the sum
__device__ __forceinline__ float excess(float e)
{
    const float s = e * e * (0.5f + e * (1.f / 6 + e * (1.f / 24 + e * (1.f / 120 + e * (1.f / 720 + e * (1.f / 5040 + e * (1.f / 40320)))))));
    return fabsf(e) < 0.25f ? s : e < 80.f ? expf(e) - 1.f - e : expf(e);  // (e = inf: not inf - inf)
}
// Loss of a frame whose token has log-probability lp, and its derivative with respect to lp (times weight and grad_scale; 0 where the loss is not finite)
__device__ __forceinline__ float loss_of(const Policy& po, const Sample& a, float lp, float& f)
{
    const float r = expf(lp - a.old_lp);
    float loss = 0.f, d = 0.f;
    if (a.A != 0.f) {  // (an advantage of 0 says nothing, whatever the ratio; NaN is not 0)
        const float plain = r * a.A, held = fminf(fmaxf(r, po.low), po.high) * a.A;
        const bool inside = plain <= held;
        loss = -(inside ? plain : held);
        d = inside ? -plain : 0.f;
    }
    if (po.kl != 0.f) {
        const float e = a.ref_lp - lp;
        loss += po.kl * excess(e);
        d -= po.kl * expm1f(e);
    }
    loss = lp - a.old_lp == lp - a.old_lp ? loss * a.w : NAN;
    f = fabsf(loss) < INFINITY ? d * a.w * po.grad_scale : 0.f;
    return loss;
}

// 2700 rows of 10001 bf16 (108 MB read and written): 26 us = 4.2 TB/s; 2900 of 32000 bf16 (371 MB): 76 us = 4.9 TB/s.
// One row by a wavefront (!MULTI, four rows a workgroup), by a workgroup, or by G workgroups; then, and where rows are few, sums has (m or -inf, s, ., .) of
// the `parts` that the row was read in before.
template <typename T, typename D, int V, bool MULTI>
__global__ __launch_bounds__(MULTI ? 1024 : 256) void policy_rows_k(const T* __restrict__ z, Policy po, Frames fr, const float4* __restrict__ sums, int parts,
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
        const Sample a = sample_of(po, fr, r, f);
        if (a.w == 0.f) {
            if (first) {
                po.frame_loss[r] = f == BAD ? NAN : 0.f;
                if (po.logprob) po.logprob[r] = f == BAD ? NAN : 0.f;
            }
            if (dz && !(how & ADD)) clear_row<T>(dz, row, V, step, n0, C, how);
            continue;
        }
        uint4 data[V];
        load_row(data, z, total, row, step, n0, C);
        const bool known = (unsigned)a.token < (unsigned)C;
        const float x = known ? Elem<T>::load(z, (size_t)r * C + a.token) : NAN;
        float m = -INFINITY, s = 0.f;
        if (MULTI && sums) {
            const float4 q = lane < parts ? sums[(size_t)r * parts + lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
            m = wave64(q.x, Max());
            s = wave64(q.y != 0.f ? q.y * expf(q.x - m) : 0.f, Sum());
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
            const float M = m * LOG2E;
            if (!(fabsf(M) < FAR)) {
                float unused;
                far_sums(z, total, row, V, step, n0, C, m, LOG2E, s, unused);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float y[N];
                    unpack(data[v], y);
#pragma unroll
                    for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f(__builtin_fmaf(y[e], LOG2E, -M));
                }
                s *= __builtin_amdgcn_exp2f(-__builtin_fmaf(m, LOG2E, -M));
            }
            s = wave64(s, Sum());
            if (MULTI) {
                if (lane == 0) red[1][wave] = s;
                __syncthreads();
                s = uniform(row16((lane & 15) < W ? red[1][lane & 15] : 0.f, Sum()));
            }
        }
        const float lp = s == s ? (s > 0.f ? (x - m) - logf(s) : known ? -INFINITY : NAN) : NAN;
        float ws;
        const float loss = loss_of(po, a, lp, ws);
        if (first) {
            po.frame_loss[r] = loss;
            if (po.logprob) po.logprob[r] = lp;
        }
        if (!dz) continue;
        if (ws == 0.f) {
            if (!(how & ADD)) clear_row<T>(dz, row, V, step, n0, C, how);
            continue;
        }
        // ws (1[c = token] - p_c): in the token's column 1 - p, from fp32 values, where p may be close to 1
        const float M0 = m * LOG2E, here = -ws * expm1f(lp);
        const bool far = !(fabsf(M0) < FAR);
        const float f0 = far ? -ws / s : -ws / s * __builtin_amdgcn_exp2f(-__builtin_fmaf(m, LOG2E, -M0));
        const int at = a.token + row.head, slot = at / (64 * N), place = at / N, elem = at & (N - 1);
        auto finish = [&](int n, float (&y)[N]) {
            if ((n >> 6) == slot)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (e == elem) y[e] = n == place ? here : y[e];
            if (n < row.nv) put(dz, row.first + (size_t)n * N, n * N - row.head, C, y, how);
        };
        if (far) {
#pragma unroll 1
            for (int v = 0; v < V; ++v) {  // from differences
                const int n = n0 + v * step;
                float y[N];
                unpack(load_vector(z, total, row, n, C), y);
#pragma unroll
                for (int e = 0; e < N; ++e) y[e] = __builtin_amdgcn_exp2f((y[e] - m) * LOG2E) * f0;
                finish(n, y);
            }
            continue;
        }
        opaque(data);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int n = n0 + v * step;
            float y[N];
            unpack(data[v], y);
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[e], LOG2E, -M0)) * f0;
            finish(n, y);
        }
    }
}

// Rows of up to 16 * NV classes, sixteen lanes each.  loss (nullable): one workgroup has all rows, FEW_ROWS at most, and adds the utterances' losses up as well.
// 24000 rows of 29 fp32: 5.4 us, and 2.8 for the utterances' losses.
template <typename T, typename D, int NV>
__global__ __launch_bounds__(1024) void policy_narrow_k(const T* __restrict__ z, Policy po, Frames fr, float* __restrict__ loss, D* __restrict__ dz, int C,
                                                        int accumulate)
{
    __shared__ float few[FEW_ROWS];
    const int l = threadIdx.x & 15;
    const unsigned per = blockDim.x / 16, stride = gridDim.x * per;
    for (unsigned r = blockIdx.x * per + (threadIdx.x >> 4); r < fr.rows; r += stride) {
        const size_t i0 = (size_t)r * C;
        const Frame f = frame_of(fr, r);
        const Sample a = sample_of(po, fr, r, f);
        float here = f == BAD ? NAN : 0.f, lp = here, ws = 0.f, g[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) g[j] = 0.f;
        if (a.w != 0.f) {
            const bool known = (unsigned)a.token < (unsigned)C;
            const float x = known ? Elem<T>::load(z, i0 + a.token) : NAN;
            float m = -INFINITY, s = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                g[j] = l + 16 * j < C ? Elem<T>::load(z, i0 + l + 16 * j) : -INFINITY;
                m = fmaxf(m, g[j]);
            }
            m = row16(m, Max());
            m = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                g[j] = __builtin_amdgcn_exp2f((g[j] - m) * LOG2E);
                s += g[j];
            }
            s = row16(s, Sum());
            lp = s == s ? (s > 0.f ? (x - m) - logf(s) : known ? -INFINITY : NAN) : NAN;
            here = loss_of(po, a, lp, ws);
            const float scale = -ws / s, own = -ws * expm1f(lp);
#pragma unroll
            for (int j = 0; j < NV; ++j) g[j] = ws == 0.f ? 0.f : l + 16 * j == a.token ? own : g[j] * scale;
        }
        if (l == 0) {
            po.frame_loss[r] = here;
            if (po.logprob) po.logprob[r] = lp;
            if (loss) few[r] = here;
        }
        if (!dz || (ws == 0.f && accumulate)) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (l + 16 * j < C) {
                const size_t i = i0 + l + 16 * j;
                Elem<D>::store(dz, i, accumulate ? Elem<D>::load(dz, i) + g[j] : g[j]);
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

// As a distillation's rows, but for those of 17 to 24 slots, which three wavefronts take here however many there are (2700 of 10001 bf16: 31 -> 28 us, 6000 of 12000 65 -> 58,
// 6000 of 6000 fp32 59 -> 52; of 16 slots 38 and 40, of 8 23 and 25).  Vector instructions take three quarters of such a row's time, so wavefronts have slots for the row and
// hardly more: with six, seven and fourteen among their numbers, and not only 4, 8 and 16, 2700 of 9000 29.3 -> 25.1 us, of 10001 30.6 -> 27.6, of 17000 47.5 -> 41.4, 400 of 50000 27 -> 24.5.
Plan plan_policy(long long rows, int C, int dtype)
{
    Plan p = plan_distill(rows, C, dtype);
    const int slots = slots_of(C, dtype);
    if (p.W == 1 && slots > 16) p.W = 3;
    if (p.W > 1) p.V = tight((slots + p.W * p.G - 1) / (p.W * p.G), {2, 4, 6, 7, 8, 10, 14, 16});
    return p;
}

template <typename T, typename D>
int launch(hipStream_t st, const void* z, const Policy& po, const Frames& fr, float* loss, void* dz, void* ws, int C, int accumulate)
{
    const int dtype = sizeof(T) == 2 ? W2L_BF16 : W2L_F32, how = how_of<D>(fr.rows, C, accumulate);
    const Plan p = plan_policy(fr.rows, C, dtype);
    bool known;
    if (p.W == 0) {
        const bool whole = fr.rows <= FEW_ROWS;  // then a launch less
        const dim3 g(whole ? 1 : grid_of(((long long)fr.rows + 15) / 16)), b(whole ? 1024 : THREADS);
        known = with_slots<2, 4, 8, 16>(p.V, [&](auto v) {
            hipLaunchKernelGGL((policy_narrow_k<T, D, decltype(v)::value>), g, b, 0, st, (const T*)z, po, fr, whole ? loss : nullptr, (D*)dz, C, accumulate);
        });
        if (whole) loss = nullptr;
    } else {
        const float4* sums = nullptr;
        int parts = 1;
        if (p.G > 1) {
            if (int rc = frame_row_sums(z, fr.in_len, (int)(fr.rows / fr.Tp), (int)fr.Tp, C, dtype, ws, &parts, st)) return rc;
            sums = (const float4*)ws;
        }
        if (p.W > 1)
            known = with_slots<2, 4, 6, 7, 8, 10, 14, 16>(p.V, [&](auto v) {
                hipLaunchKernelGGL((policy_rows_k<T, D, decltype(v)::value, true>), dim3(grid_of((long long)fr.rows * p.G)), dim3(64 * p.W), 0, st, (const T*)z,
                                   po, fr, sums, parts, (D*)dz, C, p.G, how);
            });
        else
            known = with_slots<2, 4, 6, 8, 10, 12, 14, 16>(p.V, [&](auto v) {
                hipLaunchKernelGGL((policy_rows_k<T, D, decltype(v)::value, false>), dim3(grid_of(((long long)fr.rows + 3) / 4)), dim3(256), 0, st, (const T*)z,
                                   po, fr, sums, 1, (D*)dz, C, 1, how);
            });
    }
    if (!known) return W2L_ERR_SHAPE;
    if (int rc = launch_status()) return rc;
    if (!loss) return W2L_OK;
    hipLaunchKernelGGL(utterance_loss_k, dim3(grid_of(fr.rows / fr.Tp)), dim3(THREADS), 0, st, po.frame_loss, loss, fr.rows / fr.Tp, fr.Tp);
    return launch_status();
}

}  // namespace

extern "C" size_t w2l_policy_workspace_bytes(int B, int Tp, int C, int z_dtype)
{
    if (!shape_ok(B, Tp, C, 0, 0) || !valid_dtype(z_dtype)) return 0;
    return plan_policy((long long)B * Tp, C, z_dtype).G > 1 ? w2l_token_logprob_workspace_bytes(B, Tp, C, 0, z_dtype) : 0;
}

extern "C" int w2l_policy_fwd_bwd(const void* z, const int* tokens, const float* old_logprob, const float* ref_logprob, const float* advantage,
                                  int advantage_per_frame, const float* weight, const int* in_len, float* frame_loss, float* loss, float* logprob, void* dz, int B,
                                  int Tp, int C, float clip_low, float clip_high, float kl_coef, float grad_scale, int z_dtype, int dz_dtype, int accumulate,
                                  void* workspace, size_t ws_bytes, void* stream)
{
    if (!z || !tokens || !old_logprob || !advantage || !frame_loss || (kl_coef != 0.f && !ref_logprob)) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, 0, 0) || !(clip_low >= 0.f) || !(clip_low <= 1.f) || !(clip_high >= 0.f) || !(kl_coef >= 0.f) || !(kl_coef < INFINITY) ||
        !isfinite(grad_scale))
        return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype) || !grad_dtype_ok(z_dtype, dz_dtype)) return W2L_ERR_DTYPE;
    if (!aligned16(z) || !aligned16(tokens) || !aligned16(old_logprob) || !aligned16(ref_logprob) || !aligned16(advantage) || !aligned16(weight) ||
        !aligned16(in_len) || !aligned16(frame_loss) || !aligned16(loss) || !aligned16(logprob) || !aligned16(dz))
        return W2L_ERR_ALIGN;
    const size_t rows = (size_t)B * Tp, need = w2l_policy_workspace_bytes(B, Tp, C, z_dtype);
    if (!workspace_ok(workspace, ws_bytes, need)) return W2L_ERR_WORKSPACE;
    const Span frame{frame_loss, rows * 4}, sums{loss, (size_t)B * 4}, lps{logprob, rows * 4}, grad{dz, rows * C * dtype_size(dz_dtype)}, ws{workspace, need};
    if (!apart({{z, rows * C * dtype_size(z_dtype)}, {tokens, rows * 4}, {old_logprob, rows * 4}, {ref_logprob, rows * 4},
                {advantage, advantage_per_frame ? rows * 4 : (size_t)B * 4}, {weight, rows * 4}, {in_len, (size_t)B * 4}},
               {frame, sums, lps, grad, ws}) ||
        !apart({frame}, {sums, lps, grad, ws}) || !apart({sums}, {lps, grad, ws}) || !apart({lps}, {grad, ws}) || !apart({grad}, {ws}))
        return W2L_ERR_OVERLAP;
    const Frames fr = frames_of(in_len, B, Tp);
    const Policy po{tokens, old_logprob, ref_logprob, advantage, weight, frame_loss, logprob, 1.f - clip_low, 1.f + clip_high, kl_coef, grad_scale, advantage_per_frame};
    if (z_dtype == W2L_F32) return launch<float, float>((hipStream_t)stream, z, po, fr, loss, dz, workspace, C, accumulate);
    if (dz_dtype == W2L_F32) return launch<bf16_t, float>((hipStream_t)stream, z, po, fr, loss, dz, workspace, C, accumulate);
    return launch<bf16_t, bf16_t>((hipStream_t)stream, z, po, fr, loss, dz, workspace, C, accumulate);
}

extern "C" int w2l_policy_launch_config(int B, int Tp, int C, int z_dtype, int* wavefronts, int* groups, int* slots)
{
    if (!wavefronts || !groups || !slots) return W2L_ERR_NULL;
    if (!shape_ok(B, Tp, C, 0, 0)) return W2L_ERR_SHAPE;
    if (!valid_dtype(z_dtype)) return W2L_ERR_DTYPE;
    const Plan p = plan_policy((long long)B * Tp, C, z_dtype);
    *wavefronts = p.W;
    *groups = p.G;
    *slots = p.V;
    return W2L_OK;
}
