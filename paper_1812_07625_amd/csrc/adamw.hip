// AdamW over many tensors at once (w2l_adamw_step): one launch for up to 48 tensors, moments in 32 bits or in 8, the gradients clipped by their
// joint norm.  A value costs 18 to 30 bytes, each touched once, and 4 more where the norm reads the gradients first: memory bounds it.  107 M values with a bf16 copy,
// clipped: 584 us with moments in 32 bits (6.2 TB/s), of which the norm takes 75, and 400 in 8 (5.9 TB/s); a copy of 4 GB moves 4.8.
#include "lanes.h"

#include <algorithm>
#include <new>

using namespace w2l;

namespace {

constexpr int THREADS = 256, MOST = 48;           // MOST tensors a launch: their table is a kernel argument, of which 4 KB are to be had
// Values that share an exponent; values of a workgroup, with moments in 32 and in 8 bits (32 bits, through the caches: 4096 values take 621 us at 107 M, 2048 611, 1024 600)
constexpr int BLOCK = 256, CHUNK32 = 4 * THREADS, CHUNK8 = 16 * THREADS;
constexpr long long MOST_GROUPS = W2L_ADAMW_MAX_VALUES / CHUNK32;  // of a launch: 2^31 threads
constexpr int NORM_GROUPS = 256, NORM_CHUNK = 4096;  // workgroups a tensor's norm has at most, and values for which it has one more

struct Entry {
    float* w;
    const void* grad;
    void *m, *v;
    signed char *m_exp, *v_exp;
    bf16_t* lowp;
    long long n;
    double decay;
};
struct Table {
    Entry e[MOST];
    unsigned first[MOST + 1];  // first workgroup of every tensor, and of what follows the last
    int count, number;         // number: of the first tensor within the call
};
static_assert(sizeof(Table) <= 4000, "the table has to be a kernel argument");

// What a step's values are multiplied by: made on the host, or by adamw_now_k from what is known on the device alone
struct Scalars {
    double lr;
    float factor;        // of the gradients: grad_scale, and the clip's
    float rate, inv_root, eps;
    unsigned key;        // of the random bits
    int skip;            // the gradients' norm is not finite, or the step below 1: nothing changes
};
struct Hyper {
    double lr, beta1, beta2, eps, grad_scale, max_norm;
    long long step;
    unsigned seed;
};

// The finaliser of MurmurHash3 (A. Appleby, 2008): every bit of the result depends on every bit of x
__host__ __device__ __forceinline__ unsigned mix(unsigned x)
{
    x ^= x >> 16;
    x *= 0x85EBCA6Bu;
    x ^= x >> 13;
    x *= 0xC2B2AE35u;
    return x ^ x >> 16;
}
// power1, power2: beta1 and beta2 to the step
__host__ __device__ inline Scalars scalars_of(const Hyper& h, double power1, double power2)
{
    Scalars s;
    s.lr = h.lr;
    s.factor = (float)h.grad_scale;
    s.rate = (float)(h.lr / (1. - power1));
    s.inv_root = (float)(1. / sqrt(1. - power2));
    s.eps = (float)h.eps;
    s.key = mix(mix(h.seed) ^ (unsigned)h.step);
    s.skip = h.step < 1;
    return s;
}

// The entry of this workgroup, and its place within it.  A lane each compares the tensors' first workgroups.
__device__ __forceinline__ int entry_of(const Table& t, unsigned& within)
{
    const int lane = threadIdx.x & 63;
    const unsigned first = lane < t.count ? t.first[lane] : ~0u;
    const int i = __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= blockIdx.x)) - 1);
    within = blockIdx.x - __builtin_amdgcn_readlane(first, i);
    return i;
}

// Loads and stores past the caches, for what a step touches once: 107 M values with moments in 32 bits 578 -> 528 us, in 8 bits 332 -> 289 where the moments' bytes, of
// which a wavefront's instruction takes quarter lines, stay ordinary (321 if not); the norm after it 116 -> 75, which had waited for what was to be written back.  The
// norm's own loads stay ordinary: up to 256 MB the step finds the gradients in the memory-side cache (and beyond: 600 us, 640 past it).
template <bool PAST, typename V>
__device__ __forceinline__ V get(const void* p)
{
    if (PAST) return __builtin_nontemporal_load(static_cast<const V*>(p));
    return *static_cast<const V*>(p);
}
template <bool PAST, typename V>
__device__ __forceinline__ void set(void* p, V v)
{
    if (PAST) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else *static_cast<V*>(p) = v;
}
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef unsigned u2_t __attribute__((ext_vector_type(2)));

// ---- the gradients' norm -------------------------------------------------------------------------------------
// Squares of fp32 values are exact in 64 bits, and so is their sum to 2^-53 of itself a term: what is clipped by it does not depend on the order
template <typename G, bool PAST = false>
__device__ __forceinline__ void four(const G* p, long long i, float (&g)[4])
{
    if constexpr (sizeof(G) == 4) {
        const f4_t q = get<PAST, f4_t>(p + i);
        g[0] = q.x; g[1] = q.y; g[2] = q.z; g[3] = q.w;
    } else {
        const u2_t q = get<PAST, u2_t>(p + i);
        g[0] = __uint_as_float(q.x << 16); g[1] = __uint_as_float(q.x & 0xffff0000u);
        g[2] = __uint_as_float(q.y << 16); g[3] = __uint_as_float(q.y & 0xffff0000u);
    }
}

// sum over the workgroup, in lane 0 of its first wavefront
__device__ __forceinline__ double sum_all(double v, double* lds)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (unsigned w = 1; w < blockDim.x >> 6; ++w) v += lds[w];
    return v;
}

// sums[blockIdx.x]: the squares of a tensor's part.  first[] counts workgroups here as well: every tensor has some of its own
template <typename G>
__global__ __launch_bounds__(THREADS) void adamw_norm_k(const Table t, double* __restrict__ sums)
{
    __shared__ double lds[THREADS / 64];
    unsigned within;
    const int i = entry_of(t, within);
    const G* const grad = static_cast<const G*>(t.e[i].grad);
    const long long n = t.e[i].n, groups = t.first[i + 1] - t.first[i], n4 = n & ~3ll, step = groups * (4 * THREADS);
    double s = 0.;
    long long at = ((long long)within * THREADS + threadIdx.x) * 4;
    for (; at + 3 * step < n4; at += 4 * step) {
        float g[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) four<G>(grad, at + u * step, g[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_fma((double)g[u][e], (double)g[u][e], s);
    }
    for (; at < n4; at += step) {
        float g[4];
        four<G>(grad, at, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_fma((double)g[e], (double)g[e], s);
    }
    if (within == 0 && threadIdx.x < (n & 3)) {
        const double g = Elem<G>::load(grad, (size_t)(n4 + threadIdx.x));
        s = __builtin_fma(g, g, s);
    }
    s = sum_all(s, lds);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// The step's scalars, where they depend on what the device alone knows.  The powers of a step that only the device knows are made by a wavefront each, while the
// others sum.
__global__ __launch_bounds__(1024) void adamw_now_k(Hyper h, Scalars now, const float* lr, const int* step, const double* __restrict__ sums, int count,
                                                    float* __restrict__ grad_norm, Scalars* __restrict__ out)
{
    __shared__ double lds[16], powers[2];
    double s = 0.;
    if (lr) h.lr = *lr;
    if (step) h.step = *step;
    if ((lr || step) && (threadIdx.x == 64 || threadIdx.x == 128)) powers[threadIdx.x == 128] = pow(threadIdx.x == 64 ? h.beta1 : h.beta2, (double)h.step);
    for (int i = threadIdx.x; i < count; i += 4 * 1024) {
        double v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i + k * 1024 < count ? sums[i + k * 1024] : 0.;
#pragma unroll
        for (int k = 0; k < 4; ++k) s += v[k];
    }
    s = sum_all(s, lds);
    if (threadIdx.x != 0) return;
    double coef = 1.;
    bool finite = true;
    if (count) {
        const double norm = fabs(h.grad_scale) * sqrt(s);
        finite = norm < INFINITY;
        if (grad_norm) *grad_norm = (float)norm;
        if (h.max_norm > 0. && h.max_norm < norm + 1e-6) coef = h.max_norm / (norm + 1e-6);
    }
    if (lr || step) now = scalars_of(h, powers[0], powers[1]);
    now.factor = (float)(h.grad_scale * coef);
    if (!finite) now.skip = 1;
    *out = now;
}

// ---- moments in 8 bits ---------------------------------------------------------------------------------------
// A block of 256 values has an exponent E, the least (and at least -100) with which its largest magnitude is at most 448 * 2^E; a value is an e4m3
// number times 2^E, rounded up or down at random so that its expectation is the value.  (To the nearest, the second moment would stand still: a
// step moves it by a thousandth of itself, its numbers are an eighth apart.)  Kept is the root of the second moment, whose range is half as many
// powers of two.  The root is what has the right expectation; its square has the rounding's variance more.  A step moves a root r by d = (1 - beta2) / 2 |g^2 / v - 1| r, far
// less than the spacing s of 1/16 to 1/8 r, and moves it by s with a chance of d / s: a variance of d s, which v, forgetting 1 - beta2 of itself a step, holds
// d s / (1 - beta2) of, whatever beta2 is.  With normal gradients v settles 3 to 6 % above what it is in 32 bits, and single roots scatter by 12 to 17 %.
// A root that is not zero does not become zero, or its weight would move by the first moment over eps: below the block's least number, 2^-9 * 2^E, it
// becomes that.  (Roots below 2^-75 have squares of zero in fp32.)
__device__ __forceinline__ int exponent_of(float most)
{
    const unsigned u = __float_as_uint(most);
    const int E = (int)(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u);  // 448 = 1.75 * 2^8
    return u == 0 ? 0 : E < -100 ? -100 : E;
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }  // -126 <= e <= 127
// |x| in units of the block's least number (scale = 2^(9 - E): 0 <= u <= 448 * 512), r: 16 random bits -> the magnitude's code
__device__ __forceinline__ unsigned code_of(float u, unsigned r)
{
    const unsigned small = (unsigned)(u + (float)r * (1.f / 65536.f));            // below 2^-6 all multiples of 2^-9 are numbers
    const unsigned large = ((__float_as_uint(u) + (r << 4)) >> 20) - 1032u;       // above, those of four significant bits
    const unsigned c = u < 8.f ? small : large;
    return u < 3e38f ? (c < 126u ? c : 126u) : 127u;                              // 127: not a number, nor is infinity
}
__device__ __forceinline__ float largest_of(float most, float x)
{
    x = fabsf(x);
    return x < INFINITY ? fmaxf(most, x) : most;
}

// ---- the step ------------------------------------------------------------------------------------------------
// Moments are made of products and sums rounded one by one, as the formulas are written: a moment next to a border between two codes falls on
// the same side wherever it is computed.
struct Moments {
    float b1, c1, b2, c2;
};
__device__ __forceinline__ void advance(float g, float& m, float& v, const Moments& o)
{
#pragma clang fp contract(off)
    m = m * o.b1 + g * o.c1;
    v = v * o.b2 + (g * g) * o.c2;
}
__device__ __forceinline__ float moved(float w, float m, float root, float keep, const Scalars& s)
{
    return __builtin_fmaf(-s.rate * m, __builtin_amdgcn_rcpf(__builtin_fmaf(root, s.inv_root, s.eps)), w * keep);  // (the reciprocal to an ulp)
}

__device__ __forceinline__ u2_t low_of(f4_t x)
{
    typedef float float2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return (u2_t){__builtin_bit_cast(unsigned, __builtin_convertvector((float2_t){x.x, x.y}, bf16x2_t)),
                  __builtin_bit_cast(unsigned, __builtin_convertvector((float2_t){x.z, x.w}, bf16x2_t))};
}

template <typename G>
__global__ __launch_bounds__(THREADS) void adamw32_k(const Table t, const Scalars by_value, const Scalars* __restrict__ now, Moments o)
{
    unsigned within;
    const int i = entry_of(t, within);
    const Scalars s = now ? *now : by_value;
    if (s.skip) return;
    const Entry& e = t.e[i];
    const float keep = (float)(1. - s.lr * e.decay);
    const G* const grad = static_cast<const G*>(e.grad);
    float *const w = e.w, *const m = static_cast<float*>(e.m), *const v = static_cast<float*>(e.v);
    const long long at = (long long)within * CHUNK32 + threadIdx.x * 4;
    if (at + 4 <= e.n) {
        f4_t wq = get<true, f4_t>(w + at), mq = get<true, f4_t>(m + at), vq = get<true, f4_t>(v + at);
        float g[4];
        four<G, true>(grad, at, g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float mj = mq[j], vj = vq[j];
            advance(g[j] * s.factor, mj, vj, o);
            mq[j] = mj;
            vq[j] = vj;
            wq[j] = moved(wq[j], mj, sqrtf(vj), keep, s);
        }
        set<true>(w + at, wq);
        set<true>(m + at, mq);
        set<true>(v + at, vq);
        if (e.lowp) set<true>(e.lowp + at, low_of(wq));
    } else
        for (long long k = at; k < e.n; ++k) {
            float mk = m[k], vk = v[k];
            advance(Elem<G>::load(grad, (size_t)k) * s.factor, mk, vk, o);
            const float wk = moved(w[k], mk, sqrtf(vk), keep, s);
            m[k] = mk;
            v[k] = vk;
            w[k] = wk;
            if (e.lowp) e.lowp[k] = f32_to_bf16(wk);
        }
}

// Sixteen lanes have a block: four values at each of four places 64 apart a lane, so that a wavefront's loads are of whole lines
template <typename G>
__global__ __launch_bounds__(THREADS) void adamw8_k(const Table t, const Scalars by_value, const Scalars* __restrict__ now, Moments o)
{
    unsigned within;
    const int i = entry_of(t, within);
    const Scalars s = now ? *now : by_value;
    if (s.skip) return;
    const Entry& e = t.e[i];
    const float keep = (float)(1. - s.lr * e.decay);
    const unsigned key = mix(s.key ^ (unsigned)(t.number + i));
    const G* const grad = static_cast<const G*>(e.grad);
    float* const w = e.w;
    unsigned char *const mc = static_cast<unsigned char*>(e.m), *const vc = static_cast<unsigned char*>(e.v);
    const long long base = (long long)within * CHUNK8 + (threadIdx.x >> 4) * BLOCK, block = base / BLOCK;
    const int l = threadIdx.x & 15;
    const bool there = base < e.n, whole = base + BLOCK <= e.n;
    float wx[16], mx[16], vx[16];
    if (there) {
        float g[16];
        unsigned mq[4], vq[4];
        const float ms = __builtin_ldexpf(1.f, e.m_exp[block]), vs = __builtin_ldexpf(1.f, e.v_exp[block]);  // (-128 and -127 are exponents too: denormal numbers)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long at = base + j * 64 + l * 4;
            if (whole) {
                const f4_t q = get<true, f4_t>(w + at);
                wx[4 * j] = q.x; wx[4 * j + 1] = q.y; wx[4 * j + 2] = q.z; wx[4 * j + 3] = q.w;
                float gj[4];
                four<G, true>(grad, at, gj);
#pragma unroll
                for (int k = 0; k < 4; ++k) g[4 * j + k] = gj[k];
                mq[j] = get<false, unsigned>(mc + at);
                vq[j] = get<false, unsigned>(vc + at);
            } else {
                mq[j] = vq[j] = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool in = at + k < e.n;
                    wx[4 * j + k] = in ? w[at + k] : 0.f;
                    g[4 * j + k] = in ? Elem<G>::load(grad, (size_t)(at + k)) : 0.f;
                    mq[j] |= (in ? (unsigned)mc[at + k] : 0u) << 8 * k;
                    vq[j] |= (in ? (unsigned)vc[at + k] : 0u) << 8 * k;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            typedef float float2_t __attribute__((ext_vector_type(2)));
            const float2_t ma = __builtin_amdgcn_cvt_pk_f32_fp8(mq[j], false), mb = __builtin_amdgcn_cvt_pk_f32_fp8(mq[j], true);
            const float2_t va = __builtin_amdgcn_cvt_pk_f32_fp8(vq[j], false), vb = __builtin_amdgcn_cvt_pk_f32_fp8(vq[j], true);
            const float md[4] = {ma.x, ma.y, mb.x, mb.y}, vd[4] = {va.x, va.y, vb.x, vb.y};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float m1 = md[k] * ms, root = vd[k] * vs, v1 = root * root;
                advance(g[4 * j + k] * s.factor, m1, v1, o);
                mx[4 * j + k] = m1;
                vx[4 * j + k] = sqrtf(v1);
                wx[4 * j + k] = moved(wx[4 * j + k], m1, vx[4 * j + k], keep, s);
            }
        }
    } else
#pragma unroll
        for (int j = 0; j < 16; ++j) mx[j] = vx[j] = wx[j] = 0.f;
    float mm = 0.f, vm = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        mm = largest_of(mm, mx[j]);
        vm = largest_of(vm, vx[j]);
    }
    mm = row16(mm, Max());
    vm = row16(vm, Max());
    if (!there) return;
    const int mE = exponent_of(mm), vE = exponent_of(vm);
    const float ms = two_to(9 - mE), vs = two_to(9 - vE);
    if (l == 0) {
        e.m_exp[block] = (signed char)mE;
        e.v_exp[block] = (signed char)vE;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const long long at = base + j * 64 + l * 4;
        unsigned mq = 0, vq = 0;
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const unsigned h = mix((unsigned)((at + k) >> 1) * 0x9E3779B1u + key);  // 16 bits for each of two values: both moments of a value take the same
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const unsigned r = p ? h >> 16 : h & 0xffffu;
                const float m1 = mx[4 * j + k + p], v1 = vx[4 * j + k + p];
                unsigned mcode = code_of(fabsf(m1) * ms, r), vcode = code_of(v1 * vs, r);
                mcode |= m1 < 0.f ? 128u : 0u;
                vcode = v1 > 0.f && vcode == 0 ? 1u : vcode;
                mq |= mcode << 8 * (k + p);
                vq |= vcode << 8 * (k + p);
            }
        }
        const float* const x = wx + 4 * j;
        if (whole) {
            const f4_t wq = {x[0], x[1], x[2], x[3]};
            set<false>(mc + at, mq);
            set<false>(vc + at, vq);
            set<true>(w + at, wq);
            if (e.lowp) set<true>(e.lowp + at, low_of(wq));
        } else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (at + k < e.n) {
                    mc[at + k] = (unsigned char)(mq >> 8 * k);
                    vc[at + k] = (unsigned char)(vq >> 8 * k);
                    w[at + k] = x[k];
                    if (e.lowp) e.lowp[at + k] = f32_to_bf16(x[k]);
                }
    }
}

long long norm_groups(long long n)
{
    const long long g = (n + NORM_CHUNK - 1) / NORM_CHUNK;
    return g < 1 ? 1 : g > NORM_GROUPS ? NORM_GROUPS : g;
}
size_t workspace_of(const w2l_adamw_tensor* t, int n)
{
    size_t sums = 0;
    for (int i = 0; i < n; ++i) sums += (size_t)norm_groups(t[i].n);
    return 256 + round_up(sums * sizeof(double), 256);
}

struct Range {
    uintptr_t at, end;
    bool written;
};
// Nothing that the call writes may be read or written as anything else: two entries of one tensor would race
int overlap(const w2l_adamw_tensor* t, int n, size_t grad_size, int bits, const Range* more, int n_more)
{
    Range* const r = new (std::nothrow) Range[(size_t)n * 7 + 4];
    if (!r) return W2L_ERR_LAUNCH;
    size_t k = 0;
    auto add = [&](const void* p, size_t bytes, bool written) {
        if (p && bytes) r[k++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written};
    };
    for (int i = 0; i < n; ++i) {
        const size_t v = (size_t)t[i].n;
        add(t[i].w, v * 4, true);
        add(t[i].grad, v * grad_size, false);
        add(t[i].m, v * bits / 8, true);
        add(t[i].v, v * bits / 8, true);
        add(t[i].w_lowp, v * 2, true);
        if (bits == 8) {
            add(t[i].m_exp, (v + BLOCK - 1) / BLOCK, true);
            add(t[i].v_exp, (v + BLOCK - 1) / BLOCK, true);
        }
    }
    for (int i = 0; i < n_more; ++i)
        if (more[i].at != more[i].end && more[i].at) r[k++] = more[i];
    std::sort(r, r + k, [](const Range& a, const Range& b) { return a.at < b.at; });
    uintptr_t read = 0, written = 0;  // how far those before reach
    bool bad = false;
    for (size_t i = 0; i < k && !bad; ++i) {
        bad = r[i].at < written || (r[i].written && r[i].at < read);
        uintptr_t& end = r[i].written ? written : read;
        if (r[i].end > end) end = r[i].end;
    }
    delete[] r;
    return bad ? W2L_ERR_OVERLAP : W2L_OK;
}

template <typename G>
int launch(const w2l_adamw_tensor* t, int n, int bits, const Hyper& h, const float* lr, const int* step, float* grad_norm, void* ws, hipStream_t st)
{
    double* const sums = ws ? reinterpret_cast<double*>(static_cast<char*>(ws) + 256) : nullptr;  // (none: neither norm nor scalars from the device)
    Scalars* now = nullptr;
    const bool norm = h.max_norm > 0. || grad_norm;
    const Moments o{(float)h.beta1, (float)(1. - h.beta1), (float)h.beta2, (float)(1. - h.beta2)};
    const Scalars by_value = scalars_of(h, pow(h.beta1, (double)h.step), pow(h.beta2, (double)h.step));
    size_t count = 0;
    if (norm || lr || step) {
        now = static_cast<Scalars*>(ws);
        for (int i = 0; norm && i < n; i += MOST) {
            Table tab{};
            unsigned groups = 0;
            tab.number = i;
            tab.count = n - i < MOST ? n - i : MOST;
            for (int j = 0; j < tab.count; ++j) {
                tab.e[j].grad = t[i + j].grad;
                tab.e[j].n = t[i + j].n;
                tab.first[j] = groups;
                groups += (unsigned)norm_groups(t[i + j].n);
            }
            tab.first[tab.count] = groups;
            hipLaunchKernelGGL(adamw_norm_k<G>, dim3(groups), dim3(THREADS), 0, st, tab, sums + count);
            if (int rc = launch_status()) return rc;
            count += groups;
        }
        hipLaunchKernelGGL(adamw_now_k, dim3(1), dim3(1024), 0, st, h, by_value, lr, step, sums, (int)count, grad_norm, now);
        if (int rc = launch_status()) return rc;
    }
    const long long chunk = bits == 32 ? CHUNK32 : CHUNK8;
    for (int i = 0; i < n;) {
        Table tab{};
        unsigned groups = 0;
        tab.number = i;
        for (; tab.count < MOST && i < n; ++i, ++tab.count) {  // (a tensor has at most MOST_GROUPS by itself)
            const w2l_adamw_tensor& a = t[i];
            const long long more = (a.n + chunk - 1) / chunk;
            if (groups + more > MOST_GROUPS) break;
            tab.e[tab.count] = {a.w, a.grad, a.m, a.v, a.m_exp, a.v_exp, static_cast<bf16_t*>(a.w_lowp), a.n, a.weight_decay};
            tab.first[tab.count] = groups;
            groups += (unsigned)more;
        }
        tab.first[tab.count] = groups;
        if (!groups) continue;
        if (bits == 32) hipLaunchKernelGGL(adamw32_k<G>, dim3(groups), dim3(THREADS), 0, st, tab, by_value, now, o);
        else hipLaunchKernelGGL(adamw8_k<G>, dim3(groups), dim3(THREADS), 0, st, tab, by_value, now, o);
        if (int rc = launch_status()) return rc;
    }
    return W2L_OK;
}

}  // namespace

extern "C" size_t w2l_adamw_workspace_bytes(const w2l_adamw_tensor* tensors, int n_tensors)
{
    if (!tensors || n_tensors < 1 || n_tensors > W2L_ADAMW_MAX_TENSORS) return 0;
    for (int i = 0; i < n_tensors; ++i)
        if (tensors[i].n < 0 || tensors[i].n > W2L_ADAMW_MAX_VALUES) return 0;
    return workspace_of(tensors, n_tensors);
}

extern "C" int w2l_adamw_step(const w2l_adamw_tensor* tensors, int n_tensors, int grad_dtype, int moment_bits, long long step, double lr,
                              double beta1, double beta2, double eps, double grad_scale, double max_norm, unsigned seed, const float* lr_dev,
                              const int* step_dev, float* grad_norm, void* workspace, size_t ws_bytes, void* stream)
{
    if (!tensors) return W2L_ERR_NULL;
    if (n_tensors < 1 || n_tensors > W2L_ADAMW_MAX_TENSORS) return W2L_ERR_SHAPE;
    const bool eight = moment_bits == 8;
    for (int i = 0; i < n_tensors; ++i) {
        const w2l_adamw_tensor& a = tensors[i];
        if (a.n < 0 || a.n > W2L_ADAMW_MAX_VALUES) return W2L_ERR_SHAPE;
        if (a.n == 0) continue;
        if (!a.w || !a.grad || !a.m || !a.v || (eight && (!a.m_exp || !a.v_exp))) return W2L_ERR_NULL;
        if (!(a.weight_decay >= 0.) || !(a.weight_decay < INFINITY)) return W2L_ERR_SHAPE;
        if (!aligned16(a.w) || !aligned16(a.grad) || !aligned16(a.m) || !aligned16(a.v) || (a.w_lowp && !aligned16(a.w_lowp))) return W2L_ERR_ALIGN;
    }
    auto within = [](double v, double lo, double hi) { return v >= lo && v <= hi; };  // (not NaN)
    if ((!step_dev && step < 1) || !within(lr, 0., 3e38) || !within(beta1, 0., 1. - 1e-7) || !within(beta2, 0., 1. - 1e-7) || !within(eps, 1e-37, 3e38) ||
        !within(grad_scale, -3e38, 3e38) || !within(max_norm, 0., 3e38))
        return W2L_ERR_SHAPE;
    if (!valid_dtype(grad_dtype) || (moment_bits != 32 && !eight)) return W2L_ERR_DTYPE;
    if ((reinterpret_cast<uintptr_t>(lr_dev) | reinterpret_cast<uintptr_t>(step_dev) | reinterpret_cast<uintptr_t>(grad_norm)) & 3u) return W2L_ERR_ALIGN;
    size_t need = 0;
    if (max_norm > 0. || grad_norm || lr_dev || step_dev) {
        need = workspace_of(tensors, n_tensors);
        if (!workspace || ws_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return W2L_ERR_WORKSPACE;
    }
    auto range = [](const void* p, size_t bytes, bool written) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p);
        return Range{a, p ? a + bytes : a, written};
    };
    const Range more[4] = {range(workspace, need, true), range(grad_norm, 4, true), range(lr_dev, 4, false), range(step_dev, 4, false)};
    if (int rc = overlap(tensors, n_tensors, dtype_size(grad_dtype), moment_bits, more, 4)) return rc;
    const Hyper h{lr, beta1, beta2, eps, grad_scale, max_norm, step, seed};
    return grad_dtype == W2L_BF16 ? launch<bf16_t>(tensors, n_tensors, moment_bits, h, lr_dev, step_dev, grad_norm, workspace, (hipStream_t)stream)
                                  : launch<float>(tensors, n_tensors, moment_bits, h, lr_dev, step_dev, grad_norm, workspace, (hipStream_t)stream);
}
