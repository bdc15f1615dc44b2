// Operators over all parameters of a network in one launch: the 2-norm of the gradients with the factor that clips it,
// and an AdamW step with its two states in fp32 or in 8 bits.  Bound by HBM: every element is read and written once.
//
// A network has hundreds of tensors, most of them a few hundred elements long, so a launch per tensor would cost more than the
// step.  The tensors are cut into chunks of 4096 elements; a table in device memory, made once per network, has one 64-byte record per
// chunk with all addresses of the chunk.  A block reads its record with one scalar load (a table of tensors and a search
// would be two or more loads that depend on each other) and works on one chunk.
#include "vec_common.h"
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <vector>

namespace {

constexpr int kChunk = 4096;      // elements of a chunk: 16 per thread of a block
constexpr int kBlock = 256;       // elements that share a scale of an 8-bit state
constexpr int kNormBlocks = 1024; // four blocks per compute unit

// table record; w16, ms, vs may be null
struct alignas(64) Chunk {
    const float *g;
    float *w;
    bf16_t *w16;
    void *m, *v;
    float *ms, *vs;
    int count;     // 1 ... kChunk
    float decay;
};
static_assert(sizeof(Chunk) == 64, "one scalar load of 16 dwords");

// ---- norm ---------------------------------------------------------------------------------------------------------

// Squares and sums in 64 bits: the square of a gradient beyond 1e19 is finite, and the result does not depend on how the
// gradients are spread over the tensors.
template <bool PAST> __device__ __forceinline__ double square_sum(const Chunk &c, int t)
{
    double s = 0.0;
    const int nvec = c.count >> 2;
    float4 v[kChunk / 1024];
#pragma unroll
    for (int u = 0; u < kChunk / 1024; ++u) {
        const int i = u * 256 + t;
        v[u] = i < nvec ? load_vec<float4, PAST>(c.g + 4 * i) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int u = 0; u < kChunk / 1024; ++u) {
        s = fma((double)v[u].x, (double)v[u].x, s); s = fma((double)v[u].y, (double)v[u].y, s);
        s = fma((double)v[u].z, (double)v[u].z, s); s = fma((double)v[u].w, (double)v[u].w, s);
    }
    if (t < (c.count & 3)) { const double e = c.g[nvec * 4 + t]; s = fma(e, e, s); }
    return s;
}

// the block's sum: wavefronts by themselves, their sums in order
template <int N> __device__ __forceinline__ double block_sum(double s)
{
    __shared__ double sm[N / 64];
    s = wave_sum_fast(s);
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < N / 64; ++w) s += sm[w];
    return s;
}

__device__ __forceinline__ void write_norm(double sum, float max_norm, float *out)
{
    const double norm = sqrt(sum);
    out[0] = (float)norm;
    // a norm that is not finite gives 0, which dp_adamw_step takes for "skip this step"
    out[1] = !(norm <= 1.7e308) ? 0.f : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

// Bound by reading: 138 M elements 81 us (6.8 TB/s; through the caches 101), 25.5 M in HBM 20.6 (5.0).  A block takes every gridDim-th chunk; a chunk's
// four vectors per thread are on their way together.
template <bool PAST> __global__ __launch_bounds__(256) void k_norm_partial(const Chunk *__restrict__ table, long long n_chunks, double *__restrict__ partial)
{
    double s = 0.0;
    for (long long i = blockIdx.x; i < n_chunks; i += gridDim.x) s += square_sum<PAST>(table[i], threadIdx.x);
    s = block_sum<256>(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void k_norm_final(const double *__restrict__ partial, int n, float max_norm, float *__restrict__ out)
{
    double v[kNormBlocks / 256], s = 0.0;
#pragma unroll
    for (int u = 0; u < kNormBlocks / 256; ++u) {
        const int i = u * 256 + threadIdx.x;
        v[u] = i < n ? partial[i] : 0.0;
    }
#pragma unroll
    for (int u = 0; u < kNormBlocks / 256; ++u) s += v[u];
    s = block_sum<256>(s);
    if (threadIdx.x == 0) write_norm(s, max_norm, out);
}

// A short list in one block, a chunk to every four wavefronts: no second kernel to wait for (8 chunks 6.0 -> 3.3 us, 24: 6.1 -> 5.2; 32: 6.2 by both).
constexpr int kNormShort = 24;
__global__ __launch_bounds__(1024) void k_norm_short(const Chunk *__restrict__ table, int n_chunks, float max_norm, float *__restrict__ out)
{
    double s = 0.0;
    for (int i = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8); i < n_chunks; i += 4) s += square_sum<false>(table[i], threadIdx.x & 255);
    s = block_sum<1024>(s);
    if (threadIdx.x == 0) write_norm(s, max_norm, out);
}

int norm_blocks(long long n_chunks) { return (int)std::max(1ll, std::min<long long>(n_chunks, kNormBlocks)); }

// ---- AdamW --------------------------------------------------------------------------------------------------------

struct AdamArgs {
    float beta1, beta2, one_minus_beta1, one_minus_beta2;
    float step_size;        // lr / (1 - beta1^step)
    float inv_root_bc2;     // 1 / sqrt(1 - beta2^step)
    float eps, lr;
    unsigned long long seed;
};

// The step's factor on the gradients; a step whose factor is 0 or NaN is skipped as a whole.
__device__ __forceinline__ bool step_factor(const float *scale, float &s)
{
    s = scale != nullptr ? *scale : 1.f;
    return fabsf(s) > 0.f;
}

// Each product and sum is rounded by itself, as the definition is written: an 8-bit state then follows from its definition to the
// last code, whoever computes it (a fused multiply-add would tip one random rounding in 10^6 the other way).  The kernels are bound by memory either way.
__device__ __forceinline__ void adam_moments(const AdamArgs &a, float g, float &m, float &v)
{
#pragma clang fp contract(off)
    m = a.beta1 * m + a.one_minus_beta1 * g;
    v = a.beta2 * v + a.one_minus_beta2 * (g * g);
}
__device__ __forceinline__ float adam_weight(const AdamArgs &a, float keep, float w, float m, float root)
{
    return fmaf(-a.step_size * m, __builtin_amdgcn_rcpf(fmaf(root, a.inv_root_bc2, a.eps)), keep * w);   // one unit in the last place of the update
}

// Bound by HBM, 30 bytes per element with the bf16 copy (28 without): 138 M elements 749 us (5.5 TB/s), 25.5 M 140 (5.5; through the caches 147).  All sixteen vectors of a
// thread are read before the first is used.  PAST: 1: weights and states go past the caches, 2: gradients too.
template <int PAST> __global__ __launch_bounds__(256) void k_adamw(const Chunk *__restrict__ table, AdamArgs a, const float *__restrict__ scale)
{
    const Chunk c = table[blockIdx.x];
    float s;
    if (!step_factor(scale, s)) return;
    const int t = threadIdx.x, nvec = c.count >> 2;
    const float keep = fmaf(-a.lr, c.decay, 1.f);
    float *m32 = (float *)c.m, *v32 = (float *)c.v;
    constexpr int U = kChunk / 1024;
    float4 g[U], w[U], m[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = u * 256 + t;
        if (i < nvec) {
            g[u] = load_vec<float4, PAST == 2>(c.g + 4 * i);
            m[u] = load_vec<float4, PAST != 0>(m32 + 4 * i);
            v[u] = load_vec<float4, PAST != 0>(v32 + 4 * i);
            w[u] = load_vec<float4, PAST != 0>(c.w + 4 * i);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = u * 256 + t;
        if (i >= nvec) continue;
        const float ge[4] = {g[u].x * s, g[u].y * s, g[u].z * s, g[u].w * s};
        float *me = &m[u].x, *ve = &v[u].x, *we = &w[u].x;
        Pack<bf16_t, 4> o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            adam_moments(a, ge[e], me[e], ve[e]);
            we[e] = adam_weight(a, keep, we[e], me[e], sqrtf(ve[e]));
            o.v[e] = from_f32<bf16_t>(we[e]);
        }
        store_vec<float4, PAST != 0>(m32 + 4 * i, m[u]);
        store_vec<float4, PAST != 0>(v32 + 4 * i, v[u]);
        store_vec<float4, PAST != 0>(c.w + 4 * i, w[u]);
        if (c.w16 != nullptr) reinterpret_cast<Pack<bf16_t, 4> *>(c.w16)[i] = o;
    }
    if (t < (c.count & 3)) {
        const int i = nvec * 4 + t;
        float me = m32[i], ve = v32[i];
        adam_moments(a, c.g[i] * s, me, ve);
        const float we = adam_weight(a, keep, c.w[i], me, sqrtf(ve));
        m32[i] = me; v32[i] = ve; c.w[i] = we;
        if (c.w16 != nullptr) c.w16[i] = from_f32<bf16_t>(we);
    }
}

// ---- 8-bit states -------------------------------------------------------------------------------------------------
//
// m and sqrt(v) (whose range is half of v's in the exponent) are held as e4m3 floats with one fp32 scale for each 256
// elements, value = float8 * scale, the largest magnitude of a block at 448.  Rounding is stochastic: a step changes v
// by 0.1 % at beta2 = 0.999 while neighbouring e4m3 values are 6 to 12 % apart, so rounding to the nearest would leave
// most values where they are for good; taking the upper neighbour with the probability of the distance keeps them right on average.
// The 16 random bits of each value are fields of a SplitMix64 output (published: Steele, Lea, Flood 2014) whose counter
// is the element's place in the list, so the result depends on the seed and the list alone and on no launch shape.

__device__ __forceinline__ unsigned long long splitmix64(unsigned long long seed, unsigned long long counter)
{
    unsigned long long z = seed + (counter + 1) * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// e4m3 code of a in [0, 448 (1 + 2^-21)]: up from the lower neighbour with probability (distance + rnd16 / 2^16 >= 1).  Normal values
// add the random bits below the three fraction bits that stay; below 2^-6 the values are multiples of 2^-9.
__device__ __forceinline__ unsigned encode8(float a, unsigned rnd16)
{
    const int normal = (int)((__float_as_uint(a) + (rnd16 << 4)) >> 20) - 960;
    const int small = (int)(a * 512.f + (float)rnd16 * (1.f / 65536.f));
    return (unsigned)min(a < 0.015625f ? small : normal, 126);
}

// scale, and 448 / largest (as reciprocal times 448, each rounded), from the bits of a block's largest magnitude.  Not finite: the scale is NaN, as fp32 states would be.
// Below 2e-36, where 1 / largest times 448 overflows: the block is zero.
__device__ __forceinline__ float scale8(unsigned top_bits, float &inv)
{
    const float top = __uint_as_float(top_bits);
    if (top_bits >= 0x7f800000u) { inv = 0.f; return __uint_as_float(0x7fc00000u); }
    if (top < 2e-36f) { inv = 0.f; return 0.f; }
    inv = (1.f / top) * 448.f;
    return top * (1.f / 448.f);
}

// One lane's four elements of a block of 256: the new states in m, root, the new weights in w.
struct Four { float g[4], w[4]; unsigned m8, v8; };

__device__ __forceinline__ void update_four(const AdamArgs &a, float s, float keep, float mscale, float vscale, Four &f, float (&m)[4], float (&root)[4])
{
    auto each = [&](int e, float m0, float r0) {
        m[e] = m0 * mscale;
        const float r = r0 * vscale;
        float v = r * r;
        adam_moments(a, f.g[e] * s, m[e], v);
        root[e] = sqrtf(v);
        f.w[e] = adam_weight(a, keep, f.w[e], m[e], root[e]);
    };
    each(0, __builtin_amdgcn_cvt_f32_fp8(f.m8, 0), __builtin_amdgcn_cvt_f32_fp8(f.v8, 0));
    each(1, __builtin_amdgcn_cvt_f32_fp8(f.m8, 1), __builtin_amdgcn_cvt_f32_fp8(f.v8, 1));
    each(2, __builtin_amdgcn_cvt_f32_fp8(f.m8, 2), __builtin_amdgcn_cvt_f32_fp8(f.v8, 2));
    each(3, __builtin_amdgcn_cvt_f32_fp8(f.m8, 3), __builtin_amdgcn_cvt_f32_fp8(f.v8, 3));
}

// The wavefront's 256 states as codes in f and the scales.  pair: number of the lane's first pair of elements in the list.
__device__ __forceinline__ void store_four(const AdamArgs &a, unsigned long long pair, const float (&m)[4], const float (&root)[4], Four &f, float &mscale, float &vscale)
{
    unsigned mtop = 0, rtop = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        mtop = max(mtop, __float_as_uint(fabsf(m[e])));
        rtop = max(rtop, __float_as_uint(fabsf(root[e])));
    }
    float minv, rinv;
    mscale = scale8(wave_max_fast(mtop), minv);
    vscale = scale8(wave_max_fast(rtop), rinv);
    f.m8 = f.v8 = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned long long r = splitmix64(a.seed, pair + (e >> 1)) >> (32 * (e & 1));
        unsigned code = encode8(fabsf(m[e]) * minv, (unsigned)r & 0xffffu);
        if (m[e] < 0.f) code |= 0x80u;
        f.m8 |= code << (8 * e);
        // a positive sqrt(v) stays positive: as 0 it would let the next step's update grow
        const float ra = root[e] * rinv;
        code = encode8(ra, (unsigned)(r >> 16) & 0xffffu);
        f.v8 |= (ra > 0.f ? max(code, 1u) : code) << (8 * e);
    }
}

// A wavefront works on 256 elements that share scales, four per lane; a block's four wavefronts on four times four of them.  A whole chunk's
// loads are issued together; a tensor's last chunk goes 256 elements at a time, with bounds.  18 bytes and 97 vector instructions per element: bound by HBM
// (25.5 M elements 83 us, 5.5 TB/s; through the caches 90) with the vector units busy for two thirds of that; PAST as above.
template <int PAST> __global__ __launch_bounds__(256) void k_adamw8(const Chunk *__restrict__ table, AdamArgs a, const float *__restrict__ scale)
{
    const Chunk c = table[blockIdx.x];
    float s;
    if (!step_factor(scale, s)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float keep = fmaf(-a.lr, c.decay, 1.f);
    unsigned char *m8 = (unsigned char *)c.m, *v8 = (unsigned char *)c.v;
    const unsigned long long first = (unsigned long long)blockIdx.x * kChunk;
    if (c.count == kChunk) {
        constexpr int U = kChunk / kBlock / 4;
        Four f[U];
        float ms[U], vs[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = wave + 4 * u, i = b * kBlock + lane * 4;
            *reinterpret_cast<float4 *>(f[u].g) = load_vec<float4, PAST == 2>(c.g + i);
            *reinterpret_cast<float4 *>(f[u].w) = load_vec<float4, PAST != 0>(c.w + i);
            f[u].m8 = load_vec<unsigned, PAST != 0>(m8 + i);
            f[u].v8 = load_vec<unsigned, PAST != 0>(v8 + i);
            ms[u] = c.ms[b];
            vs[u] = c.vs[b];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = wave + 4 * u, i = b * kBlock + lane * 4;
            float m[4], root[4];
            update_four(a, s, keep, ms[u], vs[u], f[u], m, root);
            store_vec<float4, PAST != 0>(c.w + i, *reinterpret_cast<float4 *>(f[u].w));
            if (c.w16 != nullptr) {
                Pack<bf16_t, 4> o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o.v[e] = from_f32<bf16_t>(f[u].w[e]);
                *reinterpret_cast<Pack<bf16_t, 4> *>(c.w16 + i) = o;
            }
            float mscale, vscale;
            store_four(a, (first + (unsigned)i) >> 1, m, root, f[u], mscale, vscale);
            store_vec<unsigned, PAST != 0>(m8 + i, f[u].m8);
            store_vec<unsigned, PAST != 0>(v8 + i, f[u].v8);
            if (lane == 0) { c.ms[b] = mscale; c.vs[b] = vscale; }
        }
        return;
    }
    for (int b = wave; b * kBlock < c.count; b += 4) {
        const int i = b * kBlock + lane * 4;
        Four f = {};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < c.count) {
                f.g[e] = c.g[i + e];
                f.w[e] = c.w[i + e];
                f.m8 |= (unsigned)m8[i + e] << (8 * e);
                f.v8 |= (unsigned)v8[i + e] << (8 * e);
            }
        float m[4], root[4], mscale = c.ms[b], vscale = c.vs[b];
        update_four(a, s, keep, mscale, vscale, f, m, root);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e >= c.count) m[e] = root[e] = 0.f;   // also with a scale that is NaN
        store_four(a, (first + (unsigned)i) >> 1, m, root, f, mscale, vscale);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < c.count) {
                c.w[i + e] = f.w[e];
                m8[i + e] = (unsigned char)(f.m8 >> (8 * e));
                v8[i + e] = (unsigned char)(f.v8 >> (8 * e));
                if (c.w16 != nullptr) c.w16[i + e] = from_f32<bf16_t>(f.w[e]);
            }
        if (lane == 0) { c.ms[b] = mscale; c.vs[b] = vscale; }
    }
}

// ---- checks -------------------------------------------------------------------------------------------------------

constexpr int64_t kMaxCount = (int64_t)1 << 40;
constexpr int64_t kMaxChunks = (1 << 24) - 1;   // a grid has fewer than 2^32 threads

struct Range { uintptr_t lo, hi; int param; bool written; };

dp_status check_param(const dp_param &p, int i, int state, bool &updates)
{
    if (p.count < 0 || p.count > kMaxCount) { dp_set_error("parameter %d: count %lld", i, (long long)p.count); return DP_ERR_BAD_DESC; }
    if (p.count == 0) return DP_OK;
    if (p.grad == nullptr) { dp_set_error("parameter %d: grad is NULL", i); return DP_ERR_NULL; }
    const bool any = p.w32 != nullptr || p.w_bf16 != nullptr || p.m != nullptr || p.v != nullptr || p.m_scale != nullptr || p.v_scale != nullptr;
    if (!any) updates = false;
    else if (p.w32 == nullptr || p.m == nullptr || p.v == nullptr || (state == DP_STATE_Q8 && (p.m_scale == nullptr || p.v_scale == nullptr))) {
        dp_set_error("parameter %d: w32, m, v%s are needed together", i, state == DP_STATE_Q8 ? ", m_scale, v_scale" : "");
        return DP_ERR_NULL;
    }
    if (!aligned16(p.grad) || !aligned16(p.w32) || !aligned16(p.w_bf16) || !aligned16(p.m) || !aligned16(p.v) || !aligned16(p.m_scale) || !aligned16(p.v_scale)) {
        dp_set_error("parameter %d: pointers must be 16-byte aligned", i);
        return DP_ERR_BAD_DESC;
    }
    if (!std::isfinite(p.weight_decay) || p.weight_decay < 0.f) { dp_set_error("parameter %d: weight_decay must be finite and not negative", i); return DP_ERR_BAD_DESC; }
    return DP_OK;
}

// memory that a step writes: whatever else of the list lies there would race with it; gradients may be the same for several parameters
dp_status check_overlap(const dp_param *params, int n, int state)
{
    std::vector<Range> r;
    auto add = [&](const void *p, int64_t bytes, int i, bool written = true) {
        if (p != nullptr) r.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, i, written});
    };
    for (int i = 0; i < n; ++i) {
        const dp_param &p = params[i];
        if (p.count == 0) continue;
        const int64_t state_bytes = state == DP_STATE_Q8 ? p.count : 4 * p.count, scales = 4 * ((p.count + kBlock - 1) / kBlock);
        add(p.w32, 4 * p.count, i); add(p.w_bf16, 2 * p.count, i); add(p.m, state_bytes, i); add(p.v, state_bytes, i);
        if (state == DP_STATE_Q8) { add(p.m_scale, scales, i); add(p.v_scale, scales, i); }
        add(p.grad, 4 * p.count, i, false);
    }
    std::sort(r.begin(), r.end(), [](const Range &x, const Range &y) { return x.lo < y.lo; });
    // by ascending start: the range that reaches furthest, of those that are written and of all
    const Range *written = nullptr, *any = nullptr;
    for (const Range &k : r) {
        const Range *other = k.written ? any : written;
        if (other != nullptr && k.lo < other->hi) { dp_set_error("parameters %d and %d share memory that a step writes", other->param, k.param); return DP_ERR_BAD_DESC; }
        if (k.written && (written == nullptr || k.hi > written->hi)) written = &k;
        if (any == nullptr || k.hi > any->hi) any = &k;
    }
    return DP_OK;
}

int64_t chunks_of(int64_t count) { return (count + kChunk - 1) / kChunk; }

dp_status check_list(const dp_param_list *list)
{
    if (list == nullptr) { dp_set_error("parameter list is NULL"); return DP_ERR_NULL; }
    if (list->n_chunks < 0 || list->n_chunks > kMaxChunks || (list->state != DP_STATE_F32 && list->state != DP_STATE_Q8)) {
        dp_set_error("not a list that dp_param_table_build has filled in");
        return DP_ERR_BAD_DESC;
    }
    if (list->n_chunks > 0 && list->table == nullptr) { dp_set_error("parameter list: no table"); return DP_ERR_NULL; }
    if ((reinterpret_cast<uintptr_t>(list->table) & 63u) != 0) { dp_set_error("parameter list: the table must be 64-byte aligned"); return DP_ERR_BAD_DESC; }
    return DP_OK;
}

// What a step has read is pushed out of the memory-side cache (256 MB) before the next step comes, once it is larger; written there all the
// same, it leaves dirty lines that are written back while the next kernels read.  Gradients come from the backward pass and are
// read twice.  Step of a copy into the gradients, norm, AdamW and a reading of the new weights, us, cached / states past / all past:
//   9 M elements 78 / 82 / 82; 14 M 127 / 115 / 118; 25.5 M 230 / 200 / 207; 33 M 293 / 256 / 262; 45 M 387 / 371 / 356; 138 M 1193 / 1136 / 1122
//   8-bit states 9 M 68 / 68 / 68; 18 M 122 / 111 / 113; 25.5 M 174 / 159 / 160; 33 M 218 / 196 / 198; 45 M 288 / 273 / 264; 138 M 858 / 820 / 817
// The bf16 copies of the weights stay in the caches: the next forward pass reads them, and their stores made no difference.
bool states_past(const dp_param_list *list) { return list->n_elements > (int64_t)10 << 20; }
bool gradients_past(const dp_param_list *list) { return list->n_elements > (int64_t)32 << 20; }

}  // namespace

extern "C" size_t dp_param_table_bytes(const dp_param *params, int32_t n_params)
{
    if (params == nullptr || n_params < 0) return 0;
    int64_t chunks = 0;
    for (int i = 0; i < n_params; ++i) {
        if (params[i].count < 0 || params[i].count > kMaxCount) return 0;
        chunks += chunks_of(params[i].count);
    }
    return (size_t)chunks * sizeof(Chunk);
}

extern "C" dp_status dp_param_table_build(const dp_param *params, int32_t n_params, int32_t state, void *host_table, size_t host_table_bytes,
                                          const void *device_table, dp_param_list *list)
{
    if (list == nullptr || (params == nullptr && n_params != 0)) { dp_set_error("parameter table: null pointer"); return DP_ERR_NULL; }
    if (n_params < 0) { dp_set_error("parameter table: negative number of parameters"); return DP_ERR_BAD_DESC; }
    if (state != DP_STATE_F32 && state != DP_STATE_Q8) { dp_set_error("parameter table: unknown state format %d", state); return DP_ERR_UNSUPPORTED; }
    bool updates = true;
    int64_t chunks = 0, elements = 0;
    for (int i = 0; i < n_params; ++i) {
        const dp_status s = check_param(params[i], i, state, updates);
        if (s != DP_OK) return s;
        chunks += chunks_of(params[i].count);
        elements += params[i].count;
    }
    if (chunks > kMaxChunks) { dp_set_error("parameter table: too many elements"); return DP_ERR_BAD_DESC; }
    if (chunks > 0 && (host_table == nullptr || device_table == nullptr)) { dp_set_error("parameter table: null pointer"); return DP_ERR_NULL; }
    if ((reinterpret_cast<uintptr_t>(device_table) & 63u) != 0) { dp_set_error("parameter table: the device address must be 64-byte aligned"); return DP_ERR_BAD_DESC; }
    if (host_table_bytes < (size_t)chunks * sizeof(Chunk)) {
        dp_set_error("parameter table: needs %zu bytes, got %zu", (size_t)chunks * sizeof(Chunk), host_table_bytes);
        return DP_ERR_WORKSPACE;
    }
    if (updates) {
        dp_status s;
        try { s = check_overlap(params, n_params, state); }
        catch (...) { dp_set_error("parameter table: out of host memory"); return DP_ERR_HIP; }
        if (s != DP_OK) return s;
    }
    unsigned char *out = (unsigned char *)host_table;
    const int64_t es = state == DP_STATE_Q8 ? 1 : 4;
    for (int i = 0; i < n_params; ++i) {
        const dp_param &p = params[i];
        for (int64_t at = 0; at < p.count; at += kChunk, out += sizeof(Chunk)) {
            Chunk c = {};
            c.g = p.grad + at;
            if (updates) {
                c.w = p.w32 + at;
                c.w16 = p.w_bf16 != nullptr ? (bf16_t *)p.w_bf16 + at : nullptr;
                c.m = (char *)p.m + at * es;
                c.v = (char *)p.v + at * es;
                if (state == DP_STATE_Q8) { c.ms = p.m_scale + at / kBlock; c.vs = p.v_scale + at / kBlock; }
            }
            c.count = (int)std::min<int64_t>(kChunk, p.count - at);
            c.decay = p.weight_decay;
            __builtin_memcpy(out, &c, sizeof c);
        }
    }
    list->table = device_table;
    list->n_chunks = chunks;
    list->n_elements = elements;
    list->n_params = n_params;
    list->state = state;
    list->updates = updates ? 1 : 0;
    list->reserved = 0;
    return DP_OK;
}

extern "C" size_t dp_grad_norm_workspace_bytes(const dp_param_list *list)
{
    if (list == nullptr || list->n_chunks < 0) return 0;
    return (size_t)norm_blocks(list->n_chunks) * sizeof(double);
}

extern "C" dp_status dp_grad_norm(const dp_param_list *list, float max_norm, float *norm_and_scale, void *ws, size_t ws_bytes, void *hip_stream)
{
    const dp_status s = check_list(list);
    if (s != DP_OK) return s;
    if (norm_and_scale == nullptr) { dp_set_error("gradient norm: no output"); return DP_ERR_NULL; }
    if (!(max_norm > 0.f)) { dp_set_error("gradient norm: max_norm must be positive (INFINITY: no clipping)"); return DP_ERR_BAD_DESC; }
    if (!aligned16(norm_and_scale) || !aligned16(ws)) { dp_set_error("gradient norm: pointers must be 16-byte aligned"); return DP_ERR_BAD_DESC; }
    const size_t need = dp_grad_norm_workspace_bytes(list);
    if (ws == nullptr || ws_bytes < need) { dp_set_error("gradient norm needs %zu workspace bytes, got %zu", need, ws == nullptr ? (size_t)0 : ws_bytes); return DP_ERR_WORKSPACE; }
    hipStream_t st = (hipStream_t)hip_stream;
    if (list->n_chunks <= kNormShort) {
        hipLaunchKernelGGL(k_norm_short, dim3(1), dim3(1024), 0, st, (const Chunk *)list->table, (int)list->n_chunks, max_norm, norm_and_scale);
        return launched("gradient norm");
    }
    const int blocks = norm_blocks(list->n_chunks);
    hipLaunchKernelGGL(gradients_past(list) ? k_norm_partial<true> : k_norm_partial<false>, dim3(blocks), dim3(256), 0, st, (const Chunk *)list->table, (long long)list->n_chunks, (double *)ws);
    hipLaunchKernelGGL(k_norm_final, dim3(1), dim3(256), 0, st, (const double *)ws, blocks, max_norm, norm_and_scale);
    return launched("gradient norm");
}

extern "C" dp_status dp_adamw_step(const dp_param_list *list, const dp_adamw_hyper *h, const float *grad_scale, void *hip_stream)
{
    const dp_status s = check_list(list);
    if (s != DP_OK) return s;
    if (h == nullptr) { dp_set_error("AdamW: hyper-parameters are NULL"); return DP_ERR_NULL; }
    if (!list->updates && list->n_chunks > 0) { dp_set_error("AdamW: the list has gradients only"); return DP_ERR_NULL; }
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0)) { dp_set_error("AdamW: beta1 and beta2 must be in [0, 1)"); return DP_ERR_BAD_DESC; }
    // without eps an element that never had a gradient would become 0 / 0, and the reciprocal of a subnormal one is infinite
    if (!std::isfinite((float)h->lr) || !((float)h->eps >= FLT_MIN) || !std::isfinite((float)h->eps)) { dp_set_error("AdamW: lr must be finite in fp32, eps finite and at least 2^-126"); return DP_ERR_BAD_DESC; }
    if (h->step < 1) { dp_set_error("AdamW: steps count from 1"); return DP_ERR_BAD_DESC; }
    if ((reinterpret_cast<uintptr_t>(grad_scale) & 3u) != 0) { dp_set_error("AdamW: grad_scale must be 4-byte aligned"); return DP_ERR_BAD_DESC; }
    if (list->n_chunks == 0) return DP_OK;
    AdamArgs a;
    a.beta1 = (float)h->beta1; a.beta2 = (float)h->beta2;
    a.one_minus_beta1 = (float)(1.0 - h->beta1); a.one_minus_beta2 = (float)(1.0 - h->beta2);
    a.step_size = (float)(h->lr / (1.0 - std::pow(h->beta1, (double)h->step)));
    a.inv_root_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, (double)h->step)));
    a.eps = (float)h->eps; a.lr = (float)h->lr;
    a.seed = h->seed;
    const dim3 grid((unsigned)list->n_chunks), block(256);
    const bool q8 = list->state == DP_STATE_Q8;
    const int past = gradients_past(list) ? 2 : states_past(list) ? 1 : 0;
    auto *kernel = q8 ? (past == 2 ? k_adamw8<2> : past == 1 ? k_adamw8<1> : k_adamw8<0>) : past == 2 ? k_adamw<2> : past == 1 ? k_adamw<1> : k_adamw<0>;
    hipLaunchKernelGGL(kernel, grid, block, 0, (hipStream_t)hip_stream, (const Chunk *)list->table, a, grad_scale);
    return launched("AdamW step");
}
