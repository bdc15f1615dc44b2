// Log-probabilities, entropy and the likeliest classes of rows of scores, and the gradient of the first two.  Bound by HBM: the
// scores are read once forward, read and written once backward.
//
// With m the row's maximum, d = z - m, s = sum exp(d), t = sum d exp(d):
//   lse = m + log s,  log p_j = d_j - log s,  entropy = log s - t / s.
// Each thread keeps m, s, t of what it has read; a larger maximum m' turns them into s f and (t + s (m - m')) f with f = exp(m - m').
#include "vec_common.h"
#include <algorithm>

namespace {

constexpr int NT = 256;

struct LpArgs {
    const void *z;
    const int *ids;
    float *logp, *entropy, *lse, *top_logp;
    int *top_ids;
    int rows, classes, k;
    long long stride;
};

// Orders scores as whole numbers, larger first: value, then the lower index.  -0 counts as 0, a NaN ranks above everything.
__device__ __forceinline__ unsigned long long key_of(float z, int index)
{
    z += 0.f;
    unsigned u = z != z ? 0x7fffffffu : __float_as_uint(z);
    u ^= (unsigned)((int)u >> 31) | 0x80000000u;
    return (unsigned long long)u << 32 | (unsigned)~index;
}
__device__ __forceinline__ float score_of(unsigned long long key)
{
    unsigned u = (unsigned)(key >> 32);
    u ^= (u >> 31) != 0 ? 0x80000000u : 0xffffffffu;
    return __uint_as_float(u);
}
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)~(unsigned)key; }

struct Soft { float m, s, t; };   // maximum, sum exp, sum (z - m) exp

__device__ __forceinline__ void add_score(Soft &a, float z)
{
    if (z > a.m) {
        const float f = __expf(a.m - z);   // m = -inf at first: f = 0 and s = t = 0
        a.t = f > 0.f ? fmaf(a.s, a.m - z, a.t) * f : 0.f;   // s (m - z) may pass the range where f is 0
        a.s *= f;
        a.m = z;
    }
    if (z != -INFINITY) {
        const float d = z - a.m, e = __expf(d);
        a.s += e;
        if (!(d < -200.f)) a.t = fmaf(d, e, a.t);   // below, e is 0, and d may be -inf
    }
}
__device__ __forceinline__ void join(Soft &a, const Soft &b)
{
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) { a.s += b.s; a.t += b.t; return; }   // nothing yet on either side, or NaN sums
    const float da = a.m - m, db = b.m - m, fa = __expf(da), fb = __expf(db);
    const float ta = fa > 0.f ? fmaf(a.s, da, a.t) * fa : 0.f, tb = fb > 0.f ? fmaf(b.s, db, b.t) * fb : 0.f;
    a.s = a.s * fa + b.s * fb;   // a NaN sum stays one
    a.t = ta + tb;
    a.m = m;
}
__device__ __forceinline__ void wave_join(Soft &a)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const Soft b = {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)};
        // the same order on both sides: the lanes agree in every bit
        Soft lo = (threadIdx.x & o) ? b : a;
        join(lo, (threadIdx.x & o) ? a : b);
        a = lo;
    }
}
__device__ __forceinline__ unsigned long long wave_top(unsigned long long v)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const unsigned long long w = (unsigned long long)__shfl_xor((long long)v, o, 64);
        v = v > w ? v : w;
    }
    return v;
}

template <typename T>
__global__ __launch_bounds__(NT) void k_logprobs(LpArgs a)
{
    __shared__ Soft part[NT / 64];
    __shared__ unsigned long long best[2][NT / 64];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r = blockIdx.x;
    const T *z = (const T *)a.z + (size_t)r * a.stride;
    Soft mine = {-INFINITY, 0.f, 0.f};
    for (int c = t; c < a.classes; c += NT) add_score(mine, as_f32(z[c]));
    wave_join(mine);
    if (lane == 0) part[wave] = mine;
    __syncthreads();
    Soft all = part[0];
    for (int w = 1; w < NT / 64; ++w) join(all, part[w]);
    const bool none = all.m == -INFINITY && all.s == 0.f;
    const float log_s = logf(all.s), lse = none ? -INFINITY : all.m + log_s;
    if (t == 0) {
        if (a.lse != nullptr) a.lse[r] = lse;
        if (a.entropy != nullptr) a.entropy[r] = none ? 0.f : log_s - all.t / all.s;
        if (a.logp != nullptr) {
            const int id = a.ids[r];
            a.logp[r] = id < 0 || id >= a.classes ? 0.f : none ? -INFINITY : as_f32(z[id]) - lse;
        }
    }
    unsigned long long last = ~0ull;
    for (int j = 0; j < a.k; ++j) {   // the largest below the one before
        unsigned long long top = 0;
        for (int c = t; c < a.classes; c += NT) {
            const unsigned long long key = key_of(as_f32(z[c]), c);
            if (key < last && key > top) top = key;
        }
        top = wave_top(top);
        if (lane == 0) best[j & 1][wave] = top;
        __syncthreads();
        last = best[j & 1][0];
        for (int w = 1; w < NT / 64; ++w) last = last > best[j & 1][w] ? last : best[j & 1][w];
        if (t == 0) {
            a.top_ids[(size_t)r * a.k + j] = index_of(last);
            a.top_logp[(size_t)r * a.k + j] = none ? -INFINITY : score_of(last) - lse;
        }
    }
}

struct LpGradArgs {
    const void *z;
    const int *ids;
    const float *lse, *entropy, *dlogp, *dentropy;
    void *dz;
    int rows, classes;
    long long stride;
};

template <typename T>
__global__ __launch_bounds__(NT) void k_logprobs_grad(LpGradArgs a)
{
    const int r = blockIdx.x;
    const T *z = (const T *)a.z + (size_t)r * a.stride;
    T *dz = (T *)a.dz + (size_t)r * a.stride;
    const float lse = a.lse[r], h = a.entropy != nullptr ? a.entropy[r] : 0.f, de = a.dentropy != nullptr ? a.dentropy[r] : 0.f;
    const int id = a.ids != nullptr ? a.ids[r] : -1;
    const float dl = a.dlogp != nullptr && id >= 0 && id < a.classes ? a.dlogp[r] : 0.f;
    for (int c = threadIdx.x; c < a.classes; c += NT) {
        const float lp = as_f32(z[c]) - lse, p = __expf(lp);
        // p (log p + h) is 0 where p is, also for log p = -inf
        float g = -p * dl - de * (lp < -200.f ? 0.f : p * (lp + h));
        if (c == id) g += dl;
        dz[c] = from_f32<T>(lse == -INFINITY ? 0.f : g);
    }
}

long long stride_of(const dp_logprobs_desc &d) { return d.row_stride != 0 ? (long long)d.row_stride : d.classes; }

dp_status check_desc(const dp_logprobs_desc *d)
{
    if (d == nullptr) { dp_set_error("log-probabilities: descriptor is NULL"); return DP_ERR_NULL; }
    if (d->io_dtype != DP_F32 && d->io_dtype != DP_BF16) { dp_set_error("log-probabilities: unknown io_dtype %d", d->io_dtype); return DP_ERR_UNSUPPORTED; }
    if (d->rows < 0 || d->classes < 1) { dp_set_error("log-probabilities: rows must not be negative, classes positive"); return DP_ERR_BAD_DESC; }
    // a grid has fewer than 2^32 threads; class numbers of a block's last steps pass the row's end
    if (d->rows > (1 << 23) || d->classes > (1 << 30)) { dp_set_error("log-probabilities: rows > 2^23 or classes > 2^30"); return DP_ERR_BAD_DESC; }
    if (d->row_stride != 0 && d->row_stride < d->classes) { dp_set_error("log-probabilities: row_stride is smaller than a row"); return DP_ERR_BAD_DESC; }
    if (stride_of(*d) > (1ll << 40)) { dp_set_error("log-probabilities: row_stride too large"); return DP_ERR_BAD_DESC; }
    if (d->top_k < 0 || d->top_k > DP_LOGPROBS_MAX_TOP || d->top_k > d->classes) {
        dp_set_error("log-probabilities: top_k must be in 0 ... min(classes, %d)", DP_LOGPROBS_MAX_TOP);
        return DP_ERR_BAD_DESC;
    }
    return DP_OK;
}

bool misaligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

dp_status check_scores(const dp_logprobs_desc &d, const void *z)
{
    if (z == nullptr) { dp_set_error("log-probabilities: the scores are NULL"); return DP_ERR_NULL; }
    if (misaligned(z, d.io_dtype == DP_BF16 ? 2 : 4)) { dp_set_error("log-probabilities: scores must be aligned to their type"); return DP_ERR_BAD_DESC; }
    return DP_OK;
}

}  // namespace

extern "C" size_t dp_logprobs_workspace_bytes(const dp_logprobs_desc *desc)
{
    (void)desc;
    return 0;
}

extern "C" dp_status dp_logprobs_fwd(const dp_logprobs_desc *desc, const void *z, const int32_t *ids, float *logp, float *entropy, float *lse,
                                     float *top_logp, int32_t *top_ids, void *ws, size_t ws_bytes, void *hip_stream)
{
    dp_status s = check_desc(desc);
    if (s != DP_OK) return s;
    const dp_logprobs_desc &d = *desc;
    if (d.rows == 0) return DP_OK;
    if ((s = check_scores(d, z)) != DP_OK) return s;
    if (d.top_k > 0 && (top_logp == nullptr || top_ids == nullptr)) { dp_set_error("log-probabilities: top_k needs top_logp and top_ids"); return DP_ERR_NULL; }
    if (logp != nullptr && ids == nullptr) { dp_set_error("log-probabilities: logp needs ids"); return DP_ERR_NULL; }
    if (logp == nullptr && entropy == nullptr && lse == nullptr && d.top_k == 0) { dp_set_error("log-probabilities: no output requested"); return DP_ERR_NULL; }
    for (const void *p : {(const void *)ids, (const void *)logp, (const void *)entropy, (const void *)lse, (const void *)top_logp, (const void *)top_ids})
        if (misaligned(p, 4)) { dp_set_error("log-probabilities: pointers must be 4-byte aligned"); return DP_ERR_BAD_DESC; }
    (void)ws; (void)ws_bytes;
    const LpArgs a = {z, ids, logp, entropy, lse, top_logp, top_ids, d.rows, d.classes, d.top_k, stride_of(d)};
    if (d.io_dtype == DP_BF16) hipLaunchKernelGGL(k_logprobs<bf16_t>, dim3(d.rows), dim3(NT), 0, (hipStream_t)hip_stream, a);
    else hipLaunchKernelGGL(k_logprobs<float>, dim3(d.rows), dim3(NT), 0, (hipStream_t)hip_stream, a);
    return launched("log-probabilities");
}

extern "C" dp_status dp_logprobs_bwd(const dp_logprobs_desc *desc, const void *z, const int32_t *ids, const float *lse, const float *entropy,
                                     const float *dlogp, const float *dentropy, void *dz, void *hip_stream)
{
    dp_status s = check_desc(desc);
    if (s != DP_OK) return s;
    const dp_logprobs_desc &d = *desc;
    if (d.rows == 0) return DP_OK;
    if ((s = check_scores(d, z)) != DP_OK || (s = check_scores(d, dz)) != DP_OK) return s;
    if (lse == nullptr) { dp_set_error("log-probabilities' gradient: lse is NULL"); return DP_ERR_NULL; }
    if (dlogp == nullptr && dentropy == nullptr) { dp_set_error("log-probabilities' gradient: neither dlogp nor dentropy is given"); return DP_ERR_NULL; }
    if ((dlogp != nullptr && ids == nullptr) || (dentropy != nullptr && entropy == nullptr)) {
        dp_set_error("log-probabilities' gradient: dlogp needs ids, dentropy needs entropy");
        return DP_ERR_NULL;
    }
    for (const void *p : {(const void *)ids, (const void *)lse, (const void *)entropy, (const void *)dlogp, (const void *)dentropy})
        if (misaligned(p, 4)) { dp_set_error("log-probabilities' gradient: pointers must be 4-byte aligned"); return DP_ERR_BAD_DESC; }
    const LpGradArgs a = {z, ids, lse, entropy, dlogp, dentropy, dz, d.rows, d.classes, stride_of(d)};
    if (d.io_dtype == DP_BF16) hipLaunchKernelGGL(k_logprobs_grad<bf16_t>, dim3(d.rows), dim3(NT), 0, (hipStream_t)hip_stream, a);
    else hipLaunchKernelGGL(k_logprobs_grad<float>, dim3(d.rows), dim3(NT), 0, (hipStream_t)hip_stream, a);
    return launched("log-probabilities' gradient");
}
