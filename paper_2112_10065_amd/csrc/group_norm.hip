// Group normalisation with an activation, NHWC, forward and backward.  Bound by HBM: the operations per element are few.
//
// Both directions are a reduction over (pixels x channels of a group) per sample, then a pointwise pass that needs its result.
// In NHWC a group is a narrow column of channels, so a block takes whole rows: each thread keeps one vector of channels (16 bytes)
// and walks pixels.  Partial results per channel meet in `part` [sample][split][channel], two floats each:
//   forward    mean and sum of squared deviations of the split's pixels: never a difference of large sums, whatever offset x has
//   backward   A = sum g and B = sum g * xhat of the split's pixels
// The second kernel combines the partials of the groups that its channels belong to, in a fixed order, and applies them; in the
// backward pass its first blocks sum dgamma and dbeta over samples and splits instead.
#include "vec_common.h"
#include <algorithm>
#include <cmath>

namespace {

constexpr int NT = 256;
enum { ACT_NONE = 0, ACT_MASK = 1, ACT_SILU = 2, ACT_RELU = 3 };   // MASK: backward of a ReLU by its saved output

struct GnArgs {
    const void *x, *dy, *y_saved;
    const float *gamma, *beta, *mean_in, *rstd_in;
    void *out;                       // y or dx
    float *mean_out, *rstd_out;      // forward, may be null
    float *dgamma, *dbeta;           // backward, may be null
    float2 *part;
    int n, hw, c, groups, cg;
    int cs, slabs;                   // channels of a slab (the last one may be narrower), slabs
    int splits, split_pixels;        // pixels of a split (the last one may be shorter)
    int chunks, chunk_pixels;        // the same for the second kernel's blocks
    int grad_blocks;                 // blocks of the second kernel that sum dgamma / dbeta
    float eps, inv_count;            // 1 / (hw * cg)
};

template <typename T, int V> __device__ __forceinline__ void load(const T *p, float (&v)[V])
{
    const Pack<T, V> q = *reinterpret_cast<const Pack<T, V> *>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = as_f32(q.v[e]);
}

__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + __expf(-u)); }

// What a thread's vector of channels needs for the pixel loop.
template <int V> struct ChannelConst { float mean[V], rstd[V], gamma[V], beta[V]; };

template <int V> __device__ __forceinline__ void affine(const GnArgs &a, int ch, ChannelConst<V> &k)
{
#pragma unroll
    for (int e = 0; e < V; ++e) {
        k.gamma[e] = a.gamma != nullptr ? a.gamma[ch + e] : 1.f;
        k.beta[e] = a.beta != nullptr ? a.beta[ch + e] : 0.f;
    }
}

// g = dy * derivative of the activation, and xhat, of one vector
template <int V, int ACT> __device__ __forceinline__ void gradient(const ChannelConst<V> &k, const float (&x)[V], const float (&dy)[V], const float (&ys)[V],
                                                                   float (&g)[V], float (&xh)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) {
        xh[e] = (x[e] - k.mean[e]) * k.rstd[e];
        g[e] = dy[e];
        if (ACT == ACT_MASK) g[e] = ys[e] > 0.f ? dy[e] : 0.f;
        if (ACT == ACT_SILU) {
            const float u = fmaf(xh[e], k.gamma[e], k.beta[e]), q = sigmoid(u);
            g[e] = dy[e] * (q * fmaf(u, 1.f - q, 1.f));
        }
    }
}

// Adds `v` of the threads that have the same channel vector (thread t: vector t % cvs, row t / cvs) and leaves the sums of the
// slab's channels in sum[0 .. cvs * V).  Fixed order.  sm: NT * V floats.
template <int V> __device__ __forceinline__ void add_rows(const float (&v)[V], int cvs, int rows, float *sm, float *sum)
{
    const int t = threadIdx.x;
    __syncthreads();
    if (t < rows * cvs)
#pragma unroll
        for (int e = 0; e < V; ++e) sm[t * V + e] = v[e];
    __syncthreads();
    const int width = cvs * V;
    for (int j = t; j < width; j += NT) {
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += sm[r * width + j];
        sum[j] = s;
    }
    __syncthreads();
}

// First kernel.  Block = (sample, slab of channels, split of the pixels).
template <typename T, int V, bool BWD, int ACT>
__global__ __launch_bounds__(NT) void k_gn_reduce(GnArgs a)
{
    __shared__ float sm[NT * V], sum0[NT * V], sum1[NT * V];
    const int t = threadIdx.x;
    int id = blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int slab = id % a.slabs, n = id / a.slabs;
    const int ch0 = slab * a.cs, cvs = min(a.cs, a.c - ch0) / V, rows = NT / cvs;
    const int row = t / cvs, ch = ch0 + (t - row * cvs) * V;
    const int p0 = split * a.split_pixels, p1 = min(a.hw, p0 + a.split_pixels);
    const bool active = row < rows;
    const size_t base = (size_t)n * a.hw * a.c + ch;
    const T *x = (const T *)a.x + base;
    float2 *part = a.part + ((size_t)n * a.splits + split) * a.c + ch0;

    if (!BWD) {
        // running count, mean, sum of squared deviations; eight pixels at a time, whose own mean is subtracted first
        float mean[V] = {}, m2[V] = {}, cnt = 0.f;
        if (active) {
            int p = p0 + row;
            for (; p + 7 * rows < p1; p += 8 * rows) {
                Pack<T, V> q[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) q[u] = *reinterpret_cast<const Pack<T, V> *>(x + (size_t)(p + u * rows) * a.c);
                const float total = cnt + 8.f, w = 8.f / total, wn = cnt * w;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float s = 0.f, d2 = 0.f;
#pragma unroll
                    for (int u = 0; u < 8; ++u) s += as_f32(q[u].v[e]);
                    const float mc = s * 0.125f;
#pragma unroll
                    for (int u = 0; u < 8; ++u) { const float d = as_f32(q[u].v[e]) - mc; d2 = fmaf(d, d, d2); }
                    const float delta = mc - mean[e];
                    mean[e] = fmaf(delta, w, mean[e]);
                    m2[e] += fmaf(delta * delta, wn, d2);
                }
                cnt = total;
            }
            for (; p < p1; p += rows) {
                float v[V];
                load<T, V>(x + (size_t)p * a.c, v);
                const float total = cnt + 1.f, w = 1.f / total, wn = cnt * w;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float delta = v[e] - mean[e];
                    mean[e] = fmaf(delta, w, mean[e]);
                    m2[e] = fmaf(delta * delta, wn, m2[e]);
                }
                cnt = total;
            }
        }
        // over the rows: the mean first, then the deviations from it
        const float inv = 1.f / (float)(p1 - p0);
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = mean[e] * cnt;
        add_rows<V>(v, cvs, rows, sm, sum0);
        if (active)
#pragma unroll
            for (int e = 0; e < V; ++e) { const float d = mean[e] - sum0[ch - ch0 + e] * inv; v[e] = fmaf(d * d, cnt, m2[e]); }
        add_rows<V>(v, cvs, rows, sm, sum1);
        for (int j = t; j < cvs * V; j += NT) part[j] = make_float2(sum0[j] * inv, sum1[j]);
        return;
    }

    ChannelConst<V> k;
    float A[V] = {}, B[V] = {};
    if (active) {
        affine<V>(a, ch, k);
#pragma unroll
        for (int e = 0; e < V; ++e) { const int g = n * a.groups + (ch + e) / a.cg; k.mean[e] = a.mean_in[g]; k.rstd[e] = a.rstd_in[g]; }
        const T *dy = (const T *)a.dy + base, *ys = (const T *)a.y_saved + base;
        constexpr int U = 4;
        for (int p = p0 + row; p < p1; p += U * rows) {
            Pack<T, V> qx[U], qd[U], qy[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const size_t o = (size_t)min(p + u * rows, p1 - 1) * a.c;
                qx[u] = *reinterpret_cast<const Pack<T, V> *>(x + o);
                qd[u] = *reinterpret_cast<const Pack<T, V> *>(dy + o);
                if (ACT == ACT_MASK) qy[u] = *reinterpret_cast<const Pack<T, V> *>(ys + o);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u * rows >= p1) continue;
                float vx[V], vd[V], vy[V] = {}, g[V], xh[V];
#pragma unroll
                for (int e = 0; e < V; ++e) { vx[e] = as_f32(qx[u].v[e]); vd[e] = as_f32(qd[u].v[e]); if (ACT == ACT_MASK) vy[e] = as_f32(qy[u].v[e]); }
                gradient<V, ACT>(k, vx, vd, vy, g, xh);
#pragma unroll
                for (int e = 0; e < V; ++e) { A[e] += g[e]; B[e] = fmaf(g[e], xh[e], B[e]); }
            }
        }
    }
    add_rows<V>(A, cvs, rows, sm, sum0);
    add_rows<V>(B, cvs, rows, sm, sum1);
    for (int j = t; j < cvs * V; j += NT) part[j] = make_float2(sum0[j], sum1[j]);
}

// dgamma, dbeta of 32 channels: eight threads each take every eighth (sample, split), their sums are added in order
__device__ __forceinline__ void sum_gradients(const GnArgs &a, float *sm)
{
    const int cl = threadIdx.x & 31, part = threadIdx.x >> 5, ch = blockIdx.x * 32 + cl;
    float s0 = 0.f, s1 = 0.f;
    if (ch < a.c) {
        const int total = a.n * a.splits;
        int i = part;
        for (; i + 56 < total; i += 64) {
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = a.part[(size_t)(i + 8 * u) * a.c + ch];
#pragma unroll
            for (int u = 0; u < 8; ++u) { s0 += v[u].x; s1 += v[u].y; }
        }
        for (; i < total; i += 8) { const float2 v = a.part[(size_t)i * a.c + ch]; s0 += v.x; s1 += v.y; }
    }
    sm[threadIdx.x] = s0;
    sm[NT + threadIdx.x] = s1;
    __syncthreads();
    if (part == 0 && ch < a.c) {
        s0 = s1 = 0.f;
        for (int r = 0; r < 8; ++r) { s0 += sm[r * 32 + cl]; s1 += sm[NT + r * 32 + cl]; }
        if (a.dbeta != nullptr) a.dbeta[ch] = s0;
        if (a.dgamma != nullptr) a.dgamma[ch] = s1;
    }
}

// The two results of each group that channels [ch0, ch0 + width) belong to, from all partials of the group, in st[2 * (group - first)]:
// forward mean and rstd, backward mean(t) and mean(t * xhat).  `per` threads (a power of two within a wavefront) share a group.
template <bool BWD>
__device__ __forceinline__ void group_results(const GnArgs &a, int n, int ch0, int width, float *st)
{
    const int g0 = ch0 / a.cg, gs = (ch0 + width - 1) / a.cg - g0 + 1;
    int per = 64;
    while (per > 1 && per * gs > NT) per >>= 1;
    const int sub = threadIdx.x & (per - 1), step = NT / per;
    const int entries = a.cg * a.splits;
    const float2 *part = a.part + (size_t)n * a.splits * a.c;
    for (int gb = 0; gb < gs; gb += step) {
        const int gi = gb + threadIdx.x / per, g = g0 + gi;
        if (gi >= gs) continue;   // whole teams of `per` lanes
        const float2 *pg = part + g * a.cg;
        float s0 = 0.f, s1 = 0.f, s2 = 0.f;
        const float shift = BWD ? 0.f : pg[0].x;   // deviations from one of the means, so that the sums below stay small
        for (int i = sub; i < entries; i += per) {
            const int split = i / a.cg, c = i - split * a.cg;
            const float2 v = pg[(size_t)split * a.c + c];
            if (BWD) {
                const float gamma = a.gamma != nullptr ? a.gamma[g * a.cg + c] : 1.f;
                s0 = fmaf(gamma, v.x, s0);
                s1 = fmaf(gamma, v.y, s1);
            } else {
                const float d = v.x - shift, w = (float)(min(a.hw, (split + 1) * a.split_pixels) - split * a.split_pixels);
                s0 = fmaf(w, d, s0);
                s1 = fmaf(w * d, d, s1);
                s2 += v.y;
            }
        }
        for (int o = per >> 1; o >= 1; o >>= 1) {
            s0 += __shfl_xor(s0, o, 64);
            s1 += __shfl_xor(s1, o, 64);
            if (!BWD) s2 += __shfl_xor(s2, o, 64);
        }
        if (sub == 0) {
            if (BWD) {
                st[2 * gi] = s0 * a.inv_count;
                st[2 * gi + 1] = s1 * a.inv_count;
            } else {
                const float off = s0 * a.inv_count;
                float var = (s2 + s1 - s0 * off) * a.inv_count;
                if (var < 0.f) var = 0.f;   // a NaN stays one
                st[2 * gi] = shift + off;
                st[2 * gi + 1] = 1.f / sqrtf(var + a.eps);
            }
        }
    }
    __syncthreads();
}

// Second kernel.  Block = (sample, slab of channels, chunk of pixels).
template <typename T, int V, bool BWD, int ACT>
__global__ __launch_bounds__(NT) void k_gn_apply(GnArgs a)
{
    __shared__ float st[2 * NT * V];
    const int t = threadIdx.x;
    if (BWD && (int)blockIdx.x < a.grad_blocks) { sum_gradients(a, st); return; }
    int id = (int)blockIdx.x - a.grad_blocks;
    const int chunk = id % a.chunks;
    id /= a.chunks;
    const int slab = id % a.slabs, n = id / a.slabs;
    const int ch0 = slab * a.cs, width = min(a.cs, a.c - ch0), cvs = width / V, rows = NT / cvs;
    group_results<BWD>(a, n, ch0, width, st);
    if (!BWD && chunk == 0) {   // the statistics of the groups that begin in this slab
        const int g0 = ch0 / a.cg, gs = (ch0 + width - 1) / a.cg - g0 + 1;
        for (int gi = t; gi < gs; gi += NT) {
            if ((g0 + gi) * a.cg < ch0) continue;
            if (a.mean_out != nullptr) a.mean_out[n * a.groups + g0 + gi] = st[2 * gi];
            if (a.rstd_out != nullptr) a.rstd_out[n * a.groups + g0 + gi] = st[2 * gi + 1];
        }
    }
    const int row = t / cvs, ch = ch0 + (t - row * cvs) * V;
    if (row >= rows) return;
    ChannelConst<V> k;
    affine<V>(a, ch, k);
    float mt[V], mtx[V];   // forward: rstd * gamma in mt
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int gi = (ch + e) / a.cg - ch0 / a.cg;
        if (BWD) {
            mt[e] = st[2 * gi];
            mtx[e] = st[2 * gi + 1];
            const int g = n * a.groups + (ch + e) / a.cg;
            k.mean[e] = a.mean_in[g];
            k.rstd[e] = a.rstd_in[g];
        } else {
            k.mean[e] = st[2 * gi];
            k.rstd[e] = st[2 * gi + 1];
        }
    }
    const size_t base = (size_t)n * a.hw * a.c + ch;
    const T *x = (const T *)a.x + base, *dy = (const T *)a.dy + base, *ys = (const T *)a.y_saved + base;
    T *out = (T *)a.out + base;
    const int p0 = chunk * a.chunk_pixels, p1 = min(a.hw, p0 + a.chunk_pixels);
    constexpr int U = 4;
    for (int p = p0 + row; p < p1; p += U * rows) {
        Pack<T, V> qx[U], qd[U], qy[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t o = (size_t)min(p + u * rows, p1 - 1) * a.c;
            qx[u] = *reinterpret_cast<const Pack<T, V> *>(x + o);
            if (BWD) qd[u] = *reinterpret_cast<const Pack<T, V> *>(dy + o);
            if (BWD && ACT == ACT_MASK) qy[u] = *reinterpret_cast<const Pack<T, V> *>(ys + o);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * rows >= p1) continue;
            Pack<T, V> r;
            float vx[V];
#pragma unroll
            for (int e = 0; e < V; ++e) vx[e] = as_f32(qx[u].v[e]);
            if (BWD) {
                float vd[V], vy[V] = {}, g[V], xh[V];
#pragma unroll
                for (int e = 0; e < V; ++e) { vd[e] = as_f32(qd[u].v[e]); if (ACT == ACT_MASK) vy[e] = as_f32(qy[u].v[e]); }
                gradient<V, ACT>(k, vx, vd, vy, g, xh);
#pragma unroll
                for (int e = 0; e < V; ++e) r.v[e] = from_f32<T>(k.rstd[e] * (fmaf(g[e], k.gamma[e], -mt[e]) - xh[e] * mtx[e]));
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float u1 = fmaf((vx[e] - k.mean[e]) * k.rstd[e], k.gamma[e], k.beta[e]);
                    if (ACT == ACT_RELU) u1 = u1 > 0.f ? u1 : u1 == u1 ? 0.f : u1;   // a NaN stays one
                    if (ACT == ACT_SILU) u1 *= sigmoid(u1);
                    r.v[e] = from_f32<T>(u1);
                }
            }
            *reinterpret_cast<Pack<T, V> *>(out + (size_t)(p + u * rows) * a.c) = r;
        }
    }
}

// ---- launch shapes ------------------------------------------------------------------------------------------------

int vector_of(const dp_group_norm_desc &d)
{
    const int v = d.io_dtype == DP_BF16 ? 8 : 4;
    return d.c % v == 0 ? v : 1;
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Slabs of at most NT vectors, of equal width where possible.  Splits: about four blocks per compute unit, at least eight pixels per
// thread, and few enough that a block of the second kernel reads at most 8192 partials (64 KB, from L2) or one split's.
void shape(const dp_group_norm_desc &d, bool bwd, GnArgs &a)
{
    const int V = vector_of(d);
    a.n = d.n; a.hw = d.h * d.w; a.c = d.c; a.groups = d.groups; a.cg = d.c / d.groups;
    a.eps = d.eps;
    a.inv_count = (float)(1.0 / ((double)a.hw * a.cg));
    const int vectors = d.c / V;
    a.slabs = ceil_div(vectors, NT);
    a.cs = ceil_div(vectors, a.slabs) * V;
    a.slabs = ceil_div(d.c, a.cs);
    const int rows = NT / (a.cs / V);
    int64_t splits = ceil_div(1024, (int64_t)a.n * a.slabs);
    splits = std::min<int64_t>(splits, ceil_div(a.hw, 8 * rows));
    splits = std::min<int64_t>(splits, std::max(1, 8192 / a.c));
    a.split_pixels = ceil_div(a.hw, splits);
    a.splits = ceil_div(a.hw, a.split_pixels);
    int64_t chunks = ceil_div(2048, (int64_t)a.n * a.slabs);
    chunks = std::min<int64_t>(chunks, ceil_div(a.hw, 8 * rows));
    a.chunk_pixels = ceil_div(a.hw, chunks);
    a.chunks = ceil_div(a.hw, a.chunk_pixels);
    a.grad_blocks = bwd ? ceil_div(a.c, 32) : 0;
}

size_t part_bytes(const GnArgs &a) { return (size_t)a.n * a.splits * a.c * sizeof(float2); }

template <typename T, int V, bool BWD, int ACT>
void launch(const GnArgs &a, bool apply, hipStream_t st)
{
    hipLaunchKernelGGL((k_gn_reduce<T, V, BWD, BWD ? ACT : ACT_NONE>), dim3(a.n * a.slabs * a.splits), dim3(NT), 0, st, a);
    const int blocks = a.grad_blocks + (apply ? a.n * a.slabs * a.chunks : 0);
    hipLaunchKernelGGL((k_gn_apply<T, V, BWD, ACT>), dim3(blocks), dim3(NT), 0, st, a);
}

template <typename T, int V, bool BWD>
void launch_act(const GnArgs &a, int act, bool apply, hipStream_t st)
{
    if (act == ACT_SILU) launch<T, V, BWD, ACT_SILU>(a, apply, st);
    else if (act == ACT_NONE) launch<T, V, BWD, ACT_NONE>(a, apply, st);
    else if (BWD) launch<T, V, true, ACT_MASK>(a, apply, st);
    else launch<T, V, false, ACT_RELU>(a, apply, st);
}

template <bool BWD>
void launch_type(const dp_group_norm_desc &d, const GnArgs &a, int act, bool apply, hipStream_t st)
{
    const int v = vector_of(d);
    if (d.io_dtype == DP_BF16) {
        if (v == 8) launch_act<bf16_t, 8, BWD>(a, act, apply, st);
        else launch_act<bf16_t, 1, BWD>(a, act, apply, st);
    } else {
        if (v == 4) launch_act<float, 4, BWD>(a, act, apply, st);
        else launch_act<float, 1, BWD>(a, act, apply, st);
    }
}

// ---- checks -------------------------------------------------------------------------------------------------------

dp_status check_desc(const dp_group_norm_desc *d)
{
    if (d == nullptr) { dp_set_error("group norm: descriptor is NULL"); return DP_ERR_NULL; }
    if (d->io_dtype != DP_F32 && d->io_dtype != DP_BF16) { dp_set_error("group norm: unknown io_dtype %d", d->io_dtype); return DP_ERR_UNSUPPORTED; }
    if (d->flags != 0 && d->flags != DP_RELU && d->flags != DP_SILU) { dp_set_error("group norm: flags 0x%x: one of DP_RELU, DP_SILU or none", d->flags); return DP_ERR_UNSUPPORTED; }
    if (d->n < 1 || d->h < 1 || d->w < 1 || d->c < 1) { dp_set_error("group norm: n, h, w, c must be positive"); return DP_ERR_BAD_DESC; }
    if (d->groups < 1 || d->c % d->groups != 0) { dp_set_error("group norm: %d groups do not divide %d channels", d->groups, d->c); return DP_ERR_BAD_DESC; }
    const int64_t limit = (int64_t)1 << 31;
    const int64_t hw = (int64_t)d->h * d->w;
    if (hw >= limit || hw * d->c >= limit || hw * d->c * d->n >= limit) { dp_set_error("group norm: a tensor must hold fewer than 2^31 elements"); return DP_ERR_BAD_DESC; }
    // pixel numbers of a block's last steps pass h * w; a grid has fewer than 2^32 threads
    if (hw > ((int64_t)1 << 30) || (int64_t)d->n * ceil_div(d->c, NT) > (1 << 23)) { dp_set_error("group norm: h * w > 2^30 or n * ceil(c / 256) > 2^23"); return DP_ERR_BAD_DESC; }
    if (!(d->eps > 0.f) || !std::isfinite(d->eps)) { dp_set_error("group norm: eps must be positive"); return DP_ERR_BAD_DESC; }
    return DP_OK;
}

dp_status check_ptrs(const char *what, std::initializer_list<const void *> needed, std::initializer_list<const void *> optional, const void *ws,
                     size_t ws_bytes, size_t need)
{
    for (const void *p : needed) {
        if (p == nullptr) { dp_set_error("%s: null pointer", what); return DP_ERR_NULL; }
        if (!aligned16(p)) { dp_set_error("%s: pointers must be 16-byte aligned", what); return DP_ERR_BAD_DESC; }
    }
    for (const void *p : optional)
        if (!aligned16(p)) { dp_set_error("%s: pointers must be 16-byte aligned", what); return DP_ERR_BAD_DESC; }
    if (!aligned16(ws)) { dp_set_error("%s: the workspace must be 16-byte aligned", what); return DP_ERR_BAD_DESC; }
    if (need > 0 && (ws == nullptr || ws_bytes < need)) {
        dp_set_error("%s needs %zu workspace bytes, got %zu", what, need, ws == nullptr ? (size_t)0 : ws_bytes);
        return DP_ERR_WORKSPACE;
    }
    return DP_OK;
}

}  // namespace

extern "C" size_t dp_group_norm_workspace_bytes(const dp_group_norm_desc *desc, int pass)
{
    if (check_desc(desc) != DP_OK || (pass != DP_PASS_FWD && pass != DP_PASS_DGRAD)) return 0;
    GnArgs a = {};
    shape(*desc, pass == DP_PASS_DGRAD, a);
    return part_bytes(a);
}

extern "C" dp_status dp_group_norm_fwd(const dp_group_norm_desc *desc, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                                       float *rstd, void *ws, size_t ws_bytes, void *hip_stream)
{
    dp_status s = check_desc(desc);
    if (s != DP_OK) return s;
    GnArgs a = {};
    shape(*desc, false, a);
    s = check_ptrs("group norm forward", {x, y}, {gamma, beta, mean, rstd}, ws, ws_bytes, part_bytes(a));
    if (s != DP_OK) return s;
    a.x = x; a.gamma = gamma; a.beta = beta; a.out = y; a.mean_out = mean; a.rstd_out = rstd; a.part = (float2 *)ws;
    launch_type<false>(*desc, a, desc->flags == DP_RELU ? ACT_RELU : desc->flags == DP_SILU ? ACT_SILU : ACT_NONE, true, (hipStream_t)hip_stream);
    return launched("group norm forward");
}

extern "C" dp_status dp_group_norm_bwd(const dp_group_norm_desc *desc, const void *x, const void *dy, const void *y_saved, const float *gamma,
                                       const float *beta, const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *ws,
                                       size_t ws_bytes, void *hip_stream)
{
    dp_status s = check_desc(desc);
    if (s != DP_OK) return s;
    if (dx == nullptr && dgamma == nullptr && dbeta == nullptr) { dp_set_error("group norm backward: no output requested"); return DP_ERR_NULL; }
    GnArgs a = {};
    shape(*desc, true, a);
    if (dgamma == nullptr && dbeta == nullptr) a.grad_blocks = 0;
    s = check_ptrs("group norm backward", {x, dy, mean, rstd}, {y_saved, gamma, beta, dx, dgamma, dbeta}, ws, ws_bytes, part_bytes(a));
    if (s != DP_OK) return s;
    a.x = x; a.dy = dy; a.y_saved = y_saved; a.gamma = gamma; a.beta = beta; a.mean_in = mean; a.rstd_in = rstd;
    a.out = dx; a.dgamma = dgamma; a.dbeta = dbeta; a.part = (float2 *)ws;
    launch_type<true>(*desc, a, desc->flags == DP_SILU ? ACT_SILU : desc->flags == DP_RELU && y_saved != nullptr ? ACT_MASK : ACT_NONE, dx != nullptr, (hipStream_t)hip_stream);
    return launched("group norm backward");
}
