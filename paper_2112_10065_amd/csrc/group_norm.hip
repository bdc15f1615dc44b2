// Group normalisation with an activation, NHWC, forward and backward.  Bound by HBM: the operations per element are few.
//
// Both directions are a reduction over (pixels x channels of a group) per sample, then a pointwise pass that needs its result.
// In NHWC a group is a narrow column of channels, so a block takes whole rows of a slab of channels: each thread keeps one vector of
// channels (16 bytes) and walks pixels.  A slab is some whole groups, or, for groups wider than a block, a part of one; a group's part in
// a slab is a cell.  Partial results go to scratch memory, two floats per [sample][split of the pixels][cell]:
//   forward    mean and sum of squared deviations of the cell: never a difference of large sums, whatever offset x, its channels or a few pixels have
//   backward   sum t and sum t * xhat, t = g * gamma; and per [sample][split][channel] sum g and sum g * xhat, for dgamma and dbeta
// The second kernel adds up the partials of its groups in a fixed order and applies them; in the backward pass its first
// blocks sum dgamma and dbeta instead.
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
    float2 *part, *chan;             // partials of cells, of channels (backward): chan[entry][channel]
    float2 *runs;                    // sums of runs of entries, if there are many
    int entries, run;                // entries of chan, entries of a run
    int n, hw, c, groups, cg;
    int cs, slabs;                   // channels of a slab (the last one of all, or of a group, may be narrower), slabs
    int per_group, cells;            // slabs of a group (1: a slab is whole groups), cells in all
    int splits, split_pixels;        // pixels of a split (the last one may be shorter)
    int chunks, chunk_pixels;        // the same for the second kernel's blocks
    int grad_blocks;                 // blocks of the second kernel that sum dgamma / dbeta
    float eps, inv_count;            // 1 / (hw * cg)
    int past;                        // the second kernel's stores (1), loads too (2) go past the caches
    int units, units_each, cvs;      // one-kernel form: units in all, units of an eighth of them; vectors of a unit's row
};

struct Slab { int ch0, width, g0, gs, cell0; };   // first channel, channels, first group, groups, first cell
__device__ __forceinline__ Slab slab_of(const GnArgs &a, int slab)
{
    Slab s;
    if (a.per_group == 1) {
        s.ch0 = slab * a.cs;
        s.width = min(a.cs, a.c - s.ch0);
        s.g0 = s.ch0 / a.cg;
        s.gs = s.width / a.cg;
        s.cell0 = s.g0;
    } else {
        s.g0 = slab / a.per_group;
        const int off = (slab - s.g0 * a.per_group) * a.cs;
        s.ch0 = s.g0 * a.cg + off;
        s.width = min(a.cs, a.cg - off);
        s.gs = 1;
        s.cell0 = slab;
    }
    return s;
}

// 1 / (1 + exp(-u)); in fp32 tensors to the last bits, down to exp(-88).  bf16 ones lose nothing by the product's rounding.
template <typename T> __device__ __forceinline__ float sigmoid(float u)
{
    const float x = sizeof(T) == 2 ? __builtin_amdgcn_exp2f(-u * kLog2e) : exp_full(__builtin_amdgcn_fmed3f(-u, -128.f, 88.f));
    return __builtin_amdgcn_rcpf(1.f + x);
}

template <int V> __device__ __forceinline__ void load_floats(const float *p, float none, float (&v)[V])
{
    if (p == nullptr) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = none;
    } else if (V % 4 == 0) {
#pragma unroll
        for (int e = 0; e < V; e += 4) *reinterpret_cast<float4 *>(&v[e]) = *reinterpret_cast<const float4 *>(p + e);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = p[e];
    }
}

// f(e, group of channel ch + e): one division for the vector
template <int V, typename F> __device__ __forceinline__ void for_groups(int ch, int cg, F &&f)
{
    int g = ch / cg, r = ch - g * cg;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        f(e, g);
        if (++r == cg) { r = 0; ++g; }
    }
}

// g = dy * derivative of the activation at u = xm * scale + beta
template <typename T, int ACT> __device__ __forceinline__ float gradient(float dy, float ys, float xm, float scale, float beta)
{
    if (ACT == ACT_MASK) return ys > 0.f ? dy : 0.f;
    if (ACT == ACT_SILU) {
        const float u = fmaf(xm, scale, beta), q = sigmoid<T>(u);
        return dy * (q * fmaf(u, 1.f - q, 1.f));
    }
    return dy;
}
template <typename T, int ACT> __device__ __forceinline__ float activation(float u)
{
    if (ACT == ACT_RELU) return u > 0.f ? u : u == u ? 0.f : u;   // a NaN stays one
    if (ACT == ACT_SILU) return u * sigmoid<T>(u);
    return u;
}

// Adds `v` of the threads that have the same channel vector (thread t: vector t % cvs, row t / cvs) and leaves the sums of the slab's
// channels in sm[0 .. cvs * V).  Fixed order.  X: float or float2.  sm: N * V values, N threads; a column is read and written by the same threads.
__device__ __forceinline__ void add_to(float &s, float v) { s += v; }
__device__ __forceinline__ void add_to(float2 &s, const float2 &v) { s.x += v.x; s.y += v.y; }
template <int N, int V, typename X> __device__ __forceinline__ void add_rows(const X (&v)[V], int cvs, int rows, X *sm)
{
    const int t = threadIdx.x, width = cvs * V;
    if (t < rows * cvs)
#pragma unroll
        for (int e = 0; e < V; ++e) sm[t * V + e] = v[e];
    __syncthreads();
    int parts = 1;
    while (2 * parts * width <= N && 2 * parts <= rows) parts *= 2;
    if (parts == 1) {
        for (int i = t; i < width; i += N) {
            X s = {};
            for (int r = 0; r < rows; ++r) add_to(s, sm[r * width + i]);
            sm[i] = s;
        }
    } else {   // `parts` threads to a channel, the first of them adds their sums
        const int part = t / width, j = t - part * width;
        X s = {};
        if (part < parts)
            for (int r = part; r < rows; r += parts) add_to(s, sm[r * width + j]);
        __syncthreads();
        if (part < parts) sm[t] = s;
        __syncthreads();
        if (t < width) {
            s = sm[t];
            for (int q = 1; q < parts; ++q) add_to(s, sm[q * width + t]);
            sm[t] = s;
        }
    }
    __syncthreads();
}

// f(g, sub, per, sum) for each of gs groups of about `entries` entries each, by all lanes of a team of `per` up to 64 lanes, this one the sub-th; sum(v) adds
// up the team's.
template <int N, typename F> __device__ __forceinline__ void for_teams(int gs, int entries, F &&f)
{
    int per = 64;
    while (per > 1 && (per * gs > N || per >= 2 * entries)) per >>= 1;
    const int sub = threadIdx.x & (per - 1), step = N / per;
    for (int g = threadIdx.x / per; g < gs; g += step)   // whole teams
        f(g, sub, per, [&](float v) {
            for (int o = per >> 1; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
            return v;
        });
}

// First kernel.  Block = (sample, slab of channels, split of the pixels).  Bound by HBM: 32 x 224 x 224 x 64 bf16 forward 39 us (205 MB, 5.3 TB/s); backward with
// SiLU the vector instructions (19 per element) are nearly as long: 32 x 56 x 56 x 256 23.2 us (103 MB, 4.4 TB/s).
template <typename T, int V, bool BWD, int ACT>
__global__ __launch_bounds__(NT) void k_gn_reduce(GnArgs a)
{
    __shared__ float2 sum[BWD ? 1 : NT * V];          // forward: both sums of a channel together
    __shared__ float near[BWD ? 1 : NT * V], sum0[BWD ? NT * V : 1], sum1[BWD ? NT * V : 1];
    const int t = threadIdx.x;
    int id = blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int n = id / a.slabs;
    const Slab s = slab_of(a, id - n * a.slabs);
    const int cvs = s.width / V, rows = NT / cvs, row = t / cvs, j0 = (t - row * cvs) * V, ch = s.ch0 + j0;
    const int p0 = split * a.split_pixels, p1 = min(a.hw, p0 + a.split_pixels);
    const bool active = row < rows;
    const size_t base = (size_t)n * a.hw * a.c + ch;
    const T *x = (const T *)a.x + base;
    const size_t at = (size_t)n * a.splits + split;
    float2 *part = a.part + at * a.cells + s.cell0;
    const int cell_width = s.width / s.gs;

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
                    float sum = 0.f, d2 = 0.f;
#pragma unroll
                    for (int u = 0; u < 8; ++u) sum += as_f32(q[u].v[e]);
                    const float mc = sum * 0.125f;
#pragma unroll
                    for (int u = 0; u < 8; ++u) { const float d = as_f32(q[u].v[e]) - mc; d2 = fmaf(d, d, d2); }
                    const float delta = mc - mean[e];
                    mean[e] = fmaf(delta, w, mean[e]);
                    m2[e] += fmaf(delta * delta, wn, d2);
                }
                cnt = total;
            }
            for (; p < p1; p += rows) {
                const Pack<T, V> q = *reinterpret_cast<const Pack<T, V> *>(x + (size_t)p * a.c);
                const float total = cnt + 1.f, w = 1.f / total, wn = cnt * w;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float delta = as_f32(q.v[e]) - mean[e];
                    mean[e] = fmaf(delta, w, mean[e]);
                    m2[e] = fmaf(delta * delta, wn, m2[e]);
                }
                cnt = total;
            }
        }
        // over the rows: deviations from a value near the channel's mean, the first row's mean; a row that lies apart adds its distance's square for
        // all rows, up to rows / cnt times the sum of squares itself, so where that is more than four times, eight rows' mean
        const int width = s.width, firsts = (int64_t)4 * (p1 - p0) < (int64_t)rows * rows ? min(min(rows, 8), p1 - p0) : 1;
        if (row < firsts)
#pragma unroll
            for (int e = 0; e < V; ++e) near[row * width + j0 + e] = mean[e];
        __syncthreads();
        if (firsts > 1) {
            for (int j = t; j < width; j += NT) {
                float all = near[j];
                for (int r = 1; r < firsts; ++r) all += near[r * width + j];
                near[j] = all / (float)firsts;
            }
            __syncthreads();
        }
        float2 v[V];
        if (active)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = mean[e] - near[j0 + e];
                v[e] = make_float2(cnt * d, fmaf(cnt * d, d, m2[e]));
            }
        add_rows<NT, V>(v, cvs, rows, sum);
        // over the channels of a cell: their mean first, then the deviations from it (a channel that lies apart is one of up to 2048)
        const float count = (float)(p1 - p0), inv = 1.f / count, inv_width = 1.f / (float)cell_width;
        for_teams<NT>(s.gs, cell_width, [&](int g, int sub, int per, auto &&team_sum_of) {
            const int first = g * cell_width;
            const float at = near[first];
            float off = 0.f, dev = 0.f;
            for (int i = first + sub; i < first + cell_width; i += per) off += (near[i] - at) + sum[i].x * inv;
            off = team_sum_of(off) * inv_width;
            for (int i = first + sub; i < first + cell_width; i += per) {
                const float o = sum[i].x * inv, d = (near[i] - at) + o - off, own = fmaf(-sum[i].x, o, sum[i].y);
                dev += fmaf(count * d, d, own < 0.f ? 0.f : own);   // a NaN stays one
            }
            dev = team_sum_of(dev);
            if (sub == 0) part[g] = make_float2(at + off, dev);
        });
        return;
    }

    float A[V] = {}, B[V] = {}, rstd[V], gamma[V];
    if (active) {
        float mean[V], beta[V], scale[V];
        load_floats<V>(a.gamma != nullptr ? a.gamma + ch : nullptr, 1.f, gamma);
        load_floats<V>(a.beta != nullptr ? a.beta + ch : nullptr, 0.f, beta);
        for_groups<V>(ch, a.cg, [&](int e, int g) { mean[e] = a.mean_in[n * a.groups + g]; rstd[e] = a.rstd_in[n * a.groups + g]; scale[e] = rstd[e] * gamma[e]; });
        const T *dy = (const T *)a.dy + base, *ys = (const T *)a.y_saved + base;
        constexpr int U = 4;
        // sums of 64 pixels, added up: a chain of thousands of one sign would lose 2^-13 (32 x 56 x 56 x 256 21.9 -> 23.2 us; with the sums in LDS instead of registers the
        // same, and 4 x 224 x 224 x 64 32.8 -> 35.7)
        for (int p = p0 + row; p < p1;) {
            const int end = min(p1, p + 64 * rows);
            float A64[V] = {}, B64[V] = {};
            for (; p < end; p += U * rows) {
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
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float xm = as_f32(qx[u].v[e]) - mean[e];
                        const float g = gradient<T, ACT>(as_f32(qd[u].v[e]), ACT == ACT_MASK ? as_f32(qy[u].v[e]) : 0.f, xm, scale[e], beta[e]);
                        A64[e] += g;
                        B64[e] = fmaf(g, xm, B64[e]);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) { A[e] += A64[e]; B[e] += B64[e]; }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) B[e] *= rstd[e];
    }
    // one after the other: in pairs, as forward, the two sums measured slower (1 x 224 x 224 x 64: 22.5 -> 27.5 us)
    add_rows<NT, V>(A, cvs, rows, sum0);
    add_rows<NT, V>(B, cvs, rows, sum1);
    for (int j = t; j < s.width; j += NT) a.chan[at * a.c + s.ch0 + j] = make_float2(sum0[j], sum1[j]);
    for_teams<NT>(s.gs, cell_width, [&](int g, int sub, int per, auto &&team_sum_of) {
        float k0 = 0.f, k1 = 0.f;
        for (int j = g * cell_width + sub; j < (g + 1) * cell_width; j += per) {
            const float gm = a.gamma != nullptr ? a.gamma[s.ch0 + j] : 1.f;
            k0 = fmaf(gm, sum0[j], k0);
            k1 = fmaf(gm, sum1[j], k1);
        }
        k0 = team_sum_of(k0);
        k1 = team_sum_of(k1);
        if (sub == 0) part[g] = make_float2(k0, k1);
    });
}

// Sums of entries [first, end) of chan for 32 channels, in 64 bits (a chain may be hundreds of terms of one sign long): eight threads each take every eighth
// entry, their sums are added in order by the first, which gets them.  sm: 2 * NT floats.
__device__ __forceinline__ bool sum_entries(const float2 *chan, int c, int ch, int first, int end, float *sm, float2 &sum)
{
    const int cl = threadIdx.x & 31, part = threadIdx.x >> 5;
    double s0 = 0.0, s1 = 0.0;
    if (ch < c) {
        int i = first + part;
        for (; i + 56 < end; i += 64) {
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = chan[(size_t)(i + 8 * u) * c + ch];
#pragma unroll
            for (int u = 0; u < 8; ++u) { s0 += (double)v[u].x; s1 += (double)v[u].y; }
        }
        for (; i < end; i += 8) { const float2 v = chan[(size_t)i * c + ch]; s0 += (double)v.x; s1 += (double)v.y; }
    }
    sm[threadIdx.x] = (float)s0;
    sm[NT + threadIdx.x] = (float)s1;
    __syncthreads();
    sum = make_float2(0.f, 0.f);
    if (part != 0 || ch >= c) return false;
    for (int r = 0; r < 8; ++r) { sum.x += sm[r * 32 + cl]; sum.y += sm[NT + r * 32 + cl]; }
    return true;
}

// dgamma, dbeta of 32 channels
__device__ __forceinline__ void sum_gradients(const GnArgs &a, float *sm)
{
    const int ch = blockIdx.x * 32 + (threadIdx.x & 31);
    float2 sum;
    if (!sum_entries(a.chan, a.c, ch, 0, a.entries, sm, sum)) return;
    if (a.dbeta != nullptr) a.dbeta[ch] = sum.x;
    if (a.dgamma != nullptr) a.dgamma[ch] = sum.y;
}

// Many entries in two steps: a run of them to a block.
__global__ __launch_bounds__(NT) void k_gn_runs(GnArgs a)
{
    __shared__ float sm[2 * NT];
    const int run = blockIdx.x / a.grad_blocks, ch = (blockIdx.x - run * a.grad_blocks) * 32 + (threadIdx.x & 31), first = run * a.run;
    float2 sum;
    if (sum_entries(a.chan, a.c, ch, first, min(a.entries, first + a.run), sm, sum)) a.runs[(size_t)run * a.c + ch] = sum;
}

// The two results of each of a slab's groups in st[2 * (group - first)]: forward mean and rstd, backward mean(t) and mean(t * xhat).
// Teams of up to 64 lanes share a group, eight partials to a lane at a time: they come from other dies, and the wait is the cost.
template <bool BWD>
__device__ __forceinline__ void group_results(const GnArgs &a, int n, const Slab &s, float *st)
{
    constexpr int U = 8;
    const int entries = a.splits * a.per_group;
    int per = 64;
    while (per > 1 && (per * s.gs > NT || per >= 2 * entries)) per >>= 1;
    const int sub = threadIdx.x & (per - 1), step = NT / per;
    const float2 *part = a.part + (size_t)n * a.splits * a.cells + s.g0 * a.per_group;
    for (int g = threadIdx.x / per; g < s.gs; g += step) {   // whole teams
        const float2 *pg = part + g * a.per_group;
        // f(partial, number of values behind it) for this lane's entries
        auto each = [&](auto &&f) {
            for (int i0 = sub; i0 < entries; i0 += U * per) {
                float2 v[U];
                float w[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = min(i0 + u * per, entries - 1), split = a.per_group == 1 ? i : i / a.per_group, sub_cell = i - split * a.per_group;
                    v[u] = pg[(size_t)split * a.cells + sub_cell];
                    const int width = a.per_group == 1 ? a.cg : min(a.cs, a.cg - sub_cell * a.cs);
                    w[u] = (float)(min(a.hw, (split + 1) * a.split_pixels) - split * a.split_pixels) * (float)width;
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i0 + u * per < entries) f(v[u], w[u]);
            }
        };
        auto team = [&](float v) {
            for (int o = per >> 1; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
            return v;
        };
        float k0 = 0.f, k1 = 0.f;
        if (BWD) {
            each([&](const float2 &v, float) { k0 += v.x; k1 += v.y; });
            k0 = team(k0);
            k1 = team(k1);
            if (sub != 0) continue;
            st[2 * g] = k0 * a.inv_count;
            st[2 * g + 1] = k1 * a.inv_count;
        } else {
            // deviations from one of the means, so that the sums stay small; if that one lies apart, once more from the mean
            const float shift = pg->x;
            float k2 = 0.f;
            each([&](const float2 &v, float w) {
                const float d = v.x - shift;
                k0 = fmaf(w, d, k0);
                k1 = fmaf(w * d, d, k1);
                k2 += v.y;
            });
            k0 = team(k0);
            k1 = team(k1);
            k2 = team(k2);
            const float off = k0 * a.inv_count;
            float dev = k2 + fmaf(-k0, off, k1);
            if (k1 > 4.f * dev) {   // the same for the whole team
                dev = 0.f;
                each([&](const float2 &v, float w) {
                    const float d = v.x - shift - off;
                    dev += fmaf(w * d, d, v.y);
                });
                dev = team(dev);
            }
            if (sub != 0) continue;
            st[2 * g] = shift + off;
            st[2 * g + 1] = 1.f / sqrtf(fmaf(dev, a.inv_count, a.eps));   // a NaN stays one
        }
    }
    __syncthreads();
}

// Second kernel.  Block = (sample, slab of channels, chunk of pixels).  PAST: 1: stores go past the caches, 2: loads too.
// Bound by HBM: 32 x 224 x 224 x 64 bf16 forward 67 us (411 MB, 6.1 TB/s), 32 x 56 x 56 x 256 backward 29 (154 MB, 5.3 TB/s).
template <typename T, int V, bool BWD, int ACT, int PAST>
__global__ __launch_bounds__(NT) void k_gn_apply(GnArgs a)
{
    __shared__ float st[2 * NT * V];
    const int t = threadIdx.x;
    if (BWD && (int)blockIdx.x < a.grad_blocks) { sum_gradients(a, st); return; }
    int id = (int)blockIdx.x - a.grad_blocks;
    const int chunk = id % a.chunks;
    id /= a.chunks;
    const int n = id / a.slabs;
    const Slab s = slab_of(a, id - n * a.slabs);
    const int cvs = s.width / V, rows = NT / cvs, row = t / cvs, ch = s.ch0 + (t - row * cvs) * V;
    const size_t base = (size_t)n * a.hw * a.c + ch;
    const T *x = (const T *)a.x + base, *dy = (const T *)a.dy + base, *ys = (const T *)a.y_saved + base;
    T *out = (T *)a.out + base;
    const int p0 = chunk * a.chunk_pixels + row, p1 = row < rows ? min(a.hw, (chunk + 1) * a.chunk_pixels) : 0;
    constexpr int U = 4;
    Pack<T, V> qx[U], qd[U], qy[U];
    auto fetch = [&](int p) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t o = (size_t)min(p + u * rows, p1 - 1) * a.c;
            qx[u] = load_vec<Pack<T, V>, PAST == 2>(x + o);
            if (BWD) qd[u] = load_vec<Pack<T, V>, PAST == 2>(dy + o);
            if (BWD && ACT == ACT_MASK) qy[u] = load_vec<Pack<T, V>, PAST == 2>(ys + o);
        }
    };
    if (p0 < p1) fetch(p0);   // on their way while the partials are added up
    group_results<BWD>(a, n, s, st);
    if (!BWD && chunk == 0 && s.ch0 == s.g0 * a.cg) {   // the slab in which its groups begin
        for (int g = t; g < s.gs; g += NT) {
            if (a.mean_out != nullptr) a.mean_out[n * a.groups + s.g0 + g] = st[2 * g];
            if (a.rstd_out != nullptr) a.rstd_out[n * a.groups + s.g0 + g] = st[2 * g + 1];
        }
    }
    if (p0 >= p1) return;
    // forward  y = act((x - mean) * scale + beta);  backward  dx = g * scale - (off + (x - mean) * slope)
    float mean[V], scale[V], beta[V], off[V], slope[V];
    load_floats<V>(a.gamma != nullptr ? a.gamma + ch : nullptr, 1.f, scale);
    load_floats<V>(a.beta != nullptr ? a.beta + ch : nullptr, 0.f, beta);
    for_groups<V>(ch, a.cg, [&](int e, int g) {
        const float s0 = st[2 * (g - s.g0)], s1 = st[2 * (g - s.g0) + 1];
        if (BWD) {
            const float rstd = a.rstd_in[n * a.groups + g];
            mean[e] = a.mean_in[n * a.groups + g];
            scale[e] *= rstd;
            off[e] = rstd * s0;
            slope[e] = rstd * rstd * s1;
        } else {
            mean[e] = s0;
            scale[e] *= s1;
        }
    });
    for (int p = p0;;) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * rows >= p1) continue;
            Pack<T, V> r;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xm = as_f32(qx[u].v[e]) - mean[e];
                if (BWD) {
                    const float g = gradient<T, ACT>(as_f32(qd[u].v[e]), ACT == ACT_MASK ? as_f32(qy[u].v[e]) : 0.f, xm, scale[e], beta[e]);
                    r.v[e] = from_f32<T>(fmaf(g, scale[e], -fmaf(xm, slope[e], off[e])));
                } else {
                    r.v[e] = from_f32<T>(activation<T, ACT>(fmaf(xm, scale[e], beta[e])));
                }
            }
            store_vec<Pack<T, V>, PAST != 0>(out + (size_t)(p + u * rows) * a.c, r);
        }
        p += U * rows;
        if (p >= p1) break;
        fetch(p);
    }
}

// ---- one kernel for small images ----------------------------------------------------------------------------------
//
// Where a group's pixels fit in the registers of a team of wavefronts, the tensor is read once and there is no second kernel to wait
// for.  A unit is the narrowest column of channels that is whole groups and whole vectors: one group of cvs vectors, or the K groups of
// one vector.  W wavefronts hold a unit, R vectors to a lane; all of them belong to the same K groups, so sums are reductions of whole wavefronts.
// Units of a cache line are handed to one die (blocks go to the eight dies in turn), whose L2 then reads the line once.

// v of all W wavefronts of the team, in order; sm: W * N floats of the team's own.  A block has one team where W > 1.
template <int W, int N> __device__ __forceinline__ void team_sum(float (&v)[N], float *sm)
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = wave_sum_fast(v[e]);
    if (W == 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    if (lane == 0)
#pragma unroll
        for (int e = 0; e < N; ++e) sm[wave * N + e] = v[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < N; ++e) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += sm[w * N + e];
        v[e] = s;
    }
}

// The same per channel of the unit (lane's vector t % cvs, cvs a power of two): every lane gets its own channels' sums.  sm: W * 64 * V floats.
template <int W, int V> __device__ __forceinline__ void team_channel_sum(float (&v)[V], int cvs, float *sm)
{
    stride_sums<V>(v, cvs);
    if (W == 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, width = cvs * V, j = (lane & (cvs - 1)) * V;
    __syncthreads();
    if (lane < cvs)
#pragma unroll
        for (int e = 0; e < V; ++e) sm[wave * width + j + e] = v[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float s = 0.f;
        for (int w = 0; w < W; ++w) s += sm[w * width + j + e];
        v[e] = s;
    }
}

template <typename T, int V, int K, bool BWD, int ACT, int W, int R>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_gn_unit(GnArgs a)
{
    constexpr int P = V / K;   // channels of a vector in one group (all of them where the group is wider)
    __shared__ float sm[W == 1 ? 1 : BWD ? W * 64 * V : W * K];
    const int block = (int)(blockIdx.x & 7) * a.units_each + (int)(blockIdx.x >> 3);
    const int unit = W == 1 ? block * 4 + (int)(threadIdx.x >> 6) : block;
    if ((int)(blockIdx.x >> 3) >= a.units_each || unit >= a.units) return;   // whole teams
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int per_sample = a.c / (K > 1 ? V : a.cg), n = unit / per_sample, ch0 = (unit - n * per_sample) * (K > 1 ? V : a.cg);
    const int cvs = K > 1 ? 1 : a.cg / V, rows = 64 * W / cvs, row = t / cvs, ch = ch0 + (t & (cvs - 1)) * V, g0 = n * a.groups + ch0 / a.cg;
    const size_t base = ((size_t)n * a.hw + row) * a.c + ch, step = (size_t)rows * a.c;
    const T *x = (const T *)a.x + base, *dy = (const T *)a.dy + base, *ys = (const T *)a.y_saved + base;
    typedef Pack<T, V> P16;
    words4 qx[R], qd[BWD ? R : 1], qy[ACT == ACT_MASK ? R : 1];   // as loaded
    auto again = [&]() {             // they stay packed between the passes: unpacked once for all they would need twice the registers
#pragma unroll
        for (int i = 0; i < R; ++i) {
            asm("" : "+v"(qx[i]));
            if (BWD) asm("" : "+v"(qd[BWD ? i : 0]));
        }
    };
    const int count = row < a.hw ? (a.hw - row + rows - 1) / rows : 0;   // this lane's pixels: row, row + rows, ...
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i < count) {
            qx[i] = *reinterpret_cast<const words4 *>(x + i * step);
            if (BWD) qd[BWD ? i : 0] = *reinterpret_cast<const words4 *>(dy + i * step);
            if (ACT == ACT_MASK) qy[ACT == ACT_MASK ? i : 0] = *reinterpret_cast<const words4 *>(ys + i * step);
        }
    float mean[K], rstd[K];
    float scale[V], beta[V];
    load_floats<V>(a.gamma != nullptr ? a.gamma + ch : nullptr, 1.f, scale);
    load_floats<V>(a.beta != nullptr ? a.beta + ch : nullptr, 0.f, beta);
    T *out = (T *)a.out + base;
    if constexpr (!BWD) {
#pragma unroll
        for (int k = 0; k < K; ++k) mean[k] = rstd[k] = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) mean[e / P] += as_f32(vx.v[e]);
            }
        again();
        team_sum<W, K>(mean, sm);
#pragma unroll
        for (int k = 0; k < K; ++k) mean[k] *= a.inv_count;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) { const float d = as_f32(vx.v[e]) - mean[e / P]; rstd[e / P] = fmaf(d, d, rstd[e / P]); }
            }
        again();
        team_sum<W, K>(rstd, sm);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            rstd[k] = 1.f / sqrtf(fmaf(rstd[k], a.inv_count, a.eps));
            if (t == 0) {
                if (a.mean_out != nullptr) a.mean_out[g0 + k] = mean[k];
                if (a.rstd_out != nullptr) a.rstd_out[g0 + k] = rstd[k];
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) scale[e] *= rstd[e / P];
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]);
                P16 r;
#pragma unroll
                for (int e = 0; e < V; ++e) r.v[e] = from_f32<T>(activation<T, ACT>(fmaf(as_f32(vx.v[e]) - mean[e / P], scale[e], beta[e])));
                *reinterpret_cast<P16 *>(out + i * step) = r;
            }
    } else {
        if (ACT == ACT_MASK)   // the mask goes into dy at once
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (i < count) {
                    const P16 q = __builtin_bit_cast(P16, qy[ACT == ACT_MASK ? i : 0]);
                    P16 vd = __builtin_bit_cast(P16, qd[i]);
#pragma unroll
                    for (int e = 0; e < V; ++e) vd.v[e] = as_f32(q.v[e]) > 0.f ? vd.v[e] : (T)0;
                    qd[i] = __builtin_bit_cast(words4, vd);
                }
#pragma unroll
        for (int k = 0; k < K; ++k) { mean[k] = a.mean_in[g0 + k]; rstd[k] = a.rstd_in[g0 + k]; }
        constexpr int G = ACT == ACT_MASK ? ACT_NONE : ACT;
        float A[V] = {}, B[V] = {}, gamma[V];
#pragma unroll
        for (int e = 0; e < V; ++e) { gamma[e] = scale[e]; scale[e] *= rstd[e / P]; }
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]), vd = __builtin_bit_cast(P16, qd[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xm = as_f32(vx.v[e]) - mean[e / P], g = gradient<T, G>(as_f32(vd.v[e]), 0.f, xm, scale[e], beta[e]);
                    A[e] += g;
                    B[e] = fmaf(g, xm, B[e]);
                }
            }
        again();
        team_channel_sum<W, V>(A, cvs, sm);
        team_channel_sum<W, V>(B, cvs, sm);
        float s0[K], s1[K];
#pragma unroll
        for (int k = 0; k < K; ++k) s0[k] = s1[k] = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            B[e] *= rstd[e / P];
            s0[e / P] = fmaf(gamma[e], A[e], s0[e / P]);
            s1[e / P] = fmaf(gamma[e], B[e], s1[e / P]);
        }
        for (int o = 1; o < cvs; o <<= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) { s0[k] += __shfl_xor(s0[k], o, 64); s1[k] += __shfl_xor(s1[k], o, 64); }
        if (t < cvs) {   // one lane for each vector of channels
            if (a.n == 1) {
                for (int e = 0; e < V; ++e) {
                    if (a.dbeta != nullptr) a.dbeta[ch + e] = A[e];
                    if (a.dgamma != nullptr) a.dgamma[ch + e] = B[e];
                }
            } else if (a.grad_blocks > 0) {
                for (int e = 0; e < V; ++e) a.chan[(size_t)n * a.c + ch + e] = make_float2(A[e], B[e]);
            }
        }
        if (a.out == nullptr) return;
        float off[K], slope[K];
#pragma unroll
        for (int k = 0; k < K; ++k) { off[k] = rstd[k] * s0[k] * a.inv_count; slope[k] = rstd[k] * rstd[k] * s1[k] * a.inv_count; }
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]), vd = __builtin_bit_cast(P16, qd[i]);
                P16 r;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xm = as_f32(vx.v[e]) - mean[e / P], g = gradient<T, G>(as_f32(vd.v[e]), 0.f, xm, scale[e], beta[e]);
                    r.v[e] = from_f32<T>(fmaf(g, scale[e], -fmaf(xm, slope[e / P], off[e / P])));
                }
                *reinterpret_cast<P16 *>(out + i * step) = r;
            }
    }
}

// The same for groups of any width: a unit is cvs vectors wide, not necessarily a power of two, and holds G groups; a vector lies in one of them or in
// two neighbours, its first `cut` channels in group `lg` of the unit.  One team to a block; lanes that whole rows of vectors do not need are idle.
template <typename T, int V, int G, bool BWD, int ACT, int W, int R>
__global__ __launch_bounds__(64 * W) void k_gn_column(GnArgs a)
{
    constexpr int N = 64 * W;
    __shared__ float2 chan[BWD ? N * V : 1];
    __shared__ float sm[BWD ? 2 * G : W * G];
    const int unit = (int)(blockIdx.x & 7) * a.units_each + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= a.units_each || unit >= a.units) return;
    const int t = threadIdx.x, cvs = a.cvs, width = cvs * V, rows = N / cvs, row = t / cvs, j0 = (t - row * cvs) * V;
    const int per_sample = a.c / width, n = unit / per_sample, ch0 = (unit - n * per_sample) * width, ch = ch0 + j0, g0 = n * a.groups + ch0 / a.cg;
    const int lg = G == 1 ? 0 : j0 / a.cg, cut = G == 1 ? V : min(V, (lg + 1) * a.cg - j0), hg = G == 1 ? 0 : min(lg + 1, G - 1);
    const size_t base = ((size_t)n * a.hw + row) * a.c + ch, step = (size_t)rows * a.c;
    const T *x = (const T *)a.x + base, *dy = (const T *)a.dy + base, *ys = (const T *)a.y_saved + base;
    typedef Pack<T, V> P16;
    words4 qx[R], qd[BWD ? R : 1], qy[ACT == ACT_MASK ? R : 1];
    auto again = [&]() {   // packed between the passes, as above
#pragma unroll
        for (int i = 0; i < R; ++i) {
            asm("" : "+v"(qx[i]));
            if (BWD) asm("" : "+v"(qd[BWD ? i : 0]));
        }
    };
    const int count = row < rows && row < a.hw ? (a.hw - row + rows - 1) / rows : 0;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i < count) {
            qx[i] = *reinterpret_cast<const words4 *>(x + i * step);
            if (BWD) qd[BWD ? i : 0] = *reinterpret_cast<const words4 *>(dy + i * step);
            if (ACT == ACT_MASK) qy[ACT == ACT_MASK ? i : 0] = *reinterpret_cast<const words4 *>(ys + i * step);
        }
    float scale[V], beta[V], mean[V];
    load_floats<V>(a.gamma != nullptr ? a.gamma + ch : nullptr, 1.f, scale);
    load_floats<V>(a.beta != nullptr ? a.beta + ch : nullptr, 0.f, beta);
    T *out = (T *)a.out + base;
    if constexpr (!BWD) {
        // the groups' sums from the channels'
        auto group_sums = [&](const float (&v)[V], float (&sums)[G]) {
            float lo = 0.f, hi = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                lo += e < cut ? v[e] : 0.f;
                hi += e < cut ? 0.f : v[e];
            }
#pragma unroll
            for (int k = 0; k < G; ++k) sums[k] = (k == lg ? lo : 0.f) + (k == lg + 1 ? hi : 0.f);
            team_sum<W, G>(sums, sm);
        };
        auto spread = [&](const float (&sums)[G], float (&v)[V]) {
            float lo = sums[0], hi = sums[0];
#pragma unroll
            for (int k = 1; k < G; ++k) { lo = k == lg ? sums[k] : lo; hi = k == hg ? sums[k] : hi; }
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = e < cut ? lo : hi;
        };
        float v[V] = {}, stat[G];
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] += as_f32(vx.v[e]);
            }
        again();
        group_sums(v, stat);
#pragma unroll
        for (int k = 0; k < G; ++k) {
            stat[k] *= a.inv_count;
            if (t == 0 && a.mean_out != nullptr) a.mean_out[g0 + k] = stat[k];
        }
        spread(stat, mean);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) { const float d = as_f32(vx.v[e]) - mean[e]; v[e] = fmaf(d, d, v[e]); }
            }
        again();
        group_sums(v, stat);
#pragma unroll
        for (int k = 0; k < G; ++k) {
            stat[k] = 1.f / sqrtf(fmaf(stat[k], a.inv_count, a.eps));
            if (t == 0 && a.rstd_out != nullptr) a.rstd_out[g0 + k] = stat[k];
        }
        spread(stat, v);
#pragma unroll
        for (int e = 0; e < V; ++e) scale[e] *= v[e];
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]);
                P16 r;
#pragma unroll
                for (int e = 0; e < V; ++e) r.v[e] = from_f32<T>(activation<T, ACT>(fmaf(as_f32(vx.v[e]) - mean[e], scale[e], beta[e])));
                *reinterpret_cast<P16 *>(out + i * step) = r;
            }
    } else {
        if (ACT == ACT_MASK)   // the mask goes into dy at once
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (i < count) {
                    const P16 q = __builtin_bit_cast(P16, qy[ACT == ACT_MASK ? i : 0]);
                    P16 vd = __builtin_bit_cast(P16, qd[i]);
#pragma unroll
                    for (int e = 0; e < V; ++e) vd.v[e] = as_f32(q.v[e]) > 0.f ? vd.v[e] : (T)0;
                    qd[i] = __builtin_bit_cast(words4, vd);
                }
        constexpr int D = ACT == ACT_MASK ? ACT_NONE : ACT;
        const float mean_lo = a.mean_in[g0 + lg], mean_hi = a.mean_in[g0 + hg], rstd_lo = a.rstd_in[g0 + lg], rstd_hi = a.rstd_in[g0 + hg];
        float A[V] = {}, B[V] = {};
#pragma unroll
        for (int e = 0; e < V; ++e) {
            mean[e] = e < cut ? mean_lo : mean_hi;
            scale[e] *= e < cut ? rstd_lo : rstd_hi;
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]), vd = __builtin_bit_cast(P16, qd[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xm = as_f32(vx.v[e]) - mean[e], g = gradient<T, D>(as_f32(vd.v[e]), 0.f, xm, scale[e], beta[e]);
                    A[e] += g;
                    B[e] = fmaf(g, xm, B[e]);
                }
            }
        again();
        float2 v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = make_float2(A[e], B[e] * (e < cut ? rstd_lo : rstd_hi));
        add_rows<N, V>(v, cvs, rows, chan);
        for (int j = t; j < width; j += N) {
            if (a.n == 1) {
                if (a.dbeta != nullptr) a.dbeta[ch0 + j] = chan[j].x;
                if (a.dgamma != nullptr) a.dgamma[ch0 + j] = chan[j].y;
            } else if (a.grad_blocks > 0) {
                a.chan[(size_t)n * a.c + ch0 + j] = chan[j];
            }
        }
        if (a.out == nullptr) return;
        for_teams<N>(G, a.cg, [&](int g, int sub, int per, auto &&team_sum_of) {
            float k0 = 0.f, k1 = 0.f;
            for (int j = g * a.cg + sub; j < (g + 1) * a.cg; j += per) {
                const float gm = a.gamma != nullptr ? a.gamma[ch0 + j] : 1.f;
                k0 = fmaf(gm, chan[j].x, k0);
                k1 = fmaf(gm, chan[j].y, k1);
            }
            k0 = team_sum_of(k0);
            k1 = team_sum_of(k1);
            if (sub == 0) { sm[2 * g] = k0 * a.inv_count; sm[2 * g + 1] = k1 * a.inv_count; }
        });
        __syncthreads();
        const float off_lo = rstd_lo * sm[2 * lg], off_hi = rstd_hi * sm[2 * hg], slope_lo = rstd_lo * rstd_lo * sm[2 * lg + 1], slope_hi = rstd_hi * rstd_hi * sm[2 * hg + 1];
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < count) {
                const P16 vx = __builtin_bit_cast(P16, qx[i]), vd = __builtin_bit_cast(P16, qd[i]);
                P16 r;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xm = as_f32(vx.v[e]) - mean[e], g = gradient<T, D>(as_f32(vd.v[e]), 0.f, xm, scale[e], beta[e]);
                    r.v[e] = from_f32<T>(fmaf(g, scale[e], -fmaf(xm, e < cut ? slope_lo : slope_hi, e < cut ? off_lo : off_hi)));
                }
                *reinterpret_cast<P16 *>(out + i * step) = r;
            }
    }
}

// dgamma, dbeta from the units' sums
__global__ __launch_bounds__(NT) void k_gn_sums(GnArgs a)
{
    __shared__ float sm[2 * NT];
    sum_gradients(a, sm);
}

// ---- launch shapes ------------------------------------------------------------------------------------------------

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
int gcd(int a, int b) { return b == 0 ? a : gcd(b, a % b); }

// Slabs for vectors of V channels: as many whole groups as fit in `cap` channels, at most what a block's threads cover, or equal parts of a wider
// group.  False: a group boundary falls inside a vector that a slab cannot avoid.
bool slabs_for(int V, int cap, GnArgs &a)
{
    const int unit = V / gcd(V, a.cg);   // groups that fill whole vectors
    a.per_group = 1;
    if (a.c % V != 0) return false;
    if (unit * a.cg <= cap) {
        const int64_t width = (int64_t)unit * a.cg;
        a.slabs = ceil_div(a.c, cap / width * width);
        a.cs = (int)(ceil_div(ceil_div(a.c, width), a.slabs) * width);
        a.slabs = ceil_div(a.c, a.cs);
        a.cells = a.groups;
        return true;
    }
    if (unit != 1) return false;
    a.per_group = ceil_div(a.cg, cap);
    a.cs = ceil_div(a.cg / V, a.per_group) * V;
    a.per_group = ceil_div(a.cg, a.cs);
    a.slabs = a.cells = a.groups * a.per_group;
    return true;
}

// Vectors where they fit, single channels else.  Splits: about four blocks per compute unit, at least eight pixels per thread (four at a time
// backward where blocks are few: 4 x 73 x 80 x 80 fp32 14.2 -> 12.7 us, but 32 x 56 x 56 x 64 23.1 -> 24.4), and few enough
// that a block of the second kernel reads at most 2048 partials: 16 KB that come from other dies (4096: 4 x 224 x 224 x 64 forward 23 -> 27 us),
// 4096 where a sample is 16 MB or more and the first kernel's blocks are too long otherwise (2 x 400 x 400 x 64 backward 75 -> 61 us).
// Where that leaves the first kernel without a block for every compute unit, as with very many narrow groups, slabs are narrower, down to a cache line (us, slabs as wide as
// a block / narrower: bf16 1 x 224 x 224 x 2048 of 2048 groups forward 3500 / 111, backward 11900 / 211, 1 x 128 x 128 x 512 of 512 71 / 18, 221 / 27; fp32 1 x 112 x 112 x 256 of 256
// 33 / 14, 110 / 18, 1 x 224 x 224 x 64 of 32 16.5 / 15.8, 28 / 20; bf16 1 x 200 x 200 x 96 of 32 16.0 / 16.5, 25 / 20).
// The second kernel's threads have at least eight pixels too where blocks are many (8 x 56 x 56 x 256 backward 19.4 -> 16.9 us), else four (1 x 80 x 80
// x 64: with eight 12.5 -> 13.9).
// The second kernel has half as many blocks for tensors up to 64 MB (4 x 224 x 224 x 64 backward 43.5 -> 38.8 us; 16 x: 118.5 -> 122).
// Past the caches: outputs above 32 MB, which would be written back while the next kernel reads (32 x 224 x 224 x 64 forward 133 -> 113 us;
// 25 MB: no difference), and the second reading of inputs above 150 MB, which have left the memory-side cache (113 -> 105; 103 MB: 50.7 -> 53.4).
int shape(const dp_group_norm_desc &d, bool bwd, GnArgs &a)
{
    a.n = d.n; a.hw = d.h * d.w; a.c = d.c; a.groups = d.groups; a.cg = d.c / d.groups;
    a.eps = d.eps;
    a.inv_count = (float)(1.0 / ((double)a.hw * a.cg));
    int V = d.io_dtype == DP_BF16 ? 8 : 4;
    if (!slabs_for(V, NT * V, a)) slabs_for(V = 1, NT, a);
    const int64_t sample_bytes = (int64_t)a.hw * a.c * (d.io_dtype == DP_BF16 ? 2 : 4), bytes = a.n * sample_bytes;
    const int line = d.io_dtype == DP_BF16 ? 64 : 32, partials = sample_bytes >= (16 << 20) ? 4096 : 2048;
    for (int cap = NT * V / 2; a.per_group == 1 && cap >= std::max(line, V / gcd(V, a.cg) * a.cg); cap /= 2) {
        const int most = std::max(1, partials / (a.cs / a.cg));
        if (most >= ceil_div(a.hw, 8 * (NT / (a.cs / V))) || (int64_t)a.n * a.slabs * most >= 256) break;
        slabs_for(V, cap, a);
    }
    const int rows = NT / (a.cs / V), slab_groups = a.per_group == 1 ? a.cs / a.cg : a.per_group;
    const bool plenty = (int64_t)a.n * a.slabs * ceil_div(a.hw, 8 * rows) >= 256;   // eight pixels a thread leave a block for every compute unit
    int64_t splits = ceil_div(1024, (int64_t)a.n * a.slabs);
    splits = std::min<int64_t>(splits, ceil_div(a.hw, (plenty || !bwd ? 8 : 4) * rows));
    splits = std::min<int64_t>(splits, std::max(1, partials / slab_groups));
    a.split_pixels = ceil_div(a.hw, splits);
    a.splits = ceil_div(a.hw, a.split_pixels);
    int64_t chunks = ceil_div(bytes > (64 << 20) ? 2048 : 1024, (int64_t)a.n * a.slabs);
    chunks = std::min<int64_t>(chunks, ceil_div(a.hw, (plenty ? 8 : 4) * rows));
    a.chunk_pixels = ceil_div(a.hw, chunks);
    a.chunks = ceil_div(a.hw, a.chunk_pixels);
    a.grad_blocks = bwd ? ceil_div(a.c, 32) : 0;
    a.past = bytes * (bwd ? 2 : 1) > (150 << 20) ? 2 : bytes > (32 << 20) ? 1 : 0;
    return V;
}

// The one-kernel form: wavefronts to a unit (0: two kernels), vectors to a lane, groups of a unit.  k_gn_unit where groups are a power of two of
// whole vectors or divide one.  Measured in both forms (bf16, us, two kernels / one):
//   up to 8 vectors a lane of four wavefronts   8 x 28 x 28 x 512 forward 13.3 / 5.7, backward 16.9 / 13.0; 1 x 14 x 14 x 512 11.1 / 3.5, 11.5 / 5.1
//   1024 units and more: a wavefront each (32 x 14 x 14 x 1024 forward 17 / 8.3); fewer: four (1 x 14 x 14 x 512 forward 4.9 -> 3.8)
//   forward eight instead of four, half as many vectors to a lane: 1 x 28 x 28 x 512 5.1 -> 4.2, 16 x 28 x 28 x 512 9.3 -> 8.7; backward has more to
//     exchange (16 x 28 x 28 x 512 14.9 -> 16.9)
//   backward of 1024 units of four wavefronts: the pieces of a unit are a fraction of a cache line, and the L2s lose the rest of it
//     (32 x 28 x 28 x 256, 16-byte pieces 21 / 23; x 512, 32-byte pieces 33.6 / 27.8, with the saved output 39 / 43)
//   9 to 16 vectors of four wavefronts: forward eight hold them (8 x 56 x 56 x 256 17.1 / 13.0, but 32 x 56 x 56 x 256 33 / 48); backward pieces of 32 bytes
//     and more (8 x 40 x 40 x 512 20.3 / 15.5, with the saved output 23.5 / 19.0; 16 x: 29.8 / 24.8, 39 / 41; 16-byte pieces 8 x 64 x 64 x 128 16.6 / 19.2)
// k_gn_column for the other widths, if a vector lies in two groups at most:
//   8 x 16 x 16 x 1280 of 32 groups forward 12.1 / 5.1, backward 15.8 / 9.6; 1 x 8 x 8 x 320 9.2 / 4.6, 10.1 / 4.9; 32 x 14 x 14 x 768 15.1 / 7.4, 18.0 / 12.7
//   9 to 16 vectors: 32 x 28 x 28 x 320 forward 19.9 / 11.2, backward 22.6 / 16.5, but 1024 units 128 x 28 x 28 x 320 36.9 / 40.0, 60 / 65
//   forward sixteen wavefronts: 32 x 32 x 32 x 320 21.1 / 13.6, 1 x 32 x 32 x 320 10.9 / 9.0; at the limit of their registers and alone a compute unit
//     draws its piece for too long (40 x 40 x 320: 8 units 10.1 / 10.7, 64 units 14.9 / 12.1)
// fp32, half the channels to a vector, by the same limits: in 23 of these shapes both ways the one kernel is never slower where it is taken (8 x 28 x 28 x 512 forward 14.7 / 7.1,
//   backward 18.4 / 13.1, 32 x 28 x 28 x 256 18.4 / 13.5, 28.5 / 24.5, 32 x 14 x 14 x 768 17.5 / 9.4, 25.9 / 19.1, 32 x 32 x 32 x 320 forward 25.3 / 21.2)
struct UnitForm { int waves, vectors, groups, cvs; };   // cvs > 0: k_gn_column
UnitForm unit_form(const GnArgs &a, int V, bool bwd, bool mask)
{
    UnitForm f = {0, 0, 1, 0};
    if (V == 1) return f;
    const int g = gcd(V, a.cg), width = a.cg / g * V, cvs = width / V;   // channels of the narrowest column of whole groups and vectors
    const int64_t units = (int64_t)a.n * (a.c / width);
    if (cvs > 64 || units > (1 << 22)) return f;   // a grid has fewer than 2^32 threads
    const int w1 = ceil_div(a.hw, 64 / cvs), w4 = ceil_div(a.hw, 256 / cvs), w8 = ceil_div(a.hw, 512 / cvs), w16 = ceil_div(a.hw, 1024 / cvs);
    f.groups = V / g;
    if ((f.groups == 1 && (cvs & (cvs - 1)) == 0) || cvs == 1) {
        if (w1 <= 8 && units >= 1024) { f.waves = 1; f.vectors = 8; }
        else if (!bwd && w4 <= 8) { f.waves = 8; f.vectors = 4; }
        else if (bwd && w4 <= 8 && (units < 1024 || (cvs > 1 && !mask))) { f.waves = 4; f.vectors = 8; }
        else if (!bwd && w4 <= 16 && units <= 512) { f.waves = 8; f.vectors = 8; }
        else if (bwd && w8 <= 8 && cvs > 1 && units <= (mask ? 256 : 512)) { f.waves = 8; f.vectors = 8; }
    } else if (f.groups <= 4 && V - g <= a.cg) {   // a vector lies in two groups at most
        f.cvs = cvs;
        if (!bwd && w8 <= 4) { f.waves = 8; f.vectors = 4; }
        else if (bwd && w4 <= 8) { f.waves = 4; f.vectors = 8; }
        else if (!bwd && w8 <= 8 && units <= 512) { f.waves = 8; f.vectors = 8; }
        else if (!bwd && w16 <= 8 && (w16 <= 6 || units >= 32) && units <= 512) { f.waves = 16; f.vectors = 8; }
        else if (bwd && w8 <= 8 && units <= 512) { f.waves = 8; f.vectors = 8; }
    }
    return f;
}

// Entries of the channels' sums of which a block adds up all, and the length of a run beyond (backward, bf16, one step / two: 2049 x 14 x 14 x 64 62 / 52 us, 3000 x 7 x 7 x 64
// 48 / 33, 1048576 x 1 x 1 x 32 11.7 / 3.7 ms; below, the second kernel has other blocks beside the one).
constexpr int kEntries = 2048, kRun = 256, kRuns = 1024;
int run_length(int entries) { return std::max(kRun, ceil_div(entries, kRuns)); }
size_t runs_bytes(int entries, int c) { return entries <= kEntries ? 0 : (size_t)ceil_div(entries, run_length(entries)) * c * sizeof(float2); }
// dgamma and dbeta are wanted: leaves at most kRuns entries to sum_gradients
void sum_runs(GnArgs &a, int entries, hipStream_t st)
{
    a.entries = entries;
    if (entries <= kEntries || a.grad_blocks == 0) return;
    a.run = run_length(entries);
    const int runs = ceil_div(entries, a.run);
    hipLaunchKernelGGL(k_gn_runs, dim3(a.grad_blocks * runs), dim3(NT), 0, st, a);
    a.chan = a.runs;
    a.entries = runs;
}

size_t cell_bytes(const GnArgs &a) { return ((size_t)a.n * a.splits * a.cells * sizeof(float2) + 15) / 16 * 16; }
size_t chan_bytes(const GnArgs &a) { return (size_t)a.n * a.splits * a.c * sizeof(float2); }
size_t part_bytes(const GnArgs &a, bool bwd) { return cell_bytes(a) + (bwd ? chan_bytes(a) + runs_bytes(a.n * a.splits, a.c) : 0); }

template <typename T, int V, int K, bool BWD, int ACT>
void launch_unit(GnArgs a, const UnitForm &f, hipStream_t st)
{
    a.units = a.n * (a.c / std::max(a.cg, V));
    const int blocks = f.waves == 1 ? (a.units + 3) / 4 : a.units;
    a.units_each = (blocks + 7) / 8;
    const dim3 grid(8 * a.units_each);
    if (f.waves == 1) hipLaunchKernelGGL((k_gn_unit<T, V, K, BWD, ACT, 1, 8>), grid, dim3(256), 0, st, a);
    else if constexpr (BWD) {
        if (f.waves == 4) hipLaunchKernelGGL((k_gn_unit<T, V, K, BWD, ACT, 4, 8>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_gn_unit<T, V, K, BWD, ACT, 8, 8>), grid, dim3(512), 0, st, a);
    }
    else if (f.vectors == 4) hipLaunchKernelGGL((k_gn_unit<T, V, K, BWD, ACT, 8, 4>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_gn_unit<T, V, K, BWD, ACT, 8, 8>), grid, dim3(512), 0, st, a);
    if (BWD && a.grad_blocks > 0 && a.n > 1) {
        sum_runs(a, a.n, st);
        hipLaunchKernelGGL(k_gn_sums, dim3(a.grad_blocks), dim3(NT), 0, st, a);
    }
}

template <typename T, int V, int G, bool BWD, int ACT>
void launch_column(GnArgs a, const UnitForm &f, hipStream_t st)
{
    a.cvs = f.cvs;
    a.units = a.n * (a.c / (f.cvs * V));
    a.units_each = (a.units + 7) / 8;
    const dim3 grid(8 * a.units_each);
    if constexpr (BWD) {
        if (f.waves == 4) hipLaunchKernelGGL((k_gn_column<T, V, G, BWD, ACT, 4, 8>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_gn_column<T, V, G, BWD, ACT, 8, 8>), grid, dim3(512), 0, st, a);
    }
    else if (f.vectors == 4) hipLaunchKernelGGL((k_gn_column<T, V, G, BWD, ACT, 8, 4>), grid, dim3(512), 0, st, a);
    else if (f.waves == 8) hipLaunchKernelGGL((k_gn_column<T, V, G, BWD, ACT, 8, 8>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_gn_column<T, V, G, BWD, ACT, 16, 8>), grid, dim3(1024), 0, st, a);
    if (BWD && a.grad_blocks > 0 && a.n > 1) {
        sum_runs(a, a.n, st);
        hipLaunchKernelGGL(k_gn_sums, dim3(a.grad_blocks), dim3(NT), 0, st, a);
    }
}

template <typename T, int V, bool BWD, int ACT>
void launch(GnArgs a, bool apply, hipStream_t st)
{
    if constexpr (V > 1) {
        const UnitForm f = unit_form(a, V, BWD, ACT == ACT_MASK);
        if (f.waves > 0 && f.cvs > 0) {
            if (f.groups == 1) return launch_column<T, V, 1, BWD, ACT>(a, f, st);
            if (f.groups == 2) return launch_column<T, V, 2, BWD, ACT>(a, f, st);
            return launch_column<T, V, 4, BWD, ACT>(a, f, st);
        }
        if (f.waves > 0) {
            if (f.groups == 1) return launch_unit<T, V, 1, BWD, ACT>(a, f, st);
            if (f.groups == 2) return launch_unit<T, V, 2, BWD, ACT>(a, f, st);
            if (f.groups == 4) return launch_unit<T, V, 4, BWD, ACT>(a, f, st);
            if constexpr (V == 8) return launch_unit<T, V, 8, BWD, ACT>(a, f, st);
        }
    }
    hipLaunchKernelGGL((k_gn_reduce<T, V, BWD, BWD ? ACT : ACT_NONE>), dim3(a.n * a.slabs * a.splits), dim3(NT), 0, st, a);
    if (BWD) sum_runs(a, a.n * a.splits, st);
    const int blocks = a.grad_blocks + (apply ? a.n * a.slabs * a.chunks : 0);
    if constexpr (V > 1) {
        if (a.past == 2) hipLaunchKernelGGL((k_gn_apply<T, V, BWD, ACT, 2>), dim3(blocks), dim3(NT), 0, st, a);
        else if (a.past == 1) hipLaunchKernelGGL((k_gn_apply<T, V, BWD, ACT, 1>), dim3(blocks), dim3(NT), 0, st, a);
        if (a.past != 0) return;
    }
    hipLaunchKernelGGL((k_gn_apply<T, V, BWD, ACT, 0>), dim3(blocks), dim3(NT), 0, st, a);
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
void launch_type(const dp_group_norm_desc &d, int V, const GnArgs &a, int act, bool apply, hipStream_t st)
{
    if (d.io_dtype == DP_BF16) {
        if (V == 8) launch_act<bf16_t, 8, BWD>(a, act, apply, st);
        else launch_act<bf16_t, 1, BWD>(a, act, apply, st);
    } else {
        if (V == 4) launch_act<float, 4, BWD>(a, act, apply, st);
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
    if (hw > ((int64_t)1 << 30) || (int64_t)d->n * ceil_div(d->c, NT) > (1 << 22)) { dp_set_error("group norm: h * w > 2^30 or n * ceil(c / 256) > 2^22"); return DP_ERR_BAD_DESC; }
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
    return part_bytes(a, pass == DP_PASS_DGRAD);
}

extern "C" dp_status dp_group_norm_fwd(const dp_group_norm_desc *desc, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                                       float *rstd, void *ws, size_t ws_bytes, void *hip_stream)
{
    dp_status s = check_desc(desc);
    if (s != DP_OK) return s;
    GnArgs a = {};
    const int V = shape(*desc, false, a);
    s = check_ptrs("group norm forward", {x, y}, {gamma, beta, mean, rstd}, ws, ws_bytes, part_bytes(a, false));
    if (s != DP_OK) return s;
    a.x = x; a.gamma = gamma; a.beta = beta; a.out = y; a.mean_out = mean; a.rstd_out = rstd; a.part = (float2 *)ws;
    launch_type<false>(*desc, V, a, desc->flags == DP_RELU ? ACT_RELU : desc->flags == DP_SILU ? ACT_SILU : ACT_NONE, true, (hipStream_t)hip_stream);
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
    const int V = shape(*desc, true, a);
    if (dgamma == nullptr && dbeta == nullptr) a.grad_blocks = 0;
    s = check_ptrs("group norm backward", {x, dy, mean, rstd}, {y_saved, gamma, beta, dx, dgamma, dbeta}, ws, ws_bytes, part_bytes(a, true));
    if (s != DP_OK) return s;
    a.x = x; a.dy = dy; a.y_saved = y_saved; a.gamma = gamma; a.beta = beta; a.mean_in = mean; a.rstd_in = rstd;
    a.out = dx; a.dgamma = dgamma; a.dbeta = dbeta; a.part = (float2 *)ws; a.chan = (float2 *)((char *)ws + cell_bytes(a));
    a.runs = (float2 *)((char *)a.chan + chan_bytes(a));
    launch_type<true>(*desc, V, a, desc->flags == DP_SILU ? ACT_SILU : desc->flags == DP_RELU && y_saved != nullptr ? ACT_MASK : ACT_NONE, dx != nullptr, (hipStream_t)hip_stream);
    return launched("group norm backward");
}
