// Norm of every head of queries and keys over its own channels, and the rotation of pairs of channels by the token's place on up to three axes.
// Bound by HBM: forward reads and writes each element once, backward reads two and writes one.
//
//   u = x r gamma, r = 1/sqrt(mean x^2 + eps);   y = R(angle) u
//   backward, g = R(-angle) dy, t = g gamma:   dgamma = sum g x r,   dx = r (t - x r^2 mean(t x))
//
// A rotation is written per channel: y_c = C_c u_c + S_c u_partner(c) with S of opposite signs in the two channels of a pair, and C = 1, S = 0 behind
// the turned channels.  A wavefront takes one row: its lanes compute the row's angles once, then hold C and S of their own eight channels in registers
// while they go over the heads, several heads at a time.
//
// 16 x 28 x 28 tokens, 32 heads of 128 bf16, backward: 67 us for 308 MB (4.6 TB/s; a large copy reaches 4.8-5.2) and 4.5 for the sums of dgamma.  32 x 14 x 14 tokens, 24 heads of 64,
// forward: 14 us for 39 MB: a wavefront has one row, and a launch's start and a row's waits (its place, then one turn of heads after the other) are half of it.  With four
// turns under way at once (backward two) they took 17 and 63.
#include "vec_common.h"
#include <algorithm>

namespace {

constexpr int NT = 256, WAVES = NT / 64, V = 8;   // V channels per lane
constexpr int kMaxDim = 256, kMaxAxes = 3;
constexpr int kBlocks = 4096, kNormGradBlocks = 768;   // at most; of the norm's gradient three to a compute unit, each of which leaves one partial sum of dgamma

struct QkSide {
    const void *x, *dy;      // forward: x alone
    void *out;               // y or dx
    const float *gamma;
    long long x_stride, dy_stride, out_stride;
    int heads;
};

struct QkArgs {
    QkSide q, k;
    const float *pos;
    const double *freq;
    float *part;             // [block][2][dim] sums of dgamma, or NULL
    int rows, dim, axes, pairs[kMaxAxes], turned;   // turned: pairs of all axes
    int parts;               // a row's heads are dealt out to this many wavefronts
    float eps;
};

template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[V])
{
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < V / W; ++h) {
        Pack<T, W> w;
#pragma unroll
        for (int e = 0; e < W; ++e) w.v[e] = from_f32<T>(v[W * h + e]);
        *reinterpret_cast<Pack<T, W> *>(p + W * h) = w;
    }
}

// Sum over neighbouring LPH lanes, in each of them.
template <int LPH> __device__ __forceinline__ float head_sum(float v)
{
    if constexpr (LPH >= 2) v += moved<0xb1, 0xf>(v, 0.f);     // lanes 1 0 3 2
    if constexpr (LPH >= 4) v += moved<0x4e, 0xf>(v, 0.f);     // lanes 2 3 0 1
    if constexpr (LPH >= 8) v += moved<0x141, 0xf>(v, 0.f);    // eights mirrored
    if constexpr (LPH >= 16) v += moved<0x140, 0xf>(v, 0.f);   // sixteens mirrored
    if constexpr (LPH >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

// cos and sin of 2 pi turns: the nearest quarter is taken off in 64 bits, what is left (within pi / 4) goes through the Taylor series, whose next terms are
// below 3e-9; error 1e-7 at the most, whatever the place, beside that of `turns`: three roundings of 2^-53 of the angle (the frequency in turns, its factor, the product), below 1e-7 up to
// angles of 3e8.
__device__ __forceinline__ void cos_sin_turns(double turns, float &c, float &s)
{
    const double rest = turns - rint(turns), quarter = rint(4.0 * rest);
    const float a = (float)((rest - 0.25 * quarter) * 6.283185307179586), a2 = a * a;
    const float sn = a * fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
    const float cs = fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const int n = (int)quarter;   // -2 ... 2; NaN: 0, and a is NaN
    const bool odd = (n & 1) != 0;
    c = odd ? sn : cs;
    s = odd ? cs : sn;
    c = n == 1 || n == 2 || n == -2 ? -c : c;
    s = n == -1 || n == 2 || n == -2 ? -s : s;
}

__device__ __forceinline__ void add_by(float (&v)[V], int o)
{
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] += __shfl_xor(v[e], o, 64);
}

// LDS of one wavefront: the row's table, then the heads in flight.
__device__ __forceinline__ void own_lds_written() { __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront"); __builtin_amdgcn_wave_barrier(); __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront"); }

// Eight channels as they lie in memory.
template <typename T> struct Raw { words4 w[sizeof(T) * V / 16]; };
template <typename T> __device__ __forceinline__ void load_raw(const T *p, Raw<T> &r)
{
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) * V / 16; ++h) r.w[h] = *reinterpret_cast<const words4 *>(p + h * (16 / sizeof(T)));
}
template <typename T> __device__ __forceinline__ void unpack(const Raw<T> &r, float (&v)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) {
        if constexpr (sizeof(T) == 2) v[e] = __uint_as_float((e & 1) ? r.w[0][e / 2] & 0xffff0000u : r.w[0][e / 2] << 16);
        else v[e] = __uint_as_float(r.w[e / 4][e % 4]);
    }
}

template <typename T, int LPH, bool HALVES, bool NORM, bool BWD> __global__ __launch_bounds__(NT) void k_qk_rotary(QkArgs a)
{
    constexpr int GROUPS = 64 / LPH, ROOM = LPH * V;   // heads at a time; channels of a head with those of idle lanes
    constexpr bool READ_X = NORM || !BWD;
    __shared__ alignas(16) float s_cs[WAVES][2][kMaxDim / 2];
    __shared__ alignas(16) float s_x[WAVES][HALVES ? GROUPS * ROOM : 1];
    __shared__ float s_g[BWD && NORM ? WAVES * 2 * ROOM : 1];
    // uniform for the compiler: 32 x 14 x 14 rows forward 15.3 -> 13.8 us, 4099 fp32 8.8 -> 8.0; but the norm's gradient (16 x 28 x 28 rows) 66 -> 79
    const int wave = BWD && NORM ? threadIdx.x >> 6 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = lane / LPH, c0 = (lane % LPH) * V;
    const bool live = c0 < a.dim;
    float *cs = s_cs[wave][0], *sn = s_cs[wave][1];
    const int P = a.turned;
    const bool whole = HALVES && P % V == 0;   // a lane's partners are one other lane's channels
    const bool all_turned = 2 * P == a.dim;
    const float inv_dim = 1.f / a.dim;

    float sum_q[V], sum_k[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum_q[e] = sum_k[e] = 0.f;
    const int turns_q = (a.q.heads + GROUPS - 1) / GROUPS, turns_k = (a.k.heads + GROUPS - 1) / GROUPS;
    const unsigned units = (unsigned)a.rows * a.parts, step = gridDim.x * WAVES, parts = a.parts;   // below 2^31: only few rows are cut
    // what comes next is always under way: the heads that follow, at the row's end the next row's first ones, and its place
    Raw<T> nx = {}, ndy = {};
    auto fetch = [&](const QkSide &side, int row, int head) {
        if (!live || head >= side.heads) return;
        const int at = head * a.dim + c0;
        if constexpr (READ_X) load_raw(reinterpret_cast<const T *>(side.x) + row * side.x_stride + at, nx);
        if constexpr (BWD) load_raw(reinterpret_cast<const T *>(side.dy) + row * side.dy_stride + at, ndy);
    };
    auto first_key_turn = [&](int part) { return part < turns_q ? (turns_q - part + a.parts - 1) / a.parts * a.parts + part - turns_q : part - turns_q; };
    auto axis_of = [&](int p) { return p < a.pairs[0] ? 0 : p < a.pairs[0] + a.pairs[1] ? 1 : 2; };
    constexpr int PAIRS = LPH * V / 2 > 64 ? 2 : 1;   // of a lane: p = lane, lane + 64
    double freq[PAIRS];
    float pos[PAIRS] = {};
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) freq[i] = lane + 64 * i < P ? a.freq[lane + 64 * i] * 0.15915494309189535 : 0.0;   // turns, not radians
    auto fetch_row = [&](unsigned unit) {
        if (unit >= units) return;
        const int row = unit / parts, part = unit % parts;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) if (lane + 64 * i < P) pos[i] = a.pos[(long long)row * a.axes + axis_of(lane + 64 * i)];
        if (part < turns_q) fetch(a.q, row, part * GROUPS + group);
        else fetch(a.k, row, first_key_turn(part) * GROUPS + group);
    };
    unsigned unit = blockIdx.x * WAVES + wave;
    fetch_row(unit);
    for (; unit < units; unit += step) {
        const int row = unit / parts, part = unit % parts, first_k = first_key_turn(part);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) if (lane + 64 * i < P) cos_sin_turns((double)pos[i] * freq[i], cs[lane + 64 * i], sn[lane + 64 * i]);
        own_lds_written();
        float C[V], S[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = c0 + e;
            const bool first = HALVES ? c < P : (c & 1) == 0, turned = c < 2 * P;
            const int p = HALVES ? (first ? c : c - P) : c >> 1;
            C[e] = turned ? cs[turned ? p : 0] : 1.f;
            const float s = turned ? sn[turned ? p : 0] : 0.f;
            S[e] = first != BWD ? -s : s;   // the gradient turns back
        }
        own_lds_written();
        auto side = [&](const QkSide &sd, int t, int turns, auto &&after_last, float (&sum)[V]) {
            float gamma[V];
#pragma unroll
            for (int e = 0; e < V; ++e) gamma[e] = NORM && live && sd.gamma != nullptr ? sd.gamma[c0 + e] : 1.f;
            for (; t < turns; t += a.parts) {
                const int head = t * GROUPS + group;
                const bool on = live && head < sd.heads;
                float x[V], dy[V], y[V];
                unpack(nx, x);
                unpack(ndy, dy);
                if (!on) {   // what a fetch left out is an older head's
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] = dy[e] = 0.f;
                }
                if (t + a.parts < turns) fetch(sd, row, head + a.parts * GROUPS);
                else after_last();
                float r = 1.f, ss = 0.f;
                if constexpr (NORM) {
#pragma unroll
                    for (int e = 0; e < V; ++e) ss = fmaf(x[e], x[e], ss);
                    r = __builtin_amdgcn_rsqf(fmaf(head_sum<LPH>(ss), inv_dim, a.eps));
                }
                float u[V], w[V];   // what is turned, and its partners
#pragma unroll
                for (int e = 0; e < V; ++e) u[e] = BWD ? dy[e] : NORM ? x[e] * r * gamma[e] : x[e];
                if constexpr (HALVES) {
                    float *mine = s_x[wave] + group * ROOM;
#pragma unroll
                    for (int e = 0; e < V; e += 4) *reinterpret_cast<float4 *>(mine + c0 + e) = make_float4(u[e], u[e + 1], u[e + 2], u[e + 3]);
                    own_lds_written();
                    if (whole) {
                        const int from = c0 < P ? c0 + P : c0 < 2 * P ? c0 - P : c0;
#pragma unroll
                        for (int e = 0; e < V; e += 4) {
                            const float4 f = *reinterpret_cast<const float4 *>(mine + from + e);
                            w[e] = f.x; w[e + 1] = f.y; w[e + 2] = f.z; w[e + 3] = f.w;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const int c = c0 + e;
                            w[e] = mine[c < P ? c + P : c < 2 * P ? c - P : c];
                        }
                    }
                    own_lds_written();
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) w[e] = u[e ^ 1];
                }
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = fmaf(C[e], u[e], S[e] * w[e]);
                if (!all_turned) {   // as they are, also infinities
#pragma unroll
                    for (int e = 0; e < V; ++e) if (c0 + e >= 2 * P) y[e] = u[e];
                }
                if constexpr (BWD && NORM) {
                    float tx = 0.f;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        sum[e] = fmaf(y[e] * x[e], r, sum[e]);
                        y[e] *= gamma[e];
                        tx = fmaf(y[e], x[e], tx);
                    }
                    const float f = head_sum<LPH>(tx) * inv_dim * r * r;
#pragma unroll
                    for (int e = 0; e < V; ++e) y[e] = r * fmaf(-x[e], f, y[e]);
                }
                if (on) store8(reinterpret_cast<T *>(sd.out) + row * sd.out_stride + head * a.dim + c0, y);
            }
        };
        if (part < turns_q) side(a.q, part, turns_q, [&] { if (first_k < turns_k) fetch(a.k, row, first_k * GROUPS + group); else fetch_row(unit + step); }, sum_q);
        if (first_k < turns_k) side(a.k, first_k, turns_k, [&] { fetch_row(unit + step); }, sum_k);
    }
    if constexpr (BWD && NORM) {
        if (a.part == nullptr) return;
        // the heads of a wavefront, then the wavefronts of the block
#pragma unroll
        for (int o = LPH; o < 64; o *= 2) { add_by(sum_q, o); add_by(sum_k, o); }
        if (group == 0) {
#pragma unroll
            for (int e = 0; e < V; ++e) { s_g[(wave * 2) * ROOM + c0 + e] = sum_q[e]; s_g[(wave * 2 + 1) * ROOM + c0 + e] = sum_k[e]; }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * a.dim; i += NT) {
            const int which = i >= a.dim, c = i - which * a.dim;
            float s = 0.f;
            for (int w = 0; w < WAVES; ++w) s += s_g[(w * 2 + which) * ROOM + c];
            a.part[(long long)blockIdx.x * 2 * a.dim + i] = s;
        }
    }
}

// dgamma of eight channels: 128 threads to each go over the blocks' sums, in 64 bits.
constexpr int kSumThreads = 1024, kSumChannels = 8;
__global__ __launch_bounds__(kSumThreads) void k_qk_rotary_dgamma(const float *part, int blocks, int dim, float *dgamma_q, float *dgamma_k)
{
    __shared__ double s[kSumThreads];
    const int i = blockIdx.x * kSumChannels + (threadIdx.x & (kSumChannels - 1));
    double sum = 0;
#pragma unroll 8
    for (int b = threadIdx.x / kSumChannels; b < blocks; b += kSumThreads / kSumChannels) sum += part[(long long)b * 2 * dim + i];
    s[threadIdx.x] = sum;
    __syncthreads();
    for (int o = kSumThreads / 2; o >= kSumChannels; o /= 2) {
        if (threadIdx.x < o) s[threadIdx.x] = sum = sum + s[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x >= kSumChannels) return;
    float *to = i < dim ? dgamma_q : dgamma_k;
    if (to != nullptr) to[i < dim ? i : i - dim] = (float)sum;
}

// ---- entry points -------------------------------------------------------------------------------------------------

const char *const kName = "norm and rotary position";

long long width(const dp_qk_rotary_desc &d, bool keys) { return (long long)(keys ? d.kv_heads : d.heads) * d.dim; }

dp_status check_desc(const dp_qk_rotary_desc *desc)
{
    if (desc == nullptr) { dp_set_error("%s: descriptor is NULL", kName); return DP_ERR_NULL; }
    const dp_qk_rotary_desc &d = *desc;
    if (d.io_dtype != DP_BF16 && d.io_dtype != DP_F32) { dp_set_error("%s: unknown io_dtype %d", kName, d.io_dtype); return DP_ERR_UNSUPPORTED; }
    if ((d.flags & ~(DP_QK_NORM | DP_ROTARY_HALVES)) != 0) { dp_set_error("%s: unknown flags 0x%x", kName, d.flags); return DP_ERR_UNSUPPORTED; }
    if (d.rows < 0 || d.heads < 1 || d.kv_heads < 0) { dp_set_error("%s: %d rows, %d and %d heads", kName, d.rows, d.heads, d.kv_heads); return DP_ERR_BAD_DESC; }
    if (d.dim < 8 || d.dim > kMaxDim || d.dim % 8 != 0) { dp_set_error("%s: dim %d is not a multiple of 8 up to %d", kName, d.dim, kMaxDim); return DP_ERR_BAD_DESC; }
    if (d.axes < 1 || d.axes > kMaxAxes) { dp_set_error("%s: %d axes", kName, d.axes); return DP_ERR_BAD_DESC; }
    long long turned = 0;
    for (int i = 0; i < d.axes; ++i) {
        if (d.pairs[i] < 0) { dp_set_error("%s: %d pairs on axis %d", kName, d.pairs[i], i); return DP_ERR_BAD_DESC; }
        turned += d.pairs[i];
    }
    if (2 * turned > d.dim) { dp_set_error("%s: %lld pairs in %d channels", kName, turned, d.dim); return DP_ERR_BAD_DESC; }
    if ((d.flags & DP_QK_NORM) != 0 && !(d.eps >= 1.17549435e-38f && d.eps < INFINITY)) { dp_set_error("%s: eps must be 2^-126 or more", kName); return DP_ERR_BAD_DESC; }
    if (width(d, false) + width(d, true) > INT32_MAX) { dp_set_error("%s: a row has 2^31 elements or more", kName); return DP_ERR_BAD_DESC; }
    const int vec = d.io_dtype == DP_BF16 ? 8 : 4;
    const long long q[] = {d.q_stride, d.q_out_stride, d.dq_stride}, k[] = {d.k_stride, d.k_out_stride, d.dk_stride};
    for (int i = 0; i < 3; ++i)
        if ((q[i] != 0 && (q[i] < width(d, false) || q[i] % vec != 0)) || (k[i] != 0 && (k[i] < width(d, true) || k[i] % vec != 0)) ||
            q[i] > (1ll << 40) || k[i] > (1ll << 40)) {
            dp_set_error("%s: strides must be whole multiples of 16 bytes and hold the heads", kName);
            return DP_ERR_BAD_DESC;
        }
    return DP_OK;
}

long long stride_or(long long stride, long long dense) { return stride != 0 ? stride : dense; }

bool turns(const dp_qk_rotary_desc &d) { return d.pairs[0] > 0 || (d.axes > 1 && d.pairs[1] > 0) || (d.axes > 2 && d.pairs[2] > 0); }   // else pos and freq are not read

struct Launch { int blocks, parts; };

// Wavefronts of a row: one goes over all its heads unless rows are few (at 8 rows of 28 heads of 128 channels the row's last head is then seven waits for memory away
// instead of one).  The norm's gradient has as many blocks as the card holds, which go on from row to row with the next one's first heads under way (16 x 28 x 28 rows of 32
// heads of 128: 66 us, 72 with 2048 blocks); the others are better off with a wavefront to a row (4099 rows of 12 heads of 72 fp32: 8.1 us, 9.4 with 768 blocks).
Launch launch_of(const dp_qk_rotary_desc &d, bool norm_grad)
{
    int lph = 2;
    while (lph * V < d.dim) lph *= 2;
    const int groups = 64 / lph, turns = (d.heads + groups - 1) / groups + (d.kv_heads + groups - 1) / groups;
    const long long wanted = 256 * 16;
    Launch l;
    l.parts = (int)std::min<long long>(turns, std::max<long long>(1, wanted / std::max(1, d.rows)));
    const long long waves = (long long)d.rows * l.parts;
    l.blocks = (int)std::min<long long>((waves + WAVES - 1) / WAVES, norm_grad ? kNormGradBlocks : kBlocks);
    return l;
}

size_t sums_bytes(const dp_qk_rotary_desc &d) { return (size_t)launch_of(d, true).blocks * 2 * d.dim * sizeof(float); }

template <typename T, int LPH, bool HALVES> auto pick(bool norm, bool bwd)
{
    return bwd ? (norm ? k_qk_rotary<T, LPH, HALVES, true, true> : k_qk_rotary<T, LPH, HALVES, false, true>)
               : (norm ? k_qk_rotary<T, LPH, HALVES, true, false> : k_qk_rotary<T, LPH, HALVES, false, false>);
}
template <typename T, bool HALVES> auto pick(int dim, bool norm, bool bwd)
{
    return dim <= 16 ? pick<T, 2, HALVES>(norm, bwd) : dim <= 32 ? pick<T, 4, HALVES>(norm, bwd) : dim <= 64 ? pick<T, 8, HALVES>(norm, bwd)
         : dim <= 128 ? pick<T, 16, HALVES>(norm, bwd) : pick<T, 32, HALVES>(norm, bwd);
}

dp_status run(const dp_qk_rotary_desc &d, QkArgs &a, bool bwd, hipStream_t st)
{
    const bool norm = (d.flags & DP_QK_NORM) != 0, halves = (d.flags & DP_ROTARY_HALVES) != 0, bf = d.io_dtype == DP_BF16;
    a.rows = d.rows; a.dim = d.dim; a.axes = d.axes; a.eps = d.eps;
    a.turned = 0;
    for (int i = 0; i < kMaxAxes; ++i) { a.pairs[i] = i < d.axes ? d.pairs[i] : 0; a.turned += a.pairs[i]; }
    a.q.heads = d.heads; a.k.heads = d.kv_heads;
    const Launch l = launch_of(d, norm && bwd);
    a.parts = l.parts;
    auto *kernel = bf ? (halves ? pick<bf16_t, true>(d.dim, norm, bwd) : pick<bf16_t, false>(d.dim, norm, bwd))
                      : (halves ? pick<float, true>(d.dim, norm, bwd) : pick<float, false>(d.dim, norm, bwd));
    hipLaunchKernelGGL(kernel, dim3(l.blocks), dim3(NT), 0, st, a);
    return launched(kName);
}

dp_status check_pointers(std::initializer_list<const void *> needed, std::initializer_list<const void *> given)
{
    for (const void *p : needed) if (p == nullptr) { dp_set_error("%s: a required pointer is NULL", kName); return DP_ERR_NULL; }
    for (auto &list : {needed, given})
        for (const void *p : list) if (!aligned16(p)) { dp_set_error("%s: pointers must be 16-byte aligned", kName); return DP_ERR_BAD_DESC; }
    return DP_OK;
}

}  // namespace

extern "C" size_t dp_qk_rotary_workspace_bytes(const dp_qk_rotary_desc *desc, int pass)
{
    if (check_desc(desc) != DP_OK || pass != DP_PASS_DGRAD || desc->rows == 0 || (desc->flags & DP_QK_NORM) == 0) return 0;
    return sums_bytes(*desc);
}

extern "C" dp_status dp_qk_rotary_fwd(const dp_qk_rotary_desc *desc, const void *q, const void *k, const float *gamma_q, const float *gamma_k,
                                      const float *pos, const double *freq, void *q_out, void *k_out, void *hip_stream)
{
    dp_status s = check_desc(desc);
    if (s != DP_OK) return s;
    const dp_qk_rotary_desc &d = *desc;
    if (d.rows == 0) return DP_OK;
    const bool keys = d.kv_heads > 0;
    if ((s = check_pointers({q, q_out}, {gamma_q, gamma_k, pos, freq})) != DP_OK || (turns(d) && (s = check_pointers({pos, freq}, {})) != DP_OK) || (keys && (s = check_pointers({k, k_out}, {})) != DP_OK)) return s;
    const long long wq = width(d, false), wk = width(d, true);
    QkArgs a = {};
    a.q = {q, nullptr, q_out, gamma_q, stride_or(d.q_stride, wq), 0, stride_or(d.q_out_stride, wq), 0};
    a.k = {k, nullptr, k_out, gamma_k, stride_or(d.k_stride, wk), 0, stride_or(d.k_out_stride, wk), 0};
    if ((q == q_out && a.q.x_stride != a.q.out_stride) || (keys && k == k_out && a.k.x_stride != a.k.out_stride)) {
        dp_set_error("%s: in place, a result's stride must be its input's", kName);
        return DP_ERR_BAD_DESC;
    }
    a.pos = pos; a.freq = freq;
    return run(d, a, false, (hipStream_t)hip_stream);
}

extern "C" dp_status dp_qk_rotary_bwd(const dp_qk_rotary_desc *desc, const void *q, const void *k, const float *gamma_q, const float *gamma_k,
                                      const float *pos, const double *freq, const void *dq_out, const void *dk_out, void *dq, void *dk,
                                      float *dgamma_q, float *dgamma_k, void *ws, size_t ws_bytes, void *hip_stream)
{
    dp_status s = check_desc(desc);
    if (s != DP_OK) return s;
    const dp_qk_rotary_desc &d = *desc;
    hipStream_t st = (hipStream_t)hip_stream;
    const bool norm = (d.flags & DP_QK_NORM) != 0, keys = d.kv_heads > 0, sums = dgamma_q != nullptr || dgamma_k != nullptr;
    if (sums && !norm) { dp_set_error("%s: dgamma without DP_QK_NORM", kName); return DP_ERR_UNSUPPORTED; }
    if (d.rows > 0) {
        if ((s = check_pointers({dq_out, dq}, {q, k, gamma_q, gamma_k, pos, freq})) != DP_OK || (turns(d) && (s = check_pointers({pos, freq}, {})) != DP_OK) || (keys && (s = check_pointers({dk_out, dk}, {})) != DP_OK) ||
            (norm && (s = check_pointers({q}, {})) != DP_OK) || (norm && keys && (s = check_pointers({k}, {})) != DP_OK)) return s;
    }
    if ((s = check_pointers({}, {dgamma_q, dgamma_k, ws})) != DP_OK) return s;
    const long long wq = width(d, false), wk = width(d, true);
    QkArgs a = {};
    a.q = {q, dq_out, dq, gamma_q, stride_or(d.q_stride, wq), stride_or(d.q_out_stride, wq), stride_or(d.dq_stride, wq), 0};
    a.k = {k, dk_out, dk, gamma_k, stride_or(d.k_stride, wk), stride_or(d.k_out_stride, wk), stride_or(d.dk_stride, wk), 0};
    if ((dq_out == dq && a.q.dy_stride != a.q.out_stride) || (keys && dk_out == dk && a.k.dy_stride != a.k.out_stride) ||
        (norm && q == dq && a.q.x_stride != a.q.out_stride) || (norm && keys && k == dk && a.k.x_stride != a.k.out_stride)) {
        dp_set_error("%s: in place, a result's stride must be its input's", kName);
        return DP_ERR_BAD_DESC;
    }
    const size_t need = sums && d.rows > 0 ? sums_bytes(d) : 0;
    if (need > 0 && (ws == nullptr || ws_bytes < need)) {
        dp_set_error("%s: the gradient needs %zu workspace bytes, got %zu", kName, need, ws == nullptr ? (size_t)0 : ws_bytes);
        return DP_ERR_WORKSPACE;
    }
    a.pos = pos; a.freq = freq;
    a.part = sums ? (float *)ws : nullptr;
    if (d.rows > 0 && (s = run(d, a, true, st)) != DP_OK) return s;
    if (!sums) return DP_OK;
    // without rows the gradients are zero
    hipLaunchKernelGGL(k_qk_rotary_dgamma, dim3(2 * d.dim / kSumChannels), dim3(kSumThreads), 0, st, (const float *)ws, d.rows > 0 ? launch_of(d, true).blocks : 0, d.dim, dgamma_q, dgamma_k);
    return launched(kName);
}
