// Attention, forward: o = softmax(scale q k^T) v, one pass over the keys with the running maximum and sum of every query's softmax.
//
// Columns of a wavefront are pairs (query, head) of the heads that share one head of keys, so that a single token's heads are read against the
// cache together and neighbouring columns share their keys.  Per tile of keys: S = K q (lane: one query, half of the tile's keys in registers), p = exp2(S scale2 - m),
// o += V^T p.  m is a maximum of S scale2 that may be up to 8 short of the true one: p <= 2^8 costs 32-bit sums nothing, and o is rescaled
// only in the few tiles where the maximum grows by more.  p is rounded to bf16 as an operand of the second product (its sum is not): 2^-9 of each value at random, a third of the
// rounding of o itself.
//
// Long sequences are bound by the matrix cores and the power they draw: 8192 x 8192, 16 heads of 128, bf16, 507-536 us or 1025-1085 TFLOP/s (a product of 8192^3
// reaches 1235), matrix instructions in 59 % of the cycles at the 1.6 GHz that the card then keeps.  S a tile ahead, between the exponentials, and eight wavefronts to a tile changed nothing
// there.  Fewer heads' channels leave more cycles to the exponentials: 24 x 1024 tokens, 16 heads, 64 channels 126 us (819 TFLOP/s), 80 160, 96 177.  Two or three blocks share a compute
// unit, one exponentiates while another multiplies.  Single tokens are bound by memory: 16 sequences of up to 8192 keys, 8 heads of 128, 352 MB in 71 us.
#include "attention_common.h"
#include <algorithm>
#include <cmath>

namespace {

constexpr float kSlack = 8.f;

// Wavefronts of a block: CW of them side by side in columns, 4 / CW share the keys of each tile among them.
// With split keys there are many blocks, and two of them on a compute unit with one tile each load more than one with two.
template <typename T, int DP, int CW, bool SPLIT> struct Shape {
    static constexpr int RW = 4 / CW, NB = sizeof(T) == 2 && CW == 4 ? 2 : 1, KT = RW * NB * 32, BYTES = KT * Tile<T, DP>::RB;   // NB: blocks of 32 keys of a wavefront
    static constexpr int STAGES = 4 * BYTES <= (SPLIT ? 65536 : 131072) ? 2 : 1;
};

template <typename T, int DP, int CW, bool SPLIT> __global__ __launch_bounds__(256, CW == 4 && sizeof(T) == 2 && DP <= 96 ? 3 : (CW == 4 || SPLIT) && (sizeof(T) == 2 || DP <= 64) ? 2 : 1) void k_attention(AttnArgs a)
{
    using L = Tile<T, DP>;
    using S = Shape<T, DP, CW, SPLIT>;
    constexpr int RW = S::RW, NB = S::NB, KT = S::KT, DB = L::DB, BYTES = S::BYTES, STAGES = S::STAGES, COLS = CW * 32;
    constexpr int ROOM = 2 * STAGES * BYTES > (RW > 1 ? 4 * DB * 4096 : 0) ? 2 * STAGES * BYTES : 4 * DB * 4096;
    __shared__ alignas(1024) char s_tiles[ROOM];   // K and V of each stage
    __shared__ float2 s_ml[RW > 1 ? 256 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, wc = wave % CW, wr = wave / CW;
    const Item item = item_of<COLS, SPLIT, true, CW == 4 && sizeof(T) == 2 ? DP <= 96 ? 3 : 2 : 1>(a, a.q, a.shared, blockIdx.x, gridDim.x);
    if (!item.any) return;
    const int b = item.b, hk = item.hk, split = item.split;
    const int col0 = item.tile * COLS;
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rq.own * a.shared) return;

    const int wcol = col0 + wc * 32, col = wcol + (lane & 31), i = col / a.shared, head = hk * a.shared + col % a.shared;
    const bool own = i < rq.own, on = i < rq.used;
    const int ahead = rk.used - rq.used, last = rq.used * a.shared - 1;
    // the keys that the block's queries see, and the wavefront's (lengths are at most 2^28 and bounds 2^30: no sum here passes 31 bits)
    int lo = 0, hi = 0;
    const int i0 = col0 / a.shared, i1 = min(col0 + COLS - 1, last) / a.shared, w0 = wcol / a.shared, w1 = min(wcol + 31, last) / a.shared;
    if (col0 <= last) {
        lo = max(0, i0 + ahead - a.left);
        hi = min(rk.used, i1 + ahead + a.right + 1);
    }
    if (SPLIT) {
        lo += split * a.split_keys;
        hi = min(hi, lo + a.split_keys);
    }
    const int first = lo, keys = max(0, hi - lo);
    const long long row = rq.first + i;

    // the lane's keys, counted from the wavefront's place in the first tile
    const int mine = wr * NB * 32;
    const int seen0 = max(i + ahead - a.left - first, 0);
    const unsigned seen = on ? (unsigned)max(min(i + ahead + a.right + 1 - first, keys) - seen0, 0) : 0u;
    // a wavefront's keys from t on are seen by all of its queries if all0 <= t <= all1, by none if t <= none0 or t >= none1
    const int all0 = max(w1 + ahead - a.left - first, 0), all1 = max(min(w0 + ahead + a.right + 1 - first, keys) - NB * 32, -1);
    const int none0 = max(w0 + ahead - a.left - first, 0) - NB * 32, none1 = min(w1 + ahead + a.right + 1 - first, keys);

    f32x16 acc[DB];
    clear(acc);
    float m = -INFINITY, mu = 0.f, l = 0.f;
    if (keys > 0) {
        using Copy = TileCopy<T, DP, KT, 256>;
        Copy ck, cv;
        ck.init(threadIdx.x, a.dim, a.k_stride);
        cv.init(threadIdx.x, a.dim, a.v_stride);
        const T *kp = reinterpret_cast<const T *>(a.kp) + (rk.first + first) * a.k_stride + (long long)hk * a.dim;
        const T *vp = reinterpret_cast<const T *>(a.vp) + (rk.first + first) * a.v_stride + (long long)hk * a.dim;
        const unsigned base = lds_offset(s_tiles);
        TileLane<T, DP> tl;
        tl.init(lane);
        ck.issue(kp, keys, a.dim, a.k_stride, base, wave);
        cv.issue(vp, keys, a.dim, a.v_stride, base + STAGES * BYTES, wave);
        u32x4 q[L::SLICES];
        load_column<T, DP>(reinterpret_cast<const T *>(a.qp) + row * a.q_stride + (long long)head * a.dim, on, a.dim, half, q);
        unsigned stage = 0;
        for (int t = 0; t < keys; t += KT) {
            const bool more = t + KT < keys;
            if (STAGES == 2) wait_vmcnt<0>();
            else wait_vmcnt<Copy::N>();     // K alone
            __builtin_amdgcn_s_barrier();   // the tile has arrived, and the one before is done with
            const unsigned kt = base + stage + mine * L::RB, vt = kt + STAGES * BYTES;
            const auto next_k = [&] {
                kp += KT * a.k_stride;
                ck.issue(kp, keys - t - KT, a.dim, a.k_stride, base + stage, wave);
            };
            const auto next_v = [&] {
                vp += KT * a.v_stride;
                cv.issue(vp, keys - t - KT, a.dim, a.v_stride, base + STAGES * BYTES + stage, wave);
            };
            if (STAGES == 2 && more) {
                stage ^= BYTES;
                next_k();
                next_v();
            }
            const int w = t + mine;
            const bool some = w > none0 && w < none1;
            f32x16 s[NB];
            if (some) {
                clear(s);
                First<T, DP, NB, DP == 96 ? 6 : 8> kq;
                kq.begin(kt + tl.row, tl.x);
                kq.run(kt + tl.row, tl.x, q, s);
            }
            if constexpr (STAGES == 1) {    // K's room takes the next keys, then V has to be there
                __builtin_amdgcn_s_barrier();
                if (more) { next_k(); wait_vmcnt<Copy::N>(); }
                else wait_vmcnt<0>();
                __builtin_amdgcn_s_barrier();
            }
            if (some) {
                Second<T, DP, NB * 2> pv;
                pv.begin(vt, tl);
                if (w < all0 || w > all1) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            if ((unsigned)(w + 32 * nb + 8 * (v >> 2) + 4 * half + (v & 3) - seen0) >= seen) s[nb][v] = -INFINITY;
                }
                float mx = s[0][0];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[nb][v]);
                mx = fmaxf(mx, other_half(mx)) * a.scale2;
                if (__any(mx > m + kSlack)) {
                    const float mn = fmaxf(m, mx), f = mn == m ? 1.f : __builtin_amdgcn_exp2f(m - mn);
                    m = mn;
                    mu = m == -INFINITY ? 0.f : m;
                    l *= f;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int v = 0; v < 16; ++v) acc[db][v] *= f;
                }
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        s[nb][v] = __builtin_amdgcn_exp2f(fmaf(s[nb][v], a.scale2, -mu));
                        sum[v & 3] += s[nb][v];
                    }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                pv.run(vt, tl, [&](auto sc) { constexpr int sl = decltype(sc)::value; return column<T>(s[sl / 2], sl % 2); }, acc);
            }
            if (STAGES == 1 && more) {
                __builtin_amdgcn_s_barrier();
                next_v();
            }
        }
    }
    l += other_half(l);
    if constexpr (RW > 1) {   // the wavefronts' results brought to one maximum and added up
        s_ml[wave * 64 + lane] = make_float2(m, l);
        __syncthreads();
        float most = m;
#pragma unroll
        for (int w = 0; w < 4; ++w) most = fmaxf(most, s_ml[w * 64 + lane].x);
        l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 ml = s_ml[w * 64 + lane];
            l += ml.x == most ? ml.y : ml.y * __builtin_amdgcn_exp2f(ml.x - most);
        }
        const float f = m == most ? 1.f : __builtin_amdgcn_exp2f(m - most);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[db][v] *= f;
        m = most;
        sum_waves<4>(acc, reinterpret_cast<float *>(s_tiles), wave, lane);
    }
    if (!own) return;
    const bool some = on && l != 0.f;
    const long long at = (long long)head * a.q.rows + row, part = split * (long long)a.heads * a.q.rows + at;
    const float f = SPLIT ? 1.f : some ? 1.f / l : 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        if (RW > 1 && db != wr) continue;
        if (!some) {
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
        }
        if constexpr (SPLIT) { if (some) store_block<float>(acc[db], f, a.part_o + part * a.dim, db * 32, a.dim, half); }
        else store_block<T>(acc[db], f, reinterpret_cast<T *>(a.op) + row * a.o_stride + (long long)head * a.dim, db * 32, a.dim, half);
    }
    if (half == 0 && wr == 0) {
        if constexpr (SPLIT) *reinterpret_cast<float2 *>(a.part_ml + 2 * part) = make_float2(m, on ? l : 0.f);
        else if (a.lse != nullptr) a.lse[at] = some ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    }
}

// Splits of the keys put together: 32 lanes to a column, four channels each; for the statistics a lane has splits lane and lane + 32.
constexpr int kJoinThreads = 256, kMaxSplits = 64;
template <typename T> __global__ __launch_bounds__(kJoinThreads) void k_attention_join(AttnArgs a)
{
    const int hb = blockIdx.x / a.tiles, b = hb % a.n, hk = hb / a.n, lane = threadIdx.x & 31;
    const int col = (blockIdx.x % a.tiles) * (kJoinThreads / 32) + (threadIdx.x >> 5), i = col / a.shared, head = hk * a.shared + col % a.shared;
    const Rows rq = rows_of(a.q, b);
    const bool own = i < rq.own;
    const int splits = a.ragged ? parts_of(a, b) : a.splits;
    const long long row = rq.first + i, at = (long long)head * a.q.rows + row, step = (long long)a.heads * a.q.rows;
    float2 ml[2] = {{-INFINITY, 0.f}, {-INFINITY, 0.f}};
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (own && lane + 32 * h < splits) ml[h] = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (at + (lane + 32 * h) * step));
    float m = fmaxf(ml[0].y != 0.f ? ml[0].x : -INFINITY, ml[1].y != 0.f ? ml[1].x : -INFINITY);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor(m, o, 32));
    float f[2], l = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        f[h] = ml[h].y == 0.f ? 0.f : ml[h].x == m ? 1.f : __builtin_amdgcn_exp2f(ml[h].x - m);
        l += f[h] * ml[h].y;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) l += __shfl_xor(l, o, 32);
    const int c = lane * 4;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < splits; s0 += 8) {   // eight at a time are under way
        f32x4 v[8];
        float g[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int s = s0 + u;
            g[u] = __shfl(s < 32 ? f[0] : f[1], s & 31, 32);
            v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (own && s < splits && g[u] != 0.f && c < a.dim) v[u] = *reinterpret_cast<const f32x4 *>(a.part_o + (at + s * step) * a.dim + c);   // 0: its o was not written, or vanishes
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(g[u], v[u][e], o[e]);
    }
    if (!own) return;
    const float inv = l != 0.f ? 1.f / l : 0.f;
    if (c < a.dim) {
        T *to = reinterpret_cast<T *>(a.op) + row * a.o_stride + (long long)head * a.dim + c;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2 *>(to) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
        else *reinterpret_cast<f32x4 *>(to) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    }
    if (lane == 0 && a.lse != nullptr) a.lse[at] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// ---- entry points -------------------------------------------------------------------------------------------------

const char *const kName = "attention";

long long rows_or(long long rows, long long dense) { return rows != 0 ? rows : dense; }

struct Form { int cw, splits, split_keys, span; };   // wavefronts side by side in a block; blocks that the keys of a column are dealt out to, each one's keys, and all of them at most

// Four wavefronts side by side share the copies of a tile of keys; where that takes longer (attn_wide) the four of them take the same 32 columns and share the keys, and if that leaves
// compute units without work too, blocks share them.
Form form_of(const dp_attention_desc &d)
{
    const long long shared = d.heads / d.kv_heads, cols = d.q_len * shared, rows = rows_or(d.q_rows, (long long)d.n * d.q_len);
    if (attn_wide(d, d.q_len, rows, shared, attn_seen(d, d.kv_len, 128 / (int)std::min<long long>(shared, 128)))) return {4, 1, 0, 0};
    const long long blocks = std::max<long long>(1, d.kv_heads * attn_tiles(d.n, d.q_len, rows, shared, 32));
    constexpr int kt = 128;
    // keys that a block looks at: of its queries; behind the last query's place there are none
    const long long queries = std::min<long long>(d.q_len, 32 / shared + (32 % shared != 0 ? 2 : 0)), behind = std::max<long long>(0, d.right < 0 ? d.q_len - 1 : std::min(d.right, d.q_len - 1));
    const long long span = d.left < 0 ? d.kv_len : std::min<long long>(d.kv_len, d.left + behind + queries);
    const long long most = std::min<long long>(kMaxSplits, (span + 4 * kt - 1) / (4 * kt));   // four tiles at least: the join takes as long as two
    // A single token's columns fit one block, which waits for memory most of the time: four rounds of blocks at least.  Others compute, and are split only to give every compute unit work
    // (2000 causal tokens fp32, 8 heads of 128 over 2, 500 blocks: 113 us, 205 in four parts; bf16 33 and 53).
    const long long want = std::min<long long>(most, (cols <= 32 ? 2048 : 512) / blocks);
    if (want < 2) return {1, 1, 0, 0};
    // whole tiles, from the first key on that a block's queries see (one token that sees 4096 of 131072 keys, 32 heads of 128 over 8: 9.0 us, 35.9 where the parts are of all keys and one of nine holds those)
    const long long per = ((span + want - 1) / want + kt - 1) / kt * kt;
    return {1, (int)((span + per - 1) / per), (int)per, (int)span};
}

size_t split_bytes(const dp_attention_desc &d, const Form &f)
{
    if (f.splits < 2) return 0;
    return (size_t)f.splits * d.heads * (size_t)rows_or(d.q_rows, (long long)d.n * d.q_len) * (d.dim + 2) * sizeof(float);
}

template <typename T> void launch(const AttnArgs &a, const Form &f, unsigned blocks, hipStream_t st)
{
    for_dim(a.dim, [&](auto dc) {
        constexpr int DP = decltype(dc)::value;
        auto *kernel = f.cw == 4 ? k_attention<T, DP, 4, false> : f.splits == 1 ? k_attention<T, DP, 1, false> : k_attention<T, DP, 1, true>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, a);
    });
}

}  // namespace

dp_status attn_check(const dp_attention_desc *desc, const dp_attention_seqs *seqs, bool gradient)
{
    if (desc == nullptr) { dp_set_error("%s: descriptor is NULL", kName); return DP_ERR_NULL; }
    const dp_attention_desc &d = *desc;
    if (d.io_dtype != DP_BF16 && d.io_dtype != DP_F32) { dp_set_error("%s: unknown io_dtype %d", kName, d.io_dtype); return DP_ERR_UNSUPPORTED; }
    if (d.n < 0 || d.q_len < 0 || d.kv_len < 0 || d.q_len > (1 << 28) || d.kv_len > (1 << 28)) {
        dp_set_error("%s: %d sequences of %d and %d", kName, d.n, d.q_len, d.kv_len);
        return DP_ERR_BAD_DESC;
    }
    if (d.heads < 1 || d.kv_heads < 1 || d.heads % d.kv_heads != 0) { dp_set_error("%s: %d heads of queries, %d of keys", kName, d.heads, d.kv_heads); return DP_ERR_BAD_DESC; }
    if (d.dim < 8 || d.dim > 128 || d.dim % 8 != 0) { dp_set_error("%s: dim %d is not a multiple of 8 up to 128", kName, d.dim); return DP_ERR_BAD_DESC; }
    if (d.left < -1 || d.right < -1) { dp_set_error("%s: window %d, %d", kName, d.left, d.right); return DP_ERR_BAD_DESC; }
    if (!(d.scale >= 0.f && d.scale <= 0x1p126f)) { dp_set_error("%s: scale must be above 0 and at most 2^126 (0: 1/sqrt(dim))", kName); return DP_ERR_BAD_DESC; }
    const long long wq = (long long)d.heads * d.dim, wk = (long long)d.kv_heads * d.dim;
    const int vec = d.io_dtype == DP_BF16 ? 8 : 4;
    const long long strides[] = {d.q_stride, d.o_stride, d.k_stride, d.v_stride}, widths[] = {wq, wq, wk, wk};
    for (int i = 0; i < 4; ++i) {
        const long long s = strides[i] != 0 ? strides[i] : widths[i];
        if (s < widths[i] || s % vec != 0 || s > (1 << 22)) {
            dp_set_error("%s: strides must be whole multiples of 16 bytes, hold the heads, and be at most 2^22 elements", kName);
            return DP_ERR_BAD_DESC;
        }
    }
    const bool q_packed = seqs != nullptr && seqs->q_starts != nullptr, kv_packed = seqs != nullptr && seqs->kv_starts != nullptr;
    if (seqs != nullptr) {
        if ((q_packed && seqs->q_lens != nullptr) || (kv_packed && seqs->kv_lens != nullptr)) {
            dp_set_error("%s: starts and lengths of one side exclude each other", kName);
            return DP_ERR_UNSUPPORTED;
        }
        for (const void *p : {(const void *)seqs->q_starts, (const void *)seqs->kv_starts, (const void *)seqs->q_lens, (const void *)seqs->kv_lens})
            if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) { dp_set_error("%s: starts and lengths must be 4-byte aligned", kName); return DP_ERR_BAD_DESC; }
    }
    const long long q_dense = (long long)d.n * d.q_len, kv_dense = (long long)d.n * d.kv_len;
    if (d.q_rows < 0 || d.kv_rows < 0 || d.q_rows > (1ll << 31) || d.kv_rows > (1ll << 31) || rows_or(d.q_rows, q_dense) > (1ll << 31) || rows_or(d.kv_rows, kv_dense) > (1ll << 31) ||
        (!q_packed && rows_or(d.q_rows, q_dense) < q_dense) || (!kv_packed && rows_or(d.kv_rows, kv_dense) < kv_dense)) {
        dp_set_error("%s: %lld and %lld rows do not hold the sequences, or are more than 2^31", kName, (long long)d.q_rows, (long long)d.kv_rows);
        return DP_ERR_BAD_DESC;
    }
    // a launch has fewer than 2^32 threads, 512 to a block at the most (blocks of 32 columns: attn_wide); columns of queries, and of keys for dk and dv
    const double shared = d.heads / d.kv_heads, most = std::max<double>(d.q_len * shared, gradient ? d.kv_len : 0);
    if (d.q_len * shared >= (double)(1 << 30) || (double)d.n * d.kv_heads * (std::floor(most / 128) + 1) >= (double)(1 << 23)) {
        dp_set_error("%s: too many sequences, heads and tokens for one launch", kName);
        return DP_ERR_BAD_DESC;
    }
    return DP_OK;
}

void attn_args(const dp_attention_desc &d, const dp_attention_seqs *seqs, AttnArgs &a)
{
    a = {};
    a.q = {seqs != nullptr ? seqs->q_starts : nullptr, seqs != nullptr ? seqs->q_lens : nullptr, d.q_len, rows_or(d.q_rows, (long long)d.n * d.q_len)};
    a.kv = {seqs != nullptr ? seqs->kv_starts : nullptr, seqs != nullptr ? seqs->kv_lens : nullptr, d.kv_len, rows_or(d.kv_rows, (long long)d.n * d.kv_len)};
    a.n = d.n; a.heads = d.heads; a.kv_heads = d.kv_heads; a.shared = d.heads / d.kv_heads; a.dim = d.dim;
    a.left = d.left < 0 ? kFar : std::min(d.left, kFar);
    a.right = d.right < 0 ? kFar : std::min(d.right, kFar);
    a.scale = d.scale != 0.f ? d.scale : (float)(1.0 / std::sqrt((double)d.dim));
    a.scale2 = (float)((d.scale != 0.f ? (double)d.scale : 1.0 / std::sqrt((double)d.dim)) * 1.4426950408889634);
    const long long wq = (long long)d.heads * d.dim, wk = (long long)d.kv_heads * d.dim;
    a.q_stride = d.q_stride != 0 ? d.q_stride : wq;
    a.k_stride = d.k_stride != 0 ? d.k_stride : wk;
    a.v_stride = d.v_stride != 0 ? d.v_stride : wk;
    a.o_stride = d.o_stride != 0 ? d.o_stride : wq;
    a.splits = 1;
    a.causal = (d.left < 0) != (d.right < 0);
    a.ragged = seqs != nullptr && d.n <= kMostRagged && (seqs->q_starts != nullptr || seqs->kv_starts != nullptr || seqs->q_lens != nullptr || seqs->kv_lens != nullptr);
}

dp_status attn_pointers(std::initializer_list<const void *> needed, const void *lse, const void *ws)
{
    for (const void *p : needed) if (p == nullptr) { dp_set_error("%s: a required pointer is NULL", kName); return DP_ERR_NULL; }
    for (const void *p : needed) if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) { dp_set_error("%s: pointers must be 16-byte aligned", kName); return DP_ERR_BAD_DESC; }
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0 || (reinterpret_cast<uintptr_t>(ws) & 15u) != 0) { dp_set_error("%s: lse must be 4-byte, the workspace 16-byte aligned", kName); return DP_ERR_BAD_DESC; }
    return DP_OK;
}

dp_status attn_apart(std::initializer_list<const void *> results, std::initializer_list<const void *> inputs)
{
    for (const void *r : results)
        for (const void *i : inputs)
            if (r == i && r != nullptr) { dp_set_error("%s: a result may not take the place of an input", kName); return DP_ERR_BAD_DESC; }
    return DP_OK;
}

dp_status attn_workspace(size_t need, const void *ws, size_t ws_bytes)
{
    if (need == 0 || (ws != nullptr && ws_bytes >= need)) return DP_OK;
    dp_set_error("%s needs %zu workspace bytes, got %zu", kName, need, ws == nullptr ? (size_t)0 : ws_bytes);
    return DP_ERR_WORKSPACE;
}

dp_status attn_launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return DP_OK;
    dp_set_error("%s launch: %s", what, hipGetErrorString(e));
    return DP_ERR_HIP;
}

extern "C" size_t dp_attention_workspace_bytes(const dp_attention_desc *desc, int pass)
{
    // packed rows may be fewer than n q_len: checked with starts
    const int32_t none = 0;
    const dp_attention_seqs packed = {&none, &none, nullptr, nullptr};
    if (attn_check(desc, &packed, pass != DP_PASS_FWD) != DP_OK) return 0;
    const dp_attention_desc &d = *desc;
    if (pass == DP_PASS_FWD) return split_bytes(d, form_of(d));
    if (pass == DP_PASS_DGRAD) return attn_bwd_bytes(d);
    return 0;
}

extern "C" dp_status dp_attention_fwd(const dp_attention_desc *desc, const void *q, const void *k, const void *v, void *o, float *lse,
                                      const dp_attention_seqs *seqs, void *ws, size_t ws_bytes, void *hip_stream)
{
    dp_status s = attn_check(desc, seqs, false);
    if (s != DP_OK) return s;
    const dp_attention_desc &d = *desc;
    AttnArgs a;
    attn_args(d, seqs, a);
    if (d.n == 0 || d.q_len == 0 || a.q.rows == 0) return DP_OK;
    if ((s = attn_pointers({q, o}, lse, ws)) != DP_OK || (d.kv_len > 0 && a.kv.rows > 0 && (s = attn_pointers({k, v}, nullptr, nullptr)) != DP_OK)) return s;
    if ((s = attn_apart({o}, {q, k, v})) != DP_OK) return s;
    const Form f = form_of(d);
    if ((s = attn_workspace(split_bytes(d, f), ws, ws_bytes)) != DP_OK) return s;
    a.qp = q; a.kp = k; a.vp = v; a.op = o; a.lse = lse;
    a.splits = f.splits;
    a.split_keys = f.split_keys;
    a.span = f.span;
    a.part_o = (float *)ws;
    if (f.splits > 1) a.part_ml = a.part_o + (long long)f.splits * d.heads * a.q.rows * d.dim;
    const long long cols = (long long)d.q_len * a.shared, groups = (long long)d.n * d.kv_heads;
    a.tiles = (int)((cols + 32 * f.cw - 1) / (32 * f.cw));
    hipStream_t st = (hipStream_t)hip_stream;
    const bool bf = d.io_dtype == DP_BF16;
    const unsigned blocks = attn_blocks(a, a.q, a.shared, 32 * f.cw);
    if (bf) launch<bf16_t>(a, f, blocks, st);
    else launch<float>(a, f, blocks, st);
    if (f.splits > 1) {
        a.tiles = (int)((std::min<long long>(d.q_len, a.q.rows) * a.shared + kJoinThreads / 32 - 1) / (kJoinThreads / 32));
        hipLaunchKernelGGL(bf ? k_attention_join<bf16_t> : k_attention_join<float>, dim3((unsigned)(groups * a.tiles)), dim3(kJoinThreads), 0, st, a);
    }
    return attn_launched(kName);
}
