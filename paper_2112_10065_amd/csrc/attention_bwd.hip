// Attention, backward.  With p_ij = exp(s_ij - lse_i) recomputed from the forward call's lse, dp_ij = dout_i . v_j and delta_i = dout_i . o_i:
//   dv_j = sum_i p_ij dout_i;   ds_ij = p_ij (dp_ij - delta_i);   dq_i = scale sum_j ds_ij k_j;   dk_j = scale sum_i ds_ij q_i
// Two kernels, each with its sums in registers from the first to the last tile: one holds queries and lets keys pass (dq; it computes delta and leaves it for the other),
// one holds keys and lets the queries of all heads that share them pass (dk, dv).  p and dp are computed in both, seven products for the five that the formulas
// have, in return for sums without atomics in a fixed order and without partial sums in memory (dq's would be 32 bits per query and block of keys).
#include "attention_common.h"
#include <algorithm>

namespace {

template <typename T> constexpr int kRows = sizeof(T) == 2 ? 64 : 32;   // of a tile

template <typename T, int DP> __global__ __launch_bounds__(256, sizeof(T) == 2 || DP <= 64 ? 2 : 1) void k_attention_dq(AttnArgs a)
{
    using L = Tile<T, DP>;
    constexpr int KT = kRows<T>, DB = DP / 32, BYTES = KT * L::RB, COLS = 128;
    __shared__ alignas(1024) char s_tiles[4 * BYTES];   // K and V, two stages of each
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int id = logical_block(blockIdx.x, gridDim.x);
    const int bh = id / a.tiles, hk = bh % a.kv_heads, b = bh / a.kv_heads;
    const int col0 = (a.tiles - 1 - id % a.tiles) * COLS;
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rq.own * a.shared) return;
    const int col = col0 + wave * 32 + (lane & 31), i = col / a.shared, head = hk * a.shared + col % a.shared;
    const bool own = i < rq.own, on = i < rq.used;
    const int ahead = rk.used - rq.used, wcol = col0 + wave * 32, last = rq.used * a.shared - 1;
    long long lo = 0, hi = 0;
    const long long i0 = col0 / a.shared, i1 = min(col0 + COLS - 1, last) / a.shared, w0 = wcol / a.shared, w1 = min(wcol + 31, last) / a.shared;
    if (col0 <= last) {
        lo = max(0ll, i0 + ahead - a.left);
        hi = min((long long)rk.used, i1 + ahead + a.right + 1);
    }
    const int first = (int)lo, keys = (int)max(0ll, hi - lo);
    const long long row = rq.first + i, stat = (long long)head * a.q.rows + row;

    u32x4 q[L::SLICES], g[L::SLICES];
    load_column<T, DP>(reinterpret_cast<const T *>(a.qp) + row * a.q_stride + (long long)head * a.dim, on, a.dim, half, q);
    float delta = 0.f, lse2 = INFINITY;
    {
        u32x4 o[L::SLICES];
        const long long at = row * a.o_stride + (long long)head * a.dim;
        load_column<T, DP>(reinterpret_cast<const T *>(a.dout) + at, on, a.dim, half, g);
        load_column<T, DP>(reinterpret_cast<const T *>(a.op_in) + at, on, a.dim, half, o);
#pragma unroll
        for (int s = 0; s < L::SLICES; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (sizeof(T) == 2) {
                    delta = fmaf(__uint_as_float(g[s][e] << 16), __uint_as_float(o[s][e] << 16), delta);
                    delta = fmaf(__uint_as_float(g[s][e] & 0xffff0000u), __uint_as_float(o[s][e] & 0xffff0000u), delta);
                } else delta = fmaf(__uint_as_float(g[s][e]), __uint_as_float(o[s][e]), delta);
            }
        delta += other_half(delta);
        if (on) {
            const float x = a.lse_in[stat];
            lse2 = x == -INFINITY ? INFINITY : x * kLog2e;
        }
        if (on && half == 0) { a.lse2[stat] = lse2; a.delta[stat] = delta; }
    }
    const long long see0 = max((long long)i + ahead - a.left - first, 0ll), see1 = min((long long)i + ahead + a.right + 1 - first, (long long)keys);
    const int seen0 = (int)min(see0, (long long)kFar);
    const unsigned seen = on ? (unsigned)max(see1 - seen0, 0ll) : 0u;
    const int all0 = (int)min(max(w1 + ahead - a.left - first, 0ll), (long long)kFar), all1 = (int)max(min(w0 + ahead + a.right + 1 - first, (long long)keys) - KT, -1ll);
    const int none0 = (int)(min(max(w0 + ahead - a.left - first, 0ll), (long long)kFar) - KT), none1 = (int)min(w1 + ahead + a.right + 1 - first, (long long)kFar);

    f32x16 acc[DB];
    clear(acc);
    if (keys > 0) {
        TileCopy<T, DP, KT, 256> ck, cv;
        ck.init(threadIdx.x, a.dim, a.k_stride);
        cv.init(threadIdx.x, a.dim, a.v_stride);
        const T *kp = reinterpret_cast<const T *>(a.kp) + (rk.first + first) * a.k_stride + (long long)hk * a.dim;
        const T *vp = reinterpret_cast<const T *>(a.vp) + (rk.first + first) * a.v_stride + (long long)hk * a.dim;
        const unsigned base = lds_offset(s_tiles);
        TileLane<T, DP> tl;
        tl.init(lane);
        ck.issue(kp, keys, a.dim, a.k_stride, base, wave);
        cv.issue(vp, keys, a.dim, a.v_stride, base + 2 * BYTES, wave);
        unsigned stage = 0;
        for (int t = 0; t < keys; t += KT, stage ^= BYTES) {
            wait_vmcnt<0>();
            __builtin_amdgcn_s_barrier();   // the tile has arrived, and the one before is done with
            if (t + KT < keys) {
                kp += KT * a.k_stride;
                vp += KT * a.v_stride;
                ck.issue(kp, keys - t - KT, a.dim, a.k_stride, base + (stage ^ BYTES), wave);
                cv.issue(vp, keys - t - KT, a.dim, a.v_stride, base + 2 * BYTES + (stage ^ BYTES), wave);
            }
            if (t <= none0 || t >= none1) continue;
            const bool edge = t < all0 || t > all1;
#pragma unroll
            for (int nb = 0; nb < KT / 32; ++nb) {
                const unsigned kt = base + stage + nb * 32 * L::RB, vt = base + 2 * BYTES + stage + nb * 32 * L::RB;
                f32x16 s[1], dp[1];
                clear(s);
                clear(dp);
                First<T, DP, 1, 6> kq, vg;
                kq.begin(kt + tl.row, tl.x);
                kq.run(kt + tl.row, tl.x, q, s);
                vg.begin(vt + tl.row, tl.x);
                vg.run(vt + tl.row, tl.x, g, dp);
                Second<T, DP, 2> ks;
                ks.begin(kt, tl);
                if (edge) {
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if ((unsigned)(t + 32 * nb + 8 * (v >> 2) + 4 * half + (v & 3) - seen0) >= seen) s[0][v] = -INFINITY;
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[0][v], a.scale2, -lse2));
                    s[0][v] = p * (dp[0][v] - delta);
                }
                ks.run(kt, tl, [&](auto sc) { return column<T>(s[0], decltype(sc)::value); }, acc);
            }
        }
    }
    if (!own) return;
    if (!on || lse2 == INFINITY) clear(acc);
    store_column<T, DB>(acc, a.scale, reinterpret_cast<T *>(a.dq) + row * a.q_stride + (long long)head * a.dim, a.dim, half);
}

template <typename T, int DP> __global__ __launch_bounds__(256, 1) void k_attention_dkv(AttnArgs a)
{
    using L = Tile<T, DP>;
    constexpr int QT = kRows<T>, DB = DP / 32, BYTES = QT * L::RB, COLS = 128;
    __shared__ alignas(1024) char s_tiles[4 * BYTES];   // q and dout, two stages of each
    __shared__ alignas(16) float s_stats[2][2][64];     // [stage][lse2, delta]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int id = logical_block(blockIdx.x, gridDim.x);
    const int bh = id / a.tiles, hk = bh % a.kv_heads, b = bh / a.kv_heads;
    const int col0 = (id % a.tiles) * COLS;             // causal: the longest first
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rk.own) return;
    const int j = col0 + wave * 32 + (lane & 31);
    const bool own = j < rk.own, on = j < rk.used;
    const long long ahead = rk.used - rq.used;
    // the queries that see the block's keys, and the wavefront's
    const int last = rk.used - 1, wcol = col0 + wave * 32;
    long long lo = 0, hi = 0;
    const long long j1 = min(col0 + COLS - 1, last), w0 = wcol, w1 = min(wcol + 31, last);
    if (col0 <= last) {
        lo = max(0ll, col0 - a.right - ahead);
        hi = min((long long)rq.used, j1 + a.left - ahead + 1);
    }
    const int first = (int)min(lo, (long long)kFar), count = (int)max(0ll, hi - lo);
    const long long row = rk.first + j;
    const long long see0 = max(j - a.right - ahead - first, 0ll), see1 = min(j + a.left - ahead + 1 - first, (long long)count);
    const int seen0 = (int)min(see0, (long long)kFar);
    const unsigned seen = on ? (unsigned)max(see1 - seen0, 0ll) : 0u;
    const int all0 = (int)min(max(w1 - a.right - ahead - first, 0ll), (long long)kFar), all1 = (int)max(min(w0 + a.left - ahead + 1 - first, (long long)kFar) - QT, -1ll);
    const int none0 = (int)(min(max(w0 - a.right - ahead - first, 0ll), (long long)kFar) - QT), none1 = (int)min(w1 + a.left - ahead + 1 - first, (long long)kFar);

    f32x16 dk[DB], dv[DB];
    clear(dk);
    clear(dv);
    if (count > 0) {
        u32x4 kc[L::SLICES], vc[L::SLICES];
        load_column<T, DP>(reinterpret_cast<const T *>(a.kp) + row * a.k_stride + (long long)hk * a.dim, on, a.dim, half, kc);
        load_column<T, DP>(reinterpret_cast<const T *>(a.vp) + row * a.v_stride + (long long)hk * a.dim, on, a.dim, half, vc);
        TileCopy<T, DP, QT, 256> cq, cg;
        cq.init(threadIdx.x, a.dim, a.q_stride);
        cg.init(threadIdx.x, a.dim, a.o_stride);
        const unsigned base = lds_offset(s_tiles), stats = lds_offset(s_stats);
        TileLane<T, DP> tl;
        tl.init(lane);
        const int tiles = (count + QT - 1) / QT, all = tiles * a.shared;
        // tile n: queries first + (n % tiles) QT ... of the n / tiles-th head; rows behind the last query arrive as zeros, also their statistics: nothing is added then
        int ih = hk * a.shared, it = 0;
        auto issue = [&](unsigned stage, int slot) {
            const long long at = rq.first + first + it;
            const int rows = count - it;
            cq.issue(reinterpret_cast<const T *>(a.qp) + at * a.q_stride + (long long)ih * a.dim, rows, a.dim, a.q_stride, base + stage, wave);
            cg.issue(reinterpret_cast<const T *>(a.dout) + at * a.o_stride + (long long)ih * a.dim, rows, a.dim, a.o_stride, base + 2 * BYTES + stage, wave);
            if (wave < 2) {
                const auto r = make_rsrc((wave == 0 ? a.lse2 : a.delta) + (long long)ih * a.q.rows + at, (unsigned)min(rows, QT) * 4);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void)(size_t)(stats + slot * 512 + wave * 256), 4, lane * 4, 0, 0, 0);
            }
            it += QT;
            if (it >= count) { it = 0; ++ih; }
        };
        issue(0, 0);
        unsigned stage = 0;
        int t = 0;
        for (int n = 0; n < all; ++n, stage ^= BYTES, t = t + QT >= count ? 0 : t + QT) {
            wait_vmcnt<0>();
            __builtin_amdgcn_s_barrier();   // the tile has arrived, and the one before is done with
            const int slot = stage != 0;
            if (n + 1 < all) issue(stage ^ BYTES, slot ^ 1);
            if (t <= none0 || t >= none1) continue;
            const bool edge = t < all0 || t > all1;
#pragma unroll
            for (int nb = 0; nb < QT / 32; ++nb) {
                const unsigned qt = base + stage + nb * 32 * L::RB, gt = base + 2 * BYTES + stage + nb * 32 * L::RB, st = stats + slot * 512 + nb * 128 + half * 16;
                f32x16 s[1], dp[1];
                clear(s);
                clear(dp);
                u32x4 l2[4], de[4];   // of rows 8 g + 4 half ...
                l2[0] = lds_read16<0>(st); l2[1] = lds_read16<32>(st); l2[2] = lds_read16<64>(st); l2[3] = lds_read16<96>(st);
                de[0] = lds_read16<256>(st); de[1] = lds_read16<288>(st); de[2] = lds_read16<320>(st); de[3] = lds_read16<352>(st);
                First<T, DP, 1, 6> qk, gv;
                qk.begin(qt + tl.row, tl.x);
                qk.run(qt + tl.row, tl.x, kc, s);
#pragma unroll
                for (int e = 0; e < 4; ++e) { tie(l2[e]); tie(de[e]); }   // older than the reads that were waited for
                gv.begin(gt + tl.row, tl.x);
                gv.run(gt + tl.row, tl.x, vc, dp);
                Second<T, DP, 2> gp, qs;
                gp.begin(gt, tl);
                if (edge) {
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if ((unsigned)(t + 32 * nb + 8 * (v >> 2) + 4 * half + (v & 3) - seen0) >= seen) s[0][v] = -INFINITY;
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[0][v], a.scale2, -__uint_as_float(l2[v >> 2][v & 3])));
                    dp[0][v] = p * (dp[0][v] - __uint_as_float(de[v >> 2][v & 3]));
                    s[0][v] = p;
                }
                gp.run(gt, tl, [&](auto sc) { return column<T>(s[0], decltype(sc)::value); }, dv);
                qs.begin(qt, tl);
                qs.run(qt, tl, [&](auto sc) { return column<T>(dp[0], decltype(sc)::value); }, dk);
            }
        }
    }
    if (!own) return;
    if (!on) { clear(dk); clear(dv); }
    store_column<T, DB>(dk, a.scale, reinterpret_cast<T *>(a.dk) + row * a.k_stride + (long long)hk * a.dim, a.dim, half);
    store_column<T, DB>(dv, 1.f, reinterpret_cast<T *>(a.dv) + row * a.v_stride + (long long)hk * a.dim, a.dim, half);
}

template <typename T, int DP> void launch(AttnArgs &a, unsigned groups, hipStream_t st)
{
    const auto tiles = [](long long cols) { return (int)((cols + 127) / 128); };
    a.tiles = tiles((long long)a.q.len * a.shared);
    if (a.tiles > 0 && a.q.rows > 0) hipLaunchKernelGGL((k_attention_dq<T, DP>), dim3(groups * a.tiles), dim3(256), 0, st, a);
    a.tiles = tiles(a.kv.len);
    if (a.tiles > 0 && a.kv.rows > 0) hipLaunchKernelGGL((k_attention_dkv<T, DP>), dim3(groups * a.tiles), dim3(256), 0, st, a);
}
template <typename T> void launch(AttnArgs &a, unsigned groups, hipStream_t st)
{
    if (a.dim <= 32) launch<T, 32>(a, groups, st);
    else if (a.dim <= 64) launch<T, 64>(a, groups, st);
    else if (a.dim <= 96) launch<T, 96>(a, groups, st);
    else launch<T, 128>(a, groups, st);
}

size_t stat_bytes(const dp_attention_desc &d)
{
    const size_t rows = (size_t)(d.q_rows != 0 ? d.q_rows : (long long)d.n * d.q_len);
    return ((size_t)d.heads * rows * sizeof(float) + 15) / 16 * 16;
}

}  // namespace

size_t attn_bwd_bytes(const dp_attention_desc &d) { return 2 * stat_bytes(d); }

extern "C" dp_status dp_attention_bwd(const dp_attention_desc *desc, const void *q, const void *k, const void *v, const void *o, const void *dout,
                                      const float *lse, void *dq, void *dk, void *dv, const dp_attention_seqs *seqs, void *ws, size_t ws_bytes,
                                      void *hip_stream)
{
    dp_status s = attn_check(desc, seqs);
    if (s != DP_OK) return s;
    const dp_attention_desc &d = *desc;
    AttnArgs a;
    attn_args(d, seqs, a);
    const bool queries = d.n > 0 && d.q_len > 0 && a.q.rows > 0, keys = d.n > 0 && d.kv_len > 0 && a.kv.rows > 0;
    if (!queries && !keys) return DP_OK;
    if (queries && ((s = attn_pointers({q, o, dout, dq, lse}, nullptr, ws)) != DP_OK || (s = attn_workspace(attn_bwd_bytes(d), ws, ws_bytes)) != DP_OK)) return s;
    if (keys && (s = attn_pointers({k, v, dk, dv}, nullptr, nullptr)) != DP_OK) return s;
    a.qp = q; a.kp = k; a.vp = v; a.op_in = o; a.dout = dout; a.lse_in = lse;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.lse2 = (float *)ws;
    a.delta = (float *)((char *)ws + stat_bytes(d));
    const unsigned groups = (unsigned)((long long)d.n * d.kv_heads);
    if (d.io_dtype == DP_BF16) launch<bf16_t>(a, groups, (hipStream_t)hip_stream);
    else launch<float>(a, groups, (hipStream_t)hip_stream);
    return attn_launched("attention's gradient");
}
