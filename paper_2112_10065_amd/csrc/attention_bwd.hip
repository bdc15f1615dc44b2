// Attention, backward.  With p_ij = exp(s_ij - lse_i) recomputed from the forward call's lse, dp_ij = dout_i . v_j and delta_i = dout_i . o_i:
//   dv_j = sum_i p_ij dout_i;   ds_ij = p_ij (dp_ij - delta_i);   dq_i = scale sum_j ds_ij k_j;   dk_j = scale sum_i ds_ij q_i
// Two kernels, each with its sums in registers from the first to the last tile: one holds queries and lets keys pass (dq; it computes delta and leaves it for the other),
// one holds keys and lets the queries of all heads that share them pass (dk, dv).  p and dp are computed in both, seven products for the five that the formulas
// have, in return for sums without atomics in a fixed order and without partial sums in memory (dq's would be 32 bits per query and block of keys).
#include "attention_common.h"
#include <algorithm>

namespace {

// Wavefronts of a block: CW of them side by side in columns, 4 / CW share the rows of each tile among them.
template <typename T, int DP, int CW> struct Shape {
    static constexpr int RW = 4 / CW, NB = sizeof(T) == 2 && CW == 4 ? 2 : 1, RT = RW * NB * 32, BYTES = RT * Tile<T, DP>::RB;   // NB: blocks of 32 rows of a wavefront
    static constexpr int STAGES = 4 * BYTES <= 131072 ? 2 : 1;
};

template <typename T, int DP, int CW> __global__ __launch_bounds__(256, CW == 4 && (sizeof(T) == 2 || DP <= 64) ? 2 : 1) void k_attention_dq(AttnArgs a)
{
    using L = Tile<T, DP>;
    using S = Shape<T, DP, CW>;
    constexpr int RW = S::RW, NB = S::NB, KT = S::RT, DB = L::DB, BYTES = S::BYTES, STAGES = S::STAGES, COLS = CW * 32;
    constexpr int ROOM = 2 * STAGES * BYTES > (RW > 1 ? 4 * DB * 4096 : 0) ? 2 * STAGES * BYTES : 4 * DB * 4096;
    __shared__ alignas(1024) char s_tiles[ROOM];   // K and V of each stage
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, wc = wave % CW, wr = wave / CW;
    const int id = logical_block(blockIdx.x, gridDim.x);
    const int hb = id / a.tiles, b = hb % a.n, hk = hb / a.n;
    const int col0 = (a.tiles - 1 - id % a.tiles) * COLS;
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rq.own * a.shared) return;
    const int wcol = col0 + wc * 32, col = wcol + (lane & 31), i = col / a.shared, head = hk * a.shared + col % a.shared;
    const bool own = i < rq.own, on = i < rq.used;
    const int ahead = rk.used - rq.used, last = rq.used * a.shared - 1;
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
        if (on && half == 0 && wr == 0) { a.lse2[stat] = lse2; a.delta[stat] = delta; }
    }
    const int mine = wr * NB * 32;
    const long long see0 = max((long long)i + ahead - a.left - first, 0ll), see1 = min((long long)i + ahead + a.right + 1 - first, (long long)keys);
    const int seen0 = (int)min(see0, (long long)kFar);
    const unsigned seen = on ? (unsigned)max(see1 - seen0, 0ll) : 0u;
    // keys t ... t + 31 are seen by all of the wavefront's queries if all0 <= t <= all1, by none if t <= none0 or t >= none1
    const int all0 = (int)min(max(w1 + ahead - a.left - first, 0ll), (long long)kFar), all1 = (int)max(min(w0 + ahead + a.right + 1 - first, (long long)keys) - 32, -1ll);
    const int none0 = (int)(min(max(w0 + ahead - a.left - first, 0ll), (long long)kFar) - 32), none1 = (int)min(min(w1 + ahead + a.right + 1 - first, (long long)keys), (long long)kFar);

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
        cv.issue(vp, keys, a.dim, a.v_stride, base + STAGES * BYTES, wave);
        unsigned stage = 0;
        for (int t = 0; t < keys; t += KT) {
            wait_vmcnt<0>();
            __builtin_amdgcn_s_barrier();   // the tile has arrived, and the one before is done with
            const unsigned at = base + stage;
            const auto next = [&] {
                if (t + KT >= keys) return;
                if (STAGES == 2) stage ^= BYTES;
                kp += KT * a.k_stride;
                vp += KT * a.v_stride;
                ck.issue(kp, keys - t - KT, a.dim, a.k_stride, base + stage, wave);
                cv.issue(vp, keys - t - KT, a.dim, a.v_stride, base + STAGES * BYTES + stage, wave);
            };
            if constexpr (STAGES == 2) next();
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int w = t + mine + 32 * nb;
                if (w <= none0 || w >= none1) continue;
                const unsigned kt = at + (mine + nb * 32) * L::RB, vt = kt + STAGES * BYTES;
                f32x16 s[1], dp[1];
                clear(s);
                clear(dp);
                TwoFirst<T, DP, 8> kv;
                kv.begin(kt + tl.row, vt + tl.row, tl.x);
                kv.run(kt + tl.row, vt + tl.row, tl.x, q, g, s[0], dp[0], [](auto) {});
                Second<T, DP, 2> ks;
                ks.begin(kt, tl);
                if (w < all0 || w > all1) {
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if ((unsigned)(w + 8 * (v >> 2) + 4 * half + (v & 3) - seen0) >= seen) s[0][v] = -INFINITY;
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) s[0][v] = __builtin_amdgcn_exp2f(fmaf(s[0][v], a.scale2, -lse2)) * (dp[0][v] - delta);
                ks.run(kt, tl, [&](auto sc) { return column<T>(s[0], decltype(sc)::value); }, acc);
            }
            if constexpr (STAGES == 1) {
                __builtin_amdgcn_s_barrier();
                next();
            }
        }
    }
    if constexpr (RW > 1) {
        __syncthreads();
        sum_waves<4>(acc, reinterpret_cast<float *>(s_tiles), wave, lane);
    }
    if (!own) return;
    const bool some = on && lse2 != INFINITY;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        if (RW > 1 && db != wr) continue;
        if (!some) {
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
        }
        store_block<T>(acc[db], a.scale, reinterpret_cast<T *>(a.dq) + row * a.q_stride + (long long)head * a.dim, db * 32, a.dim, half);
    }
}

// dk and dv.  PIPE: one wavefront on each SIMD (its sums and operands take most of the registers), so nothing else runs while it exponentiates: the
// products of the next 32 queries are put between the exponentials of these.
template <typename T, int DP, int CW> constexpr bool kPipe = sizeof(T) == 2 && CW == 4 && DP > 64;
template <typename T, int DP, int CW> struct KvShape : Shape<T, DP, CW> {};
template <int DP> struct KvShape<bf16_t, DP, 4> {
    static constexpr bool P = kPipe<bf16_t, DP, 4>;
    static constexpr int RW = 1, NB = P ? 1 : 2, RT = NB * 32, BYTES = RT * Tile<bf16_t, DP>::RB, STAGES = P ? 4 : 2;
};

template <typename T, int DP, int CW> __global__ __launch_bounds__(256, sizeof(T) == 2 && CW == 4 && DP <= 64 ? 2 : 1) void k_attention_dkv(AttnArgs a)
{
    using L = Tile<T, DP>;
    using S = KvShape<T, DP, CW>;
    constexpr bool PIPE = kPipe<T, DP, CW>;
    constexpr int RW = S::RW, NB = S::NB, QT = S::RT, DB = L::DB, BYTES = S::BYTES, STAGES = S::STAGES, COLS = CW * 32;
    constexpr int ROOM = 2 * STAGES * BYTES > (RW > 1 ? 4 * DB * 4096 : 0) ? 2 * STAGES * BYTES : 4 * DB * 4096;
    __shared__ alignas(1024) char s_tiles[ROOM];                  // q and dout of each stage
    __shared__ alignas(16) float s_stats[STAGES][2][QT < 64 ? 64 : QT];   // lse2 and delta
    constexpr unsigned STATS = sizeof(s_stats[0]), SIDE = STATS / 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, wc = wave % CW, wr = wave / CW;
    const int id = logical_block(blockIdx.x, gridDim.x);
    const int hb = id / a.tiles, b = hb % a.n, hk = hb / a.n;
    const int col0 = (id % a.tiles) * COLS;             // causal: the longest first
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rk.own) return;
    const int wcol = col0 + wc * 32, j = wcol + (lane & 31);
    const bool own = j < rk.own, on = j < rk.used;
    const long long ahead = rk.used - rq.used;
    // the queries that see the block's keys, and the wavefront's
    const int last = rk.used - 1;
    long long lo = 0, hi = 0;
    const long long j1 = min(col0 + COLS - 1, last), w0 = wcol, w1 = min(wcol + 31, last);
    if (col0 <= last) {
        lo = max(0ll, col0 - a.right - ahead);
        hi = min((long long)rq.used, j1 + a.left - ahead + 1);
    }
    const int first = (int)min(lo, (long long)kFar), count = (int)max(0ll, hi - lo);
    const long long row = rk.first + j;
    const int mine = wr * NB * 32;
    const long long see0 = max(j - a.right - ahead - first, 0ll), see1 = min(j + a.left - ahead + 1 - first, (long long)count);
    const int seen0 = (int)min(see0, (long long)kFar);
    const unsigned seen = on ? (unsigned)max(see1 - seen0, 0ll) : 0u;
    // queries t ... t + 31 see all of the wavefront's keys if all0 <= t <= all1 (those behind the last one add zeros), none of them if t <= none0 or t >= none1
    const int all0 = (int)min(max(w1 - a.right - ahead - first, 0ll), (long long)kFar), all1 = (int)max(min(w0 + a.left - ahead + 1 - first, (long long)kFar) - 32, -1ll);
    const int none0 = (int)(min(max(w0 - a.right - ahead - first, 0ll), (long long)kFar) - 32), none1 = (int)min(min(w1 + a.left - ahead + 1 - first, (long long)count), (long long)kFar);

    f32x16 sum[2 * DB];   // dk, then dv
    clear(sum);
    f32x16(&dk)[DB] = *reinterpret_cast<f32x16(*)[DB]>(&sum[0]);
    f32x16(&dv)[DB] = *reinterpret_cast<f32x16(*)[DB]>(&sum[DB]);
    if (count > 0) {
        u32x4 kc[L::SLICES], vc[L::SLICES];
        load_column<T, DP>(reinterpret_cast<const T *>(a.kp) + row * a.k_stride + (long long)hk * a.dim, on, a.dim, half, kc);
        load_column<T, DP>(reinterpret_cast<const T *>(a.vp) + row * a.v_stride + (long long)hk * a.dim, on, a.dim, half, vc);
        using Copy = TileCopy<T, DP, QT, 256>;
        Copy cq, cg;
        cq.init(threadIdx.x, a.dim, a.q_stride);
        cg.init(threadIdx.x, a.dim, a.o_stride);
        const unsigned base = lds_offset(s_tiles), stats = lds_offset(s_stats);
        TileLane<T, DP> tl;
        tl.init(lane);
        const int tiles = (count + QT - 1) / QT, all = tiles * a.shared;
        // tile n: queries first + (n % tiles) QT ... of the n / tiles-th head; rows behind the last query arrive as zeros, also their statistics: nothing is added then
        int ih = hk * a.shared, it = 0, slot_in = 0;
        constexpr int STAT_COPIES = QT > 64 ? QT / 64 : 1;
        auto issue = [&] {
            const long long at = rq.first + first + it;
            const int rows = count - it;
            cq.issue(reinterpret_cast<const T *>(a.qp) + at * a.q_stride + (long long)ih * a.dim, rows, a.dim, a.q_stride, base + slot_in * BYTES, wave);
            cg.issue(reinterpret_cast<const T *>(a.dout) + at * a.o_stride + (long long)ih * a.dim, rows, a.dim, a.o_stride, base + (STAGES + slot_in) * BYTES, wave);
            // wavefronts 0 and 2 copy the same, 1 and 3 too: each has as many copies under way as the others
            const auto r = make_rsrc(((wave & 1) == 0 ? a.lse2 : a.delta) + (long long)ih * a.q.rows + at, (unsigned)min(rows, QT) * 4);
#pragma unroll
            for (int c = 0; c < STAT_COPIES; ++c)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void)(size_t)(stats + slot_in * STATS + (wave & 1) * SIDE + c * 256), 4, (c * 64 + lane) * 4, 0, 0, 0);
            slot_in = slot_in + 1 == STAGES ? 0 : slot_in + 1;
            it += QT;
            if (it >= count) { it = 0; ++ih; }
        };
        u32x4 l2[4], de[4];   // statistics of rows 8 g + 4 half ...
        const auto read_stats = [&](unsigned st) {
            l2[0] = lds_read16<0>(st); l2[1] = lds_read16<32>(st); l2[2] = lds_read16<64>(st); l2[3] = lds_read16<96>(st);
            de[0] = lds_read16<SIDE>(st); de[1] = lds_read16<SIDE + 32>(st); de[2] = lds_read16<SIDE + 64>(st); de[3] = lds_read16<SIDE + 96>(st);
        };
        const auto stats_there = [&] {
#pragma unroll
            for (int e = 0; e < 4; ++e) { tie(l2[e]); tie(de[e]); }
        };
        const auto hide = [&](f32x16 &s, int w) {
            if (w >= all0 && w <= all1) return;
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if ((unsigned)(w + 8 * (v >> 2) + 4 * half + (v & 3) - seen0) >= seen) s[v] = -INFINITY;
        };
        const auto soften = [&](f32x16 &s, f32x16 &dp, int v) {   // s -> p, dp -> ds
            const float p = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale2, -__uint_as_float(l2[v >> 2][v & 3])));
            dp[v] = p * (dp[v] - __uint_as_float(de[v >> 2][v & 3]));
            s[v] = p;
        };
        if constexpr (PIPE) {
            constexpr int COPIES = 2 * Copy::N + 1;
            issue();
            if (all > 1) issue();
            if (all > 2) issue();
            if (all > 2) wait_vmcnt<2 * COPIES>();
            else if (all > 1) wait_vmcnt<COPIES>();
            else wait_vmcnt<0>();
            __builtin_amdgcn_s_barrier();
            f32x16 s[2], dp[2];
            clear(s);
            clear(dp);
            TwoFirst<T, DP, 6> ab;
            read_stats(stats + half * 16);
            ab.begin(base + tl.row, base + STAGES * BYTES + tl.row, tl.x);
            ab.run(base + tl.row, base + STAGES * BYTES + tl.row, tl.x, kc, vc, s[0], dp[0], [](auto) {});
            stats_there();
            int slot = 0, t = 0;
            hide(s[0], 0);
            const auto step = [&](int n, f32x16 &sc, f32x16 &dc, f32x16 &sn, f32x16 &dn) {
                const unsigned qt = base + slot * BYTES, gt = qt + STAGES * BYTES;
                u32x4 p[2], ds[2];
                if (n + 1 < all) {
                    // the next tile has arrived, and the one before this is done with: its room takes the third from here
                    if (n + 2 < all) wait_vmcnt<COPIES>();
                    else wait_vmcnt<0>();
                    __builtin_amdgcn_s_barrier();
                    if (n + 3 < all) issue();
                    slot = slot + 1 == STAGES ? 0 : slot + 1;
                    t = t + QT >= count ? 0 : t + QT;
                    const unsigned qn = base + slot * BYTES + tl.row, gn = qn + STAGES * BYTES;
#pragma unroll
                    for (int v = 0; v < 16; ++v) sn[v] = dn[v] = 0.f;
                    ab.begin(qn, gn, tl.x);
                    ab.run(qn, gn, tl.x, kc, vc, sn, dn, [&](auto ic) {
                        constexpr int i = decltype(ic)::value, N = 2 * L::SLICES;
#pragma unroll
                        for (int v = i * 16 / N; v < (i + 1) * 16 / N; ++v) soften(sc, dc, v);
                    });
                    hide(sn, t);
#pragma unroll
                    for (int h = 0; h < 2; ++h) { p[h] = column<T>(sc, h); ds[h] = column<T>(dc, h); }
                    read_stats(stats + slot * STATS + half * 16);
                } else {
#pragma unroll
                    for (int v = 0; v < 16; ++v) soften(sc, dc, v);
#pragma unroll
                    for (int h = 0; h < 2; ++h) { p[h] = column<T>(sc, h); ds[h] = column<T>(dc, h); }
                }
                Second<T, DP, 2> gp, qs;
                gp.begin(gt, tl);
                gp.run(gt, tl, [&](auto sl) { return p[decltype(sl)::value]; }, dv);
                qs.begin(qt, tl);
                qs.run(qt, tl, [&](auto sl) { return ds[decltype(sl)::value]; }, dk);
                stats_there();   // older than the reads that were waited for
            };
            for (int n = 0; n < all; ++n) {
                step(n, s[0], dp[0], s[1], dp[1]);
                s[0] = s[1];
                dp[0] = dp[1];
            }
        } else {
            issue();
            int slot = 0, t = 0;
            for (int n = 0; n < all; ++n) {
                wait_vmcnt<0>();
                __builtin_amdgcn_s_barrier();   // the tile has arrived, and the one before is done with
                if (STAGES == 2 && n + 1 < all) issue();
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const int w = t + mine + 32 * nb;
                    if (w <= none0 || w >= none1) continue;
                    const unsigned at = (mine + nb * 32) * L::RB, qt = base + slot * BYTES + at, gt = base + (STAGES + slot) * BYTES + at;
                    f32x16 s[1], dp[1];
                    clear(s);
                    clear(dp);
                    read_stats(stats + slot * STATS + (mine + nb * 32) * 4 + half * 16);
                    TwoFirst<T, DP, 6> ab;
                    ab.begin(qt + tl.row, gt + tl.row, tl.x);
                    ab.run(qt + tl.row, gt + tl.row, tl.x, kc, vc, s[0], dp[0], [](auto) {});
                    stats_there();   // older than the reads that were waited for
                    Second<T, DP, 2> gp, qs;
                    gp.begin(gt, tl);
                    hide(s[0], w);
#pragma unroll
                    for (int v = 0; v < 16; ++v) soften(s[0], dp[0], v);
                    gp.run(gt, tl, [&](auto sc) { return column<T>(s[0], decltype(sc)::value); }, dv);
                    qs.begin(qt, tl);
                    qs.run(qt, tl, [&](auto sc) { return column<T>(dp[0], decltype(sc)::value); }, dk);
                }
                if (STAGES == 1 && n + 1 < all) {
                    __builtin_amdgcn_s_barrier();
                    issue();
                }
                if (STAGES == 2) slot ^= 1;
                t = t + QT >= count ? 0 : t + QT;
            }
        }
    }
    if constexpr (RW > 1) {   // one after the other: the room of dk's sums takes dv's
        __syncthreads();
        sum_waves<4>(dk, reinterpret_cast<float *>(s_tiles), wave, lane);
        __syncthreads();
        sum_waves<4>(dv, reinterpret_cast<float *>(s_tiles), wave, lane);
    }
    if (!own) return;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        if (RW > 1 && db != wr) continue;
        if (!on) {
#pragma unroll
            for (int v = 0; v < 16; ++v) dk[db][v] = dv[db][v] = 0.f;
        }
        store_block<T>(dk[db], a.scale, reinterpret_cast<T *>(a.dk) + row * a.k_stride + (long long)hk * a.dim, db * 32, a.dim, half);
        store_block<T>(dv[db], 1.f, reinterpret_cast<T *>(a.dv) + row * a.v_stride + (long long)hk * a.dim, db * 32, a.dim, half);
    }
}

// Four wavefronts side by side where such blocks fill the card; else they take the same 32 columns and share the rows of the other side.
template <typename T> void launch(AttnArgs &a, long long groups, hipStream_t st)
{
    for_dim(a.dim, [&](auto dc) {
        constexpr int DP = decltype(dc)::value;
        const auto wide = [&](long long cols) { return cols > 32 && groups * ((cols + 127) / 128) >= 256; };
        const long long qc = (long long)a.q.len * a.shared, kc = a.kv.len;
        const bool wq = wide(qc), wk = wide(kc);
        a.tiles = (int)((qc + (wq ? 127 : 31)) / (wq ? 128 : 32));
        if (a.tiles > 0 && a.q.rows > 0) hipLaunchKernelGGL((wq ? k_attention_dq<T, DP, 4> : k_attention_dq<T, DP, 1>), dim3((unsigned)(groups * a.tiles)), dim3(256), 0, st, a);
        a.tiles = (int)((kc + (wk ? 127 : 31)) / (wk ? 128 : 32));
        if (a.tiles > 0 && a.kv.rows > 0) hipLaunchKernelGGL((wk ? k_attention_dkv<T, DP, 4> : k_attention_dkv<T, DP, 1>), dim3((unsigned)(groups * a.tiles)), dim3(256), 0, st, a);
    });
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
    const long long groups = (long long)d.n * d.kv_heads;
    if (d.io_dtype == DP_BF16) launch<bf16_t>(a, groups, (hipStream_t)hip_stream);
    else launch<float>(a, groups, (hipStream_t)hip_stream);
    return attn_launched("attention's gradient");
}
