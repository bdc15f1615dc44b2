// Attention, backward.  With p_ij = exp(s_ij - lse_i) recomputed from the forward call's lse, dp_ij = dout_i . v_j and delta_i = dout_i . o_i:
//   dv_j = sum_i p_ij dout_i;   ds_ij = p_ij (dp_ij - delta_i);   dq_i = scale sum_j ds_ij k_j;   dk_j = scale sum_i ds_ij q_i
// Two kernels, each with its sums in registers from the first to the last tile: one holds queries and lets keys pass (dq; it computes delta and leaves it for the other),
// one holds keys and lets the queries of all heads that share them pass (dk, dv).  p and dp are computed in both, seven products for the five that the formulas
// have, in return for sums without atomics in a fixed order and without partial sums in memory (dq's would be 32 bits per query and block of keys: 2 GB written and read for two
// sequences of 4096 causal tokens, 0.8 ms, where the two products take 0.25).
// With bf16, p and ds are rounded as operands of the second products; p, dp and delta themselves stay in 32 bits.
//
// Bound by the matrix cores: two sequences of 4096 causal tokens, 32 heads of 128 over 8: dq 385-403 us (1.02-1.07 PFLOP/s of the products that it computes), dk and dv 543-590 (0.93-1.01).
// Short sequences wait: 32 x 197 tokens, 12 heads of 64, 20 + 26 us for four tiles a block in one round and one and a half.
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
    const Item item = item_of<COLS, false, true, CW == 4 && sizeof(T) == 2 ? 2 : 1>(a, a.q, a.shared, blockIdx.x, gridDim.x);
    if (!item.any) return;
    const int b = item.b, hk = item.hk, col0 = item.tile * COLS;
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rq.own * a.shared) return;
    const int wcol = col0 + wc * 32, col = wcol + (lane & 31), i = col / a.shared, head = hk * a.shared + col % a.shared;
    const bool own = i < rq.own, on = i < rq.used;
    const int ahead = rk.used - rq.used, last = rq.used * a.shared - 1;
    int lo = 0, hi = 0;   // lengths are at most 2^28 and bounds 2^30: no sum here passes 31 bits
    const int i0 = col0 / a.shared, i1 = min(col0 + COLS - 1, last) / a.shared, w0 = wcol / a.shared, w1 = min(wcol + 31, last) / a.shared;
    if (col0 <= last) {
        lo = max(0, i0 + ahead - a.left);
        hi = min(rk.used, i1 + ahead + a.right + 1);
    }
    const int first = lo, keys = max(0, hi - lo);
    const long long row = rq.first + i, stat = (long long)head * a.q.rows + row;

    TileCopy<T, DP, KT, 256> ck, cv;
    ck.init(threadIdx.x, a.dim, a.k_stride);
    cv.init(threadIdx.x, a.dim, a.v_stride);
    const T *kp = reinterpret_cast<const T *>(a.kp) + (rk.first + first) * a.k_stride + (long long)hk * a.dim;
    const T *vp = reinterpret_cast<const T *>(a.vp) + (rk.first + first) * a.v_stride + (long long)hk * a.dim;
    const unsigned base = lds_offset(s_tiles);
    TileLane<T, DP> tl;
    tl.init(lane);
    if (keys > 0) {   // under way while the queries' rows are loaded
        ck.issue(kp, keys, a.dim, a.k_stride, base, wave);
        cv.issue(vp, keys, a.dim, a.v_stride, base + STAGES * BYTES, wave);
    }
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
        if (on && half == 0 && wr == 0) { a.lse2[stat] = lse2; a.delta[stat] = -delta; }
    }
    const int mine = wr * NB * 32;
    const int seen0 = max(i + ahead - a.left - first, 0);
    const unsigned seen = on ? (unsigned)max(min(i + ahead + a.right + 1 - first, keys) - seen0, 0) : 0u;
    // keys t ... t + 31 are seen by all of the wavefront's queries if all0 <= t <= all1, by none if t <= none0 or t >= none1
    const int all0 = max(w1 + ahead - a.left - first, 0), all1 = max(min(w0 + ahead + a.right + 1 - first, keys) - 32, -1);
    const int none0 = max(w0 + ahead - a.left - first, 0) - 32, none1 = min(w1 + ahead + a.right + 1 - first, keys);

    f32x16 acc[DB];
    clear(acc);
    if (keys > 0) {
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
                kv.run(kt + tl.row, vt + tl.row, tl.x, q, g, s[0], dp[0]);
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

// The rows (queries) that a block of keys, from col0 on, is seen by, and the wavefront's part of them.
struct Seen { int first, count, seen0, all0, all1, none0, none1; unsigned seen; };
template <int COLS> DEVFN Seen seen_by(const AttnArgs &a, const Rows &rq, const Rows &rk, int col0, int wcol, int j)
{
    const int ahead = rk.used - rq.used, w0 = wcol, last = rk.used - 1, j1 = min(col0 + COLS - 1, last), w1 = min(w0 + 31, last);
    int lo = 0, hi = 0;   // lengths are at most 2^28 and bounds 2^30: no sum here passes 31 bits
    if (col0 <= last) {
        lo = max(0, col0 - a.right - ahead);
        hi = min(rq.used, j1 + a.left - ahead + 1);
    }
    Seen s;
    s.first = lo;
    s.count = max(0, hi - lo);
    s.seen0 = max(j - a.right - ahead - s.first, 0);
    s.seen = j < rk.used ? (unsigned)max(min(j + a.left - ahead + 1 - s.first, s.count) - s.seen0, 0) : 0u;
    // queries t ... t + 31 see all of the wavefront's keys if all0 <= t <= all1 (those behind the last one add zeros), none of them if t <= none0 or t >= none1
    s.all0 = max(w1 - a.right - ahead - s.first, 0);
    s.all1 = max(w0 + a.left - ahead + 1 - s.first - 32, -1);
    s.none0 = max(w0 - a.right - ahead - s.first, 0) - 32;
    s.none1 = min(w1 + a.left - ahead + 1 - s.first, s.count);
    return s;
}
DEVFN void hide(f32x16 &s, const Seen &w, int t, int half)
{
    if (t >= w.all0 && t <= w.all1) return;
#pragma unroll
    for (int v = 0; v < 16; ++v)
        if ((unsigned)(t + 8 * (v >> 2) + 4 * half + (v & 3) - w.seen0) >= w.seen) s[v] = -INFINITY;
}

// With SPLIT: where part `part` of `parts` of `total` tiles begins.
template <bool SPLIT> DEVFN int part_of(int total, int part, int parts) { return SPLIT ? (int)((long long)total * part / parts) : 0; }

// dk and dv for 128 keys of wide heads.  Both sums and the operands k and v take more registers than each of two wavefronts on a SIMD has, and one alone has nothing to run
// beside its exponentials; so two share 32 keys.  Of each tile of 64 queries each makes p and ds for its half of the queries, and then one adds up dk, the other dv, over all of
// them: what the other wavefront's half needs of p or ds goes through LDS, already rounded, lane by lane.  The sums are one tile behind the products, so that
// a wavefront's exponentials lie between matrix products that do not wait for them.
template <int DP, bool SPLIT> __global__ __launch_bounds__(512, 2) void k_attention_dkv(AttnArgs a)
{
    using T = bf16_t;
    using L = Tile<T, DP>;
    constexpr int QT = 64, DB = L::DB, BYTES = QT * L::RB, STAGES = 3, COLS = 128;
    using Copy = TileCopy<T, DP, QT, 256>;
    __shared__ alignas(1024) char s_tiles[2 * STAGES * BYTES];   // q and dout of each stage
    __shared__ alignas(16) float s_stats[STAGES][2][QT];         // lse2 and -delta
    __shared__ alignas(16) u32x4 s_packs[2][8][2][64];           // [tile][wavefront][slice][lane]: the first's p, the second's ds
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, pair = wave & 3, second = wave >> 2;
    const int blocks = SPLIT ? gridDim.x / a.kv_parts : gridDim.x, part = SPLIT ? blockIdx.x / blocks : 0;
    const Item item = item_of<COLS, false, false>(a, a.kv, 1, SPLIT ? blockIdx.x % blocks : blockIdx.x, blocks);
    if (!item.any) return;
    const int b = item.b, hk = item.hk, col0 = item.tile * COLS;
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rk.own) return;
    const int wcol = col0 + pair * 32, j = wcol + (lane & 31);
    const bool own = j < rk.own, on = j < rk.used;
    const Seen w = seen_by<COLS>(a, rq, rk, col0, wcol, j);
    const long long row = rk.first + j;

    f32x16 sum[DB];   // the first's dk, the second's dv
    clear(sum);
    // a part may have nothing to add up
    if (w.count > 0 && (!SPLIT || part_of<SPLIT>((w.count + QT - 1) / QT * a.shared, part + 1, a.kv_parts) > part_of<SPLIT>((w.count + QT - 1) / QT * a.shared, part, a.kv_parts))) {
        const unsigned tiles_q = lds_offset(s_tiles), tiles_g = tiles_q + STAGES * BYTES, stats = lds_offset(s_stats), packs = lds_offset(s_packs) + lane * 16;
        const long long stride = second ? a.o_stride : a.q_stride;
        const T *source = reinterpret_cast<const T *>(second ? a.dout : a.qp);
        const float *stat_from = second ? a.delta : a.lse2;
        Copy copy;
        copy.init(threadIdx.x & 255, a.dim, stride);
        TileLane<T, DP> tl;
        tl.init(lane);
        // tiles of all heads, one head's behind the other's; with SPLIT a part of them
        const int tiles = (w.count + QT - 1) / QT, total = tiles * a.shared, from = part_of<SPLIT>(total, part, a.kv_parts), all = SPLIT ? part_of<SPLIT>(total, part + 1, a.kv_parts) - from : total;
        // tile n: queries first + QT (n % tiles) ... of the n / tiles-th head, n from `from` on; rows behind the last query arrive as zeros, also their statistics: nothing is added then.
        // The first wavefronts copy q and lse2, the second dout and -delta.
        int ih = hk * a.shared + from / tiles, it = from % tiles * QT, slot_in = 0;
        auto issue = [&] {
            const long long at = rq.first + w.first + it;
            const int rows = w.count - it;
            copy.issue(source + at * stride + (long long)ih * a.dim, rows, a.dim, stride, (second ? tiles_g : tiles_q) + slot_in * BYTES, pair);
            if (pair == 0) {
                const auto r = make_rsrc(stat_from + (long long)ih * a.q.rows + at, (unsigned)min(rows, QT) * 4);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void)(size_t)(stats + (slot_in * 2 + second) * QT * 4), 4, lane * 4, 0, 0, 0);
            }
            slot_in = slot_in + 1 == STAGES ? 0 : slot_in + 1;
            it += QT;
            if (it >= w.count) { it = 0; ++ih; }
        };
        issue();
        u32x4 kc[L::SLICES], vc[L::SLICES];
        load_column<T, DP>(reinterpret_cast<const T *>(a.kp) + row * a.k_stride + (long long)hk * a.dim, on, a.dim, half, kc);
        load_column<T, DP>(reinterpret_cast<const T *>(a.vp) + row * a.v_stride + (long long)hk * a.dim, on, a.dim, half, vc);
        u32x4 mine[2];   // ds (the first's) or p (the second's) of the own half of the tile before
        int t = from % tiles * QT, slot = 0, before = 0;
        f32x16 s, dp;
        u32x4 l2[4];     // of rows 8 g + 4 half ... of the own half
        const auto arrive = [&](int n) {   // tile n, and the packs of tile n - 1; tile n - 2 is done with: its room takes tile n + 1
            wait_vmcnt<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            if (n + 1 < all) issue();
        };
        const auto products = [&] {
            const unsigned qt = tiles_q + slot * BYTES + second * 32 * L::RB + tl.row, gt = qt + STAGES * BYTES, st = stats + slot * 2 * QT * 4 + second * 128 + half * 16;
            u32x4 de[4];
            de[0] = lds_read16<QT * 4>(st); de[1] = lds_read16<QT * 4 + 32>(st); de[2] = lds_read16<QT * 4 + 64>(st); de[3] = lds_read16<QT * 4 + 96>(st);
            l2[0] = lds_read16<0>(st); l2[1] = lds_read16<32>(st); l2[2] = lds_read16<64>(st); l2[3] = lds_read16<96>(st);
            TwoFirst<T, DP, 6> ab;
            ab.begin(qt, gt, tl.x);
            wait_reads<1, 6>();
#pragma unroll
            for (int e = 0; e < 4; ++e) { tie(de[e]); tie(l2[e]); }
#pragma unroll
            for (int v = 0; v < 16; ++v) { s[v] = 0.f; dp[v] = __uint_as_float(de[v >> 2][v & 3]); }   // dp - delta: the sum begins at -delta
            ab.run(qt, gt, tl.x, kc, vc, s, dp);
            hide(s, w, t + 32 * second, half);
        };
        const auto soften = [&](int v) {   // s -> p, dp -> ds
            s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale2, -__uint_as_float(l2[v >> 2][v & 3])));
            dp[v] *= s[v];
        };
        const auto pack = [&](int n) {
            const unsigned pk = packs + (n & 1) * sizeof(s_packs[0]) + wave * sizeof(s_packs[0][0]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 p = column<T>(s, h), ds = column<T>(dp, h);
                mine[h] = second ? p : ds;
                lds_write16(pk + h * 1024, second ? ds : p);
            }
            before = slot;
            slot = slot + 1 == STAGES ? 0 : slot + 1;
            t = t + QT >= w.count ? 0 : t + QT;
        };
        // the sums of tile n: the own half of its queries, then the other's; beside(i), i = 0 ... 4 DB - 1
        const auto add = [&](int n, auto &&beside) {
            const unsigned yt = (second ? tiles_g : tiles_q) + before * BYTES, pk = packs + (n & 1) * sizeof(s_packs[0]) + (wave ^ 4) * sizeof(s_packs[0][0]);
            u32x4 other[2];
            other[0] = lds_read16<0>(pk);
            other[1] = lds_read16<1024>(pk);
            const unsigned at = yt + second * 32 * L::RB, back = yt + (second ^ 1) * 32 * L::RB;
            Second<T, DP, 2> x, y;
            x.begin(at, tl);
            wait_reads<1, decltype(x)::READS>();
            tie(other[0]);
            tie(other[1]);
            x.run_beside(at, tl, [&](auto sl) { return mine[decltype(sl)::value]; }, sum, [&](auto i) { beside(std::integral_constant<int, decltype(i)::value>{}); });
            y.begin(back, tl);
            y.run_beside(back, tl, [&](auto sl) { return other[decltype(sl)::value]; }, sum, [&](auto i) { beside(std::integral_constant<int, decltype(i)::value + 2 * DB>{}); });
        };
        arrive(0);
        products();
#pragma unroll
        for (int v = 0; v < 16; ++v) soften(v);
        pack(0);
        for (int n = 1; n < all; ++n) {
            arrive(n);
            products();
            add(n - 1, [&](auto ic) {
                constexpr int i = decltype(ic)::value, N = 4 * DB;
#pragma unroll
                for (int v = i * 16 / N; v < (i + 1) * 16 / N; ++v) soften(v);
            });
            pack(n);
        }
        arrive(all);
        add(all - 1, [](auto) {});
    }
    if (!own) return;
    if (!on) clear(sum);
    if constexpr (SPLIT) {
        store_column<float, DB>(sum, second ? 1.f : a.scale, (second ? a.part_dv : a.part_dk) + ((part * a.kv.rows + row) * a.kv_heads + hk) * a.dim, a.dim, half);
    } else if (second) store_column<T, DB>(sum, 1.f, reinterpret_cast<T *>(a.dv) + row * a.v_stride + (long long)hk * a.dim, a.dim, half);
    else store_column<T, DB>(sum, a.scale, reinterpret_cast<T *>(a.dk) + row * a.k_stride + (long long)hk * a.dim, a.dim, half);
}

// dk and dv with both sums in one wavefront: for 32 keys, where there are few (four wavefronts share each tile of queries), and for 128 of narrow heads, whose sums leave room, or
// in fp32, where the matrix products take sixteen times as long as with bf16 and hide the rest.
template <typename T, int DP, int CW, bool SPLIT> __global__ __launch_bounds__(256, CW == 4 && sizeof(T) == 2 ? 2 : 1) void k_attention_dkv_whole(AttnArgs a)
{
    using L = Tile<T, DP>;
    using S = Shape<T, DP, CW>;
    constexpr int RW = S::RW, NB = S::NB, QT = S::RT, DB = L::DB, BYTES = S::BYTES, STAGES = S::STAGES, COLS = CW * 32;
    constexpr int ROOM = 2 * STAGES * BYTES > (RW > 1 ? 4 * DB * 4096 : 0) ? 2 * STAGES * BYTES : 4 * DB * 4096, SIDE = QT < 64 ? 64 : QT;
    __shared__ alignas(1024) char s_tiles[ROOM];              // q and dout of each stage
    __shared__ alignas(16) float s_stats[STAGES][2][SIDE];    // lse2 and delta
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int blocks = SPLIT ? gridDim.x / a.kv_parts : gridDim.x, part = SPLIT ? blockIdx.x / blocks : 0;
    const Item item = item_of<COLS, false, false>(a, a.kv, 1, SPLIT ? blockIdx.x % blocks : blockIdx.x, blocks);
    if (!item.any) return;
    const int b = item.b, hk = item.hk, col0 = item.tile * COLS, wcol = col0 + wave % CW * 32, wr = wave / CW;
    const Rows rq = rows_of(a.q, b), rk = rows_of(a.kv, b);
    if (col0 >= rk.own) return;
    const int j = wcol + (lane & 31);
    const bool own = j < rk.own, on = j < rk.used;
    const Seen w = seen_by<COLS>(a, rq, rk, col0, wcol, j);
    const long long row = rk.first + j;
    const int mine = wr * NB * 32;

    f32x16 dk[DB], dv[DB];
    clear(dk);
    clear(dv);
    if (w.count > 0) {
        TileCopy<T, DP, QT, 256> cq, cg;
        cq.init(threadIdx.x, a.dim, a.q_stride);
        cg.init(threadIdx.x, a.dim, a.o_stride);
        const unsigned base = lds_offset(s_tiles), stats = lds_offset(s_stats);
        TileLane<T, DP> tl;
        tl.init(lane);
        const int tiles = (w.count + QT - 1) / QT, total = tiles * a.shared;
        const int from = part_of<SPLIT>(total, part, a.kv_parts), all = SPLIT ? part_of<SPLIT>(total, part + 1, a.kv_parts) - from : total;   // a part of the tiles, all heads' one behind the other
        int ih = hk * a.shared + from / tiles, it = from % tiles * QT, slot_in = 0;
        auto issue = [&] {
            const long long at = rq.first + w.first + it;
            const int rows = w.count - it;
            cq.issue(reinterpret_cast<const T *>(a.qp) + at * a.q_stride + (long long)ih * a.dim, rows, a.dim, a.q_stride, base + slot_in * BYTES, wave);
            cg.issue(reinterpret_cast<const T *>(a.dout) + at * a.o_stride + (long long)ih * a.dim, rows, a.dim, a.o_stride, base + (STAGES + slot_in) * BYTES, wave);
            // wavefronts 0 and 1: lse2, 64 rows each; 2 and 3: delta
            if ((wave & 1) * 64 < QT) {
                const auto r = make_rsrc((wave < 2 ? a.lse2 : a.delta) + (long long)ih * a.q.rows + at, (unsigned)min(rows, QT) * 4);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void)(size_t)(stats + ((slot_in * 2 + (wave >> 1)) * SIDE + (wave & 1) * 64) * 4), 4, ((wave & 1) * 64 + lane) * 4, 0, 0, 0);
            }
            if (STAGES == 2) slot_in ^= 1;
            it += QT;
            if (it >= w.count) { it = 0; ++ih; }
        };
        static_assert(QT <= 128, "two wavefronts copy a statistic");
        if (!SPLIT || all > 0) issue();
        u32x4 kc[L::SLICES], vc[L::SLICES];
        load_column<T, DP>(reinterpret_cast<const T *>(a.kp) + row * a.k_stride + (long long)hk * a.dim, on, a.dim, half, kc);
        load_column<T, DP>(reinterpret_cast<const T *>(a.vp) + row * a.v_stride + (long long)hk * a.dim, on, a.dim, half, vc);
        int slot = 0, t = from % tiles * QT;
        for (int n = 0; n < all; ++n) {
            wait_vmcnt<0>();
            __builtin_amdgcn_s_barrier();   // the tile has arrived, and the one before is done with
            if (STAGES == 2 && n + 1 < all) issue();
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int in = mine + 32 * nb, at = t + in;
                if (at <= w.none0 || at >= w.none1) continue;
                const unsigned qt = base + slot * BYTES + in * L::RB, gt = qt + STAGES * BYTES, st = stats + (slot * 2 * SIDE + in) * 4 + half * 16;
                f32x16 s[1], dp[1];
                clear(s);
                u32x4 l2[4], de[4];   // of rows 8 g + 4 half ...
                de[0] = lds_read16<SIDE * 4>(st); de[1] = lds_read16<SIDE * 4 + 32>(st); de[2] = lds_read16<SIDE * 4 + 64>(st); de[3] = lds_read16<SIDE * 4 + 96>(st);
                l2[0] = lds_read16<0>(st); l2[1] = lds_read16<32>(st); l2[2] = lds_read16<64>(st); l2[3] = lds_read16<96>(st);
                TwoFirst<T, DP, 6> ab;
                ab.begin(qt + tl.row, gt + tl.row, tl.x);
                wait_reads<1, decltype(ab)::D>();
#pragma unroll
                for (int e = 0; e < 4; ++e) { tie(l2[e]); tie(de[e]); }
#pragma unroll
                for (int v = 0; v < 16; ++v) dp[0][v] = __uint_as_float(de[v >> 2][v & 3]);   // dp - delta: the sum begins at -delta
                ab.run(qt + tl.row, gt + tl.row, tl.x, kc, vc, s[0], dp[0]);
                Second<T, DP, 2> gp, qs;
                gp.begin(gt, tl);
                hide(s[0], w, at, half);
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    s[0][v] = __builtin_amdgcn_exp2f(fmaf(s[0][v], a.scale2, -__uint_as_float(l2[v >> 2][v & 3])));
                    dp[0][v] *= s[0][v];
                }
                gp.run(gt, tl, [&](auto sc) { return column<T>(s[0], decltype(sc)::value); }, dv);
                qs.begin(qt, tl);
                qs.run(qt, tl, [&](auto sc) { return column<T>(dp[0], decltype(sc)::value); }, dk);
            }
            if (STAGES == 1 && n + 1 < all) {
                __builtin_amdgcn_s_barrier();
                issue();
            }
            if (STAGES == 2) slot ^= 1;
            t = t + QT >= w.count ? 0 : t + QT;
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
        if constexpr (SPLIT) {
            const long long at = ((part * a.kv.rows + row) * a.kv_heads + hk) * a.dim;
            store_block<float>(dk[db], a.scale, a.part_dk + at, db * 32, a.dim, half);
            store_block<float>(dv[db], 1.f, a.part_dv + at, db * 32, a.dim, half);
        } else {
            store_block<T>(dk[db], a.scale, reinterpret_cast<T *>(a.dk) + row * a.k_stride + (long long)hk * a.dim, db * 32, a.dim, half);
            store_block<T>(dv[db], 1.f, reinterpret_cast<T *>(a.dv) + row * a.v_stride + (long long)hk * a.dim, db * 32, a.dim, half);
        }
    }
}

// The parts' sums added up, in their order: 32 lanes to a row of one head, four channels each.
constexpr int kSumThreads = 256;
template <typename T> __global__ __launch_bounds__(kSumThreads) void k_attention_dkv_sum(AttnArgs a)
{
    const int b = blockIdx.x / a.tiles, col = (blockIdx.x % a.tiles) * (kSumThreads / 32) + (threadIdx.x >> 5), j = col / a.kv_heads, hk = col % a.kv_heads, c = (threadIdx.x & 31) * 4;
    const Rows rk = rows_of(a.kv, b);
    if (j >= rk.own || c >= a.dim) return;
    const long long row = rk.first + j, step = a.kv.rows * a.kv_heads * a.dim, at = (row * a.kv_heads + hk) * a.dim + c;
    f32x4 dk = {0.f, 0.f, 0.f, 0.f}, dv = dk;
#pragma unroll 4
    for (int p = 0; p < a.kv_parts; ++p) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part_dk + at + p * step), y = *reinterpret_cast<const f32x4 *>(a.part_dv + at + p * step);
#pragma unroll
        for (int e = 0; e < 4; ++e) { dk[e] += x[e]; dv[e] += y[e]; }
    }
    T *to_k = reinterpret_cast<T *>(a.dk) + row * a.k_stride + (long long)hk * a.dim + c, *to_v = reinterpret_cast<T *>(a.dv) + row * a.v_stride + (long long)hk * a.dim + c;
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u32x2 *>(to_k) = u32x2{pack_bf16(dk[0], dk[1]), pack_bf16(dk[2], dk[3])};
        *reinterpret_cast<u32x2 *>(to_v) = u32x2{pack_bf16(dv[0], dv[1]), pack_bf16(dv[2], dv[3])};
    } else {
        *reinterpret_cast<f32x4 *>(to_k) = dk;
        *reinterpret_cast<f32x4 *>(to_v) = dv;
    }
}

// Blocks of dk and dv: of 128 columns or of 32, and how many share the queries of a column.
struct DkvForm { bool wide; int parts; };

// As attn_wide says, unless an estimate of microseconds finds that the queries dealt out to several blocks take less, the sums' kernel included; where a causal mask makes blocks of different lengths that evens
// them out too.  Measured whole and so (us): causal, 8192 tokens, 8 heads of 128 over 2 491 / 424, of 64 293 / 219, 4096 tokens, 32 heads of 128 over 8 435 / 376, 2000 tokens, 8 over 2 95 / 45, fp32
// 4096 tokens 1198 / 750; all to all, 8192 tokens, 4 over 1 392 / 271.  Not: two sequences of 4096 tokens, 32 over 8, 525 / 662.
DkvForm dkv_form(const dp_attention_desc &d)
{
    const long long rows = d.kv_rows != 0 ? d.kv_rows : (long long)d.n * d.kv_len, shared = d.heads / d.kv_heads;
    const bool bf = d.io_dtype == DP_BF16, causal = (d.left < 0) != (d.right < 0);
    const DkvForm plain = {attn_wide(d, d.kv_len, rows, 1, shared * attn_seen(d, d.q_len, 128)), 1};
    if (d.q_len == 0 || rows == 0 || d.n > kMostRagged) return plain;
    const int size = d.dim <= 64 ? 0 : d.dim <= 96 ? 1 : 2;
    // of a tile, 64 rows to 128 columns or 128 to 32, on a busy card; on one whose compute units have a block of 128 columns each
    constexpr double t_wide[2][3] = {{9.6, 13, 18.8}, {1.25, 1.8, 2}}, t_few[2][3] = {{5.1, 7.5, 9.3}, {1.14, 1.37, 1.55}}, t_alone[3] = {1.2, 1.4, 1.55};
    const double sums = (double)rows * d.kv_heads * d.dim * 8 / 2.5e6;   // written, then read
    DkvForm best = plain;
    double limit = 0;
    for (const bool wide : {plain.wide, !plain.wide}) {
        if (wide && !plain.wide && (!bf || d.kv_len <= 32)) continue;
        const long long tiles = wide ? (attn_seen(d, d.q_len, 128) + 63) / 64 : (attn_seen(d, d.q_len, 32) + 127) / 128, longest = tiles * shared;
        const double blocks = (double)d.kv_heads * attn_tiles(d.n, d.kv_len, rows, 1, wide ? 128 : 32), t = wide ? t_wide[bf][size] : t_few[bf][size], alone = wide && bf ? t_alone[size] : t;
        const double seen = attn_share(d);
        for (int p = wide == plain.wide ? 1 : 2; p <= 16 && p <= longest && blocks * p <= 2048; ++p) {
            // causal: what a unit has on average, and what the last blocks leave idle
            const double even = t * (double)(long long)(blocks * p / 256 + 0.999) / p;
            const double busy = causal ? attn_between(seen, t * blocks * (0.5 + 0.5 / tiles) / 256 + (p == 1 ? 0.1 : wide ? 0.4 : 0.5 * t) / p, even) : even;
            const double us = (8 + longest * std::max(alone / p, busy) + (p > 1 ? 4 + p * sums : 0)) * (p > 1 && blocks * p > 256 ? 1.03 : 1);
            if (wide == plain.wide && p == 1) {
                if (us < 25) return plain;
                limit = 0.9 * us;
            } else if (us < limit) {
                limit = us;
                best = {wide, p};
            }
        }
        if (limit == 0) return plain;   // more blocks than need be
    }
    return best;
}

template <typename T, int DP> auto dkv_kernel(bool wide_one, bool split, int &threads)
{
    threads = 256;
    if (!wide_one) return split ? k_attention_dkv_whole<T, DP, 1, true> : k_attention_dkv_whole<T, DP, 1, false>;
    if constexpr (sizeof(T) == 4 || DP <= 96) return split ? k_attention_dkv_whole<T, DP, 4, true> : k_attention_dkv_whole<T, DP, 4, false>;
    else {
        threads = 512;
        return split ? k_attention_dkv<DP, true> : k_attention_dkv<DP, false>;
    }
}

template <typename T> void launch(const dp_attention_desc &d, AttnArgs &a, bool wk, hipStream_t st)
{
    for_dim(a.dim, [&](auto dc) {
        constexpr int DP = decltype(dc)::value;
        const long long qc = (long long)a.q.len * a.shared, kc = a.kv.len;
        const bool wq = attn_wide(d, a.q.len, a.q.rows, a.shared, attn_seen(d, a.kv.len, std::max(1, 128 / a.shared)));
        a.tiles = (int)((qc + (wq ? 127 : 31)) / (wq ? 128 : 32));
        if (a.tiles > 0 && a.q.rows > 0) hipLaunchKernelGGL((wq ? k_attention_dq<T, DP, 4> : k_attention_dq<T, DP, 1>), dim3(attn_blocks(a, a.q, a.shared, wq ? 128 : 32)), dim3(256), 0, st, a);
        a.tiles = (int)((kc + (wk ? 127 : 31)) / (wk ? 128 : 32));
        if (a.tiles == 0 || a.kv.rows == 0) return;
        int threads;
        auto *kernel = dkv_kernel<T, DP>(wk, a.kv_parts > 1, threads);
        hipLaunchKernelGGL(kernel, dim3(attn_blocks(a, a.kv, 1, wk ? 128 : 32) * a.kv_parts), dim3(threads), 0, st, a);
        if (a.kv_parts == 1) return;
        a.tiles = (int)((std::min<long long>(kc, a.kv.rows) * a.kv_heads + kSumThreads / 32 - 1) / (kSumThreads / 32));
        hipLaunchKernelGGL(k_attention_dkv_sum<T>, dim3((unsigned)((long long)a.n * a.tiles)), dim3(kSumThreads), 0, st, a);
    });
}

size_t stat_bytes(const dp_attention_desc &d)
{
    const size_t rows = (size_t)(d.q_rows != 0 ? d.q_rows : (long long)d.n * d.q_len);
    return ((size_t)d.heads * rows * sizeof(float) + 15) / 16 * 16;
}

size_t sum_bytes(const dp_attention_desc &d, const DkvForm &f)   // of dk's, or of dv's parts
{
    return f.parts == 1 ? 0 : (size_t)f.parts * (size_t)(d.kv_rows != 0 ? d.kv_rows : (long long)d.n * d.kv_len) * d.kv_heads * d.dim * sizeof(float);
}

}  // namespace

size_t attn_bwd_bytes(const dp_attention_desc &d) { return 2 * (stat_bytes(d) + sum_bytes(d, dkv_form(d))); }

extern "C" dp_status dp_attention_bwd(const dp_attention_desc *desc, const void *q, const void *k, const void *v, const void *o, const void *dout,
                                      const float *lse, void *dq, void *dk, void *dv, const dp_attention_seqs *seqs, void *ws, size_t ws_bytes,
                                      void *hip_stream)
{
    dp_status s = attn_check(desc, seqs, true);
    if (s != DP_OK) return s;
    const dp_attention_desc &d = *desc;
    AttnArgs a;
    attn_args(d, seqs, a);
    const bool queries = d.n > 0 && d.q_len > 0 && a.q.rows > 0, keys = d.n > 0 && d.kv_len > 0 && a.kv.rows > 0;
    if (!queries && !keys) return DP_OK;
    if (queries && (s = attn_pointers({q, o, dout, dq}, lse, nullptr)) != DP_OK) return s;
    if (queries && lse == nullptr) { dp_set_error("attention's gradient: lse is NULL"); return DP_ERR_NULL; }
    if (keys && (s = attn_pointers({k, v, dk, dv}, nullptr, nullptr)) != DP_OK) return s;
    const DkvForm f = dkv_form(d);
    // dk and dv are made behind dq, from all inputs but o
    if ((s = attn_apart({queries ? dq : nullptr, keys ? dk : nullptr, keys ? dv : nullptr}, {q, k, v, o, dout, lse})) != DP_OK || (s = attn_pointers({}, nullptr, ws)) != DP_OK || (s = attn_workspace(2 * (stat_bytes(d) + sum_bytes(d, f)), ws, ws_bytes)) != DP_OK) return s;
    a.qp = q; a.kp = k; a.vp = v; a.op_in = o; a.dout = dout; a.lse_in = lse;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.lse2 = (float *)ws;
    a.delta = (float *)((char *)ws + stat_bytes(d));
    a.kv_parts = f.parts;
    a.part_dk = (float *)((char *)ws + 2 * stat_bytes(d));
    a.part_dv = (float *)((char *)a.part_dk + sum_bytes(d, f));
    if (d.io_dtype == DP_BF16) launch<bf16_t>(d, a, f.wide, (hipStream_t)hip_stream);
    else launch<float>(d, a, f.wide, (hipStream_t)hip_stream);
    return attn_launched("attention's gradient");
}
