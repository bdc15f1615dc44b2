// What the attention kernels share: the call's arguments, the sequences, tiles of rows in LDS and the two kinds of matrix-core products on them.
//
// Every kernel keeps 32 columns per wavefront in registers (queries forward and for dq, keys for dk and dv) and lets tiles of rows of the other side pass
// through LDS.  A product of the first kind, rows x columns over a head's channels, gives lane l the 16 rows 8 (v / 4) + 4 (l / 32) + v % 4 of column
// l % 32.  Those registers are as they stand the second operand of a product of the second kind, channels x columns over rows: the order of a reduction
// is free, so its first operand, the tile transposed, is read from LDS in the same order of rows.  Softmax is then a matter of single lanes, and nothing is
// exchanged but one value between the two halves of a wavefront.
#pragma once
#include "../../include/dp.h"
#include "dma_common.h"
#include <algorithm>
#include <initializer_list>

void dp_set_error(const char *fmt, ...);   // dp_api.hip

struct AttnSide {
    const int *starts, *lens;
    int len;                // the longest sequence's
    long long rows;
};

struct AttnArgs {
    AttnSide q, kv;
    int n, heads, kv_heads, shared, dim;   // shared: heads of queries to one of keys
    int left, right;                       // no bound: kFar
    float scale, scale2;                   // scale2 = scale log2(e)
    long long q_stride, k_stride, v_stride, o_stride;
    const void *qp, *kp, *vp, *op_in, *dout;
    void *op;
    float *lse;
    const float *lse_in;
    void *dq, *dk, *dv;
    float *lse2, *delta;                   // backward's workspace: lse log2(e) (+inf: sees nothing) and -sum dout o, [heads][q_rows]
    int tiles;                             // of a sequence and head of keys
    int splits, split_keys, span;          // forward: the keys that a block's queries see, at most span, dealt out to so many blocks, split_keys each
    bool causal;                           // a bound on one side alone: tiles of a sequence see more or fewer rows
    bool ragged;                           // lengths differ: blocks are numbered by the work there is
    float *part_o, *part_ml;               // [split][head][q_rows][dim] and [split][head][q_rows][2]
    int kv_parts;                          // backward: the queries of a block of keys dealt out to so many blocks,
    float *part_dk, *part_dv;              // which leave their sums in [part][kv_rows][kv_heads][dim]
};

namespace {

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr int kFar = 1 << 30;
// Rows of one sequence: where they begin, how many are in use, and how many are its own to be written.
struct Rows { long long first; int used, own; };
DEVFN Rows rows_of(const AttnSide &s, int b)
{
    Rows r;
    if (s.starts != nullptr) {
        const long long lo = min(max((long long)s.starts[b], 0ll), s.rows), hi = min(max((long long)s.starts[b + 1], lo), s.rows);
        r.first = lo;
        r.used = r.own = (int)min(hi - lo, (long long)s.len);
    } else {
        r.first = (long long)b * s.len;
        r.own = s.len;
        r.used = s.lens != nullptr ? min(max(s.lens[b], 0), s.len) : s.len;
    }
    return r;
}

// Forward, split keys: how many parts the keys of a sequence have, where sequences differ.
DEVFN int parts_of(const AttnArgs &a, int b) { return (min(rows_of(a.kv, b).used, a.span) + a.split_keys - 1) / a.split_keys; }

// What a block does: sequence, head of keys, tile of columns and part of the keys.
struct Item { int b, hk, tile, split; bool any; };

DEVFN int prefix_sum(int v)   // over the lanes up to this one
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // one, two, four, eight lanes up
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // the last lane of a row to the next row
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
    return v;
}

// The number of block `block` of `of` among the tiles of `groups` heads, one head's behind the other's, where tiles of a head take different times.  A contiguous eighth for each die
// is as much work for all of them only if it holds whole heads; else as many dies as hold whole ones together take the tiles in turn (8192 causal tokens, 8 heads of 128 over 2: forward
// 226 -> 178 us, dq 319 -> 242, dk and dv 695 -> 480).
DEVFN int dealt(int block, int of, int groups)
{
    if (groups % 8 == 0) return logical_block(block, of);
    const int dies = of % 8 != 0 ? 8 : groups % 4 == 0 ? 2 : groups % 2 == 0 ? 4 : 8, die = block & 7;
    return die / dies * (of / 8 * dies) + (block >> 3) * dies + die % dies;
}

// Block 256 ... 511 of a launch of `of`: the one in its place where each die takes its blocks of these, as many as there are, in reverse.
inline __host__ __device__ int second_reversed(int block, int of)
{
    const int die = block & 7, there = ((of < 512 ? of : 512) - 256 - die + 7) >> 3;
    return (63 + there - (block >> 3)) << 3 | die;
}

// The grid has room for sequences of the longest length.  Whole sequences: tile by tile, head by head, a contiguous eighth for each die, so that the tiles of one head read their
// rows from one L2 (with a causal mask: dealt).  Lengths that differ: the same over the tiles that there are, counted by each block for itself (a lane to a sequence), since tiles of nothing, numbered
// among the others, would leave some dies with much more work than others (9 sequences of up to 1500 of 4 heads of keys, dk and dv: 73 us, 53 this way).  Tiles that hold padding alone come last.
// `mult` columns to a row of `side`; SPLIT: every part of the keys that a sequence has; LAST_FIRST: a causal mask makes a sequence's last tiles the longest.  Where all blocks of such a call
// are on the card at once, SLOTS to a compute unit, each die's second 32, or as many as there are, are taken in reverse, so that a long one shares its unit with a short one (4096 causal tokens, 16 heads
// of 128: 105 -> 97 us forward, dq 147 -> 136; 12 heads, 384 blocks, 108 -> 81 and 149 -> 112).
constexpr int kMostRagged = 256;   // sequences: more of them are counted for longer than it helps
template <int COLS, bool SPLIT, bool LAST_FIRST, int SLOTS = 1> DEVFN Item item_of(const AttnArgs &a, const AttnSide &side, int mult, int block, int of)
{
    Item r;
    if (!a.ragged) {
        if (SLOTS > 1 && LAST_FIRST && of <= 256 * SLOTS && a.causal && (block & 256) != 0) block = second_reversed(block, of);
        int id = a.causal ? dealt(block, of, a.n * a.kv_heads) : logical_block(block, of);
        r.split = SPLIT ? id % a.splits : 0;
        if (SPLIT) id /= a.splits;
        const int hb = id / a.tiles;
        r.tile = LAST_FIRST ? a.tiles - 1 - id % a.tiles : id % a.tiles;
        r.b = hb % a.n;
        r.hk = hb / a.n;
        r.any = true;
        return r;
    }
    const int lane = threadIdx.x & 63;
    // parts, and tiles with rows in use and in all, of sequence b
    const auto count = [&](int b, int list, int &parts, int &used) {
        parts = used = 0;
        if (b >= a.n) return 0;
        const Rows rows = rows_of(side, b);
        parts = SPLIT ? parts_of(a, b) : 1;
        const int own = (int)(((long long)rows.own * mult + COLS - 1) / COLS);
        used = SPLIT ? own : (int)(((long long)rows.used * mult + COLS - 1) / COLS);
        return (list == 0 ? used : own - used) * parts;
    };
    int id = block, parts, used;
    for (int list = 0; list < (SPLIT ? 1 : 2); ++list) {
        int total = 0;
        for (int base = 0; base < a.n; base += 64) total += __builtin_amdgcn_readlane(prefix_sum(count(base + lane, list, parts, used)), 63);
        const int blocks = total * a.kv_heads;
        if (id >= blocks) { id -= blocks; continue; }
        id = logical_block(id, blocks);
        r.hk = id / total;
        id %= total;
        for (int base = 0; base < a.n; base += 64) {
            const int c = count(base + lane, list, parts, used), sum = prefix_sum(c);
            const unsigned long long found = __ballot(sum > id);
            if (found == 0) { id -= __builtin_amdgcn_readlane(sum, 63); continue; }
            const int l = __ffsll(found) - 1;
            id -= __builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(c, l);
            parts = __builtin_amdgcn_readlane(parts, l);
            r.b = base + l;
            r.split = id % parts;
            used = __builtin_amdgcn_readlane(used, l);
            r.tile = list != 0 ? used + id : LAST_FIRST ? used - 1 - id / parts : id / parts;
            break;
        }
        r.any = true;
        return r;
    }
    r.any = false;
    return r;
}

// Halves of a wavefront: v of lane l and lane l ^ 32.
DEVFN float other_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// A tile in LDS: rows of RB bytes (whole blocks of 32 channels; those behind the head's own are zero) in chunks of 16 bytes, chunk c of row r at c ^ swizzle(r).  The 64 banks
// hold sixteen chunks, so chunk c' of row r lies in banks (CR r + c') % 16: the swizzle makes reads of one chunk of 16 rows, and transposed reads of four chunks
// of four rows, touch every bank once.  Where CR is an odd multiple of four, four rows lie apart by themselves and the swizzle stays within four chunks (FLAT).
template <typename T, int DP> struct Tile {
    static constexpr int E = 16 / sizeof(T);                              // elements of a chunk
    static constexpr int SLICES = DP / (2 * E);                           // of the first kind of product
    static constexpr int DB = (DP + 31) / 32;                             // blocks of 32 channels of the second
    static constexpr int RB = DB * 32 * (int)sizeof(T), CR = RB / 16;     // CR: chunks of a row
    static constexpr bool FLAT = CR % 8 == 4;
    static DEVFN int swizzle(int r)
    {
        if constexpr (FLAT) return (r >> 2) & 3;
        else if constexpr (CR % 16 == 8) return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
        else if constexpr (CR == 16) return (r & 3) << 2 | ((r >> 2) & 3);
        else return r & 15;
    }
};

// One block's copies of ROWS rows of a matrix into a tile, THREADS threads taking part.  Rows behind the last one and channels behind the head's own become zero.
template <typename T, int DP, int ROWS, int THREADS> struct TileCopy {
    using L = Tile<T, DP>;
    static constexpr int N = ROWS * L::CR / THREADS;   // 16-byte copies of a thread
    static_assert(ROWS * L::CR % THREADS == 0, "whole copies");
    unsigned off[N];
    DEVFN void init(int tid, int dim, long long stride)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = i * THREADS + tid, row = p / L::CR, c = (p % L::CR) ^ L::swizzle(row);
            off[i] = c * L::E < dim ? (unsigned)(row * (int)stride * (int)sizeof(T) + c * 16) : OOR;
        }
    }
    // rows: how many there are from `base` on (at least 1)
    DEVFN void issue(const T *base, int rows, int dim, long long stride, unsigned lds, int wave) const
    {
        const unsigned bytes = (unsigned)(min(rows, ROWS) - 1) * (unsigned)(stride * (int)sizeof(T)) + (unsigned)dim * (unsigned)sizeof(T);
        const auto r = make_rsrc(base, bytes);
#pragma unroll
        for (int i = 0; i < N; ++i) dma16(r, lds + (i * THREADS + wave * 64) * 16, off[i]);
    }
};

template <typename T> struct Mma;
template <> struct Mma<bf16_t> {
    static DEVFN void first(const u32x4 &a, const u32x4 &b, f32x16 &c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma<float> {
    static DEVFN void first(const u32x4 &a, const u32x4 &b, f32x16 &c)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    }
};

// Waits until LEFT items of NR reads each are under way at most (reads from LDS arrive in their order, so the older ones are there), and the
// mark of a register that such a read fills: nothing that uses it is moved in front of the wait.
template <int NR, int LEFT> DEVFN void wait_reads()
{
    constexpr int n = NR * LEFT < 15 ? NR * LEFT : 15;
    asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(n));
}
DEVFN void tie(u32x4 &v) { asm volatile("" : "+v"(v)); }
DEVFN void tie(u32x2 &v) { asm volatile("" : "+v"(v)); }
DEVFN void tie(float &v) { asm volatile("" : "+v"(v)); }

// First kind: acc[block] (32 rows each) += tile rows x `cols`, over the channels.  NB blocks of 32 rows from row `addr` on.
template <typename T, int DP, int NB, int DEPTH> struct First {
    using L = Tile<T, DP>;
    static constexpr int N = NB * L::SLICES, D = DEPTH < N ? DEPTH : N;
    u32x4 buf[D];
    template <int I> DEVFN void read(unsigned base, unsigned x)   // base: the lane's row in block 0; x: its swizzled chunk of slice 0, in bytes
    {
        constexpr int block = I % NB, s = I / NB;   // neighbours in time add to different sums
        if constexpr (L::FLAT) buf[I % D] = lds_read16<block * 32 * L::RB + s / 2 * 64>(base + (x ^ (unsigned)(s % 2 * 32)));
        else buf[I % D] = lds_read16<block * 32 * L::RB>(base + (x ^ (unsigned)(s * 32)));
    }
    DEVFN void begin(unsigned base, unsigned x) { for_constant<D>([&](auto i) { read<decltype(i)::value>(base, x); }); }
    DEVFN void run(unsigned base, unsigned x, const u32x4 (&cols)[L::SLICES], f32x16 (&acc)[NB])
    {
        for_constant<N>([&](auto ic) {
            constexpr int i = decltype(ic)::value, left = (N - i < D ? N - i : D) - 1;
            wait_reads<1, left>();
            tie(buf[i % D]);
            Mma<T>::first(buf[i % D], cols[i / NB], acc[i % NB]);
            if constexpr (i + D < N) read<i + D>(base, x);
        });
    }
};

// Two products of the first kind on two tiles of 32 rows, their slices in turn: sa += rows a x ca, sb += rows b x cb.
template <typename T, int DP, int DEPTH> struct TwoFirst {
    using L = Tile<T, DP>;
    static constexpr int N = 2 * L::SLICES, D = DEPTH < N ? DEPTH : N;
    u32x4 buf[D];
    template <int I> DEVFN void read(unsigned a, unsigned b, unsigned x)
    {
        constexpr int s = I / 2;
        if constexpr (L::FLAT) buf[I % D] = lds_read16<s / 2 * 64>((I % 2 == 0 ? a : b) + (x ^ (unsigned)(s % 2 * 32)));
        else buf[I % D] = lds_read16<0>((I % 2 == 0 ? a : b) + (x ^ (unsigned)(s * 32)));
    }
    DEVFN void begin(unsigned a, unsigned b, unsigned x) { for_constant<D>([&](auto i) { read<decltype(i)::value>(a, b, x); }); }
    DEVFN void run(unsigned a, unsigned b, unsigned x, const u32x4 (&ca)[L::SLICES], const u32x4 (&cb)[L::SLICES], f32x16 &sa, f32x16 &sb)
    {
        for_constant<N>([&](auto ic) {
            constexpr int i = decltype(ic)::value, left = (N - i < D ? N - i : D) - 1;
            wait_reads<1, left>();
            tie(buf[i % D]);
            if constexpr (i % 2 == 0) Mma<T>::first(buf[i % D], ca[i / 2], sa);
            else Mma<T>::first(buf[i % D], cb[i / 2], sb);
            if constexpr (i + D < N) read<i + D>(a, b, x);
        });
    }
};

// The lane's addresses in a tile.
template <typename T, int DP> struct TileLane {
    using L = Tile<T, DP>;
    unsigned row, x;          // first kind: own row's offset, swizzled chunk of slice 0
    unsigned lo, hi;          // second kind, bf16: rows 4 (l / 32) + (l % 16) / 4 of a slice of 16, and 8 further (relative to 8 rows further)
    DEVFN void init(int lane)
    {
        const int r = lane & 31, h = lane >> 5;
        row = r * L::RB;
        x = (unsigned)(h ^ L::swizzle(r)) * 16;
        if constexpr (sizeof(T) == 2) {
            const int j = lane & 15, rr = 4 * h + (j >> 2), c = ((lane >> 4) & 1) * 2 + ((j & 3) >> 1);
            lo = rr * L::RB + (unsigned)(c ^ L::swizzle(rr)) * 16 + (j & 1) * 8;
            hi = rr * L::RB + (unsigned)(c ^ L::swizzle(rr + 8)) * 16 + (j & 1) * 8;
        } else {
            lo = 4 * h * L::RB + (r & 3) * 4;   // the chunk, r / 4, is swizzled by each row
            hi = h;
        }
    }
};

// Second kind: acc[db] (32 channels each) += tile^T x cols, over NS slices of 16 rows.
template <typename T, int DP, int NS> struct Second;
template <int DP, int NS> struct Second<bf16_t, DP, NS> {
    using L = Tile<bf16_t, DP>;
    static constexpr int DB = L::DB, N = NS * DB, D = N < 6 ? N : 6, READS = 2 * D;   // READS: under way behind begin()
    u32x2 lo[D], hi[D];
    // a channel block of 32 is 64 bytes on: bits above the two lowest of the chunk's number, which the swizzle may have set
    template <int I> DEVFN void read(unsigned tile, const TileLane<bf16_t, DP> &l)
    {
        constexpr int s = I / DB, db = I % DB;
        if constexpr (L::FLAT) {
            lo[I % D] = lds_read_tr<s * 16 * L::RB + db * 64>(tile + l.lo);
            hi[I % D] = lds_read_tr<(s * 16 + 8) * L::RB + db * 64>(tile + l.hi);
        } else {
            lo[I % D] = lds_read_tr<s * 16 * L::RB>(tile + (l.lo ^ (unsigned)(db * 64)));
            hi[I % D] = lds_read_tr<(s * 16 + 8) * L::RB>(tile + (l.hi ^ (unsigned)(db * 64)));
        }
    }
    DEVFN void begin(unsigned tile, const TileLane<bf16_t, DP> &l) { for_constant<D>([&](auto i) { read<decltype(i)::value>(tile, l); }); }
    template <int I, typename F> DEVFN void item(unsigned tile, const TileLane<bf16_t, DP> &l, F &&cols, f32x16 (&acc)[DB])
    {
        constexpr int left = (N - I < D ? N - I : D) - 1;
        wait_reads<2, left>();
        tie(lo[I % D]);
        tie(hi[I % D]);
        const u32x4 a = {lo[I % D].x, lo[I % D].y, hi[I % D].x, hi[I % D].y};
        Mma<bf16_t>::first(a, cols(std::integral_constant<int, I / DB>{}), acc[I % DB]);
        if constexpr (I + D < N) read<I + D>(tile, l);
    }
    // cols(s): the eight rows of slice s of the lane's column, packed
    template <typename F> DEVFN void run(unsigned tile, const TileLane<bf16_t, DP> &l, F &&cols, f32x16 (&acc)[DB])
    {
        for_constant<N>([&](auto i) { item<decltype(i)::value>(tile, l, cols, acc); });
    }
    // between(i): what the vector unit does beside matrix product i of N; kept in this order
    template <typename F, typename G> DEVFN void run_beside(unsigned tile, const TileLane<bf16_t, DP> &l, F &&cols, f32x16 (&acc)[DB], G &&between)
    {
        for_constant<N>([&](auto i) {
            item<decltype(i)::value>(tile, l, cols, acc);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        });
    }
};
template <int OFF> DEVFN float lds_read4(unsigned addr)
{
    float v;
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int DP, int NS> struct Second<float, DP, NS> {
    using L = Tile<float, DP>;
    static constexpr int DB = L::DB, N = NS * DB, READS = 8;
    float buf[2][8];   // an item's reads are under way while the products of the one before run
    // register v of a lane's column is row 8 (v / 4) + 4 half + v % 4: one 32x32x2 product takes v of both halves
    template <int I> DEVFN void read(unsigned tile, const TileLane<float, DP> &l, int chunk)
    {
        constexpr int s = I / DB, db = I % DB;
        for_constant<8>([&](auto ec) {
            constexpr int e = decltype(ec)::value, row = s * 16 + 8 * (e / 4) + e % 4;   // and 4 h
            buf[I % 2][e] = lds_read4<row * L::RB>(tile + l.lo + (unsigned)(((db * 8 + chunk) ^ L::swizzle(row + 4 * (int)l.hi)) * 16));
        });
    }
    static DEVFN int own_chunk()
    {
        int chunk = (threadIdx.x & 31) >> 2;
        asm volatile("" : "+v"(chunk));   // addresses are made where they are used: kept for the whole loop they would take registers that the sums need
        return chunk;
    }
    DEVFN void begin(unsigned tile, const TileLane<float, DP> &l) { read<0>(tile, l, own_chunk()); }
    template <typename F> DEVFN void run(unsigned tile, const TileLane<float, DP> &l, F &&cols, f32x16 (&acc)[DB])
    {
        const int chunk = own_chunk();
        for_constant<N>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            if constexpr (i + 1 < N) read<i + 1>(tile, l, chunk);
            wait_reads<8, (i + 1 < N ? 1 : 0)>();
#pragma unroll
            for (int e = 0; e < 8; ++e) tie(buf[i % 2][e]);
            const auto c = cols(std::integral_constant<int, i / DB>{});
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x2f32(buf[i % 2][e], c[e], acc[i % DB], 0, 0, 0);
        });
    }
};

// Eight registers of a column (slice s: 8 s ... 8 s + 7) as the second operand of a product of the second kind.
typedef __attribute__((ext_vector_type(8))) float f32x8;
template <typename T> DEVFN auto column(const f32x16 &v, int half)
{
    const int b = 8 * half;
    if constexpr (sizeof(T) == 2) return u32x4{pack_bf16(v[b], v[b + 1]), pack_bf16(v[b + 2], v[b + 3]), pack_bf16(v[b + 4], v[b + 5]), pack_bf16(v[b + 6], v[b + 7])};
    else return f32x8{v[b], v[b + 1], v[b + 2], v[b + 3], v[b + 4], v[b + 5], v[b + 6], v[b + 7]};
}

// The lane's column of a matrix as the second operand of products of the first kind: chunks l / 32, l / 32 + 2, ... of its row; zero where there is none.
template <typename T, int DP> DEVFN void load_column(const T *row, bool on, int dim, int half, u32x4 (&v)[Tile<T, DP>::SLICES])
{
    using L = Tile<T, DP>;
#pragma unroll
    for (int s = 0; s < L::SLICES; ++s) {
        const int c = (2 * s + half) * L::E;
        v[s] = on && c < dim ? *reinterpret_cast<const u32x4 *>(row + c) : u32x4{0, 0, 0, 0};
    }
}

// A block of a column's results, channels c0 + 8 (v / 4) + 4 half + v % 4, times f, to its row.
template <typename T> DEVFN void store_block(const f32x16 &acc, float f, T *row, int c0, int dim, int half)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int c = c0 + 8 * g + 4 * half;
        if (c >= dim) continue;
        const float v0 = acc[4 * g] * f, v1 = acc[4 * g + 1] * f, v2 = acc[4 * g + 2] * f, v3 = acc[4 * g + 3] * f;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2 *>(row + c) = u32x2{pack_bf16(v0, v1), pack_bf16(v2, v3)};
        else *reinterpret_cast<f32x4 *>(row + c) = f32x4{v0, v1, v2, v3};
    }
}
template <typename T, int DB> DEVFN void store_column(const f32x16 (&acc)[DB], float f, T *row, int dim, int half)
{
#pragma unroll
    for (int db = 0; db < DB; ++db) store_block<T>(acc[db], f, row, db * 32, dim, half);
}

// Wavefronts that went over different rows for the same columns: their sums, block i in acc of wavefront i % WAVES (the others' are left as they are).
// `room`: N blocks of 4 KB for each wavefront; free for use by all of them.
template <int WAVES, int N> DEVFN void sum_waves(f32x16 (&acc)[N], float *room, int wave, int lane)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4 *>(room + ((wave * N + i) * 4 + g) * 256 + lane * 4) = f32x4{acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i % WAVES != wave) continue;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(room + ((w * N + i) * 4 + g) * 256 + lane * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += v[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][4 * g + e] = sum[e];
        }
    }
}

template <int N> DEVFN void clear(f32x16 (&acc)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
}

}  // namespace

// f(integral_constant): the smallest size of a head's rows in LDS and registers that holds `dim` channels
template <typename F> void for_dim(int dim, F &&f)
{
    if (dim <= 32) f(std::integral_constant<int, 32>{});
    else if (dim <= 48) f(std::integral_constant<int, 48>{});
    else if (dim <= 64) f(std::integral_constant<int, 64>{});
    else if (dim <= 80) f(std::integral_constant<int, 80>{});
    else if (dim <= 96) f(std::integral_constant<int, 96>{});
    else if (dim <= 112) f(std::integral_constant<int, 112>{});
    else f(std::integral_constant<int, 128>{});
}

// attention_fwd.hip: what both passes check and take from the descriptor and the sequences
dp_status attn_check(const dp_attention_desc *desc, const dp_attention_seqs *seqs, bool gradient);
void attn_args(const dp_attention_desc &d, const dp_attention_seqs *seqs, AttnArgs &a);
dp_status attn_pointers(std::initializer_list<const void *> needed, const void *lse, const void *ws);
dp_status attn_apart(std::initializer_list<const void *> results, std::initializer_list<const void *> inputs);
dp_status attn_workspace(size_t need, const void *ws, size_t ws_bytes);
dp_status attn_launched(const char *what);
// tiles of `columns` that n sequences of up to `len` rows can have, `mult` columns to a row; packed ones have no more rows than there are in memory
inline long long attn_tiles(long long n, long long len, long long rows, long long mult, int columns)
{
    const long long all = n * ((len * mult + columns - 1) / columns), packed = rows * mult / columns + n;
    return rows < n * len && packed < all ? packed : all;
}
// The share of a sequence's pairs of a query and a key that a mask with a bound on one side leaves: a half of a square, nearly all for a few queries behind many keys.  Never below a half: where
// there are more queries than keys, the blocks that see nothing end at once and the others are as those of a square (4 x 1500 queries, 500 keys, 16 heads of 128 over 4: dk and dv 33 us, 43 as the share has it).
inline double attn_share(const dp_attention_desc &d)
{
    if ((d.left < 0) == (d.right < 0) || d.q_len == 0 || d.kv_len == 0) return 1;
    // as areas: query i sees min(i + from, kv_len) keys, if that is any (left: counted from the last query back)
    const double q = d.q_len, k = d.kv_len, from = d.right >= 0 ? k - q + d.right : d.left;
    const double whole = std::min(q, std::max(0.0, from + q - k)), first = std::max(0.0, from), rest = std::max(0.0, q - whole - std::max(0.0, -from));
    return std::max(0.5, (whole * k + rest * (first + std::min(k, first + rest)) / 2) / (q * k));
}
// Between what is true of a half and of all pairs
inline double attn_between(double share, double half, double all) { return (2 - 2 * share) * half + (2 * share - 1) * all; }
// Whether blocks are of 128 columns, four wavefronts side by side, or of 32, whose wavefronts share the other side's rows: what is shorter by this count of microseconds.  A block takes 3 for
// its beginning and its end, and t for each 64 (128 columns) or 128 (32 columns) rows of the other side; a compute unit works on one of the former at a time or as fast on several,
// on one or (narrow heads) two of the latter.  Blocks of a causal mask need attn_share of their rows on average, the first ones all.  Measured, forward in small and in large blocks (us): 2000 tokens of 8 heads of
// 64 22 / 28, 4000 causal 43 / 50, 2 x 1000 of 128 28 / 23, 8 x 197 of 12 heads of 64 11.4 / 7.8, 24 packed sequences of 16 heads of 80 267 / 75; fp32 2 x 1788 causal, 12 heads of 72, 183 / 276,
// 4 x 1024, 8 heads of 64, 107 / 82; 512 causal queries behind 32768 keys, 32 heads of 128 over 8, 630 / 518 (dq 659 / 695).
inline bool attn_wide(const dp_attention_desc &d, long long len, long long rows, long long mult, long long other)
{
    if (len * mult <= 32) return false;
    if ((double)d.n * d.kv_heads * (double)(len * mult / 32 + 1) >= (double)(1 << 23)) return true;   // a launch has fewer than 2^32 threads
    const bool bf = d.io_dtype == DP_BF16, causal = (d.left < 0) != (d.right < 0);
    const int size = d.dim <= 64 ? 0 : d.dim <= 96 ? 1 : 2;
    const double share = attn_share(d);
    constexpr double t_wide[2][3] = {{4.8, 6.5, 9.4}, {0.72, 0.9, 1.09}}, t_few[2][3] = {{2.9, 4.2, 5.9}, {0.92, 1.05, 1.19}};
    const double wide = d.kv_heads * (double)attn_tiles(d.n, len, rows, mult, 128) / 256, few = d.kv_heads * (double)attn_tiles(d.n, len, rows, mult, 32) / (bf && size == 0 ? 512 : 256);
    const auto whole = [](double x) { return (double)(long long)(x + 0.999); };
    const auto longest = [](double x) { return x > 1 ? x : 1; };
    const auto rounds = [&](double blocks, double tail, double all) { return longest(causal ? attn_between(share, 0.5 * blocks + tail, all) : all); };
    const double rounds_wide = bf ? rounds(wide, 0.25, wide) : rounds(wide, 0.75, whole(wide)), rounds_few = rounds(few, 0.25, few);
    return 3 + other / 64.0 * t_wide[bf][size] * rounds_wide <= 3 * whole(few) + other / 128.0 * t_few[bf][size] * rounds_few;
}
// rows of the other side that a block of `columns` sees, at most
inline long long attn_seen(const dp_attention_desc &d, long long len, int columns)
{
    const long long window = d.left >= 0 && d.right >= 0 ? (long long)d.left + d.right + columns : len;
    return window < len ? window : len;
}
// blocks of a call: where they are numbered by what there is, no more than that can be
inline unsigned attn_blocks(const AttnArgs &a, const AttnSide &side, long long mult, int columns)
{
    const long long tiles = a.ragged && side.starts != nullptr ? attn_tiles(a.n, side.len, side.rows, mult, columns) : (long long)a.n * a.tiles;
    return (unsigned)(tiles * a.kv_heads * a.splits);
}
size_t attn_bwd_bytes(const dp_attention_desc &d);   // attention_bwd.hip
