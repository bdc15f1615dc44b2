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

constexpr int kMaxSplits = 64;
constexpr int kCandidates = 512;   // of a block, in LDS

struct Soft { float m, s, t; };   // maximum, sum exp(d), sum d exp(d) with d = z - m; nothing yet: -FLT_MAX, 0, 0

struct LpArgs {
    const void *z;
    const int *ids;
    float *logp, *entropy, *lse, *top_logp;
    int *top_ids;
    Soft *part;                      // [row][split]
    unsigned long long *part_top;    // [row][split][k], best first; 0: none
    int rows, classes, k;
    int splits, seg;                 // classes of a split (the last one may be shorter)
    long long stride;
};

// Orders scores as whole numbers, larger first: value, then the lower index.  -0 counts as 0, a NaN ranks above everything.  No key has all
// bits set, also that of a NaN at class 0: the searches that go down from key to key begin there.
__device__ __forceinline__ unsigned order_of(float z)
{
    z += 0.f;
    const unsigned u = z != z ? 0x7ffffffeu : __float_as_uint(z);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ unsigned long long key_of(float z, int index) { return (unsigned long long)order_of(z) << 32 | (unsigned)~index; }
__device__ __forceinline__ float score_of(unsigned long long key)
{
    unsigned u = (unsigned)(key >> 32);
    u ^= (u >> 31) != 0 ? 0x80000000u : 0xffffffffu;
    return __uint_as_float(u);
}
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)~(unsigned)key; }

__device__ __forceinline__ float exp_d(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// a larger maximum
__device__ __forceinline__ void raise(Soft &a, float m)
{
    const float d = a.m - m, f = exp_d(d);
    a.t = f > 0.f ? fmaf(a.s, d, a.t) * f : 0.f;   // s d may pass the range where f is 0
    a.s *= f;
    a.m = m;
}
template <int V> __device__ __forceinline__ float add_scores(Soft &a, const float (&z)[V])   // returns their largest
{
    float m = z[0];
#pragma unroll
    for (int e = 1; e < V; ++e) m = fmaxf(m, z[e]);
    if (m > a.m) raise(a, m);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float d = z[e] - a.m, x = exp_d(d);
        a.s += x;                                   // NaN and +inf scores make this NaN
        a.t = fmaf(x, fmaxf(d, -3e38f), a.t);       // exp(-inf) * -inf counts as 0
    }
    return m;
}
__device__ __forceinline__ void join(Soft &a, const Soft &b)
{
    const float m = fmaxf(a.m, b.m);
    const float da = a.m - m, db = b.m - m, fa = exp_d(da), fb = exp_d(db);
    const float ta = fa > 0.f ? fmaf(a.s, da, a.t) * fa : 0.f, tb = fb > 0.f ? fmaf(b.s, db, b.t) * fb : 0.f;
    a.s = a.s * fa + b.s * fb;
    a.t = ta + tb;
    a.m = m;
}
// The wavefront's: its maximum, then each lane's sums brought to it.
__device__ __forceinline__ Soft wave_join(const Soft &a)
{
    const float m = wave_max_fast(a.m), d = a.m - m, f = exp_d(d);
    return {m, wave_sum_fast(a.s * f), wave_sum_fast(f > 0.f ? fmaf(a.s, d, a.t) * f : 0.f)};   // a NaN sum stays one
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

// How many of list[0 .. c) are larger than key.  Eight reads at a time: up to seven zeros stand behind the last entry.
__device__ __forceinline__ int larger(const unsigned long long *list, int c, unsigned long long key)
{
    int rank = 0;
    for (int j = 0; j < c; j += 8)
#pragma unroll
        for (int e = 0; e < 8; ++e) rank += list[j + e] > key;
    return rank;
}

// A run of scores as the block reads it: single ones in front of the first boundary of ALIGN bytes, whole vectors, up to V - 1 single ones
// behind.  Thread t takes single t of each end and vectors t, t + NT, ...
template <typename T, int ALIGN = 16> struct Run {
    static constexpr int V = 16 / sizeof(T), A = ALIGN / sizeof(T);
    const T *z;
    int n, head, vectors;
    __device__ __forceinline__ Run(const T *p, int count) : z(p), n(count)
    {
        const int off = (int)((reinterpret_cast<uintptr_t>(p) / sizeof(T)) & (A - 1));
        head = off == 0 ? 0 : min(A - off, count);
        vectors = (count - head) / V;
    }
    __device__ __forceinline__ bool aligned_like(const T *p) const { return ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0; }
    __device__ __forceinline__ int first(int v) const { return head + v * V; }
    template <bool PAST = false> __device__ __forceinline__ Pack<T, V> vector(int v) const { return load_vec<Pack<T, V>, PAST>(z + head + v * V); }
    __device__ __forceinline__ bool before(int t) const { return t < head; }
    __device__ __forceinline__ int behind(int t) const { const int i = head + vectors * V + t; return t < V && i < n ? i : -1; }
    __device__ __forceinline__ bool any(int t) const { return t < head || t < vectors || behind(t) >= 0; }
    // f(score, index) for every score of thread t
    template <typename F> __device__ __forceinline__ void each(int t, F &&f) const
    {
        if (before(t)) f(as_f32(z[t]), t);
        for (int v = t; v < vectors; v += NT) {
            const Pack<T, V> q = vector(v);
#pragma unroll
            for (int e = 0; e < V; ++e) f(as_f32(q.v[e]), first(v) + e);
        }
        const int i = behind(t);
        if (i >= 0) f(as_f32(z[i]), i);
    }
};

constexpr int U = 4;   // vectors of a thread that are on their way together

// A thread's vectors in up to kParts parts of 4 << shift each; part j of thread t has its largest score in tops[j * NT + t].
constexpr int kParts = 8;
struct Parts {
    int shift, count, log;   // log: of a part's vectors, in a single part of those there are
    __device__ __forceinline__ explicit Parts(int vectors) : shift(0)
    {
        const int steps = (vectors + U * NT - 1) / (U * NT);
        while ((steps - 1) >> shift >= kParts) ++shift;
        count = steps == 0 ? 0 : ((steps - 1) >> shift) + 1;
        log = count > 1 || vectors > 2 * NT ? shift + 2 : vectors > NT ? 1 : 0;
        static_assert(U == 4, "");
    }
};

// What thread t makes of its scores; with TOPS, the parts' largest too.
template <bool TOPS, typename T> __device__ __forceinline__ Soft scan(const Run<T> &run, const Parts &parts, float *tops)
{
    constexpr int V = Run<T>::V;
    const int t = threadIdx.x;
    Soft mine = {-3.402823466e38f, 0.f, 0.f};
    if (run.before(t)) { const float z[1] = {as_f32(run.z[t])}; add_scores<1>(mine, z); }
    if (run.behind(t) >= 0) { const float z[1] = {as_f32(run.z[run.behind(t)])}; add_scores<1>(mine, z); }
    int v = t, step = 0;
    float top = -INFINITY;
    for (; v + (U - 1) * NT < run.vectors; v += U * NT) {
        Pack<T, V> q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = run.vector(v + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = as_f32(q[u].v[e]);
            top = fmaxf(top, add_scores<V>(mine, z));
        }
        ++step;
        if (TOPS && (step & ((1 << parts.shift) - 1)) == 0) { tops[((step - 1) >> parts.shift) * NT + t] = top; top = -INFINITY; }
    }
    for (; v < run.vectors; v += NT) {
        const Pack<T, V> q = run.vector(v);
        float z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = as_f32(q.v[e]);
        top = fmaxf(top, add_scores<V>(mine, z));
    }
    // the last part, also where this thread has none of it: another one has
    if (TOPS && step >> parts.shift < parts.count) tops[(step >> parts.shift) * NT + t] = top;
    return mine;
}
// all threads' together, the same for each
__device__ __forceinline__ Soft block_join(Soft mine)
{
    __shared__ Soft part[NT / 64];
    mine = wave_join(mine);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    Soft all = part[0];
    for (int w = 1; w < NT / 64; ++w) join(all, part[w]);
    return all;
}

// The k largest keys of the block's run, best first, to put(rank, key); all threads call it.  `top`: order of the thread's largest
// score, 0 if it has none; `odd`: its scores hold a NaN or +inf.
//
// The maxima of at least k groups of threads reach `least`, so the k largest scores do; only the parts of threads that reach it are looked at again, by
// all threads together, and appended to a list in LDS; each candidate's place is the number of larger ones.  `least` is the k-th largest
// maximum to 16 bits (which is all of a bf16 score's), found bit by bit: a count over the 64 groups of four threads is one comparison of a wavefront.
// About 24 scores reach the 20th of 64 maxima; for more than 32 the threads' own 256 serve, four times the instructions.
// Looking at whole threads' scores again instead of parts: 2047 x 50001 bf16 with 20 leaders 47 -> 55 us, with 64 52 -> 72.
// Where very many scores reach it (equal ones, or ruled-out classes where fewer than k are left) the list holds those above
// it and the first k equal to it by index, and where even that does not fit, k rounds take the largest below the one before: a NaN or +inf in the row, or
// more than 512 - k scores above the k-th largest of the threads' maxima, as where all leaders are neighbours.  That is the slow case: with k = 64 and scores in
// rising order bf16 1 x 131072 118 us (in random order 12.6), 2047 x 50001 1900 (47), fp32 64 (12.6), 102 (85).
template <typename T, typename P>
__device__ __forceinline__ void block_top(const Run<T> &run, const Parts &parts, const float *part_tops, int base, int k, unsigned top, bool odd, P &&put)
{
    constexpr int V = Run<T>::V;
    __shared__ unsigned tops[NT];
    __shared__ unsigned long long list[kCandidates + 8];
    __shared__ unsigned short leaders[NT * kParts];   // thread and part
    __shared__ int count, ties, lead, some_odd;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    tops[t] = top;
    if (t == 0) { count = 0; lead = 0; some_odd = 0; }
    __syncthreads();
    if (odd) some_odd = 1;
    // a group has a thread of each wavefront: scores in rising or falling order lead in neighbouring threads
    const unsigned own[4] = {tops[lane], tops[lane + 64], tops[lane + 128], tops[lane + 192]};
    const unsigned most = max(max(own[0], own[1]), max(own[2], own[3]));
    auto threads_reach = [&](unsigned from) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) n += __popcll(__ballot(own[w] >= from));
        return n;
    };
    unsigned least = 0;
    if (k <= 32) {
        for (unsigned bit = 0x80000000u; bit >= 0x10000u; bit >>= 1)
            if (__popcll(__ballot(most >= (least | bit))) >= k) least |= bit;
    } else {
        for (unsigned bit = 0x80000000u; bit >= 0x10000u; bit >>= 1)
            if (threads_reach(least | bit) >= k) least |= bit;
    }
    auto append = [&](float z, int i, unsigned from) {
        if (order_of(z) >= from) {
            const int at = atomicAdd(&count, 1);
            if (at < kCandidates) list[at] = key_of(z, base + i);
        }
    };
    // a wavefront's vectors (`there`: this lane has one) with one addition: each is a wait
    auto append_vectors = [&](const Pack<T, V> &q, int first, bool there, unsigned from) {
        unsigned order[V];
        int hits = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            order[e] = there ? order_of(as_f32(q.v[e])) : 0u;
            hits += __popcll(__ballot(order[e] >= from));
        }
        if (hits == 0) return;
        int at = 0;
        if (lane == 0) at = atomicAdd(&count, hits);
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const unsigned long long who = __ballot(order[e] >= from);
            const int place = at + __popcll(who & ((1ull << lane) - 1));
            if (order[e] >= from && place < kCandidates) list[place] = (unsigned long long)order[e] << 32 | (unsigned)~(base + first + e);
            at += __popcll(who);
        }
    };
    // scores from `from` on: the single ones by their threads, the vectors of the parts that reach it by everybody
    auto collect = [&](unsigned from) {
        if (top >= from && top != 0) {
            for (int j = 0; j < parts.count; ++j)
                if (order_of(part_tops[j * NT + t]) >= from) leaders[atomicAdd(&lead, 1)] = (unsigned short)(j * NT + t);
            if (run.before(t)) append(as_f32(run.z[t]), t, from);
            if (run.behind(t) >= 0) append(as_f32(run.z[run.behind(t)]), run.behind(t), from);
        }
        __syncthreads();
        const int log = parts.log, total = lead << log;
        static_assert(NT == 256, "");
        for (int i0 = t - lane; i0 < total; i0 += NT) {   // whole wavefronts
            if (*(volatile int *)&count > kCandidates) break;   // it does not fit
            const int i = i0 + lane;
            Pack<T, V> q;
            int v = run.vectors;
            if (i < total) {
                const int l = leaders[i >> log];
                v = (((l >> 8) << log) + (i & ((1 << log) - 1))) * NT + (l & (NT - 1));
            }
            if (v < run.vectors) q = run.vector(v);
            append_vectors(q, run.first(v), v < run.vectors, from);
        }
        __syncthreads();
    };
    least = max(least, 1u);   // 0 is a lane without a vector
    collect(least);
    const bool slow = some_odd != 0;
    bool fits = !slow && count <= kCandidates;
    if (!slow && !fits) {
        // the largest value that k threads' maxima reach, to all its bits
        least = 0;
        for (unsigned bit = 0x80000000u; bit != 0; bit >>= 1)
            if (threads_reach(least | bit) >= k) least |= bit;
        __syncthreads();
        if (t == 0) { count = 0; lead = 0; ties = 0; }
        __syncthreads();
        collect(least + 1);   // no NaN here: least is below all bits
        fits = count <= kCandidates - k;
        if (fits && wave == 0) {   // one wavefront finds the first k in order
            int found = 0;
            const int have = count;
            for (int i0 = 0; i0 < run.n && found < k; i0 += 64) {
                const int i = i0 + lane;
                const float z = i < run.n ? as_f32(run.z[i]) : 0.f;
                const bool hit = i < run.n && order_of(z) == least;
                const unsigned long long hits = __ballot(hit);
                const int at = found + __popcll(hits & ((1ull << lane) - 1));
                if (hit && at < k) list[have + at] = key_of(z, base + i);
                found += __popcll(hits);
            }
            if (lane == 0) ties = min(found, k);
        }
        __syncthreads();
        if (fits && t == 0) count += ties;
        __syncthreads();
    }
    if (fits) {
        const int c = count;
        if (t < 8) list[c + t] = 0;
        __syncthreads();
        for (int i = t; i < c; i += NT) {
            const unsigned long long key = list[i];
            const int rank = larger(list, c, key);
            if (rank < k) put(rank, key);
        }
        for (int r = c + t; r < k; r += NT) put(r, 0ull);   // fewer scores than k
        return;
    }
    unsigned long long last = ~0ull;
    for (int j = 0; j < k; ++j) {
        unsigned long long best = 0;
        run.each(t, [&](float z, int i) {
            const unsigned long long key = key_of(z, base + i);
            if (key < last && key > best) best = key;
        });
        best = wave_top(best);
        __syncthreads();
        if (lane == 0) list[wave] = best;
        __syncthreads();
        last = list[0];
        for (int w = 1; w < NT / 64; ++w) last = last > list[w] ? last : list[w];
        if (t == 0) put(j, last);
    }
}

// log p of a class: the difference from the maximum first, which is exact where it matters, then log s (their sum, lse, cannot hold log s
// where the scores are large).  A row of nothing but ruled-out classes has -inf.
__device__ __forceinline__ float log_p(const Soft &all, float log_s, float score) { return all.s == 0.f ? -INFINITY : (score - all.m) - log_s; }

__device__ __forceinline__ void write_row(const LpArgs &a, int r, const Soft &all, float score, bool valid)
{
    const bool none = all.s == 0.f;
    const float log_s = logf(all.s);
    if (a.lse != nullptr) a.lse[r] = none ? -INFINITY : all.m + log_s;
    if (a.entropy != nullptr) a.entropy[r] = none ? 0.f : log_s - all.t / all.s;
    if (a.logp != nullptr) a.logp[r] = valid ? log_p(all, log_s, score) : 0.f;
}

// Block = (row, split of its classes).  Bound by HBM where there are many rows: 2047 x 50001 bf16 47 us with 20 leaders, 42 without (205 MB, 4.9 TB/s); one
// row of 131072 is two kernels' waits, 9.9 us.  With at most 80 scalar registers eight wavefronts share a SIMD, with more seven: 2048 x 5001 has eight
// blocks to a compute unit, and they ran in two turns (12.1 -> 14.7 us).
template <typename T>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_num_sgpr(80))) void k_logprobs(LpArgs a)
{
    const int t = threadIdx.x;
    const int r = blockIdx.x / a.splits, split = blockIdx.x - r * a.splits;
    const int c0 = split * a.seg;
    const T *row = (const T *)a.z + (size_t)r * a.stride;
    const Run<T> run(row + c0, min(a.seg, a.classes - c0));
    __shared__ float tops[kParts * NT];
    const Parts parts(run.vectors);
    const Soft mine = a.k > 0 ? scan<true>(run, parts, tops) : scan<false>(run, parts, tops);
    const unsigned top = !run.any(t) ? 0u : mine.s == 0.f ? order_of(-INFINITY) : order_of(mine.m);
    const bool odd = mine.s != mine.s;
    const Soft all = block_join(mine);
    const size_t at = (size_t)r * a.splits + split;
    if (t == 0 && a.splits > 1) a.part[at] = all;
    if (t == 0 && a.splits == 1) {
        const int id = a.logp != nullptr ? a.ids[r] : -1;
        const bool valid = id >= 0 && id < a.classes;
        write_row(a, r, all, valid ? as_f32(row[id]) : 0.f, valid);
    }
    if (a.k == 0) return;
    const float log_s = logf(all.s);
    block_top(run, parts, tops, c0, a.k, top, odd, [&](int rank, unsigned long long key) {
        if (a.splits > 1) a.part_top[at * a.k + rank] = key;
        else {
            a.top_ids[at * a.k + rank] = index_of(key);
            a.top_logp[at * a.k + rank] = log_p(all, log_s, score_of(key));
        }
    });
}

// Joins the splits of a row.  Block = row.  Each split's keys are in order: with S splits the `need`-th largest of their `each`-th
// keys, need * each >= k, bounds the k-th largest from below; with about half of the splits (the least of all of them would bound little).
// 3.8 us for 32 splits with 20 leaders: a launch, one wait for what other dies wrote, the search.
template <typename T>
__global__ __launch_bounds__(NT) void k_logprobs_join(LpArgs a)
{
    __shared__ unsigned long long heads[kMaxSplits], list[kMaxSplits * DP_LOGPROBS_MAX_TOP + 8], bound;
    __shared__ int count;
    constexpr int kAhead = 8;   // keys that a thread asks for before it knows which ones matter
    const int t = threadIdx.x, r = blockIdx.x;
    const int each = (2 * a.k + a.splits - 1) / a.splits, need = each > 0 ? (a.k + each - 1) / each : 0;
    const int total = a.splits * a.k;
    const unsigned long long *keys = a.part_top + (size_t)r * total;
    Soft mine = {-3.402823466e38f, 0.f, 0.f};
    const int s = t & 63;
    static_assert(kMaxSplits == 64, "one per lane");
    if (s < a.splits) mine = a.part[(size_t)r * a.splits + s];
    if (t < a.splits && a.k > 0) heads[t] = keys[(size_t)t * a.k + each - 1];
    unsigned long long ahead[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) ahead[u] = t + u * NT < total ? keys[t + u * NT] : 0ull;
    bool valid = false;
    float score = 0.f;
    if (t == NT - 1 && a.logp != nullptr) {
        const int id = a.ids[r];
        valid = id >= 0 && id < a.classes;
        if (valid) score = as_f32(((const T *)a.z)[(size_t)r * a.stride + id]);
    }
    if (t == 0) { count = 0; bound = 0; }
    __syncthreads();
    const Soft all = wave_join(mine);   // every wavefront the same
    if (t == NT - 1) write_row(a, r, all, score, valid);
    if (a.k == 0) return;
    if (t < a.splits) {
        const unsigned long long head = heads[t];
        int above = 0;
        for (int i = 0; i < a.splits; ++i) above += heads[i] > head || (heads[i] == head && i < t);   // equal only where 0, no key
        if (above == need - 1) bound = head;
    }
    __syncthreads();
    const unsigned long long least = bound;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (ahead[u] != 0 && ahead[u] >= least) list[atomicAdd(&count, 1)] = ahead[u];
    for (int i = t + kAhead * NT; i < total; i += NT) {
        const unsigned long long key = keys[i];
        if (key != 0 && key >= least) list[atomicAdd(&count, 1)] = key;
    }
    __syncthreads();
    const int c = count;
    if (t < 8) list[c + t] = 0;
    __syncthreads();
    const float log_s = logf(all.s);
    for (int i = t; i < c; i += NT) {
        const unsigned long long key = list[i];
        const int rank = larger(list, c, key);
        if (rank < a.k) {
            a.top_ids[(size_t)r * a.k + rank] = index_of(key);
            a.top_logp[(size_t)r * a.k + rank] = log_p(all, log_s, score_of(key));
        }
    }
}

// Short rows: a wavefront each, the row in registers (class lane + 64 j in slot j), the same steps without a barrier.  A block per
// row of 1000 classes spends its time on barriers and idle threads (bf16, 4096 rows, five leaders: 15.6 -> 6.9 us, 4.6 of them without leaders: vector instructions).
constexpr int kRowCandidates = 256;   // of a row, in LDS; a multiple of 64
template <typename T, int R>
__global__ __launch_bounds__(NT) void k_logprobs_rows(LpArgs a)
{
    __shared__ unsigned long long lists[NT / 64][kRowCandidates + 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = blockIdx.x * (NT / 64) + wave;
    if (r >= a.rows) return;   // whole wavefronts; there are no barriers
    const T *z = (const T *)a.z + (size_t)r * a.stride;
    float v[R];
#pragma unroll
    for (int j = 0; j < R; ++j) v[j] = as_f32(z[min(lane + 64 * j, a.classes - 1)]);
    const int id = a.logp != nullptr ? a.ids[r] : -1;
    const bool valid = id >= 0 && id < a.classes;
    const float score = as_f32(z[valid ? id : 0]);
#pragma unroll
    for (int j = 0; j < R; ++j) v[j] = lane + 64 * j < a.classes ? v[j] : -INFINITY;
    Soft mine = {-3.402823466e38f, 0.f, 0.f};
    add_scores<R>(mine, v);
    const Soft all = wave_join(mine);
    if (lane == 0) write_row(a, r, all, score, valid);
    if (a.k == 0) return;
    const float log_s = logf(all.s);
    auto put = [&](int rank, unsigned long long key) {
        a.top_ids[(size_t)r * a.k + rank] = index_of(key);
        a.top_logp[(size_t)r * a.k + rank] = log_p(all, log_s, score_of(key));
    };
    unsigned long long *list = lists[wave];
    const int per_lane = (a.classes - lane + 63) / 64;   // classes of this lane, may be 0
    if (all.s == all.s) {   // no NaN or +inf: the lanes' maxima are what they seem
        // by the lanes' maxima as long as half of the lanes may stay below, else by those of their even and odd classes' slots
        unsigned least = 0;
        if (a.k <= 32) {
            const unsigned top = per_lane <= 0 ? 0u : mine.s == 0.f ? order_of(-INFINITY) : order_of(mine.m);
            for (unsigned bit = 0x80000000u; bit >= 0x10000u; bit >>= 1)
                if (__popcll(__ballot(top >= (least | bit))) >= a.k) least |= bit;
        } else {
            float even = v[0], odd = v[1];   // absent ones are -inf
#pragma unroll
            for (int j = 2; j < R; j += 2) { even = fmaxf(even, v[j]); odd = fmaxf(odd, v[j + 1]); }
            const unsigned top0 = per_lane > 0 ? order_of(even) : 0u, top1 = per_lane > 1 ? order_of(odd) : 0u;
            for (unsigned bit = 0x80000000u; bit >= 0x10000u; bit >>= 1)
                if (__popcll(__ballot(top0 >= (least | bit))) + __popcll(__ballot(top1 >= (least | bit))) >= a.k) least |= bit;
        }
        const unsigned long long below = (1ull << lane) - 1;
        int c = 0;
        auto append = [&](bool hit, int j) {
            const unsigned long long hits = __ballot(hit);
            if (hits == 0) return;
            const int at = c + __popcll(hits & below);
            if (hit && at < kRowCandidates) list[at] = key_of(v[j], lane + 64 * j);
            c += __popcll(hits);
        };
        // the same bound as a score: one comparison, where the order of a score is six operations
        const float bound = least <= order_of(-INFINITY) ? -INFINITY : score_of((unsigned long long)least << 32);
#pragma unroll
        for (int j = 0; j < R; ++j) append(j < per_lane && v[j] >= bound, j);
        if (c > kRowCandidates) {   // the k-th largest score itself, those above it, and the first equal to it by index
            unsigned order[R];
#pragma unroll
            for (int j = 0; j < R; ++j) order[j] = j < per_lane ? order_of(v[j]) : 0u;
            auto reach = [&](unsigned from) {
                int n = 0;
#pragma unroll
                for (int j = 0; j < R; ++j) n += __popcll(__ballot(order[j] >= from));
                return n;
            };
            least = 0;
            for (unsigned bit = 0x80000000u; bit != 0; bit >>= 1)
                if (reach(least | bit) >= a.k) least |= bit;
            const int above = reach(least + 1);   // no NaN here: least is below all bits
            int equal = above;
            c = 0;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const unsigned long long ties = __ballot(order[j] == least);
                append(order[j] > least || (order[j] == least && equal + __popcll(ties & below) < a.k), j);
                equal += __popcll(ties);
            }
        }
        if (lane < 8) list[c + lane] = 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the list as all lanes wrote it
        for (int i = lane; i < c; i += 64) {
            const unsigned long long key = list[i];
            const int rank = larger(list, c, key);
            if (rank < a.k) put(rank, key);
        }
        return;
    }
    unsigned long long last = ~0ull;   // the largest below the one before
    for (int k = 0; k < a.k; ++k) {
        unsigned long long best = 0;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const unsigned long long key = key_of(v[j], lane + 64 * j);
            if (j < per_lane && key < last && key > best) best = key;
        }
        last = wave_top(best);
        if (lane == 0) put(k, last);
    }
}
constexpr int kShortRow = 1024;

struct LpGradArgs {
    const void *z;
    const int *ids;
    const float *lse, *entropy, *dlogp, *dentropy;
    void *dz;
    int rows, classes, splits, seg;
    long long stride;
};

// exp(d), d in [-128, 0] or a little above.  For bf16 gradients the product is enough: p is off by 6e-8 of |d|, the output's rounding by 4e-3.
template <typename T> __device__ __forceinline__ float exp_of(float d) { return sizeof(T) == 2 ? exp_d(d) : exp_full(d); }

// A row's gradient: p (-dl - de (log p + h)) = exp(d) (k0 - k1 d), d = z - lse, and dl more for the given class.
// p = exp(d) as long as lse holds its row's sum well enough: its rounding is a relative error of every p, 2^-21 below 16 (that of d itself), but 2^-17 at
// 250, where 1 - p of a confident row's class is lost.  From 16 on, p = exp(d) / S with S = sum of exp(d), which is 1 up to that error (or up to the
// number of classes, where lse is too large to hold any of it).
// sum(): S, asked for by all threads of the row or none.  It is in 64 bits: however the row is spread over blocks, it is the same to the last bit of 32.
__device__ __forceinline__ bool sums_anew(float lse) { return fabsf(lse) > 16.f && lse != -INFINITY; }
template <typename T> struct RowGrad {
    float shift, k0, k1, dl;
    int id;   // -1: none
    template <typename F> __device__ __forceinline__ RowGrad(const LpGradArgs &a, int r, F &&sum)
    {
        const float lse = a.lse[r], h = a.entropy != nullptr ? a.entropy[r] : 0.f;
        const bool none = lse == -INFINITY;
        id = a.ids != nullptr ? a.ids[r] : -1;
        const bool valid = id >= 0 && id < a.classes && !none;
        dl = a.dlogp != nullptr && valid ? a.dlogp[r] : 0.f;
        if (!valid) id = -1;
        const float de = a.dentropy != nullptr && !none ? a.dentropy[r] : 0.f;
        float log_s = 0.f, scale = lse == lse ? 1.f : lse;   // a NaN in the row makes all of it NaN
        shift = none ? 0.f : lse;                            // none: every score is -inf, p = 0
        if (sums_anew(lse)) {
            const float s = (float)sum(lse);
            log_s = logf(s);
            scale = 1.f / s;
        }
        k1 = de * scale;
        k0 = -fmaf(de, h - log_s, dl) * scale;
    }
    __device__ __forceinline__ float operator()(float z) const
    {
        const float d = fmaxf(z - shift, -128.f);   // exp(d) is 0 long before -128; k1 d must not be infinite then
        return exp_of<T>(d) * fmaf(-k1, d, k0);
    }
};

// Short rows: a wavefront each, the row in registers (class lane + 64 j in slot j).  A block to each: bf16 4096 x 1000 6.8 -> 5.8 us, 16384 x 1000
// 17.9 -> 14.0 (65 MB, 4.7 TB/s), 8192 x 512 9.3 -> 5.6, fp32 65536 x 10 51 -> 9.8.
template <typename T, int R>
__global__ __launch_bounds__(NT) void k_logprobs_grad_rows(LpGradArgs a)
{
    const int lane = threadIdx.x & 63, r = blockIdx.x * (NT / 64) + (int)(threadIdx.x >> 6);
    if (r >= a.rows) return;
    const T *z = (const T *)a.z + (size_t)r * a.stride;
    T *out = (T *)a.dz + (size_t)r * a.stride;
    float v[R];
#pragma unroll
    for (int j = 0; j < R; ++j) v[j] = as_f32(z[min(lane + 64 * j, a.classes - 1)]);
    const RowGrad<T> grad(a, r, [&](float lse) {
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < R; ++j) s += lane + 64 * j < a.classes ? (double)exp_d(v[j] - lse) : 0.0;
        return wave_sum_fast(s);
    });
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int i = lane + 64 * j;
        if (i < a.classes) out[i] = from_f32<T>(grad(v[j]) + (i == grad.id ? grad.dl : 0.f));
    }
}

// Sum of exp(z - lse) over the block's run, the same for all threads.
template <typename T> __device__ __forceinline__ double block_sum(const Run<T> &run, float lse)
{
    constexpr int V = Run<T>::V;
    __shared__ double part[NT / 64];
    const int t = threadIdx.x;
    double s = 0.0;
    auto add = [&](T z) { s += (double)exp_d(as_f32(z) - lse); };
    if (run.before(t)) add(run.z[t]);
    if (run.behind(t) >= 0) add(run.z[run.behind(t)]);
    int v = t;
    for (; v + (U - 1) * NT < run.vectors; v += U * NT) {
        Pack<T, V> q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = run.vector(v + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) add(q[u].v[e]);
    }
    for (; v < run.vectors; v += NT) {
        const Pack<T, V> q = run.vector(v);
#pragma unroll
        for (int e = 0; e < V; ++e) add(q.v[e]);
    }
    s = wave_sum_fast(s);
    if ((t & 63) == 0) part[t >> 6] = s;
    __syncthreads();
    s = part[0];
    for (int w = 1; w < NT / 64; ++w) s += part[w];
    return s;
}

// Where a row is split, the splits' sums of rows that are summed anew lie in dz itself until it is written: each split's part of dz has those of all
// splits in front (from a multiple of 8 bytes on), and only the block that reads them there writes over them.  Every block summing the whole row instead: 16 x 131072
// bf16 41 us; so 7.5, 3.7 of them this kernel's.
__device__ __forceinline__ double *sums_in_front(void *part) { return reinterpret_cast<double *>((reinterpret_cast<uintptr_t>(part) + 7) & ~(uintptr_t)7); }

template <typename T>
__global__ __launch_bounds__(NT) void k_logprobs_grad_sums(LpGradArgs a)
{
    const int t = threadIdx.x, r = blockIdx.x / a.splits, split = blockIdx.x - r * a.splits, c0 = split * a.seg;
    const float lse = a.lse[r];
    if (!sums_anew(lse)) return;
    const double s = block_sum(Run<T>((const T *)a.z + (size_t)r * a.stride + c0, min(a.seg, a.classes - c0)), lse);
    if (t < a.splits) sums_in_front((T *)a.dz + (size_t)r * a.stride + (size_t)t * a.seg)[split] = s;
}

// Block = (row, split of its classes); in place a row is one block's, which may have to read it twice.
// p (log p + entropy) is 0 where p is, also for log p = -inf.
// Bound by HBM: 2047 x 50001 bf16 64 us (411 MB, 6.4 TB/s); with its rows summed anew 97 for 78, nothing of them in the caches.
// PAST: dz goes past the caches: more than 32 MB of it would push the scores out while they are read, and be written back while the next
// kernel reads (2047 x 50001 bf16: 71 -> 69 us, and the next forward 69 -> 50).  So do the scores, whose last reading this is (66 -> 64;
// 4095 x 50001 155 -> 133).  The forward's reading stays in the caches for this one: past them it would cost 2047 x 50001 12 us here for 5 more there.
template <typename T, bool PAST>
__global__ __launch_bounds__(NT) void k_logprobs_grad(LpGradArgs a)
{
    constexpr int V = Run<T>::V;
    const int t = threadIdx.x, r = blockIdx.x / a.splits, c0 = (blockIdx.x - r * a.splits) * a.seg;
    const T *row = (const T *)a.z + (size_t)r * a.stride + c0;
    T *out = (T *)a.dz + (size_t)r * a.stride + c0;
    // from a line's boundary on, a wavefront's kilobyte is eight whole lines, also to store (2047 x 50001 bf16: 90 -> 81 us; reads alone do not care)
    const Run<T, 128> run(row, min(a.seg, a.classes - c0));
    const RowGrad<T> row_grad(a, r, [&](float lse) {
        if (a.splits == 1) return block_sum(Run<T>(row, a.classes), lse);
        static_assert(kMaxSplits == 64, "one per lane");
        const double s = wave_sum_fast((t & 63) < a.splits ? sums_in_front(out)[t & 63] : 0.0);
        __syncthreads();   // everybody has read before anybody writes there
        return s;
    });
    const int at = row_grad.id < 0 ? -1 : row_grad.id - c0;   // the given class in this run, if in [0, n)
    const float dl = row_grad.dl;
    auto grad = [&](float z) { return row_grad(z); };
    auto single = [&](int i) { out[i] = from_f32<T>(grad(as_f32(run.z[i])) + (i == at ? dl : 0.f)); };
    auto vector = [&](int v, const Pack<T, V> &q) {
        float g[V];
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = grad(as_f32(q.v[e]));
        const int e0 = at - run.first(v);
        if (e0 >= 0 && e0 < V)
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] += e == e0 ? dl : 0.f;
        Pack<T, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.v[e] = from_f32<T>(g[e]);
        store_vec<Pack<T, V>, PAST>(out + run.first(v), o);
    };
    if (run.aligned_like(out)) {
        if (run.before(t)) single(t);
        if (run.behind(t) >= 0) single(run.behind(t));
        int v = t;
        for (; v + (U - 1) * NT < run.vectors; v += U * NT) {
            Pack<T, V> q[U];
#pragma unroll
            for (int u = 0; u < U; ++u) q[u] = run.template vector<PAST>(v + u * NT);
#pragma unroll
            for (int u = 0; u < U; ++u) vector(v + u * NT, q[u]);
        }
        for (; v < run.vectors; v += NT) vector(v, run.template vector<PAST>(v));
    } else {   // dz at another offset from a 16-byte boundary than z
        for (int i = t; i < run.n; i += NT) single(i);
    }
}

// Splits of a row, in whole vectors, so that all splits of a row are aligned alike: about four blocks per compute unit, at least half of `least`
// classes each less 8 for every split (2048: the shortest last one has 1017, and the gradient's sums in front of it take 519 bytes).
void split_rows(int rows, int classes, int least, int &splits, int &seg)
{
    const int s = std::max(1, std::min({(1024 + rows - 1) / rows, (classes + least - 1) / least, kMaxSplits}));
    seg = ((classes + s - 1) / s + 7) / 8 * 8;
    splits = (classes + seg - 1) / seg;
}
// Forward, splits cost a second kernel and its wait: one block to a row where there are rows for every compute unit, and for rows that a block
// reads in the time of that (bf16, five alternatives, us, split / not: 1 x 16384 8.5 / 6.5, 1 x 32000 8.7 / 8.8; 300 x 48000 16.2 / 15.5,
// 256 x 131072 21.0 / 22.3; 512 x 131072 34 / 32.4; fp32, with twice the bytes but as many scores to weigh, 1 x 16384 8.1 / 7.3, 1 x 24576 8.4 / 8.7, 64 x 24576 9.6 / 8.8,
// 64 x 32000 10.0 / 10.1, 300 x 65536 21.8 / 20.5, 300 x 131072 33.5 / 33.9: the same limits).
void split_forward(int rows, int classes, int &splits, int &seg)
{
    splits = 1;
    seg = classes;
    if (rows < 512 && classes > (rows >= 256 ? 65536 : 24576)) split_rows(rows, classes, 4096, splits, seg);
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

// keys first: they need the wider alignment
size_t top_bytes(int rows, int splits, int k) { return (size_t)rows * splits * k * sizeof(unsigned long long); }
size_t part_bytes(int rows, int splits, int k) { return splits == 1 ? 0 : top_bytes(rows, splits, k) + (size_t)rows * splits * sizeof(Soft); }

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
    if (check_desc(desc) != DP_OK || desc->rows == 0) return 0;
    int splits, seg;
    split_forward(desc->rows, desc->classes, splits, seg);
    return part_bytes(desc->rows, splits, desc->top_k);
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
    LpArgs a = {z, ids, logp, entropy, lse, top_logp, top_ids, nullptr, nullptr, d.rows, d.classes, d.top_k, 1, d.classes, stride_of(d)};
    split_forward(d.rows, d.classes, a.splits, a.seg);
    const size_t need = part_bytes(d.rows, a.splits, d.top_k);
    if (need > 0 && (ws == nullptr || ws_bytes < need)) {
        dp_set_error("log-probabilities need %zu workspace bytes, got %zu", need, ws == nullptr ? (size_t)0 : ws_bytes);
        return DP_ERR_WORKSPACE;
    }
    if (!aligned16(ws)) { dp_set_error("log-probabilities: the workspace must be 16-byte aligned"); return DP_ERR_BAD_DESC; }
    a.part_top = (unsigned long long *)ws;
    a.part = (Soft *)((char *)ws + top_bytes(d.rows, a.splits, d.top_k));
    const bool bf = d.io_dtype == DP_BF16;
    hipStream_t st = (hipStream_t)hip_stream;
    if (d.classes <= kShortRow) {
        const dim3 grid((d.rows + NT / 64 - 1) / (NT / 64));
        auto *kernel = d.classes <= 128 ? (bf ? k_logprobs_rows<bf16_t, 2> : k_logprobs_rows<float, 2>) : d.classes <= 512 ? (bf ? k_logprobs_rows<bf16_t, 8> : k_logprobs_rows<float, 8>) :
                       (bf ? k_logprobs_rows<bf16_t, 16> : k_logprobs_rows<float, 16>);
        hipLaunchKernelGGL(kernel, grid, dim3(NT), 0, st, a);
        return launched("log-probabilities");
    }
    hipLaunchKernelGGL(bf ? k_logprobs<bf16_t> : k_logprobs<float>, dim3((unsigned)d.rows * a.splits), dim3(NT), 0, st, a);
    if (a.splits > 1) hipLaunchKernelGGL(bf ? k_logprobs_join<bf16_t> : k_logprobs_join<float>, dim3(d.rows), dim3(NT), 0, st, a);
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
    const bool bf = d.io_dtype == DP_BF16;
    LpGradArgs a = {z, ids, lse, entropy, dlogp, dentropy, dz, d.rows, d.classes, 1, d.classes, stride_of(d)};
    hipStream_t st = (hipStream_t)hip_stream;
    if (d.classes <= kShortRow) {
        const dim3 grid((d.rows + NT / 64 - 1) / (NT / 64));
        auto *kernel = d.classes <= 128 ? (bf ? k_logprobs_grad_rows<bf16_t, 2> : k_logprobs_grad_rows<float, 2>) :
                       d.classes <= 512 ? (bf ? k_logprobs_grad_rows<bf16_t, 8> : k_logprobs_grad_rows<float, 8>) :
                       (bf ? k_logprobs_grad_rows<bf16_t, 16> : k_logprobs_grad_rows<float, 16>);
        hipLaunchKernelGGL(kernel, grid, dim3(NT), 0, st, a);
        return launched("log-probabilities' gradient");
    }
    // 256 x 48000 bf16: 9.5 us, one block to a row 11.9.  In place there is no room for the splits' sums, and a row that a block sums anew has to be its own until then:
    // 16 x 131072 14.9 us in place, 5.0 beside (7.5 with all rows summed anew)
    if (dz != z) split_rows(d.rows, d.classes, 2048, a.splits, a.seg);
    const bool past = (int64_t)d.rows * d.classes * (bf ? 2 : 4) > (32 << 20);
    auto *kernel = bf ? (past ? k_logprobs_grad<bf16_t, true> : k_logprobs_grad<bf16_t, false>) : (past ? k_logprobs_grad<float, true> : k_logprobs_grad<float, false>);
    const dim3 grid((unsigned)d.rows * a.splits);
    if (a.splits > 1) hipLaunchKernelGGL(bf ? k_logprobs_grad_sums<bf16_t> : k_logprobs_grad_sums<float>, grid, dim3(NT), 0, st, a);
    hipLaunchKernelGGL(kernel, grid, dim3(NT), 0, st, a);
    return launched("log-probabilities' gradient");
}
