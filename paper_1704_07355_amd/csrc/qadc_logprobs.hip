// Log probabilities of given tokens with the entropy and the likeliest alternatives, and their gradient, on gfx950.
//
// With x = scale logits, m = max x and e = exp(x - m): lse = m + log sum e, entropy = log sum e - sum e (x - m) / sum e.  A
// thread keeps (m, s, w) = (largest logit, sum e, sum e (x - m) / log 2) of what it has read and rescales s and w where m grows,
// so that a row is read once; threads and workgroups are joined the same way.
//
// The alternatives are the k largest under one 64-bit key: the logit's bits made monotone above, the complement of the token
// below.  While the row streams by, only the largest logit of every block (32 logits of one thread) is kept.  The k-th largest of
// the threads' largest logits bounds the k-th logit from below, since k different logits reach it; the few blocks that reach it
// are read again, from the cache, and what reaches it is ordered.  Where many logits are equal to the bound, or a mask leaves fewer
// than k threads any, it is those above it, and the first of those equal to it in the row (131072 bfloat16 logits of which a mask
// leaves five, 20 alternatives: 17 us; with all that reach the bound collected first 140, and 200 in a row, 50 of them, 374 for 24).
//
// Bound by memory where there are many rows: 4096 x 65536 bfloat16 86 us (537 MB at 6.2 TB/s), its gradient 171 (1.07 GB at
// 6.3); where there are few by the join's one workgroup a row, which takes its steps one after the other: 131072 logits with 20
// alternatives 4 us for the parts and 10 for the join, 64 x 50021 with 50 alternatives 5 and 13.  (The parts and joins are kernels'
// times by the profiler; all other figures in this file are calls one after the other: 16 and 17.5 us for these two.)

#include <algorithm>
#include <type_traits>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int LP_WG = 256;
constexpr int LP_BLOCK = 32;                  // logits of a thread whose largest is kept
constexpr int LP_CHUNK = LP_WG * LP_BLOCK;    // logits of a workgroup at a time
constexpr int LP_LDS_BLOCKS = 48 * LP_WG;     // blocks of a row whose largest logits fit in LDS: 393216 logits
constexpr int LP_LIST = 1024;                 // candidates for the alternatives
constexpr int LP_READ = 512;                  // blocks that are read again by all threads together
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// A logit's bits in the order of the alternatives: -0 and +0 are equal, a NaN comes first.  0 is below every logit.
__device__ __forceinline__ uint32_t logit_bits(float logit)
{
    uint32_t u = __float_as_uint(logit + 0.0f);
    if (logit != logit) u = 0x7ffffffeu;  // (something is always above)
    return (int32_t)u < 0 ? ~u : u | 0x80000000u;
}
constexpr uint32_t MASKED = 0x007fffffu;  // of -inf, below every other logit
// (logit descending, token ascending) as one number, larger first.
__device__ __forceinline__ uint64_t alt_key(uint32_t bits, uint32_t token) { return (uint64_t)bits << 32 | (uint32_t)~token; }
__device__ __forceinline__ float alt_logit(uint64_t key)
{
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float((int32_t)u < 0 ? u & 0x7fffffffu : ~u);
}

// Statistics of a part of a row: e = 2^(c (logit - m)), c = scale / log 2, t = c (logit - m).
struct Stats {
    float m, s, w;  // largest logit, sum of e, sum of e t
};

// What a part whose largest logit is m has to be shifted by to be relative to `to` (>= m).
__device__ __forceinline__ float shift_of(float m, float to, float c)
{
    return m == to ? 0.0f : m == -INFINITY ? -INFINITY : c * (m - to);
}
__device__ __forceinline__ void rescale(Stats &a, float to, float c)
{
    const float t = shift_of(a.m, to, c), f = exp2_fast(t);
    a.w = f * fmaf(fmaxf(t, -2000.0f), a.s, a.w);  // (an empty part has s = w = 0: no infinity times zero)
    a.s *= f;
    a.m = to;
}
__device__ __forceinline__ Stats join(Stats a, Stats b, float c)
{
    const float m = fmaxf(a.m, b.m);
    rescale(a, m, c);
    rescale(b, m, c);
    return {m, a.s + b.s, a.w + b.w};
}

// Adds the LP_BLOCK logits of a thread; *top becomes the largest.  True: there was a NaN, which fmaxf passes over, or +inf.
__device__ __forceinline__ bool add_block(Stats &st, const float (&x)[LP_BLOCK], float c, float *top)
{
    float v = x[0];
#pragma unroll
    for (int e = 1; e < LP_BLOCK; ++e) v = fmaxf(v, x[e]);
    const float m = fmaxf(st.m, v), m0 = m == -INFINITY ? 0.0f : m;
    float s[2] = {0.0f, 0.0f}, w[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < LP_BLOCK; ++i) {
        const float t = c * (x[i] - m0), e = exp2_fast(t);
        s[i & 1] += e;
        w[i & 1] = fmaf(e, fmaxf(t, -2000.0f), w[i & 1]);  // (a masked logit: zero times something finite)
    }
    const float sum = s[0] + s[1];
    rescale(st, m, c);
    st.s += sum;
    st.w += w[0] + w[1];
    *top = v;
    return sum != sum;
}

// The logits of block (chunk, thread): LP_BLOCK / N packs, those of a wavefront side by side.  Packs lie at multiples of 16
// bytes in memory: a row that does not begin at one has its first pack begin `lead` logits before it (packs across those
// multiples took a quarter longer: 4096 rows of 50021 bfloat16 logits 92 us for 75).
template <typename T>
__device__ __forceinline__ int64_t pack_at(int64_t chunk, int u, int lead)
{
    return chunk * LP_CHUNK + ((int64_t)u * LP_WG + threadIdx.x) * Pack<T>::N - lead;
}
// A pack that may begin before the row or end behind it; `fill` there.
template <typename T>
__device__ __forceinline__ typename Pack<T>::V load_edge(const T *row, int64_t at, int64_t V, float fill)
{
    constexpr int N = Pack<T>::N;
    if (at >= 0 && at + N <= V) return *reinterpret_cast<const typename Pack<T>::V *>(row + at);
    typename Pack<T>::V p = (T)fill;
    if (at < V) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (at + e >= 0 && at + e < V) p[e] = row[at + e];
    }
    return p;
}
__device__ __forceinline__ int64_t chunks_of(int64_t V, int lead) { return (V + lead + LP_CHUNK - 1) / LP_CHUNK; }
template <typename T>
__device__ __forceinline__ void load_block(const T *row, int64_t chunk, int V, int lead, float (&x)[LP_BLOCK])
{
    constexpr int N = Pack<T>::N, PACKS = LP_BLOCK / N;
    typename Pack<T>::V p[PACKS];
    if ((chunk > 0 || lead == 0) && (chunk + 1) * LP_CHUNK - lead <= V) {  // (the same in all threads: loads without a wait)
#pragma unroll
        for (int u = 0; u < PACKS; ++u)
            p[u] = __builtin_nontemporal_load(reinterpret_cast<const typename Pack<T>::V *>(row + pack_at<T>(chunk, u, lead)));
    } else {
#pragma unroll
        for (int u = 0; u < PACKS; ++u) p[u] = load_edge(row, pack_at<T>(chunk, u, lead), V, -INFINITY);
    }
#pragma unroll
    for (int i = 0; i < LP_BLOCK; ++i) x[i] = (float)p[i / N][i % N];
}

// A block's largest logit in the order of the alternatives (0: it has none), where `v` is the largest that is no NaN.
template <typename T>
__device__ __forceinline__ uint32_t block_top(const T *row, int64_t chunk, int V, int lead, float v, bool odd)
{
    uint32_t bits = pack_at<T>(chunk, 0, lead) < V ? logit_bits(v) : 0u;  // (a pack before the row ends in it)
    if (odd)
#pragma unroll 1
        for (int u = 0; u < LP_BLOCK / Pack<T>::N; ++u)
#pragma unroll 1
            for (int e = 0; e < Pack<T>::N; ++e) {
                const int64_t at = pack_at<T>(chunk, u, lead) + e;
                if (at >= 0 && at < V) bits = max(bits, logit_bits((float)row[at]));
            }
    return bits;
}

// Log probabilities of a row's logits: scale (logit - m) - log s, which is as near for large logits as for small ones (as
// scale logit - lse those around 1000 were off by 6e-5), and is finite where scale m is not.
struct Row {
    float scale, m, log_s;
    bool none;  // a mask has left nothing
    __device__ __forceinline__ float log_p(float logit) const { return none ? -INFINITY : fmaf(scale, logit - m, -log_s); }
};

struct StatsLds {
    float m[LP_WG / WAVE], s[LP_WG / WAVE], w[LP_WG / WAVE];
};
struct AltLds {
    uint64_t list[LP_LIST];
    uint64_t kept[QADC_MAX_ALTERNATIVES];
    __attribute__((aligned(16))) uint32_t tops[LP_WG];  // read four at a time
    uint32_t blocks[LP_READ];
    uint32_t counts[2][LP_WG / WAVE];
    uint32_t count, block_count, bound;
};
static_assert(alignof(AltLds) == 16, "the largest logits are read 16 bytes at a time");
struct NoLds {};

// The threads' statistics joined, in every thread.
__device__ __forceinline__ Stats group_stats(Stats a, float c, StatsLds &lds)
{
    const float m = wave_max(a.m);
    rescale(a, m, c);
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    __syncthreads();
    if (lane_id() == 0) {
        lds.m[threadIdx.x >> 6] = a.m;
        lds.s[threadIdx.x >> 6] = a.s;
        lds.w[threadIdx.x >> 6] = a.w;
    }
    __syncthreads();
    a = {lds.m[0], lds.s[0], lds.w[0]};
#pragma unroll
    for (int v = 1; v < LP_WG / WAVE; ++v) a = join(a, Stats{lds.m[v], lds.s[v], lds.w[v]}, c);
    return a;
}

struct Out {
    const int32_t *tokens;
    int nt, k;
    float *logp, *lse, *entropy;
    uint32_t *top_idx;
    float *top_logp;
};

// The sum of a count that is equal within a wavefront, in every thread; `turn` alternates between calls.
__device__ __forceinline__ uint32_t group_count(uint32_t c, AltLds &lds, int turn)
{
    if (lane_id() == 0) lds.counts[turn & 1][threadIdx.x >> 6] = c;
    __syncthreads();
    uint32_t total = 0;
#pragma unroll
    for (int w = 0; w < LP_WG / WAVE; ++w) total += lds.counts[turn & 1][w];
    return total;
}

// f(chunk, its block's largest logit) for every block of this thread, the first FIRST of which it has in registers; beyond them
// eight in flight.
template <int FIRST, typename F, typename G>
__device__ __forceinline__ void each_top(int64_t chunks, const uint32_t (&first)[FIRST + 1], F top_of, G f)
{
#pragma unroll
    for (int j = 0; j < FIRST; ++j) f((int64_t)j, first[j]);  // (0 where there is no block)
    for (int64_t j = FIRST; j < chunks; j += 8) {
        uint32_t t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = j + i < chunks ? top_of(j + i) : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) f(j + i, t[i]);
    }
}
// The k alternatives of a row; top_of(chunk) is the largest logit of this thread's block.
template <int FIRST, typename T, typename F>
__device__ void write_alternatives(const T *row, int V, int lead, int64_t chunks, int k, Row of,
                                   uint32_t *top_idx, float *top_logp, AltLds &lds, const uint32_t (&first)[FIRST + 1], F top_of)
{
    constexpr int N = Pack<T>::N, PACKS = LP_BLOCK / N;
    uint32_t top = 0;
    each_top<FIRST>(chunks, first, top_of, [&](int64_t, uint32_t t) { top = max(top, t); });
    if (threadIdx.x == 0) {
        lds.count = 0;
        lds.block_count = 0;
        lds.bound = ~0u;
    }
    lds.tops[threadIdx.x] = top;
    __syncthreads();
    // The k-th largest of the threads' largest logits is the least that fewer than k of them exceed.
    int above = 0;
#pragma unroll 8
    for (int i = 0; i < LP_WG; i += 4) {
        const uint4 t = *reinterpret_cast<const uint4 *>(&lds.tops[i]);
        above += (t.x > top) + (t.y > top) + (t.z > top) + (t.w > top);
    }
    if (above < k) atomicMin(&lds.bound, top);
    __syncthreads();
    // Masked tokens come last: where the bound is no higher than theirs, what is left is ordered and the first masked ones follow.
    uint32_t bound = max(lds.bound, MASKED), from = max(bound, MASKED + 1);
    // f(bits, token) for this thread's logits that reach `least`
    const auto each = [&](uint32_t least, auto f) {
        if (top < least) return;
        for (int64_t j = 0; j < chunks; ++j) {
            if (top_of(j) < least) continue;
            for (int u = 0; u < PACKS; ++u) {
                const int64_t at = pack_at<T>(j, u, lead);
                const typename Pack<T>::V x = load_edge(row, at, V, 0.0f);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const uint32_t bits = logit_bits((float)x[e]);
                    if (bits >= least && at + e >= 0 && at + e < V) f(bits, (uint32_t)(at + e));
                }
            }
        }
    };
    const auto collect = [&](uint32_t bits, uint32_t token) {
        const uint32_t slot = atomicAdd(&lds.count, 1u);
        if (slot < LP_LIST) lds.list[slot] = alt_key(bits, token);
    };
    uint32_t n;
    int turn = 0;
    for (;;) {
        // The blocks that reach `from` are listed, then read by all threads, a pack each.
        if (top >= from)
            each_top<FIRST>(chunks, first, top_of, [&](int64_t j, uint32_t t) {
                if (t < from) return;
                const uint32_t slot = atomicAdd(&lds.block_count, 1u);
                if (slot < LP_READ) lds.blocks[slot] = (uint32_t)j * LP_WG + threadIdx.x;
            });
        __syncthreads();
        const uint32_t blocks = lds.block_count;
        if (blocks <= LP_READ) {
            for (uint32_t i = threadIdx.x; i < blocks * PACKS; i += LP_WG) {
                const uint32_t block = lds.blocks[i / PACKS];
                const int64_t at = (int64_t)(block / LP_WG) * LP_CHUNK + ((int64_t)(i % PACKS) * LP_WG + block % LP_WG) * N - lead;
                const typename Pack<T>::V x = load_edge(row, at, V, 0.0f);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const uint32_t bits = logit_bits((float)x[e]);
                    if (bits >= from && at + e >= 0 && at + e < V) collect(bits, (uint32_t)(at + e));
                }
            }
        } else if (from > bound) {
            each(from, collect);
        }
        __syncthreads();
        n = lds.count;
        if (from > bound || (blocks <= LP_READ && n <= LP_LIST)) break;
        // Too many reach the bound, as where it is the value of many tokens (a mask of the type's lowest value, a clipped row): those
        // above it alone, and of those equal to it the first in the row.
        from = bound + 1;
        __syncthreads();
        if (threadIdx.x == 0) lds.count = lds.block_count = 0;
        __syncthreads();
    }
    if (n > LP_LIST) {
        // Too many above the bound, too: the k-th logit itself, bit by bit.  Those above it are fewer than k.
        uint32_t kth = 0;
        for (int b = 31; b >= 0; --b) {
            const uint32_t trial = kth | 1u << b;
            uint32_t c = 0;
            if (trial > bound) {
                each(trial, [&](uint32_t, uint32_t) { ++c; });
                c = group_count(lane_value(wave_running_sum(c), 63), lds, turn++);
            }
            if (trial <= bound || c >= (uint32_t)k) kth = trial;
        }
        bound = kth;
        __syncthreads();
        if (threadIdx.x == 0) lds.count = 0;
        __syncthreads();
        each(bound + 1, collect);
        __syncthreads();
        n = lds.count;
    }
    for (int64_t j = 0; j < chunks && n < (uint32_t)k; ++j) {
        const bool here = top_of(j) >= bound;
        if (!__syncthreads_or(here)) continue;
        for (int u = 0; u < PACKS && n < (uint32_t)k; ++u) {
            const int64_t at = pack_at<T>(j, u, lead);
            uint32_t equal = 0;
            if (here && at < V) {
                const typename Pack<T>::V x = load_edge(row, at, V, 0.0f);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (logit_bits((float)x[e]) == bound && at + e >= 0 && at + e < V) equal |= 1u << e;
            }
            const uint32_t mine = (uint32_t)__popc(equal), running = wave_running_sum(mine);
            const uint32_t total = group_count(lane_value(running, 63), lds, turn);
            uint32_t slot = n + running - mine;
            for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) slot += lds.counts[turn & 1][w];
            for (; equal && slot < (uint32_t)k; equal &= equal - 1)
                lds.list[slot++] = alt_key(bound, (uint32_t)(at + __ffs((int)equal) - 1));
            n = min(n + total, (uint32_t)k);
            ++turn;
        }
    }
    __syncthreads();
    const uint64_t *list = lds.list;
    if (n > LP_WG) {
        // Too many to compare each with each: the k-th key, bit by bit (no two are equal, so k of them reach it).
        uint64_t kth = 0;
        for (int b = 63; b >= 0; --b) {
            const uint64_t trial = kth | 1ull << b;
            uint32_t c = 0;
            for (uint32_t i = 0; i < n; i += LP_WG)
                c += (uint32_t)__popcll(__ballot(i + threadIdx.x < n && lds.list[min(i + threadIdx.x, n - 1)] >= trial));
            if (group_count(c, lds, turn++) >= (uint32_t)k) kth = trial;
        }
        if (threadIdx.x == 0) lds.count = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n; i += LP_WG)
            if (lds.list[i] >= kth) lds.kept[atomicAdd(&lds.count, 1u)] = lds.list[i];
        __syncthreads();
        n = (uint32_t)k;
        list = lds.kept;
    }
    if (threadIdx.x < n) {
        const uint64_t key = list[threadIdx.x];
        int rank = 0;
        for (uint32_t j = 0; j < n; ++j) rank += list[j] > key;
        if (rank < k) {
            top_idx[rank] = ~(uint32_t)key;
            top_logp[rank] = of.log_p(alt_logit(key));
        }
    }
    for (int i = (int)n + threadIdx.x; i < k; i += LP_WG) {  // V < k
        top_idx[i] = 0xFFFFFFFFu;
        top_logp[i] = -INFINITY;
    }
    __syncthreads();
}

// A row's first given tokens, one a thread, and their logits.
struct Given {
    int token;
    float logit;
};
template <typename T>
__device__ __forceinline__ Given given(const T *row, int64_t r, int V, const Out &o, int t)
{
    Given g = {-1, 0.0f};
    if (t < o.nt) g.token = o.tokens[r * o.nt + t];
    if (g.token >= V) g.token = -1;
    if (g.token >= 0) g.logit = (float)row[g.token];
    return g;
}

// What follows once a row's statistics are known.
template <typename T, bool ALT, int FIRST, typename L, typename F>
__device__ __forceinline__ void write_row(const T *row, int64_t r, int V, int lead, int64_t chunks, Stats a, float scale,
                                          const Out &o, Given g, L &lds, const uint32_t (&first)[FIRST + 1], F top_of)
{
    const Row of = {scale, a.m, logf(a.s), a.m == -INFINITY && a.s == 0.0f};
    if (threadIdx.x == 0) {
        const float lse = fmaf(scale, a.m, of.log_s);  // (no float holds it: NaN, since -inf says that nothing is left)
        if (o.lse) o.lse[r] = of.none ? -INFINITY : fabsf(lse) < INFINITY ? lse : NAN;
        if (o.entropy) o.entropy[r] = of.none ? 0.0f : of.log_s - LN2 * a.w / a.s;
    }
    for (int t = threadIdx.x; t < o.nt; t += LP_WG) {
        if (t >= LP_WG) g = given(row, r, V, o, t);
        o.logp[r * o.nt + t] = g.token < 0 ? 0.0f : of.log_p(g.logit);
    }
    if constexpr (ALT)
        write_alternatives<FIRST>(row, V, lead, chunks, o.k, of, o.top_idx + r * o.k, o.top_logp + r * o.k, lds, first, top_of);
}

// A workgroup per row; four of them a compute unit (129 registers would leave three: 4096 x 65536 bfloat16, 20 alternatives 132 us
// for 115).
template <typename T, bool ALT>
__global__ __launch_bounds__(LP_WG, 4) void logprobs_row_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int V,
                                                                float scale, Out o)
{
    __shared__ StatsLds stats;
    __shared__ std::conditional_t<ALT, AltLds, NoLds> alt;
    extern __shared__ uint32_t tops[];  // [chunks][LP_WG] where there are alternatives
    const float c = scale * LOG2E;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = logits + r * ld;
        const int lead = lead_of(row);
        const int64_t chunks = chunks_of(V, lead);
        const Given g = given(row, r, V, o, threadIdx.x);
        Stats a = {-INFINITY, 0.0f, 0.0f};
        for (int64_t j = 0; j < chunks; ++j) {
            float x[LP_BLOCK], top;
            load_block(row, j, V, lead, x);
            const bool odd = add_block(a, x, c, &top);
            if constexpr (ALT) tops[j * LP_WG + threadIdx.x] = block_top(row, j, V, lead, top, odd);
        }
        a = group_stats(a, c, stats);
        const uint32_t first[1] = {};
        write_row<T, ALT, 0>(row, r, V, lead, chunks, a, scale, o, g, alt, first,
                             [&](int64_t j) { return tops[j * LP_WG + threadIdx.x]; });
    }
}

// A workgroup per `per` chunks of a row: their statistics and their blocks' largest logits into the workspace.  The rows are
// joined by a kernel of its own: joining in the last workgroup of a row to finish takes a fence over the GPU's caches in every
// one of them, which costs as much as the launch for one row (15.5 us against 15) and three times as much for 64 (60 against 20).
template <typename T, bool ALT>
__global__ __launch_bounds__(LP_WG) void logprobs_part_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int V,
                                                              float scale, int64_t stride, int parts, int per,
                                                              Stats *__restrict__ stats, uint32_t *__restrict__ tops)
{
    __shared__ StatsLds lds;
    const float c = scale * LOG2E;
    for (int64_t i = blockIdx.x; i < rows * parts; i += gridDim.x) {
        const int64_t r = i / parts, j0 = i % parts * per;
        const T *row = logits + r * ld;
        const int lead = lead_of(row);
        const int64_t j1 = min(j0 + per, chunks_of(V, lead));
        Stats a = {-INFINITY, 0.0f, 0.0f};
        for (int64_t j = j0; j < j1; ++j) {
            float x[LP_BLOCK], top;
            load_block(row, j, V, lead, x);
            const bool odd = add_block(a, x, c, &top);
            if constexpr (ALT) tops[(r * stride + j) * LP_WG + threadIdx.x] = block_top(row, j, V, lead, top, odd);
        }
        a = group_stats(a, c, lds);
        if (threadIdx.x == 0) stats[i] = a;
    }
}

template <typename T, bool ALT>
__global__ __launch_bounds__(LP_WG) void logprobs_join_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int V,
                                                              float scale, int64_t stride, int parts,
                                                              const Stats *__restrict__ stats,
                                                              const uint32_t *__restrict__ tops, Out o)
{
    __shared__ StatsLds lds;
    __shared__ std::conditional_t<ALT, AltLds, NoLds> alt;
    const float c = scale * LOG2E;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = logits + r * ld;
        const int lead = lead_of(row);
        const int64_t chunks = chunks_of(V, lead);
        const auto top_of = [&](int64_t j) { return tops[(r * stride + j) * LP_WG + threadIdx.x]; };
        constexpr int FIRST = ALT ? 16 : 0;
        uint32_t first[FIRST + 1] = {};
#pragma unroll
        for (int j = 0; j < FIRST; ++j) first[j] = j < chunks ? top_of(j) : 0u;
        Stats a = {-INFINITY, 0.0f, 0.0f};
        for (int p = threadIdx.x; p < parts; p += LP_WG) a = join(a, stats[r * parts + p], c);
        const Given g = given(row, r, V, o, threadIdx.x);
        a = group_stats(a, c, lds);
        write_row<T, ALT, FIRST>(row, r, V, lead, chunks, a, scale, o, g, alt, first, top_of);
    }
}

// exp(t), t <= 0 or thereabouts.  A float32 gradient shows the rounding of t log2(e), |t| units in its last place of a p that
// has its own size (16-bit ones do not): there what the product leaves out is put back in.
template <typename T>
__device__ __forceinline__ float exp_of(float t)
{
    const float y = t * LOG2E;
    if constexpr (sizeof(T) == 2) return exp2_fast(y);
    const float rest = fmaf(t, LOG2E, -y) + t * 1.9259629911e-8f;  // log2(e) - LOG2E = 1.92596e-8
    const float p = exp2_fast(y);
    return y > -3000.0f ? fmaf(p, rest * LN2, p) : p;  // (an infinite t: no infinity less infinity)
}

// A workgroup per `per` chunks of a row: first every logit's own share, then the given tokens', each once.  STREAM: stores past
// the caches, for gradients that they do not hold (4096 x 65536 bfloat16 176 -> 171 us, 4096 x 50021 157 -> 130; of 262 MB 1000 x
// 131072 would go from 78 to 85, 4096 x 32000 from 101 to 81).
template <typename T, bool STREAM>
__global__ __launch_bounds__(LP_WG) void logprobs_grad_kernel(const T *logits, int64_t ld, int64_t rows, int V, float scale,
                                                              int parts, int per, const int32_t *__restrict__ tokens, int nt,
                                                              const float *__restrict__ lse, const float *__restrict__ entropy,
                                                              const float *__restrict__ dlogp,
                                                              const float *__restrict__ dentropy, T *dlogits, int64_t ldd)
{
    constexpr int N = Pack<T>::N, PACKS = LP_BLOCK / N;
    __shared__ float sums[LP_WG / WAVE];
    __shared__ int tok[QADC_MAX_R];
    __shared__ float at[QADC_MAX_R], dl[QADC_MAX_R];
    for (int64_t i = blockIdx.x; i < rows * parts; i += gridDim.x) {
        const int64_t r = i / parts;
        const T *row = logits + r * ld;
        T *out = dlogits + r * ldd;
        const int lead = lead_of(out);
        const int64_t v0 = max((int64_t)0, i % parts * per * LP_CHUNK - lead);
        const int64_t v1 = min((i % parts + 1) * per * LP_CHUNK - lead, (int64_t)V);
        const float l = lse[r], dh = dentropy ? dentropy[r] : 0.0f, h = dentropy ? entropy[r] : 0.0f;
        const bool none = l == -INFINITY;
        float total = 0.0f;
        for (int t = threadIdx.x; t < nt; t += LP_WG) {
            const int v = tokens[r * nt + t];
            const bool used = v >= 0 && v < V, here = v >= v0 && v < v1;
            const float g = used ? dlogp[r * nt + t] : 0.0f;
            tok[t] = here ? v : -1;
            at[t] = here ? (float)row[v] : 0.0f;
            dl[t] = g;
            total += g;
        }
        total = wave_sum(total);
        if (lane_id() == 0) sums[threadIdx.x >> 6] = total;
        __syncthreads();
        total = 0.0f;
#pragma unroll
        for (int w = 0; w < LP_WG / WAVE; ++w) total += sums[w];
        const auto share = [&](float logit) {
            const float lp = fmaf(scale, logit, -l), p = exp_of<T>(lp);
            return p * -fmaf(dh, fmaxf(lp, -2000.0f) + h, total);  // (a masked logit: zero times something finite)
        };
        const auto value = [&](float logit) { return none ? 0.0f : scale * share(logit); };
        for (int64_t j = i % parts * per; j < (i % parts + 1) * per && j * LP_CHUNK - lead < v1; ++j) {
            typename Pack<T>::V p[PACKS];
            if ((j > 0 || lead == 0) && (j + 1) * LP_CHUNK - lead <= v1) {
#pragma unroll
                for (int u = 0; u < PACKS; ++u)
                    p[u] = __builtin_nontemporal_load(reinterpret_cast<const typename Pack<T>::V *>(row + pack_at<T>(j, u, lead)));
#pragma unroll
                for (int u = 0; u < PACKS; ++u) {
#pragma unroll
                    for (int e = 0; e < N; ++e) p[u][e] = (T)value((float)p[u][e]);
                    auto *to = reinterpret_cast<typename Pack<T>::V *>(out + pack_at<T>(j, u, lead));
                    if constexpr (STREAM) __builtin_nontemporal_store(p[u], to);
                    else *to = p[u];
                }
            } else {
#pragma unroll
                for (int u = 0; u < PACKS; ++u) p[u] = load_edge(row, pack_at<T>(j, u, lead), v1, 0.0f);
#pragma unroll
                for (int u = 0; u < PACKS; ++u) {
                    const int64_t at = pack_at<T>(j, u, lead);
                    if (at >= v1) continue;
#pragma unroll
                    for (int e = 0; e < N; ++e) p[u][e] = (T)value((float)p[u][e]);
                    if (at >= 0 && at + N <= v1) {
                        *reinterpret_cast<typename Pack<T>::V *>(out + at) = p[u];
                    } else {
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (at + e >= 0 && at + e < v1) out[at + e] = p[u][e];
                    }
                }
            }
        }
        __syncthreads();
        for (int t = threadIdx.x; t < nt; t += LP_WG) {
            if (tok[t] < 0 || none) continue;
            float own = 0.0f;
            bool first = true;
            for (int u = 0; u < nt; ++u)
                if (tok[u] == tok[t]) {
                    first = first && u >= t;
                    own += dl[u];
                }
            if (first) out[tok[t]] = (T)(scale * (own + share(at[t])));
        }
        __syncthreads();
    }
}

int check_logits(const char *who, int type, int64_t ld, int64_t rows, int V, float scale, const int32_t *tokens, int T)
{
    if (!type_ok(type)) return fail(QADC_EINVAL, "%s: unknown type %d", who, type);
    if (rows < 0 || V < 1 || ld < V) return fail(QADC_EINVAL, "%s: rows=%lld V=%d ld=%lld", who, (long long)rows, V, (long long)ld);
    if (!(scale > 0.0f) || !(scale * LOG2E < INFINITY)) return fail(QADC_EINVAL, "%s: scale=%g", who, (double)scale);
    if (T < 0 || T > QADC_MAX_R) return fail(QADC_EINVAL, "%s: T=%d", who, T);
    if (T > 0 && rows > 0 && !tokens) return fail(QADC_EINVAL, "%s: null pointer", who);
    return QADC_OK;
}

}  // namespace

constexpr int64_t LP_WHOLE = 400, LP_PARTS = 1024;

// How a call is cut: a row per workgroup where the rows alone nearly fill the chip, parts of rows otherwise.
struct Plan {
    int64_t chunks;
    int parts, per;  // workgroups a row, chunks each; parts = 1: one kernel and no workspace
    size_t tops, bytes;  // in the workspace: [rows][parts] statistics, [rows][chunks][LP_WG] largest logits
};

static Plan plan_logprobs(int64_t rows, int V, int k)
{
    Plan p;
    p.chunks = ceil_div((int64_t)V + 7, LP_CHUNK);  // (a row begins up to seven logits into its first pack)
    // Rows are cut into parts, joined by a second kernel, where there are fewer than 400 (300 x 131072, 20 alternatives: 34 us against 37 whole;
    // 500: 47 against 42; 1000: 85 against 66); then into as many as make 1024 workgroups.
    const int64_t want = rows >= LP_WHOLE ? 1 : ceil_div(LP_PARTS, rows);
    p.per = (int)ceil_div(p.chunks, std::min(p.chunks, want));
    p.parts = (int)ceil_div(p.chunks, p.per);
    if (p.parts == 1 && k > 0 && p.chunks * LP_WG > LP_LDS_BLOCKS) {  // the blocks do not fit in LDS
        p.per = (int)ceil_div(p.chunks, 2);
        p.parts = 2;
    }
    p.tops = 0;
    p.bytes = 256;
    if (p.parts > 1) {
        p.tops = align_up((size_t)rows * p.parts * sizeof(Stats), 256);
        p.bytes = p.tops + (k > 0 ? (size_t)rows * p.chunks * LP_WG * sizeof(uint32_t) : 0);
    }
    return p;
}

// Enough for these rows and for any fewer, and for shorter ones and fewer alternatives: of up to 399 rows, those that may be cut into
// parts (r rows into fewer than 1024 + r of them), and of all where they are too long for LDS.
size_t token_logprobs_workspace(int64_t rows, int V, int k)
{
    if (rows < 1 || V < 1 || k < 0 || k > QADC_MAX_ALTERNATIVES) return 0;
    const int64_t chunks = plan_logprobs(rows, V, k).chunks, few = std::min(rows, LP_WHOLE - 1);
    if (chunks == 1) return 256;
    const bool all = k > 0 && chunks * LP_WG > LP_LDS_BLOCKS;
    const int64_t parts = std::max(std::min(few * chunks, LP_PARTS + few), all ? 2 * rows : 0);
    return align_up((size_t)parts * sizeof(Stats), 256) + (k > 0 ? (size_t)(all ? rows : few) * chunks * LP_WG * sizeof(uint32_t) : 0);
}

template <typename T, bool ALT>
static void launch_logprobs(const Plan &p, const void *logits, int64_t ld, int64_t rows, int V, float scale, const Out &o,
                            void *workspace, hipStream_t st)
{
    const T *x = (const T *)logits;
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 20));
    if (p.parts == 1) {
        launch(QADC_PROF_LOGPROBS, logprobs_row_kernel<T, ALT>, grid, dim3(LP_WG),
               ALT ? (size_t)p.chunks * LP_WG * sizeof(uint32_t) : 0, st, x, ld, rows, V, scale, o);
        return;
    }
    Stats *stats = (Stats *)workspace;
    uint32_t *tops = (uint32_t *)((char *)workspace + p.tops);
    launch(QADC_PROF_LOGPROBS, logprobs_part_kernel<T, ALT>, dim3((unsigned)std::min<int64_t>(rows * p.parts, 1 << 20)),
           dim3(LP_WG), 0, st, x, ld, rows, V, scale, p.chunks, p.parts, p.per, stats, tops);
    launch(QADC_PROF_LOGPROBS, logprobs_join_kernel<T, ALT>, grid, dim3(LP_WG), 0, st, x, ld, rows, V, scale, p.chunks, p.parts,
           (const Stats *)stats, (const uint32_t *)tops, o);
}

int token_logprobs(const void *logits, int64_t ld, int type, int64_t rows, int V, float scale, const int32_t *tokens, int T,
                   int k, float *logp, float *lse, float *entropy, uint32_t *top_idx, float *top_logp, void *workspace,
                   size_t workspace_bytes, hipStream_t st)
{
    if (const int rc = check_logits("qadc_token_logprobs", type, ld, rows, V, scale, tokens, T)) return rc;
    if (k < 0 || k > QADC_MAX_ALTERNATIVES) return fail(QADC_EINVAL, "qadc_token_logprobs: k=%d", k);
    if (rows == 0) return QADC_OK;
    if (!logits || (T > 0 && !logp) || (k > 0 && (!top_idx || !top_logp)))
        return fail(QADC_EINVAL, "qadc_token_logprobs: null pointer");
    const Plan p = plan_logprobs(rows, V, k);
    if (!workspace || workspace_bytes < p.bytes)
        return fail(QADC_ENOMEM, "qadc_token_logprobs: workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
    const Out o = {tokens, T, k, logp, lse, entropy, top_idx, top_logp};
    if (k > 0) {
        QADC_BY_TYPE(type, (launch_logprobs<T, true>(p, logits, ld, rows, V, scale, o, workspace, st)));
    } else {
        QADC_BY_TYPE(type, (launch_logprobs<T, false>(p, logits, ld, rows, V, scale, o, workspace, st)));
    }
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

int token_logprobs_backward(const void *logits, int64_t ld, int type, int64_t rows, int V, float scale, const int32_t *tokens,
                            int T, const float *lse, const float *entropy, const float *dlogp, const float *dentropy,
                            void *dlogits, int64_t ldd, hipStream_t st)
{
    if (const int rc = check_logits("qadc_token_logprobs_backward", type, ld, rows, V, scale, tokens, T)) return rc;
    if (ldd < V) return fail(QADC_EINVAL, "qadc_token_logprobs_backward: ldd=%lld", (long long)ldd);
    if (rows == 0) return QADC_OK;
    if (!logits || !lse || !dlogits || (T > 0 && !dlogp) || (dentropy && !entropy))
        return fail(QADC_EINVAL, "qadc_token_logprobs_backward: null pointer");
    if (logits == dlogits && ld != ldd)
        return fail(QADC_EINVAL, "qadc_token_logprobs_backward: in place needs equal row distances");
    // (where rows begin off 16 bytes, up to seven logits into their first pack)
    const bool even = (uintptr_t)dlogits % 16 == 0 && (size_t)ldd * type_bytes(type) % 16 == 0;
    const int64_t chunks = ceil_div((int64_t)V + (even ? 0 : 7), LP_CHUNK);
    // Chunks a workgroup: one, where a row has more than two and few tokens are given (4096 x 65536 bfloat16 with one token 171 us, 192
    // with four chunks; with 16 173 for 194); up to four elsewhere: every workgroup goes through the tokens (64 of them 197 us for 212,
    // 1000 x 50021 with 1000 1060 for 2200), and of two chunks the second is rarely full (4096 x 10000 32 us for 40).
    const int64_t most = T <= 16 && chunks > 2 ? 1 : std::max<int64_t>(1, std::min<int64_t>(4, chunks * rows / 2048));
    const int parts = (int)ceil_div(chunks, most), per = (int)ceil_div(chunks, parts);
    const dim3 grid((unsigned)std::min<int64_t>(rows * parts, 1 << 20));
    const int nt = T;
    const bool stream = (size_t)rows * V * type_bytes(type) > ((size_t)384 << 20);
    QADC_BY_TYPE(type, {
        const auto kernel = stream ? &logprobs_grad_kernel<T, true> : &logprobs_grad_kernel<T, false>;
        launch(QADC_PROF_LOGPROBS, *kernel, grid, dim3(LP_WG), 0, st, (const T *)logits, ld, rows, V, scale, parts, per, tokens, nt,
               lse, entropy, dlogp, dentropy, (T *)dlogits, ldd);
    });
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
