// Low-rank adapters of many requests beside a shared projection on gfx950: y_i = base_i + s_a B_a (A_a x_i), a = ids[i].
//
// Two launches: u = A x into the workspace, cut over the inputs, then y = base + s B u.  Rows come in tiles of 256 consecutive ones;
// every wavefront groups its tile's rows by adapter with ballots, up to 16 (or 64) of one adapter to an item, so that an adapter is
// read once for all its rows of a tile, wherever they lie.  Both products are on the matrix units, with the adapter's side as the
// first operand: a lane then holds the results of one row, and rows that are not there cost no care, since their results are not
// looked at.
//
// Of 16-bit types u goes into the second product as two numbers, u rounded and what that leaves: off by 2^-16 (bfloat16) or 2^-22
// (binary16, scaled by a power of two into its range), so that only y's own rounding shows.  float32 is multiplied as float32.
//
// Bound by memory where rows are many, not reached: 8192 rows of 4096 x 4096 through rank 64, bfloat16, 29 us for the first product (67 MB
// of x, whose rows go to different lanes, so that a load of 64 lanes touches 16 rows) and 39 for the second (134 MB at 3.4 TB/s);
// 64 rows of 32 adapters of rank 16, 4096 x 16384, 5 and 10.5 us: four dependent round trips (ids, u, the pool, y) in one and a
// half rounds of workgroups; one row 3.6 and 6.0, launches and round trips.  (Kernels' times by the profiler; figures elsewhere in
// this file are calls one after the other: 67, 14.5 and 11 us.)
#include <algorithm>
#include <type_traits>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int AD_WG = 256, AD_TILE = 256;  // threads; rows of a tile, one a thread
// Rows from which on an item has 64 of them, if each adapter has as many: the pool is read a quarter as often.  4990 rows of 42 adapters of
// rank 16, 7754 x 742, 47 us for 118 with 16 rows; 400 rows of one of rank 94, 15312 x 1581 float32, 115 for 69 the other way round.
// In any order a tile of many adapters has few rows of each, and the pool is read again for every tile: 8192 rows of rank 64, 4096 x 4096, bfloat16,
// in segments and in any order: 16 adapters 81 us and 151, 32 86 and 237, 64 95 and 478, 128 120 and 860.
constexpr int64_t AD_MANY = 1024;
constexpr int AD_COLS = 64;                // outputs of a wavefront at a time
constexpr int64_t AD_GROUPS = ((int64_t)1 << 32) / AD_WG;  // of a launch, less one: their threads are counted in 32 bits

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float Quad __attribute__((ext_vector_type(4), aligned(4)));

// Eight consecutive elements.
template <typename T>
struct Eight {
    typedef T V __attribute__((ext_vector_type(8)));
    typedef T Raw __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    typedef T Lds __attribute__((ext_vector_type(8), aligned(16)));
    static __device__ __forceinline__ V zero() { return (V)(T)0.0f; }
    static __device__ __forceinline__ V load(const T *p) { return *reinterpret_cast<const Raw *>(p); }
    // n of them are there, zeros behind
    static __device__ __forceinline__ V load(const T *p, int n)
    {
        if (n >= 8) return load(p);
        V v = zero();
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) v[e] = p[e];
        return v;
    }
};

// c[i][j] += sum over k of a[i][k] b[j][k], 16 x 16 x 32: lane l holds row l % 16 of both operands, elements 8 (l / 16) .. + 7, and of
// c the column l % 16, rows 4 (l / 16) .. + 3.
__device__ __forceinline__ f32x4 mma(Eight<_Float16>::V a, Eight<_Float16>::V b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(Eight<__bf16>::V a, Eight<__bf16>::V b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(Eight<float>::V a, Eight<float>::V b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// A tile's rows by adapter, by each wavefront for itself: lane l has the adapters of rows l, 64 + l, 128 + l and 192 + l, and the rows of
// one adapter are the bits of four ballots.
struct Tile {
    static constexpr int W = AD_TILE / WAVE;
    int id[W];                      // -1: none
    unsigned long long left[W];     // rows that are there and belong to no item so far
};
struct Item {
    int id;
    unsigned long long rows[Tile::W];
    int count;
};
__device__ __forceinline__ Tile load_tile(const int32_t *ids, int64_t first, int rows, int count)
{
    Tile t;
#pragma unroll
    for (int w = 0; w < Tile::W; ++w) {
        const int i = w * WAVE + lane_id();
        int id = i < rows ? ids[first + i] : -1;
        if (id < 0 || id >= count) id = -1;
        t.id[w] = id;
        t.left[w] = __ballot(i < rows);
    }
    return t;
}
// The rows left that have the adapter of row i, one of them.
__device__ __forceinline__ Item same_as(const Tile &t, int i)
{
    Item it = {0, {}, 0};
#pragma unroll
    for (int w = 0; w < Tile::W; ++w)
        if (w == i / WAVE) it.id = (int)lane_value((unsigned)t.id[w], i % WAVE);
#pragma unroll
    for (int w = 0; w < Tile::W; ++w) {
        it.rows[w] = __ballot(t.id[w] == it.id) & t.left[w];
        it.count += __popcll(it.rows[w]);
    }
    return it;
}
// ROWS rows of an item from number `from` on, into the wavefront's list in LDS (-1 behind).
template <int ROWS>
__device__ __forceinline__ Item list_rows(const Item &it, int from, int16_t *list)
{
    __builtin_amdgcn_wave_barrier();
    if (lane_id() < ROWS) list[lane_id()] = -1;
    __builtin_amdgcn_wave_barrier();
    int before = -from;
#pragma unroll
    for (int w = 0; w < Tile::W; ++w) {
        const int place = before + (int)rank_in_mask(it.rows[w]);
        if ((it.rows[w] >> lane_id() & 1) && place >= 0 && place < ROWS) list[place] = (int16_t)(w * WAVE + lane_id());
        before += __popcll(it.rows[w]);
    }
    __builtin_amdgcn_wave_barrier();
    Item part = it;
    part.count = min(it.count - from, ROWS);
    return part;
}
// f(item) for the workgroup's items.  As many slots as rows: a workgroup has an item where its row is the first, or the one behind ROWS
// others, ... of its adapter.  Fewer: it goes over the tile's adapters, counts their items up and takes every slots-th.  (Slots
// without items are the last in a grid: between the others they left half of the compute units idle, for which it was always the turn of
// one of them: 8192 rows of rank 64, eight slots of which four had an item, 48 us for 27.)
template <int ROWS, typename F>
__device__ __forceinline__ void each_item(Tile t, int slot, int slots, int rows, int16_t *list, F f)
{
    if (ROWS == 16 && slots >= rows) {
        if (slot >= rows) return;
        const Item it = same_as(t, slot);
        int before = 0;
#pragma unroll
        for (int w = 0; w < Tile::W; ++w) {
            const unsigned long long below = w < slot / WAVE ? ~0ull : w > slot / WAVE ? 0ull : (1ull << slot % WAVE) - 1;
            before += __popcll(it.rows[w] & below);
        }
        if (before % ROWS == 0) f(list_rows<ROWS>(it, before, list));
        return;
    }
    for (int n = 0;;) {
        int i = AD_TILE;
#pragma unroll
        for (int w = Tile::W - 1; w >= 0; --w)
            if (t.left[w]) i = w * WAVE + __ffsll((long long)t.left[w]) - 1;
        if (i == AD_TILE) return;
        const Item it = same_as(t, i);
        const int items = (it.count + ROWS - 1) / ROWS;
        for (int k = (slot - n % slots + slots) % slots; k < items; k += slots) f(list_rows<ROWS>(it, k * ROWS, list));
        n += items;
#pragma unroll
        for (int w = 0; w < Tile::W; ++w) t.left[w] &= ~it.rows[w];
    }
}

struct Pool {
    const void *a, *b;
    const float *scales;
    const int32_t *ranks;
    int64_t N;
    int K, rank, count;
};
__device__ __forceinline__ int rank_of(const Pool &p, int id) { return p.ranks ? min(max(p.ranks[id], 0), p.rank) : p.rank; }

// u of the rows of an item: RT blocks of 16 ranks, RB blocks of 16 rows at a time, a quarter of the split's inputs each wavefront.
// part [split][M][wide] float32.
template <typename T, int RT, int RB>
__global__ __launch_bounds__(AD_WG) void adapters_down_kernel(Pool pool, const int32_t *__restrict__ ids, const T *__restrict__ x,
                                                              int64_t ldx, int64_t M, int slots, int splits, int per, int wide,
                                                              float *__restrict__ part)
{
    typedef Eight<T> E;
    __shared__ int16_t lists[AD_WG / WAVE][16 * RB];
    __shared__ f32x4 red[AD_WG / WAVE][RT][WAVE];
    const int tiles = (int)((M + AD_TILE - 1) / AD_TILE), split = blockIdx.x % splits, slot = blockIdx.x / splits / tiles;
    const int64_t first = (int64_t)(blockIdx.x / splits % tiles) * AD_TILE;
    const int wave = threadIdx.x >> 6, l = lane_id() % 16, g = lane_id() / 16;
    const int rows = (int)min((int64_t)AD_TILE, M - first);
    int16_t *list = lists[wave];
    const int steps = (pool.K + 31) / 32, s0 = min(steps, (split * 4 + wave) * per), s1 = min(steps, s0 + per);
    const int whole = min(s1, pool.K / 32);  // steps whose inputs are all there
    // BLOCKS: blocks of 16 rows that are looked at
    const auto take = [&](const Item &it, auto blocks) {
        constexpr int BLOCKS = decltype(blocks)::value, DEEP = BLOCKS * RT >= 16 ? 2 : 4;
        const int id = it.id;
        if (id < 0) return;
        const int r = rank_of(pool, id);
        const T *xr[BLOCKS];
        int row[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            row[b] = list[b * 16 + l];
            xr[b] = x + (first + max(row[b], 0)) * ldx;
        }
        for (int p = 0; p < r; p += 16 * RT) {
            f32x4 acc[RT][BLOCKS] = {};
            const T *ar[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) ar[t] = (const T *)pool.a + ((int64_t)id * pool.rank + min(p + 16 * t + l, r - 1)) * pool.K;
            // (rows and ranks that are not there stand for others: their results are not looked at)
            typename E::V av[DEEP][RT], xv[DEEP][BLOCKS];
            const auto load = [&](int s, int u) {
                const int k = 32 * s + 8 * g;
#pragma unroll
                for (int t = 0; t < RT; ++t) av[u][t] = E::load(ar[t] + k);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) xv[u][b] = E::load(xr[b] + k);
            };
            const auto multiply = [&](int u) {
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) acc[t][b] = mma(av[u][t], xv[u][b], acc[t][b]);
            };
            int s = s0;
            for (; s + DEEP <= whole; s += DEEP) {
#pragma unroll
                for (int u = 0; u < DEEP; ++u) load(s + u, u);
#pragma unroll
                for (int u = 0; u < DEEP; ++u) multiply(u);
            }
            for (; s < whole; ++s) {
                load(s, 0);
                multiply(0);
            }
            if (s < s1) {  // the last inputs
                const int k = 32 * s + 8 * g, n = pool.K - k;
#pragma unroll
                for (int t = 0; t < RT; ++t) av[0][t] = E::load(ar[t] + k, n);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) xv[0][b] = E::load(xr[b] + k, n);
                multiply(0);
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                __syncthreads();
#pragma unroll
                for (int t = 0; t < RT; ++t) red[wave][t][lane_id()] = acc[t][b];
                __syncthreads();
                for (int t = wave; t < RT; t += AD_WG / WAVE) {
                    f32x4 v = red[0][t][lane_id()];
#pragma unroll
                    for (int w = 1; w < AD_WG / WAVE; ++w) v += red[w][t][lane_id()];
                    const int j = p + 16 * t + 4 * g;
                    if (row[b] >= 0 && j < wide)
                        *reinterpret_cast<f32x4 *>(part + ((int64_t)split * M + first + row[b]) * wide + j) = v;
                }
            }
        }
    };
    // Of few rows fewer blocks are looked at (8192 float32 rows of rank 64, sixteen adapters in any order, 321 us; 391 with one block or four).
    each_item<16 * RB>(load_tile(ids, first, rows, pool.count), slot, slots, rows, list, [&](const Item &it) {
        if (RB > 1 && it.count <= 16) take(it, std::integral_constant<int, 1>());
        else if (RB > 2 && it.count <= 32) take(it, std::integral_constant<int, RB < 2 ? RB : 2>());
        else take(it, std::integral_constant<int, RB>());
    });
}

// A power of two that takes `most` to 2^10 .. 2^11, and its inverse.
__device__ __forceinline__ float into_half(float most, float &back)
{
    const int e = min(max((int)(__float_as_uint(most) >> 23), 20), 240) - 127 - 10;
    back = __uint_as_float((unsigned)(127 + e) << 23);
    return __uint_as_float((unsigned)(127 - e) << 23);
}

// A result of 16 rows x 64 outputs goes through LDS to where eight lanes have a row's outputs side by side: loads and stores of 16 bytes from
// 16 rows at once, four lanes of each, reached 2 TB/s.
constexpr int AD_TURN = 68;  // floats from row to row

// Ranks go in eights.  Of a pool whose rank is no multiple of eight the last eight begin at rank - 8, and those of them that the eight
// before have too are zero in u.
__device__ __forceinline__ int eight_at(int rank, int j) { return min(j, max(rank - 8, 0)); }

// y of the rows of an item, `blocks` times 64 outputs a wavefront; STEPS times 32 ranks at most.  The last block of outputs begins 64
// before the end, and writes what no other has.  SMALL: fewer than eight ranks or 64 outputs, read and written one by one (8192 rows of 4096 x
// 4096 bfloat16 in segments, four ranks 127 us where eight take 51; 64 rows of 16384 outputs 23.5 and 13.1; one row 10 and 10).  What the
// first outputs need of the pool and of base is on its way while u is added up.
template <typename T, int RB, int STEPS, bool SMALL>
__global__ __launch_bounds__(AD_WG, sizeof(T) == 2 && STEPS * RB <= 4 && !SMALL ? 3 : 2) void adapters_up_kernel(Pool pool, const int32_t *__restrict__ ids, int64_t M, int slots, int chunks,
                                                               int blocks, int splits, int wide, const float *__restrict__ part,
                                                               const T *base, int64_t ldb, T *y, int64_t ldy)
{
    typedef Eight<T> E;
    typedef typename E::V V;
    constexpr int ROWS = 16 * RB, SHARE = AD_WG / ROWS, QUADS = (8 * STEPS + SHARE - 1) / SHARE;
    constexpr bool TWO = sizeof(T) == 2;
    constexpr bool KEPT = sizeof(T) * STEPS <= 8;  // the weights of 64 outputs stay in registers for all rows
    __shared__ int16_t lists[AD_WG / WAVE][ROWS];
    __shared__ float back[ROWS];
    __shared__ f32x4 turn[AD_WG / WAVE][16 * AD_TURN / 4];
    extern __shared__ __attribute__((aligned(16))) char raw[];
    constexpr int stride = 32 * STEPS + 16 / (int)sizeof(T);
    T *hi = (T *)raw, *lo = hi + ROWS * stride;
    const int tiles = (int)((M + AD_TILE - 1) / AD_TILE), chunk = blockIdx.x % chunks, slot = blockIdx.x / chunks / tiles;
    const int64_t first = (int64_t)(blockIdx.x / chunks % tiles) * AD_TILE;
    const int wave = threadIdx.x >> 6, l = lane_id() % 16, g = lane_id() / 16;
    const int rows = (int)min((int64_t)AD_TILE, M - first);
    int16_t *list = lists[wave];
    const auto take = [&](const Item &it, auto live) {
        constexpr int LIVE = decltype(live)::value;  // blocks of 16 rows that are looked at
        const int id = it.id;
        if (id < 0 && base == y) return;
        const int r = id < 0 ? 0 : rank_of(pool, id), steps = (r + 31) / 32;
        const T *b0 = (const T *)pool.b + (int64_t)max(id, 0) * pool.N * pool.rank;
        const auto block_at = [&](int c) { return ((int64_t)(chunk * blocks + c) * (AD_WG / WAVE) + wave) * AD_COLS; };
        const auto weights = [&](int64_t n0, int s, int t) {
            const T *from = b0 + (n0 + 16 * t + l) * pool.rank;
            const int j = eight_at(pool.rank, 32 * s + 8 * g);
            V v;
            if constexpr (!SMALL) {
                v = E::load(from + j);
            } else {
                from = b0 + min(n0 + 16 * t + l, pool.N - 1) * pool.rank;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = from[min(j + e, pool.rank - 1)];
            }
            return v;
        };
        const auto cleared = [&](V v, int s) {  // (what lies beyond the rank may be anything)
            if (pool.rank % 8 == 0 && 32 * s + 32 <= r) return v;  // (the same in all lanes)
            const int j = eight_at(pool.rank, 32 * s + 8 * g), there = 32 * s + 8 * g < r ? r - j : 0;
            if constexpr (TWO) {
                typedef unsigned Words __attribute__((ext_vector_type(4)));
                Words w = __builtin_bit_cast(Words, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = there > 2 * i + 1 ? w[i] : there > 2 * i ? w[i] & 0xffffu : 0u;
                return __builtin_bit_cast(V, w);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = e < there ? v[e] : (T)0.0f;
                return v;
            }
        };
        const auto old_at = [&](int row, int64_t n) {
            V v = E::zero();
            if (base) {
                const T *from = base + (first + max(row, 0)) * ldb;
                if constexpr (!SMALL) {
                    v = E::load(from + n);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = from[min(n + e, pool.N - 1)];
                }
            }
            return v;
        };
        V w[KEPT ? STEPS : 1][4], old[LIVE][2];
        const auto fetch = [&](int64_t n0) {
            if constexpr (!SMALL) n0 = min(n0, pool.N - AD_COLS);
            if constexpr (KEPT) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int t = 0; t < 4; ++t) w[s][t] = weights(n0, s, t);
            }
#pragma unroll
            for (int b = 0; b < LIVE; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) old[b][h] = old_at(list[b * 16 + 8 * h + lane_id() / 8], n0 + lane_id() % 8 * 8);
        };
        if (block_at(0) < pool.N) fetch(block_at(0));
        __syncthreads();  // (the item before has been read)
        // u of the rows, SHARE threads a row
        {
            const int i = threadIdx.x / SHARE, own = list[i];
            const float scale = id >= 0 && pool.scales ? pool.scales[id] : 1.0f;
            f32x4 u[QUADS];
            float most = 0.0f;
#pragma unroll
            for (int q = 0; q < QUADS; ++q) {
                // places at .. at + 3 of the row hold the ranks j .. j + 3, of which the first may belong to the eight before
                const int at = 4 * (q * SHARE + (int)threadIdx.x % SHARE), j = eight_at(pool.rank, at / 8 * 8) + at % 8;
                u[q] = (f32x4)0.0f;
                if (at >= 32 * steps) continue;
                if (own >= 0 && j < r) {
                    const float *from = part + (first + own) * wide + j;
#pragma unroll 4
                    for (int s = 0; s < splits; ++s) u[q] += *reinterpret_cast<const Quad *>(from + (int64_t)s * M * wide);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    u[q][e] = j + e < r && j + e >= at / 8 * 8 ? u[q][e] * scale : 0.0f;
                    most = fmaxf(most, fabsf(u[q][e]));
                }
            }
            float f = 1.0f;
            if constexpr (std::is_same<T, _Float16>::value) {
#pragma unroll
                for (int o = 1; o < SHARE; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
                float b;
                f = into_half(most, b);
                if (threadIdx.x % SHARE == 0) back[i] = b;
            }
#pragma unroll
            for (int q = 0; q < QUADS; ++q) {
                const int j = 4 * (q * SHARE + (int)threadIdx.x % SHARE);
                if (j >= 32 * steps) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = u[q][e] * f;
                    const T h = (T)v;
                    hi[i * stride + j + e] = h;
                    if constexpr (TWO) lo[i * stride + j + e] = (T)(v - (float)h);
                }
            }
        }
        __syncthreads();
        for (int c = 0; c < blocks; ++c) {
            const int64_t from = block_at(c), n0 = SMALL ? from : min(from, pool.N - AD_COLS), n = n0 + lane_id() % 8 * 8;
            if (from >= pool.N) break;
            if (c) fetch(from);
            if constexpr (KEPT)
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int t = 0; t < 4; ++t) w[s][t] = cleared(w[s][t], s);
            const auto rows16 = [&](auto block) {
                constexpr int b = decltype(block)::value;
                f32x4 acc[4] = {};
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
                    if (s < steps) {
                        const int at = (b * 16 + l) * stride + 32 * s + 8 * g;
                        const V uh = *reinterpret_cast<const typename E::Lds *>(hi + at);
                        V ul;
                        if constexpr (TWO) ul = *reinterpret_cast<const typename E::Lds *>(lo + at);
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            V v;
                            if constexpr (KEPT) v = w[s][t];
                            else v = cleared(weights(n0, s, t), s);
                            acc[t] = mma(v, uh, acc[t]);
                            if constexpr (TWO) acc[t] = mma(v, ul, acc[t]);
                        }
                    }
                const float times = std::is_same<T, _Float16>::value ? back[b * 16 + l] : 1.0f;
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int t = 0; t < 4; ++t) turn[wave][(l * AD_TURN + 16 * t) / 4 + g] = acc[t] * times;
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int place = 8 * h + lane_id() / 8, row = list[b * 16 + place];
                    const f32x4 *sum = &turn[wave][(place * AD_TURN + lane_id() % 8 * 8) / 4];
                    const f32x4 low = sum[0], high = sum[1];
                    if (row < 0) continue;
                    V v = old[b][h];
                    if (r)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = (T)((e < 4 ? low[e % 4] : high[e % 4]) + (float)v[e]);
                    T *to = y + (first + row) * ldy + n;
                    if (!SMALL && n >= from) {
                        *reinterpret_cast<typename E::Raw *>(to) = v;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (n + e >= from && n + e < pool.N) to[e] = v[e];
                    }
                }
            };
            rows16(std::integral_constant<int, 0>());
            if constexpr (LIVE > 1)
                if (it.count > 16) rows16(std::integral_constant<int, 1>());
            if constexpr (LIVE > 2) {
                if (it.count > 32) rows16(std::integral_constant<int, 2>());
                if (it.count > 48) rows16(std::integral_constant<int, 3>());
            }
        }
    };
    each_item<ROWS>(load_tile(ids, first, rows, pool.count), slot, slots, rows, list, [&](const Item &it) {
        if (RB > 1 && it.count <= 16) take(it, std::integral_constant<int, 1>());
        else if (RB > 2 && it.count <= 32) take(it, std::integral_constant<int, RB < 2 ? RB : 2>());
        else take(it, std::integral_constant<int, RB>());
    });
}

struct AdPlan {
    int tiles, slots, splits, per, wide, chunks, blocks;
    bool many;  // 64 rows to an item
    size_t bytes;
};

AdPlan plan_adapters(int64_t M, int64_t N, int K, int rank, int count)
{
    AdPlan p;
    p.many = M >= 64 * (int64_t)count && M >= AD_MANY;
    const int each = p.many ? 64 : 16;
    p.tiles = (int)ceil_div(M, AD_TILE);
    const int rows = (int)std::min<int64_t>(M, AD_TILE);
    const int bound = std::min(rows, count + 1) + rows / each;  // items of a tile at most
    // 64 rows to an item: a tile of a few requests has four or five items (with a slot for each of up to 24, 3198 rows of 21 adapters in any
    // order 75 us for 59 in the second product).  16 rows: a workgroup for every row that may open one, unless these are four times
    // as many as the items (237 rows of one adapter, 12945 outputs, counted up 23.6 us for 33; 36 rows of 15 adapters 20 for 12).
    p.slots = p.many ? std::min(bound, 8) : bound <= std::min(20, rows / 4) ? bound : rows;
    p.slots = std::min(p.slots, std::max(1, 65536 / p.tiles));
    p.wide = (rank + 15) / 16 * 16;
    // items, where a batch's adapters are about as many as there may be
    const int64_t items = (int64_t)p.tiles * (p.many ? rows / 64 : std::min(rows, std::min(count, rows) + rows / 16));
    const int steps = (K + 31) / 32;
    const int least = std::max(1, steps / 8);  // two steps a wavefront at least
    const int read = std::max(1, 65536 / (each * p.wide * 4));  // what every workgroup of the second product reads of the first
    // More than that where a wavefront would have more than 16 steps, counted for every 64 ranks: 14336 inputs and rank 128, 2048 rows 191 us
    // with two splits and 87 with eight, 16 rows 29 with eight and 23 with fourteen; but of 4096 and 64, 4096 rows, 43 with four and 50
    // with eight.
    const int longer = std::min(p.many ? 8 : 16, steps * ((rank + 63) / 64) / 64);
    const int want = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(least, std::max(read, longer)), 768 / std::max<int64_t>(1, items)));
    p.per = (int)ceil_div(steps, 4 * want);
    p.splits = (int)ceil_div(steps, 4 * p.per);
    p.bytes = (size_t)p.splits * M * p.wide * sizeof(float);
    // Outputs a workgroup: as many as leave one round of workgroups, each of which adds u up anew (8192 rows of rank 64, 4096 outputs:
    // one block of 64 a wavefront 58 us, two 52, four 40, eight 55; 64 rows, 16384 outputs: 16, 12.6, 10.8, 13.9).
    const int64_t cols = ceil_div(N, AD_COLS * (AD_WG / WAVE));
    p.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(8, ceil_div(cols * items, p.many ? 512 : 640)));
    p.chunks = (int)ceil_div(cols, p.blocks);
    // A grid's threads are counted in 32 bits: with very many outputs a workgroup takes several of its tile's items one after the other.
    const int64_t most = (AD_GROUPS - 1) / ((int64_t)p.tiles * std::max(p.splits, p.chunks));
    p.slots = (int)std::min<int64_t>(p.slots, std::max<int64_t>(1, most));
    return p;
}

}  // namespace

static bool pool_ok(const qadc_adapters *w)
{
    return w && type_ok(w->type) && w->N >= 1 && w->N <= 1 << 30 && w->K >= 1 && w->K <= 1 << 24 && w->rank >= 1 &&
           w->rank <= QADC_MAX_RANK && w->count >= 1 && w->count <= 1 << 20;
}

// Enough for these rows and for any fewer.
size_t adapters_workspace(const qadc_adapters *w, int64_t M)
{
    if (!pool_ok(w) || M < 1 || M > 1 << 24) return 0;
    // (m rows are cut into at most 768 / (m / 256) splits, or what leaves each two steps)
    const int64_t most = std::max(1, (w->K + 31) / 32 / 8);
    return (size_t)std::min(most * M, std::max<int64_t>(M, 768 * AD_TILE)) * ((w->rank + 15) / 16 * 16) * sizeof(float);
}

template <typename T, int RB>
static void launch_adapters(const AdPlan &p, const Pool &pool, const int32_t *ids, const void *x, int64_t ldx, int64_t M, const void *base,
                            int64_t ldb, void *y, int64_t ldy, float *part, hipStream_t st)
{
    const dim3 down((unsigned)(p.tiles * p.slots * p.splits));
    if (pool.rank <= 16)
        launch(QADC_PROF_ADAPTERS, adapters_down_kernel<T, 1, RB>, down, dim3(AD_WG), 0, st, pool, ids, (const T *)x, ldx, M, p.slots,
               p.splits, p.per, p.wide, part);
    else
        launch(QADC_PROF_ADAPTERS, adapters_down_kernel<T, 4, RB>, down, dim3(AD_WG), 0, st, pool, ids, (const T *)x, ldx, M, p.slots,
               p.splits, p.per, p.wide, part);
    const auto up = [&](auto steps, auto small) {
        constexpr int S = decltype(steps)::value;
        const size_t lds = 16 * RB * (32 * S + 16 / sizeof(T)) * sizeof(T) * (sizeof(T) == 2 ? 2 : 1);
        launch(QADC_PROF_ADAPTERS, adapters_up_kernel<T, RB, S, decltype(small)::value>, dim3((unsigned)(p.tiles * p.slots * p.chunks)),
               dim3(AD_WG), lds, st, pool, ids, M, p.slots, p.chunks, p.blocks, p.splits, p.wide, (const float *)part, (const T *)base, ldb,
               (T *)y, ldy);
    };
    if (pool.N < AD_COLS) up(std::integral_constant<int, 4>(), std::true_type());
    else if (pool.rank < 8) up(std::integral_constant<int, 1>(), std::true_type());
    else if (pool.rank <= 32) up(std::integral_constant<int, 1>(), std::false_type());
    else if (pool.rank <= 64) up(std::integral_constant<int, 2>(), std::false_type());
    else up(std::integral_constant<int, 4>(), std::false_type());
}

int add_adapters(const qadc_adapters *w, const int32_t *ids, const void *x, int64_t ldx, int64_t M, const void *base, int64_t ldb, void *y,
                 int64_t ldy, void *workspace, size_t workspace_bytes, hipStream_t st)
{
    const char *who = "qadc_add_adapters";
    if (!w) return fail(QADC_EINVAL, "%s: null pointer", who);
    if (!pool_ok(w))
        return fail(QADC_EINVAL, "%s: type=%d N=%lld K=%d rank=%d count=%d", who, w->type, (long long)w->N, w->K, w->rank, w->count);
    if (M < 0 || M > 1 << 24) return fail(QADC_EINVAL, "%s: M=%lld", who, (long long)M);
    if (ldx < w->K || ldy < w->N || (base && ldb < w->N)) return fail(QADC_EINVAL, "%s: rows overlap", who);
    if (M == 0) return QADC_OK;
    if (!w->a || !w->b || !ids || !x || !y) return fail(QADC_EINVAL, "%s: null pointer", who);
    if (base == y && ldb != ldy) return fail(QADC_EINVAL, "%s: in place needs equal row distances", who);
    const AdPlan p = plan_adapters(M, w->N, w->K, w->rank, w->count);
    if ((int64_t)p.tiles * p.slots * std::max(p.splits, p.chunks) >= AD_GROUPS)
        return fail(QADC_EINVAL, "%s: M=%lld rows of N=%lld outputs are too many for one call", who, (long long)M, (long long)w->N);
    if (!workspace || workspace_bytes < p.bytes)
        return fail(QADC_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, p.bytes);
    if ((uintptr_t)workspace % 16) return fail(QADC_EINVAL, "%s: workspace is not aligned to 16 bytes", who);
    const Pool pool = {w->a, w->b, w->scales, w->ranks, w->N, w->K, w->rank, w->count};
    QADC_BY_TYPE(w->type, {
        if (p.many) launch_adapters<T, 4>(p, pool, ids, x, ldx, M, base, ldb, y, ldy, (float *)workspace, st);
        else launch_adapters<T, 1>(p, pool, ids, x, ldx, M, base, ldb, y, ldy, (float *)workspace, st);
    });
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
