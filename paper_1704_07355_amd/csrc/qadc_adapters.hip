// Low-rank adapters of many requests beside a shared projection on gfx950: y_i = base_i + s_a B_a (A_a x_i), a = ids[i].
//
// Two launches: u = A x into the workspace, cut over the inputs, then y = base + s B u.  Rows come in tiles of 256 consecutive ones;
// every workgroup groups its tile's rows by adapter, up to 16 (or 64) of one adapter to an item, so that an adapter is
// read once for all its rows of a tile, wherever they lie.  Both products are on the matrix units, with the adapter's side as the
// first operand: a lane then holds the results of one row, which differ between rows and are added where the row lies.
//
// Of 16-bit types u goes into the second product as two numbers, u rounded and what that leaves: off by 2^-16 (bfloat16) or 2^-22
// (binary16, scaled by a power of two into its range), so that only y's own rounding shows.  float32 is multiplied as float32.
#include <algorithm>
#include <type_traits>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int AD_WG = 256, AD_TILE = 256;  // threads; rows of a tile, one a thread
constexpr int AD_COLS = 64;                // outputs of a wavefront at a time

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements, of which n are there; zeros behind.
template <typename T>
struct Eight {
    typedef T V __attribute__((ext_vector_type(8)));
    typedef T Raw __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    typedef T Lds __attribute__((ext_vector_type(8), aligned(16)));
    static __device__ __forceinline__ V zero() { return (V)(T)0.0f; }
    static __device__ __forceinline__ V load(const T *p, int n)
    {
        if (n >= 8) return *reinterpret_cast<const Raw *>(p);
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

// A tile's rows by adapter: thread i has row i of the tile in item `item` at `place`; items are numbered by their first rows.
struct Items {
    int item, place;
};
struct ItemsLds {
    __attribute__((aligned(16))) int ids[AD_TILE];
    int number[AD_TILE];  // of the item that a row opens
    int id[AD_TILE];      // of an item
    int opened[AD_TILE / WAVE];
    int16_t rows[64];     // of the item at hand, -1: none
};

// ROWS of them to an item; -1 as id: no adapter.  Returns the number of items.
template <int ROWS>
__device__ __forceinline__ int group_rows(const int32_t *ids, int64_t first, int rows, int count, Items &mine, ItemsLds &lds)
{
    const int i = threadIdx.x;
    int id = -2;  // behind the last row
    if (i < rows) {
        id = ids[first + i];
        if (id < 0 || id >= count) id = -1;
    }
    lds.ids[i] = id;
    __syncthreads();
    int before = 0, opener = i;
    for (int j = 0; j < i && j < rows; j += 4) {
        const int4 v = *reinterpret_cast<const int4 *>(&lds.ids[j]);
        const int w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (w[e] == id && j + e < i) {
                if (before % ROWS == 0) opener = j + e;
                ++before;
            }
    }
    const bool opens = i < rows && before % ROWS == 0;
    if (opens) opener = i;
    const unsigned long long m = __ballot(opens);
    if (lane_id() == 0) lds.opened[i >> 6] = __popcll(m);
    __syncthreads();
    int number = (int)rank_in_mask(m), total = 0;
#pragma unroll
    for (int w = 0; w < AD_TILE / WAVE; ++w) {
        if (w < i >> 6) number += lds.opened[w];
        total += lds.opened[w];
    }
    if (opens) {
        lds.number[i] = number;
        lds.id[number] = id;
    }
    __syncthreads();
    mine.item = i < rows ? lds.number[opener] : -1;
    mine.place = before % ROWS;
    return total;
}
// The rows of an item into lds.rows; a barrier before and behind.  Returns how many there are.
template <int ROWS>
__device__ __forceinline__ void rows_of(int item, const Items &mine, ItemsLds &lds)
{
    __syncthreads();
    if (threadIdx.x < ROWS) lds.rows[threadIdx.x] = -1;
    __syncthreads();
    if (mine.item == item) lds.rows[mine.place] = (int16_t)threadIdx.x;
    __syncthreads();
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
    __shared__ ItemsLds lds;
    __shared__ f32x4 red[AD_WG / WAVE][RT][WAVE];
    const int split = blockIdx.x % splits, slot = blockIdx.x / splits % slots;
    const int64_t first = (int64_t)(blockIdx.x / splits / slots) * AD_TILE;
    const int wave = threadIdx.x >> 6, l = lane_id() % 16, g = lane_id() / 16;
    Items mine;
    const int items = group_rows<16 * RB>(ids, first, (int)min((int64_t)AD_TILE, M - first), pool.count, mine, lds);
    const int steps = (pool.K + 31) / 32, s0 = min(steps, (split * 4 + wave) * per), s1 = min(steps, s0 + per);
    for (int item = slot; item < items; item += slots) {
        const int id = lds.id[item];
        if (id < 0) continue;
        rows_of<16 * RB>(item, mine, lds);
        const int r = rank_of(pool, id);
        const T *xr[RB];
        int row[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            row[b] = lds.rows[b * 16 + l];
            xr[b] = x + (first + max(row[b], 0)) * ldx;
        }
        for (int p = 0; p < r; p += 16 * RT) {
            f32x4 acc[RT][RB] = {};
            const T *ar[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) ar[t] = (const T *)pool.a + ((int64_t)id * pool.rank + min(p + 16 * t + l, r - 1)) * pool.K;
            for (int s = s0; s < s1; ++s) {
                const int k = 32 * s + 8 * g, n = pool.K - k;
                typename E::V av[RT], xv[RB];
#pragma unroll
                for (int t = 0; t < RT; ++t) av[t] = p + 16 * t + l < r ? E::load(ar[t] + k, n) : E::zero();
#pragma unroll
                for (int b = 0; b < RB; ++b) xv[b] = row[b] >= 0 ? E::load(xr[b] + k, n) : E::zero();
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int b = 0; b < RB; ++b) acc[t][b] = mma(av[t], xv[b], acc[t][b]);
            }
#pragma unroll
            for (int b = 0; b < RB; ++b) {
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
    }
}

// A power of two that takes `most` to 2^10 .. 2^11, and its inverse.
__device__ __forceinline__ float into_half(float most, float &back)
{
    const int e = min(max((int)(__float_as_uint(most) >> 23), 20), 240) - 127 - 10;
    back = __uint_as_float((unsigned)(127 + e) << 23);
    return __uint_as_float((unsigned)(127 - e) << 23);
}

// y of the rows of an item, `blocks` times 64 outputs a wavefront.
template <typename T, int RB>
__global__ __launch_bounds__(AD_WG) void adapters_up_kernel(Pool pool, const int32_t *__restrict__ ids, int64_t M, int slots, int chunks,
                                                            int blocks, int splits, int wide, const float *__restrict__ part,
                                                            const T *base, int64_t ldb, T *y, int64_t ldy)
{
    typedef Eight<T> E;
    constexpr int ROWS = 16 * RB, SHARE = AD_WG / ROWS, QUADS = QADC_MAX_RANK / 4 / SHARE;
    constexpr bool TWO = sizeof(T) == 2;
    __shared__ ItemsLds lds;
    __shared__ float back[ROWS];
    extern __shared__ __attribute__((aligned(16))) char raw[];
    const int pad = (pool.rank + 31) / 32 * 32, stride = pad + 16 / (int)sizeof(T);
    T *hi = (T *)raw, *lo = hi + ROWS * stride;
    const int chunk = blockIdx.x % chunks, slot = blockIdx.x / chunks % slots;
    const int64_t first = (int64_t)(blockIdx.x / chunks / slots) * AD_TILE;
    const int wave = threadIdx.x >> 6, l = lane_id() % 16, g = lane_id() / 16;
    Items mine;
    const int items = group_rows<ROWS>(ids, first, (int)min((int64_t)AD_TILE, M - first), pool.count, mine, lds);
    for (int item = slot; item < items; item += slots) {
        const int id = lds.id[item];
        if (id < 0 && base == y) continue;
        rows_of<ROWS>(item, mine, lds);
        const int r = id < 0 ? 0 : rank_of(pool, id), steps = (r + 31) / 32;
        // u of the rows, SHARE threads a row
        {
            const int i = threadIdx.x / SHARE, row = lds.rows[i];
            const float scale = id >= 0 && pool.scales ? pool.scales[id] : 1.0f;
            f32x4 u[QUADS];
            float most = 0.0f;
#pragma unroll
            for (int q = 0; q < QUADS; ++q) {
                const int j = 4 * (q * SHARE + (int)threadIdx.x % SHARE);
                u[q] = (f32x4)0.0f;
                if (j >= 32 * steps) continue;
                if (row >= 0 && j < r)
                    for (int s = 0; s < splits; ++s)
                        u[q] += *reinterpret_cast<const f32x4 *>(part + ((int64_t)s * M + first + row) * wide + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    u[q][e] = j + e < r ? u[q][e] * scale : 0.0f;
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
        int row[RB];
        float times[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            row[b] = lds.rows[b * 16 + l];
            times[b] = std::is_same<T, _Float16>::value ? back[b * 16 + l] : 1.0f;
        }
        for (int c = 0; c < blocks; ++c) {
            // outputs n0 + 16 g + 4 t + e of this lane; the weights' rows go in so that the lane's sixteen lie side by side
            const int64_t n0 = ((int64_t)(chunk * blocks + c) * (AD_WG / WAVE) + wave) * AD_COLS;
            if (n0 >= pool.N) break;
            const int64_t n = n0 + 16 * g;
            const int there = (int)min((int64_t)16, pool.N - n);
            typename E::V old[RB][2];
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    old[b][h] = base && row[b] >= 0 ? E::load(base + (first + row[b]) * ldb + n + 8 * h, there - 8 * h) : E::zero();
            f32x4 acc[4][RB] = {};
            for (int s = 0; s < steps; ++s) {
                const int j = 32 * s + 8 * g;
                typename E::V w[4], uh[RB], ul[RB];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int64_t of = n0 + 16 * (l / 4) + 4 * t + l % 4;
                    w[t] = of < pool.N ? E::load((const T *)pool.b + ((int64_t)id * pool.N + of) * pool.rank + j, r - j) : E::zero();
                }
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    uh[b] = *reinterpret_cast<const typename E::Lds *>(hi + (b * 16 + l) * stride + j);
                    if constexpr (TWO) ul[b] = *reinterpret_cast<const typename E::Lds *>(lo + (b * 16 + l) * stride + j);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        acc[t][b] = mma(w[t], uh[b], acc[t][b]);
                        if constexpr (TWO) acc[t][b] = mma(w[t], ul[b], acc[t][b]);
                    }
            }
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                if (row[b] < 0) continue;
                T *to = y + (first + row[b]) * ldy + n;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    typename E::V v;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] = r ? (T)fmaf(acc[2 * h + e / 4][b][e % 4], times[b], (float)old[b][h][e]) : old[b][h][e];
                    if (there >= 8 * h + 8) {
                        *reinterpret_cast<typename E::Raw *>(to + 8 * h) = v;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (8 * h + e < there) to[8 * h + e] = v[e];
                    }
                }
            }
        }
    }
}

struct AdPlan {
    int tiles, slots, splits, per, wide, chunks, blocks;
    bool many;  // 64 rows to an item
    size_t bytes;
};

AdPlan plan_adapters(int64_t M, int64_t N, int K, int rank, int count)
{
    AdPlan p;
    p.many = M >= 64 * (int64_t)count && M >= 256;
    const int each = p.many ? 64 : 16;
    p.tiles = (int)ceil_div(M, AD_TILE);
    const int rows = (int)std::min<int64_t>(M, AD_TILE);
    const int bound = std::min(rows, std::min(count + 1, rows) + rows / each);  // items of a tile at most
    p.slots = std::min(p.many ? std::min(bound, 8) : bound, std::max(1, 16384 / p.tiles));
    p.wide = (rank + 15) / 16 * 16;
    const int steps = (K + 31) / 32;
    const int64_t wgs = (int64_t)p.tiles * std::min(bound, std::max(1, rows / each) + (p.many ? 0 : std::min(count, rows)));
    const int most = std::max(1, steps / 8);  // two steps a wavefront at least
    const int want = (int)std::max<int64_t>(1, std::min<int64_t>(most, 512 / std::max<int64_t>(1, wgs)));
    p.per = (int)ceil_div(steps, 4 * want);
    p.splits = (int)ceil_div(steps, 4 * p.per);
    p.bytes = (size_t)p.splits * M * p.wide * sizeof(float);
    const int64_t cols = ceil_div(N, AD_COLS * (AD_WG / WAVE));
    p.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(8, cols * wgs / 1024));
    p.chunks = (int)ceil_div(cols, p.blocks);
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
    // (m rows are cut into at most 512 / (m / 256) splits, or what leaves each two steps)
    const int64_t most = std::max(1, (w->K + 31) / 32 / 8);
    return (size_t)std::min(most * M, std::max<int64_t>(M, 512 * AD_TILE)) * ((w->rank + 15) / 16 * 16) * sizeof(float);
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
    const size_t pad = (pool.rank + 31) / 32 * 32, lds = 16 * RB * (pad + 16 / sizeof(T)) * sizeof(T) * (sizeof(T) == 2 ? 2 : 1);
    launch(QADC_PROF_ADAPTERS, adapters_up_kernel<T, RB>, dim3((unsigned)(p.tiles * p.slots * p.chunks)), dim3(AD_WG), lds, st, pool, ids, M,
           p.slots, p.chunks, p.blocks, p.splits, p.wide, (const float *)part, (const T *)base, ldb, (T *)y, ldy);
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
    if ((int64_t)p.tiles * p.slots * std::max(p.splits, p.chunks) > 1 << 24)
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
