// Products with 4-bit weights and group scales on gfx950.
//
// Packed weights.  A tile is 16 outputs x 128 inputs: 64 lanes x 16 bytes, lane l = 16 j + n holding of output n the inputs
// 32 s + 8 j + 0 .. 7 in its dword s = 0 .. 3, which is the order in which a matrix instruction over 16 outputs and 32 inputs
// takes them, four instructions a tile.  Of a dword's eight weights, weight 2 i is nibble i and weight 2 i + 1 nibble i + 4, so
// that one shift and one mask leave a pair in the two halves of a register.  Tiles of one block of 16 outputs follow each
// other along the inputs; behind all tiles lie the scales and the zero points, [block][set][16][per set], where a set is the
// groups of a tile (4, 2 or 1) or, of groups beyond 128 inputs, one group.  Outputs and inputs beyond N and K are zero nibbles
// with scale 0.
//
// The product.  A nibble q put into the mantissa of 16 is the 16-bit number 16 + q, exactly: no conversion, one shift and one
// and-or for a pair.  The matrix units multiply these with x (float32 x as the sum of three bfloat16 numbers) and, once for all
// outputs, a column of ones with x; with p and t the two sums over a group, the group adds s (p - (16 + z) t) to the output.

#include <algorithm>
#include <type_traits>

#include "qadc_half.h"
#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int W4_N = 16, W4_K = 128, W4_BYTES = W4_N * W4_K / 2;  // a tile

struct Shape4 {
    int64_t blocks;  // of 16 outputs
    int tiles;       // of 128 inputs
    int per;         // groups per set
    int span;        // tiles per set
    int sets;
    size_t scales, zeros, bytes;  // where the scales and zero points begin, and the end
};

__host__ __device__ inline Shape4 shape4(int64_t N, int K, int group, bool has_zeros)
{
    Shape4 s;
    s.blocks = (N + W4_N - 1) / W4_N;
    s.tiles = (K + W4_K - 1) / W4_K;
    s.per = group < W4_K ? W4_K / group : 1;
    s.span = group < W4_K ? 1 : group / W4_K;
    s.sets = (s.tiles + s.span - 1) / s.span;
    s.scales = (size_t)s.blocks * s.tiles * W4_BYTES;
    const size_t count = (size_t)s.blocks * s.sets * W4_N * s.per;
    s.zeros = s.scales + count * 2;
    s.bytes = s.zeros + (has_zeros ? count : 0);
    return s;
}

// A thread per dword of the packed weights.
__global__ __launch_bounds__(256) void pack4_codes_kernel(const uint8_t *__restrict__ codes, int64_t N, int K, int tiles,
                                                          int64_t dwords, uint32_t *__restrict__ packed)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < dwords; i += (int64_t)gridDim.x * 256) {
        const int s = (int)(i & 3), lane = (int)(i >> 2 & 63);
        const int64_t tile = i >> 8;
        const int64_t n = tile / tiles * W4_N + (lane & 15);
        const int64_t k0 = tile % tiles * W4_K + 32 * s + 8 * (lane >> 4);
        uint32_t v = 0;
        if (n < N) {
            const uint8_t *row = codes + n * (((int64_t)K + 1) / 2);
            for (int e = 0; e < 8; ++e) {
                const int64_t k = k0 + e;
                const uint32_t q = k < K ? (uint32_t)(row[k >> 1] >> (4 * (k & 1)) & 15) : 0u;
                v |= q << (4 * ((e >> 1) + 4 * (e & 1)));
            }
        }
        packed[i] = v;
    }
}

// A thread per group of an output.
__global__ __launch_bounds__(256) void pack4_scales_kernel(const uint16_t *__restrict__ scales,
                                                           const uint8_t *__restrict__ zeros, int64_t N, int groups, int sets,
                                                           int per, int64_t count, uint16_t *__restrict__ packed_scales,
                                                           uint8_t *__restrict__ packed_zeros)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t set = i / (W4_N * per), n = set / sets * W4_N + i / per % W4_N, g = set % sets * per + i % per;
        const bool in = n < N && g < groups;
        packed_scales[i] = in ? scales[n * groups + g] : (uint16_t)0;
        if (zeros) packed_zeros[i] = in ? zeros[n * groups + g] : (uint8_t)0;
    }
}

__device__ __forceinline__ float scale4(uint16_t bits, int stype)
{
    return stype == QADC_TYPE_F16 ? (float)__builtin_bit_cast(_Float16, bits) : __uint_as_float((unsigned)bits << 16);
}

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The eight weights of a dword as 16 + q, in the type that the matrix units take: nibbles into bits 6 .. 9 of a binary16 of
// exponent 4, into bits 3 .. 6 of a bfloat16.
template <bool HALF>
__device__ __forceinline__ bits16x8 weights8(unsigned v)
{
    bits16x8 w;
    if constexpr (HALF) {
        w[0] = (v << 6 & 0x03C003C0u) | 0x4C004C00u;
        w[1] = (v << 2 & 0x03C003C0u) | 0x4C004C00u;
        w[2] = (v >> 2 & 0x03C003C0u) | 0x4C004C00u;
        w[3] = (v >> 6 & 0x03C003C0u) | 0x4C004C00u;
    } else {
        w[0] = (v << 3 & 0x00780078u) | 0x41804180u;
        w[1] = (v >> 1 & 0x00780078u) | 0x41804180u;
        w[2] = (v >> 5 & 0x00780078u) | 0x41804180u;
        w[3] = (v >> 9 & 0x00780078u) | 0x41804180u;
    }
    return w;
}

template <bool HALF>
__device__ __forceinline__ f32x4 mfma16(bits16x8 a, bits16x8 b, f32x4 c)
{
    if constexpr (HALF)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight inputs of a row of x as the matrix units' operands; a float32 in three parts of eight bits each, cut off, not rounded:
// their sum is the number itself.
template <typename T>
struct Inputs {
    static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    static constexpr bool HALF = std::is_same_v<T, _Float16>;
    bits16x8 part[PARTS];

    typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    __device__ static __forceinline__ V load_last(const T *row, int64_t k, int64_t K)  // 0 beyond the row
    {
        V v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < K ? row[k + e] : (T)0.0f;
        return v;
    }
    __device__ __forceinline__ explicit Inputs(V v)
    {
        if constexpr (PARTS == 1) {
            part[0] = __builtin_bit_cast(bits16x8, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo = v[2 * i], hi = v[2 * i + 1];
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const unsigned a = __float_as_uint(lo) & 0xffff0000u, b = __float_as_uint(hi) & 0xffff0000u;
                    part[p][i] = a >> 16 | b;
                    lo -= __uint_as_float(a);
                    hi -= __uint_as_float(b);
                }
            }
        }
    }
};

// Wavefronts that may share a block: their sums, `values` a lane, fit in 64 KB.
constexpr int most_split(int values) { return values <= 8 ? 16 : 8; }

struct Args4 {
    const char *packed;
    Shape4 s;
    int64_t N, M, ldx, ldy;
    int K, stype, has_zeros;
    const float *bias;
};

// A block of NT x 16 outputs and up to 16 MT rows of x: SPLIT wavefronts, each every SPLIT-th tile of the inputs.  Of a matrix
// instruction's 16 rows, 4 q + i, the first MR of every four are rows of x (MR = 1 for up to four rows: a quarter of the work
// behind the products); the others repeat them.  STEPS: instructions per group.
template <typename T, int STEPS, int MR, int MT, int NT>
__global__ __launch_bounds__(WAVE *most_split(MT *NT *MR)) void linear4_kernel(Args4 a, const T *__restrict__ x, T *__restrict__ y, int split)
{
    constexpr int DEPTH = 2, PER = 4 / STEPS, ROWS = 4 * MR * MT;
    constexpr bool HALF = Inputs<T>::HALF, AHEAD = MT * sizeof(T) <= 4;
    extern __shared__ float lds[];
    const int lane = lane_id(), wave = threadIdx.x >> 6, n = lane & 15, j = lane >> 4;
    const int at_once = (int)(blockDim.x >> 6) / split;  // blocks of a workgroup
    const int64_t block = ((int64_t)blockIdx.x * at_once + wave / split) * NT;
    const int part = wave % split;
    const int64_t m0 = (int64_t)blockIdx.y * ROWS;
    const int tiles = a.s.tiles;

    // this lane's row of x in each m-tile, and where its weights and scales are
    const T *rows[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int i = n & 3;
        const int64_t m = m0 + t * 4 * MR + (n >> 2) * MR + (i < MR ? i : 0);
        rows[t] = x + min(m, a.M - 1) * a.ldx;
    }
    const bits16x8 *weights[NT];
    const char *scales[NT], *zeros[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t b = min(block + t, a.s.blocks - 1);
        weights[t] = reinterpret_cast<const bits16x8 *>(a.packed) + b * tiles * WAVE + lane;
        scales[t] = a.packed + a.s.scales + (b * a.s.sets * W4_N + n) * PER * 2;
        zeros[t] = a.packed + a.s.zeros + (b * a.s.sets * W4_N + n) * PER;
    }
    f32x4 sum[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) sum[t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    bits16x8 ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones[i] = HALF ? 0x3C003C00u : 0x3F803F80u;

    // The next tiles on their way: weights, scales and zero points DEPTH tiles ahead, x one.
    typedef typename Inputs<T>::V V;
    typedef std::conditional_t<PER == 4, u32x2, std::conditional_t<PER == 2, uint32_t, uint16_t>> Scales;
    typedef std::conditional_t<PER == 4, uint32_t, std::conditional_t<PER == 2, uint16_t, uint8_t>> Zeros;
    bits16x8 ring[DEPTH][NT];
    Scales ring_s[DEPTH][NT];
    Zeros ring_z[DEPTH][NT];
    const auto fetch = [&](int d, int k) {
        const int64_t set = k / a.s.span * W4_N;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            ring[d][t] = __builtin_nontemporal_load(weights[t] + (int64_t)k * WAVE);
            ring_s[d][t] = reinterpret_cast<const Scales *>(scales[t])[set];
            if (a.has_zeros) ring_z[d][t] = reinterpret_cast<const Zeros *>(zeros[t])[set];
        }
    };
    const auto fetch_x = [&](int k, V(&v)[MT][4]) {
        const int64_t at = (int64_t)k * W4_K + 8 * j;
        if ((int64_t)(k + 1) * W4_K <= a.K) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int s = 0; s < 4; ++s) v[t][s] = *reinterpret_cast<const V *>(rows[t] + at + 32 * s);
        } else {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int s = 0; s < 4; ++s) v[t][s] = Inputs<T>::load_last(rows[t], at + 32 * s, a.K);
        }
    };
    V xs[MT][4], xn[MT][4];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (part + d * split < tiles) fetch(d, part + d * split);
    if (part < tiles) fetch_x(part, xn);

    for (int k0 = part; k0 < tiles; k0 += DEPTH * split) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int k = k0 + d * split;
            if (k < tiles) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int s = 0; s < 4; ++s) xs[t][s] = xn[t][s];
                if (AHEAD && k + split < tiles) fetch_x(k + split, xn);
                bits16x8 now[NT];
                float sc[NT][PER], zp[NT][PER];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    now[t] = ring[d][t];
                    uint16_t bits[PER];
                    uint8_t z[PER];
                    __builtin_memcpy(bits, &ring_s[d][t], sizeof(bits));
                    __builtin_memcpy(z, &ring_z[d][t], sizeof(z));
#pragma unroll
                    for (int g = 0; g < PER; ++g) {
                        sc[t][g] = scale4(bits[g], a.stype);
                        zp[t][g] = a.has_zeros ? 16.0f + (float)z[g] : 24.0f;
                    }
                }
                if (k + DEPTH * split < tiles) fetch(d, k + DEPTH * split);
#pragma unroll
                for (int g = 0; g < PER; ++g) {
                    f32x4 p[MT][NT], one[MT];
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        const int step = g * STEPS + s;
                        bits16x8 w[NT];
#pragma unroll
                        for (int u = 0; u < NT; ++u) w[u] = weights8<HALF>(now[u][step]);
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            const Inputs<T> in(xs[t][step]);
#pragma unroll
                            for (int q = 0; q < Inputs<T>::PARTS; ++q) {
                                const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
                                one[t] = mfma16<HALF>(in.part[q], ones, s + q ? one[t] : none);
#pragma unroll
                                for (int u = 0; u < NT; ++u) p[t][u] = mfma16<HALF>(in.part[q], w[u], s + q ? p[t][u] : none);
                            }
                        }
                    }
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int u = 0; u < NT; ++u)
#pragma unroll
                            for (int i = 0; i < MR; ++i)
                                sum[t][u][i] = fmaf(sc[u][g], fmaf(-zp[u][g], one[t][i], p[t][u][i]), sum[t][u][i]);
                }
                if (!AHEAD && k + split < tiles) fetch_x(k + split, xn);
            }
        }
    }

    const auto write = [&](int64_t b, int t, int i, float v) {  // output n of block b, row (t, j, i)
        const int64_t m = m0 + t * 4 * MR + j * MR + i, out = b * W4_N + n;
        if (m < a.M && out < a.N) y[m * a.ldy + out] = (T)(v + (a.bias ? a.bias[out] : 0.0f));
    };
    if (split == 1) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int i = 0; i < MR; ++i) write(block + u, t, i, sum[t][u][i]);
        return;
    }
    // the wavefronts' sums, joined in their order: [wave][value][lane]
    constexpr int VALUES = MT * NT * MR;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int i = 0; i < MR; ++i) lds[(wave * VALUES + (t * NT + u) * MR + i) * WAVE + lane] = sum[t][u][i];
    __syncthreads();
    for (int v = part; v < VALUES; v += split) {
        float total = 0.0f;
        for (int p = 0; p < split; ++p) total += lds[((wave - part + p) * VALUES + v) * WAVE + lane];
        write(block + v / MR % NT, v / (MR * NT), v % MR, total);
    }
}

int check4(const char *who, int64_t N, int K, int group, int stype)
{
    if (N < 1 || N > (1ll << 31) - 16 || K < 1 || K > (1 << 24))
        return fail(QADC_EINVAL, "%s: N=%lld K=%d", who, (long long)N, K);
    if (group != 32 && group != 64 && (group < 128 || group % 128 != 0))
        return fail(QADC_EINVAL, "%s: group=%d is neither 32, 64 nor a multiple of 128", who, group);
    if (stype != QADC_TYPE_F16 && stype != QADC_TYPE_BF16) return fail(QADC_EINVAL, "%s: unknown type %d of scales", who, stype);
    return QADC_OK;
}

}  // namespace

size_t weights4_bytes(int64_t N, int K, int group, int has_zeros)
{
    if (check4("qadc_weights4_bytes", N, K, group, QADC_TYPE_F16)) return 0;
    return shape4(N, K, group, has_zeros != 0).bytes;
}

int pack_weights4(const uint8_t *codes, const void *scales, int stype, const uint8_t *zeros, int64_t N, int K, int group,
                  void *packed, hipStream_t st)
{
    if (const int rc = check4("qadc_pack_weights4", N, K, group, stype)) return rc;
    if (!codes || !scales || !packed) return fail(QADC_EINVAL, "qadc_pack_weights4: null pointer");
    if ((uintptr_t)packed % 16) return fail(QADC_EINVAL, "qadc_pack_weights4: packed is not 16-byte aligned");
    const Shape4 s = shape4(N, K, group, zeros != nullptr);
    const int64_t dwords = (int64_t)(s.scales / 4), count = s.blocks * s.sets * W4_N * s.per;
    const auto grid = [](int64_t n) { return dim3((unsigned)std::min<int64_t>(ceil_div(n, 256), 1 << 16)); };
    hipLaunchKernelGGL(pack4_codes_kernel, grid(dwords), dim3(256), 0, st, codes, N, K, s.tiles, dwords, (uint32_t *)packed);
    hipLaunchKernelGGL(pack4_scales_kernel, grid(count), dim3(256), 0, st, (const uint16_t *)scales, zeros, N,
                       (int)ceil_div(K, group), s.sets, s.per, count, (uint16_t *)((char *)packed + s.scales),
                       (uint8_t *)packed + s.zeros);
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

template <typename T, int STEPS, int MR, int MT, int NT>
static void linear4_launch(const Args4 &a, const void *x, void *y, hipStream_t st)
{
    // As many wavefronts a block as the chip holds for these outputs, but no more than there are tiles.
    constexpr int most = most_split(MT * NT * MR);
    const int64_t blocks = ceil_div(a.s.blocks, NT), rows = ceil_div(a.M, 4 * MR * MT);
    int split = 1;
    while (split < most && blocks * rows * split < 4096 && 2 * split <= a.s.tiles) split *= 2;
    const int waves = std::max(split, 4), at_once = waves / split;
    const size_t shared = split > 1 ? (size_t)waves * MT * NT * MR * WAVE * sizeof(float) : 0;
    launch(QADC_PROF_LINEAR4, linear4_kernel<T, STEPS, MR, MT, NT>, dim3((unsigned)ceil_div(blocks, at_once), (unsigned)rows),
           dim3(waves * WAVE), shared, st, a, (const T *)x, (T *)y, split);
}

template <typename T, int STEPS>
static void linear4_rows(Args4 a, const T *x, T *y, hipStream_t st)
{
    // the y dimension of a grid is 16 bits wide: rows in slabs
    const int64_t slab = 65535 * 64ll, M = a.M;
    for (int64_t m = 0; m < M; m += slab) {
        a.M = std::min(slab, M - m);
        const T *xs = x + m * a.ldx;
        T *ys = y + m * a.ldy;
        if (a.M <= 4) linear4_launch<T, STEPS, 1, 1, 2>(a, xs, ys, st);
        else if (a.M <= 16) linear4_launch<T, STEPS, 4, 1, 2>(a, xs, ys, st);
        else if (a.M <= 32) linear4_launch<T, STEPS, 4, 2, 2>(a, xs, ys, st);
        else linear4_launch<T, STEPS, 4, 4, 2>(a, xs, ys, st);
    }
}

int linear4(const qadc_weights4 *w, const void *x, int64_t ldx, int type, int64_t M, const float *bias, void *y, int64_t ldy,
            hipStream_t st)
{
    if (!w) return fail(QADC_EINVAL, "qadc_linear4: null pointer");
    if (const int rc = check4("qadc_linear4", w->N, w->K, w->group, w->stype)) return rc;
    if (!type_ok(type)) return fail(QADC_EINVAL, "qadc_linear4: unknown type %d", type);
    if (M < 0 || ldx < w->K || ldy < w->N)
        return fail(QADC_EINVAL, "qadc_linear4: M=%lld, rows %lld and %lld apart", (long long)M, (long long)ldx, (long long)ldy);
    if (M == 0) return QADC_OK;
    if (!w->packed || !x || !y) return fail(QADC_EINVAL, "qadc_linear4: null pointer");
    if ((uintptr_t)w->packed % 16) return fail(QADC_EINVAL, "qadc_linear4: packed is not 16-byte aligned");
    const Args4 a = {(const char *)w->packed, shape4(w->N, w->K, w->group, w->has_zeros != 0), w->N, M, ldx, ldy, w->K, w->stype,
                     w->has_zeros != 0, bias};
    QADC_BY_TYPE(type, {
        if (w->group == 32) linear4_rows<T, 1>(a, (const T *)x, (T *)y, st);
        else if (w->group == 64) linear4_rows<T, 2>(a, (const T *)x, (T *)y, st);
        else linear4_rows<T, 4>(a, (const T *)x, (T *)y, st);
    });
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
