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
// The product.  Of a 16-bit x: a nibble q put into the mantissa of 16 is the 16-bit number 16 + q, exactly: no conversion, one shift
// and one and-or for a pair.  The matrix units multiply these with x and, once for all outputs, a column of ones with x; with p and
// t the two sums over a group, the group adds s (p - (16 + z) t) to the output.  The sums are about ten times the result's size, which
// the rounding of a 16-bit y hides and that of a float32 would not.  So a float32 x, the sum of three bfloat16 numbers, is multiplied
// with q - z itself, a whole number that a bfloat16 holds: 24 vector instructions for 8 weights of each lane instead of 8 (16 rows
// of 4096 x 4096 13.7 us, 12.9 with 16 + q).  Up to four rows have their three parts in three rows of a matrix instruction, of whose
// 16 they need no more (one row of 131072 x 4096 68 us; with an instruction for each part 91, and 75 with 16 + q).
//
// Bound by the weights' bytes for a few rows: one row of 131072 x 4096 bfloat16 49 us (277 MB at 5.6 TB/s), of 4096 x 4096
// binary16 5.2, a launch and a round trip; beyond 16 rows by vector instructions (unpacking, 8 for 8 weights of each lane, and
// what follows a group) and by x, which every workgroup brings into LDS: 24 rows of 10007 x 5000 in groups of 32 22 us.  (These are
// the kernel's times by the profiler; figures elsewhere in this file are calls one after the other: 51, 7 and 21 us.)  64 rows of
// 131072 x 4096 141 us, 2048 of 4096 x 4096 132 (0.52 P operations/s: each 32 rows unpack the weights anew).

#include <algorithm>
#include <mutex>
#include <type_traits>

#include "qadc_half.h"
#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int W4_N = 16, W4_K = 128, W4_BYTES = W4_N * W4_K / 2;  // a tile
constexpr int64_t W4_MOST = 1ll << 30;  // outputs

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
// exponent 4, into bits 3 .. 6 of a bfloat16.  `sixteen` is a pair of 16s that the compiler does not know: a three-operand
// instruction takes one constant from outside the vector registers, not two.
template <bool HALF>
__device__ __forceinline__ bits16x8 weights8(unsigned v, unsigned sixteen)
{
    constexpr unsigned mask = HALF ? 0x03C003C0u : 0x00780078u;
    bits16x8 w;
    w[0] = ((HALF ? v << 6 : v << 3) & mask) | sixteen;
    w[1] = ((HALF ? v << 2 : v >> 1) & mask) | sixteen;
    w[2] = ((HALF ? v >> 2 : v >> 5) & mask) | sixteen;
    w[3] = ((HALF ? v >> 6 : v >> 9) & mask) | sixteen;
    return w;
}

// The eight weights of a dword as q - z, whole numbers of eight bits and a sign at most, which a bfloat16 holds.
__device__ __forceinline__ bits16x8 weights8_less(unsigned v, float zero)
{
    unsigned even = v & 0x0f0f0f0fu, odd = v >> 4 & 0x0f0f0f0fu;
    asm("" : "+v"(even), "+v"(odd));  // (bytes, which have a conversion of their own, not bit fields of v to be taken out first)
    const auto less = [&](unsigned bytes, int at) { return __float_as_uint((float)(bytes >> (8 * at) & 0xffu) - zero); };
    const auto pair = [&](unsigned bytes, int at) {  // the upper halves of the two float32
        return __builtin_amdgcn_perm(less(bytes, at + 2), less(bytes, at), 0x07060302u);
    };
    bits16x8 w;
    w[0] = pair(even, 0);
    w[1] = pair(odd, 0);
    w[2] = pair(even, 1);
    w[3] = pair(odd, 1);
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

struct Args4 {
    const char *packed;
    Shape4 s;
    int64_t N, M, ldx, ldy;
    int K, stype, has_zeros;
    const float *bias;
    int split;  // wavefronts that share a block
    int chunk;  // tiles of x in LDS at a time
    unsigned row_blocks;
};

constexpr int X_PAD = 8;  // 16 bytes between the rows of x in LDS: a fragment's rows lie in different banks

// A block of NT x 16 outputs and up to 4 MR MT rows of x: `split` wavefronts, each every split-th tile of the inputs; a workgroup
// has as many blocks as it has wavefronts for, and brings x into LDS for all of them.  Of a matrix instruction's 16 rows,
// 4 q + i, the first MR of every four are rows of x (MR = 1 for up to four rows: a quarter of the work behind the products); the
// others repeat them, or hold the parts of a float32 (SPREAD).  STEPS: instructions per group.  AGAIN: there are further rows, whose
// workgroups read the same weights.
template <typename T, int STEPS, int MR, int MT, int NT, int THREADS, bool AGAIN>
__global__ __launch_bounds__(THREADS, 4) void linear4_kernel(Args4 a, const T *__restrict__ x, T *__restrict__ y)
{
    constexpr int DEPTH = 4 / NT, PER = 4 / STEPS, ROWS = 4 * MR * MT, PARTS = Inputs<T>::PARTS;
    constexpr bool HALF = Inputs<T>::HALF, LESS = PARTS == 3, SPREAD = LESS && MR == 1;
    constexpr int FLY = sizeof(T) == 4 ? 2 : 4;
    // Four groups one after the other, each done before the next is begun where more rows share the registers (64 rows of
    // 131072 x 4096, groups of 32: 203 -> 184 us); two groups of 64 are a loop there (32 rows of 16384 x 16384 60 us, 63 unrolled).
    constexpr int UNROLL = MT == 1 || PER == 4 ? PER : 1;
    extern __shared__ float lds[];
    uint16_t *xs = reinterpret_cast<uint16_t *>(lds);  // [PARTS][rows][chunk * W4_K + X_PAD]
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, j = lane >> 4;
    const int split = a.split, at_once = THREADS / WAVE / split;
    // Workgroups go round the eight XCDs; those of different rows and the same outputs follow each other on one of them, so that
    // its cache has the weights for all (64 rows of 131072 x 4096 with the rows' workgroups far apart: 150 us).
    const unsigned turn = blockIdx.x >> 3;
    const int64_t wg = AGAIN ? turn / a.row_blocks * 8 + (blockIdx.x & 7) : blockIdx.x;
    const int64_t block = (wg * at_once + wave / split) * NT;
    const int part = wave % split, tiles = a.s.tiles;
    const int64_t m0 = AGAIN ? (int64_t)(turn % a.row_blocks) * ROWS : 0;
    const int rows = (int)min((int64_t)ROWS, a.M - m0), stride = a.chunk * W4_K + X_PAD;

    // where this lane's row of x in each m-tile lies, and its weights and scales
    int at_x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int i = n & 3, m = t * 4 * MR + (n >> 2) * MR + (i < MR ? i : 0);
        at_x[t] = (min(m, rows - 1) + (SPREAD ? min(i, PARTS - 1) * rows : 0)) * stride + 8 * j;
    }
    const char *weights[NT], *scales[NT], *zeros[NT];  // (the same in all lanes)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t b = min(block + t, a.s.blocks - 1);
        weights[t] = a.packed + b * tiles * W4_BYTES;
        scales[t] = a.packed + a.s.scales + b * a.s.sets * (W4_N * PER * 2);
        zeros[t] = a.packed + a.s.zeros + b * a.s.sets * (W4_N * PER);
    }
    // The next tiles on their way.
    typedef std::conditional_t<PER == 4, u32x2, std::conditional_t<PER == 2, uint32_t, uint16_t>> Scales;
    typedef std::conditional_t<PER == 4, uint32_t, std::conditional_t<PER == 2, uint16_t, uint8_t>> Zeros;
    bits16x8 ring[DEPTH][NT];
    Scales ring_s[DEPTH][NT];
    Zeros ring_z[DEPTH][NT];
    const auto fetch = [&](int d, int k) {
        const unsigned set = (unsigned)(k / a.s.span) * W4_N + n;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const bits16x8 *from = reinterpret_cast<const bits16x8 *>(weights[t]) + ((unsigned)k * WAVE + lane);
            if constexpr (AGAIN) ring[d][t] = *from;
            else ring[d][t] = __builtin_nontemporal_load(from);
            ring_s[d][t] = reinterpret_cast<const Scales *>(scales[t])[set];
            if (a.has_zeros) ring_z[d][t] = reinterpret_cast<const Zeros *>(zeros[t])[set];
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (part + d * split < tiles) fetch(d, part + d * split);

    f32x4 sum[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) sum[t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    bits16x8 ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones[i] = HALF ? 0x3C003C00u : 0x3F803F80u;

    // x, a chunk of tiles at a time; every wavefront comes by here once for each chunk
    int first = 0, end = 0;  // the tiles in LDS
    const auto next_chunk = [&]() {
        first = end;
        end = min(first + a.chunk, tiles);
        const unsigned packs = (unsigned)(end - first) * (W4_K / 8), all = packs * (unsigned)rows;
        const unsigned inverse = 0xffffffffu / packs + 1u;  // i / packs = i * inverse / 2^32: i * packs is far below 2^32
        const bool whole = (int64_t)end * W4_K <= a.K;
        if (first) __syncthreads();  // (the chunk before has been read)
        // FLY packs a thread in flight; past the last one it is brought again
        for (unsigned i = threadIdx.x; i < all; i += FLY * THREADS) {
            typename Inputs<T>::V v[FLY];
            unsigned to[FLY];
#pragma unroll
            for (int e = 0; e < FLY; ++e) {
                const unsigned at = min(i + e * THREADS, all - 1), r = __umulhi(at, inverse), c = (at - r * packs) * 8;
                const int64_t k = (int64_t)first * W4_K + c;
                const T *row = x + (m0 + r) * a.ldx;
                to[e] = r * stride + c;
                if (whole || k + 8 <= a.K) v[e] = *reinterpret_cast<const typename Inputs<T>::V *>(row + k);
                else v[e] = Inputs<T>::load_last(row, k, a.K);
            }
#pragma unroll
            for (int e = 0; e < FLY; ++e) {
                const Inputs<T> in(v[e]);
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    *reinterpret_cast<bits16x8 *>(xs + (unsigned)(p * rows) * stride + to[e]) = in.part[p];
            }
        }
        __syncthreads();
    };
    next_chunk();

    unsigned sixteen = HALF ? 0x4C004C00u : 0x41804180u;
    asm volatile("" : "+v"(sixteen));

    // one tile: its groups in turn, the weights, scales and zero points of the next one moved to the front each time
    const auto tile = [&](auto which, int k) {
        constexpr int d = decltype(which)::value;
        while (k >= end) next_chunk();
        bits16x8 q[NT];
        Scales sb[NT];
        Zeros zb[NT];
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            q[u] = ring[d][u];
            sb[u] = ring_s[d][u];
            zb[u] = ring_z[d][u];
        }
        if (k + DEPTH * split < tiles) fetch(d, k + DEPTH * split);
        const uint16_t *from = xs + (k - first) * W4_K;
#pragma unroll UNROLL
        for (int g = 0; g < PER; ++g, from += 32 * STEPS) {
            f32x4 p[MT][NT], one[MT];
            const auto zero = [&](int u, float more) {  // (what the nibbles are more than they stand for)
                uint8_t z;
                __builtin_memcpy(&z, &zb[u], 1);
                return a.has_zeros ? more + (float)z : more + 8.0f;
            };
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                bits16x8 w[NT];
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    if constexpr (LESS) w[u] = weights8_less(q[u][s], zero(u, 0.0f));
                    else w[u] = weights8<HALF>(q[u][s], sixteen);
                }
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int part_of = 0; part_of < (SPREAD ? 1 : PARTS); ++part_of) {
                        const bits16x8 in =
                            *reinterpret_cast<const bits16x8 *>(from + part_of * rows * stride + at_x[t] + 32 * s);
                        const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
                        const bool more = s + part_of > 0;
                        if constexpr (!LESS) one[t] = mfma16<HALF>(in, ones, more ? one[t] : none);
#pragma unroll
                        for (int u = 0; u < NT; ++u) p[t][u] = mfma16<HALF>(in, w[u], more ? p[t][u] : none);
                    }
            }
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                uint16_t bits;
                __builtin_memcpy(&bits, &sb[u], 2);
                const float sc = scale4(bits, a.stype), zp = zero(u, 16.0f);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < MR; ++i) {
                        const float of = SPREAD ? p[t][u][2] + p[t][u][1] + p[t][u][0]
                                         : LESS ? p[t][u][i]
                                                : fmaf(-zp, one[t][i], p[t][u][i]);
                        sum[t][u][i] = fmaf(sc, of, sum[t][u][i]);
                    }
                if constexpr (PER == 4) {
                    q[u] = __builtin_shufflevector(q[u], q[u], 1, 2, 3, 0);
                    sb[u] = u32x2{sb[u][0] >> 16 | sb[u][1] << 16, sb[u][1] >> 16};
                    zb[u] >>= 8;
                } else if constexpr (PER == 2) {
                    q[u] = __builtin_shufflevector(q[u], q[u], 2, 3, 0, 1);
                    sb[u] >>= 16;
                    zb[u] >>= 8;
                }
            }
            if constexpr (MT > 1 && PER == 4) __builtin_amdgcn_sched_barrier(0);
        }
    };
    int k = part;
    while (k < tiles) {
        tile(std::integral_constant<int, 0>(), k);
        if ((k += split) >= tiles) break;
        tile(std::integral_constant<int, 1>(), k);
        k += split;
        if constexpr (DEPTH == 4) {
            if (k >= tiles) break;
            tile(std::integral_constant<int, 2>(), k);
            if ((k += split) >= tiles) break;
            tile(std::integral_constant<int, 3>(), k);
            k += split;
        }
    }
    while (end < tiles) next_chunk();

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
    __syncthreads();  // (x has been read)
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
    if (N < 1 || N > W4_MOST || K < 1 || K > (1 << 24))
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

// How a product is cut: wavefronts that share a block of outputs, and the cost of that in KB of weights that a compute unit could
// have read meanwhile: those of the fullest one of the 256, and 128 KB for every round of workgroups (6 us from a workgroup's
// first load to its last store at 21.5 GB/s a compute unit).
struct Cut4 {
    int split;
    int64_t cost;
};
Cut4 cut4(int64_t blocks, int64_t row_blocks, int tiles, int nt, int waves)
{
    Cut4 best = {1, INT64_MAX};
    for (int split = 1; split <= waves && (split == 1 || split <= tiles); split *= 2) {
        const int64_t at_once = waves / split, wgs = ceil_div(blocks, at_once) * row_blocks;
        const int64_t cost = ceil_div(wgs, 256) * at_once * nt * tiles + 128 * ceil_div(wgs, 256 * (16 / waves));
        if (cost <= best.cost) best = {split, cost};
    }
    return best;
}

// A workgroup of 16 wavefronts has a compute unit and its LDS to itself, of 8 it shares them with another one.
template <typename T, int STEPS, int MR, int MT, int NT, int THREADS, bool AGAIN = false>
static int linear4_launch(Args4 a, const void *x, void *y, hipStream_t st)
{
    constexpr int WAVES = THREADS / WAVE, PARTS = Inputs<T>::PARTS;
    constexpr size_t room = THREADS == 1024 ? 156 << 10 : 78 << 10, sums = (size_t)WAVES * MT * NT * MR * WAVE * sizeof(float);
    static_assert(sums <= room, "the wavefronts' sums fit where x was");
    static std::once_flag once;
    static hipError_t attr = hipSuccess;
    const auto kernel = &linear4_kernel<T, STEPS, MR, MT, NT, THREADS, AGAIN>;
    std::call_once(once, [&] {  // more than the default limit of dynamic LDS
        attr = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)room);
    });
    QADC_HIP_TRY(attr);
    const int64_t blocks = ceil_div(a.s.blocks, NT), row_blocks = ceil_div(a.M, 4 * MR * MT);
    a.split = cut4(blocks, row_blocks, a.s.tiles, NT, WAVES).split;
    const size_t row_bytes = (size_t)std::min<int64_t>(4 * MR * MT, a.M) * PARTS * 2;
    a.chunk = (int)std::min<size_t>(a.s.tiles, (room / row_bytes - X_PAD) / W4_K);
    const size_t shared = std::max(row_bytes * (a.chunk * W4_K + X_PAD), a.split > 1 ? sums : 0);
    a.row_blocks = (unsigned)row_blocks;
    const int64_t wgs = ceil_div(blocks, WAVES / a.split);
    launch(QADC_PROF_LINEAR4, *kernel, dim3((unsigned)(AGAIN ? ceil_div(wgs, 8) * 8 * row_blocks : wgs)), dim3(THREADS),
           shared, st, a, (const T *)x, (T *)y);
    return QADC_OK;
}

// Sixteen wavefronts a workgroup (131072 x 4096, bfloat16: one row 59 us with eight, 55 with sixteen, 16 rows 63 and 59; the large x
// of 32 rows of 16384 inputs is brought in half as often: 77 and 56; 24 rows of 10007 x 5000 25 and 22), unless the last round of
// workgroups would leave much of the chip idle: there eight (one row of 40000 x 8000 35 us against 44, of float32 48 against 63).
template <typename T, int STEPS, int MR, int MT, bool AGAIN = false>
static int linear4_sized(const Args4 &a, const void *x, void *y, hipStream_t st)
{
    const int64_t blocks = ceil_div(a.s.blocks, 2), row_blocks = ceil_div(a.M, 4 * MR * MT);
    if (cut4(blocks, row_blocks, a.s.tiles, 2, 8).cost < cut4(blocks, row_blocks, a.s.tiles, 2, 16).cost)
        return linear4_launch<T, STEPS, MR, MT, 2, 512, AGAIN>(a, x, y, st);
    return linear4_launch<T, STEPS, MR, MT, 2, 1024, AGAIN>(a, x, y, st);
}

template <typename T, int STEPS>
static int linear4_rows(Args4 a, const T *x, T *y, hipStream_t st)
{
    // As many rows at a time as keep the threads of a grid within 32 bits: two an output and 32 rows (a wavefront for 32 outputs),
    // up to eight workgroups more.
    const int64_t slab = 32 * std::min<int64_t>(128, ((1ll << 32) - 1) / (2 * a.N + 8 * 1024)), M = a.M;
    for (int64_t m = 0; m < M; m += slab) {
        a.M = std::min(slab, M - m);
        const T *xs = x + m * a.ldx;
        T *ys = y + m * a.ldy;
        int rc;
        if (a.M > 32) rc = linear4_sized<T, STEPS, 4, 2, true>(a, xs, ys, st);
        else if (a.M > 16) rc = linear4_sized<T, STEPS, 4, 2>(a, xs, ys, st);
        else if (a.M > 4) rc = linear4_sized<T, STEPS, 4, 1>(a, xs, ys, st);
        // Up to four rows: two blocks a wavefront, or one where there are few outputs, for all the wavefronts that they are worth (one
        // row of 131072 x 4096 bfloat16 55.5 us with one, 51.8 with two, of 24576 x 16384 45.7 and 39.6; of 16384 x 16384 27.8 and
        // 29.0, of 4096 x 16384 10.4 and 14.7, four of 4096 x 4096 binary16 in groups of 32 6.6 and 7.8).
        else if (a.s.blocks >= 1024) rc = linear4_sized<T, STEPS, 1, 1>(a, xs, ys, st);
        else rc = linear4_launch<T, STEPS, 1, 1, 1, 1024>(a, xs, ys, st);
        if (rc != QADC_OK) return rc;
    }
    return QADC_OK;
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
                     w->has_zeros != 0, bias, 1, 1, 1};
    int rc = QADC_OK;
    QADC_BY_TYPE(type, {
        if (w->group == 32) rc = linear4_rows<T, 1>(a, (const T *)x, (T *)y, st);
        else if (w->group == 64) rc = linear4_rows<T, 2>(a, (const T *)x, (T *)y, st);
        else rc = linear4_rows<T, 4>(a, (const T *)x, (T *)y, st);
    });
    if (rc != QADC_OK) return rc;
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
