// Products with 4-bit weights and group scales on gfx950.
//
// Packed weights.  A tile is 16 outputs x 128 inputs: 64 lanes x 16 bytes, lane l = 16 j + n holding of output n the inputs
// 32 s + 8 j + 0 .. 7 in its dword s = 0 .. 3, which is the order in which a matrix instruction over 16 outputs and 32 inputs
// takes them, four instructions a tile.  Of a dword's eight weights, weight 2 i is nibble i and weight 2 i + 1 nibble i + 4, so
// that one shift and one mask leave a pair in the two halves of a register.  Tiles of one block of 16 outputs follow each
// other along the inputs; behind all tiles lie the scales, [block][group][16] of 16 bits, and the zero points,
// [block][group][16] bytes.  Outputs and inputs beyond N and K are zero nibbles with scale 0.

#include <algorithm>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int W4_N = 16, W4_K = 128, W4_BYTES = W4_N * W4_K / 2;  // a tile

struct Shape4 {
    int64_t blocks;  // of 16 outputs
    int tiles;       // of 128 inputs
    int groups;      // per output
    size_t scales, zeros, bytes;  // where the scales and zero points begin, and the end
};

__host__ __device__ inline Shape4 shape4(int64_t N, int K, int group, bool has_zeros)
{
    Shape4 s;
    s.blocks = (N + W4_N - 1) / W4_N;
    s.tiles = (K + W4_K - 1) / W4_K;
    s.groups = (int)(((int64_t)K + group - 1) / group);
    s.scales = (size_t)s.blocks * s.tiles * W4_BYTES;
    s.zeros = s.scales + (size_t)s.blocks * s.groups * W4_N * 2;
    s.bytes = s.zeros + (has_zeros ? (size_t)s.blocks * s.groups * W4_N : 0);
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
                                                           const uint8_t *__restrict__ zeros, int64_t N, int groups,
                                                           int64_t count, uint16_t *__restrict__ packed_scales,
                                                           uint8_t *__restrict__ packed_zeros)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t block = i / W4_N / groups, g = i / W4_N % groups, n = block * W4_N + i % W4_N;
        packed_scales[i] = n < N ? scales[n * groups + g] : (uint16_t)0;
        if (zeros) packed_zeros[i] = n < N ? zeros[n * groups + g] : (uint8_t)0;
    }
}

__device__ __forceinline__ float scale4(uint16_t bits, int stype)
{
    union { uint16_t u; _Float16 h; } v;
    v.u = bits;
    return stype == QADC_TYPE_F16 ? (float)v.h : __uint_as_float((unsigned)bits << 16);
}

// A workgroup per block of 16 outputs and row of x: 16 threads an output, each every sixteenth eight of the inputs.
template <typename T>
__global__ __launch_bounds__(256) void linear4_kernel(const uint32_t *__restrict__ packed, Shape4 s, int64_t N, int K, int group,
                                                      int stype, int has_zeros, const T *__restrict__ x, int64_t ldx,
                                                      const float *__restrict__ bias, T *__restrict__ y, int64_t ldy, int64_t M)
{
    __shared__ float lds[256];
    const int n = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int64_t block = blockIdx.x;
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(reinterpret_cast<const char *>(packed) + s.scales) +
                             block * s.groups * W4_N + n;
    const uint8_t *zeros = reinterpret_cast<const uint8_t *>(packed) + s.zeros + block * s.groups * W4_N + n;
    for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
        float sum = 0.0f;
        for (int64_t k = 8 * part; k < K; k += 128) {
            const int tile = (int)(k >> 7), step = (int)(k >> 5 & 3), j = (int)(k >> 3 & 3);
            const uint32_t v = packed[((block * s.tiles + tile) * 64 + 16 * j + n) * 4 + step];
            const int64_t g = k / group;
            const float sc = scale4(scales[g * W4_N], stype), z = has_zeros ? (float)zeros[g * W4_N] : 8.0f;
            float part_sum = 0.0f;
            for (int e = 0; e < 8 && k + e < K; ++e) {
                const float q = (float)(v >> (4 * ((e >> 1) + 4 * (e & 1))) & 15u);
                part_sum = fmaf(q - z, (float)x[m * ldx + k + e], part_sum);
            }
            sum = fmaf(sc, part_sum, sum);
        }
        __syncthreads();
        lds[threadIdx.x] = sum;
        __syncthreads();
        if (part == 0 && block * W4_N + n < N) {
            float t = 0.0f;
            for (int p = 0; p < 16; ++p) t += lds[16 * p + n];
            y[m * ldy + block * W4_N + n] = (T)(t + (bias ? bias[block * W4_N + n] : 0.0f));
        }
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
    const int64_t dwords = (int64_t)(s.scales / 4), count = s.blocks * s.groups * W4_N;
    const auto grid = [](int64_t n) { return dim3((unsigned)std::min<int64_t>(ceil_div(n, 256), 1 << 16)); };
    hipLaunchKernelGGL(pack4_codes_kernel, grid(dwords), dim3(256), 0, st, codes, N, K, s.tiles, dwords, (uint32_t *)packed);
    hipLaunchKernelGGL(pack4_scales_kernel, grid(count), dim3(256), 0, st, (const uint16_t *)scales, zeros, N, s.groups, count,
                       (uint16_t *)((char *)packed + s.scales), (uint8_t *)packed + s.zeros);
    QADC_HIP_TRY(hipGetLastError());
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
    const Shape4 s = shape4(w->N, w->K, w->group, w->has_zeros != 0);
    const dim3 grid((unsigned)s.blocks, (unsigned)std::min<int64_t>(M, 65535));
    QADC_BY_TYPE(type, (launch(QADC_PROF_LINEAR4, linear4_kernel<T>, grid, dim3(256), 0, st, (const uint32_t *)w->packed, s, w->N,
                               w->K, w->group, w->stype, w->has_zeros, (const T *)x, ldx, bias, (T *)y, ldy, M)));
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
