// Root-mean-square norm of the sum of two rows, its 8-bit output, and its backward pass on gfx950.
//
// Forward: h = x + residual, rounded to the rows' type, which is what goes on to the next layer and what is normalised;
// rstd = 1 / sqrt(sum h^2 / d + eps), y = h rstd w.  In 8 bits y is scaled by 448 / max |y|: the largest of |h w| times rstd is that
// of |y|, so that it is found in the same reduction as the sum of squares.  Backward: with n = h rstd and g = dy w,
// dx = rstd (g - n sum(g n) / d) + dsum, one reduction; the weight's gradient is the sum of dy n over the rows, each workgroup its
// rows in its registers, then the workgroups in a fixed order.
//
// A row of up to 16384 elements stays in the registers of its group of threads, so that everything is read once; the next row
// comes in while this one is reduced.  Longer rows are read again for the output.
//
// Bound by memory: forward with a residual 16384 x 4096 bfloat16 82 us, 6.5 TB/s read and written (float32 190); backward with the residual's
// gradient 91 us for the rows, 5.9 TB/s, and 5 for joining the workgroups' sums.  In 8 bits a call takes 84 us where y takes 87 (float32 159 and
// 187).  Without an eps ordinary rows take as long, rows with squares below float32 130 (float32 195).  Small calls are bound by the host: 5 x 4096 with a
// residual to 8 bits 14 us a call, kernel 3.4.  3001 x 1537 float32 backward: rows 14 us in three turns a workgroup, each of which exposes a
// load and a barrier, join 6.
#include <type_traits>

#include "qadc_norm_rows.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int RMS_WG = 1024;             // threads of a row beyond 16384 elements
constexpr float E4M3_MOST = 448.0f;

// The largest value over the lanes of a group of 16, 32 or 64, in every lane.
template <int G>
__device__ __forceinline__ float lanes_max(float v)
{
    if constexpr (G == WAVE) return wave_max(v);
    v = fmaxf(v, dpp_or<0x128, 0xf>(v, v));
    v = fmaxf(v, dpp_or<0x124, 0xf>(v, v));
    v = fmaxf(v, dpp_or<0x122, 0xf>(v, v));
    v = fmaxf(v, dpp_or<0x121, 0xf>(v, v));
    if constexpr (G == 32) v = fmaxf(v, __shfl_xor(v, 16));
    return v;
}

// The sum of s and the largest m of a group of G threads, in every one of them; `turn` alternates between calls.
template <int G>
__device__ __forceinline__ void group_sum_max(float &s, float &m, float *lds, int &turn)
{
    s = lanes_sum<G < WAVE ? G : WAVE>(s);
    m = lanes_max<G < WAVE ? G : WAVE>(m);
    if constexpr (G > WAVE) {
        constexpr int W = G / WAVE;
        float *buf = lds + (turn & 1) * (1024 / WAVE) * 2;
        ++turn;
        const int wave = threadIdx.x >> 6, first = wave / W * W;
        if (lane_id() == 0) {
            buf[wave * 2] = s;
            buf[wave * 2 + 1] = m;
        }
        __syncthreads();
        s = m = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            s += buf[(first + w) * 2];
            m = fmaxf(m, buf[(first + w) * 2 + 1]);
        }
    }
}

// Where eps leaves rows to themselves (TINY): float32 squares of elements below 2^-63 lose bits, and below 2^-75 are zeros.  A row whose sum is
// this small is summed again in 64 bits, and normalised as 2^64 times itself.  Kernels of their own: the ordinary ones would have 10 to 20 more
// registers.
constexpr float RMS_TINY = 0x1p-90f, RMS_UP = 0x1p64f;
constexpr float RMS_EPS_TINY = 0x1p-100f;  // from here on eps outweighs what such squares lose

// The sum of s over a group of G threads, in every one of them.  Barriers before and behind.
template <int G>
__device__ __forceinline__ double group_sum64(double s, double *lds)
{
#pragma unroll
    for (int o = (G < WAVE ? G : WAVE) / 2; o; o >>= 1) s += __shfl_xor(s, o);
    if constexpr (G > WAVE) {
        constexpr int W = G / WAVE;
        const int wave = threadIdx.x >> 6, first = wave / W * W;
        __syncthreads();
        if (lane_id() == 0) lds[wave] = s;
        __syncthreads();
        s = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) s += lds[first + w];
    }
    return s;
}

// The factor that brings a row's values into 8 bits, and the scale that takes them back.  most: the largest |y|.  A row of zeros
// has scale 0; below 448 / 2^126 the values use less of the range; a NaN stays one.
__device__ __forceinline__ float to_8bit(float most, float &scale)
{
    constexpr float LARGE = 8.507059173023462e37f;  // 2^126
    const float f = most > 0.0f ? E4M3_MOST / most : most;
    scale = f > LARGE ? 1.0f / LARGE : most / E4M3_MOST;
    return f > LARGE ? LARGE : f;
}
// Within +-448, beyond which the conversion gives NaN; a NaN stays one.
__device__ __forceinline__ float within_8bit(float v) { return v > E4M3_MOST ? E4M3_MOST : v < -E4M3_MOST ? -E4M3_MOST : v; }
// Four values as E4M3, to the nearest, ties to even.
__device__ __forceinline__ uint32_t four_8bit(float a, float b, float c, float d)
{
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(within_8bit(a), within_8bit(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(within_8bit(c), within_8bit(d), v, true);
}

// N values y into columns c .. c + N - 1 of a row of d bytes that begins anywhere.
template <int N>
__device__ __forceinline__ void store_8bit(const float (&y)[N], uint8_t *row, int c, int d)
{
    typedef uint32_t Four __attribute__((ext_vector_type(N / 4), aligned(1)));
    uint32_t q[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) q[i] = four_8bit(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    if (c + N <= d) {
        Four v;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) v[i] = q[i];
        *reinterpret_cast<Four *>(row + c) = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < d) row[c + e] = (uint8_t)(q[e / 4] >> (8 * (e % 4)));
    }
}

// The weights of a thread's columns, of the rows' type or float32.
template <typename T, int G, int E>
__device__ __forceinline__ void load_weights_of(const void *w, bool wide, int t, int d, float (&v)[E])
{
    if (wide) load_weights<T, G, E>((const float *)w, 1.0f, t, d, v);
    else load_weights<T, G, E>((const T *)w, 1.0f, t, d, v);
}

struct RmsOut {
    void *sum;        // [rows][ld_sum] of the rows' type, where there is a residual
    int64_t ld_sum;
    void *y;          // [rows][d] of the rows' type, or bytes
    float *scale;     // [rows], with bytes
    float *rstd;      // [rows] or null
    bool bytes;
};

// A group of G threads per row, THREADS / G rows of a workgroup at a time.  RES: there is a residual.
template <typename T, int G, int E, int THREADS, bool RES, bool TINY>
__global__ __launch_bounds__(THREADS) void rms_rows_kernel(const T *x, int64_t ldx, const T *res, int64_t ldr,
                                                           const void *__restrict__ weight, bool wide, int64_t rows, int d,
                                                           float eps, RmsOut o)
{
    typedef Part<T, G, E> P;
    constexpr int N = P::N;
    __shared__ float lds[4 * (1024 / WAVE)];
    __shared__ double lds64[1024 / WAVE];
    constexpr int R = THREADS / G;
    const int t = threadIdx.x % G;
    int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / G;
    const int64_t ahead = (int64_t)gridDim.x * R;
    struct Row {
        P x, res;
    } one, two;
    const auto load = [&](Row &row, int64_t at) {
        at = min(at, rows - 1);
        row.x.load(x + at * ldx, t, d);
        if constexpr (RES) row.res.load(res + at * ldr, t, d);
    };
    load(one, r);
    float w[E];
    load_weights_of<T, G, E>(weight, wide, t, d, w);
    int turns = 0;
    // a row, while the next one comes in; false behind the last (all groups of a workgroup go round together)
    const auto turn = [&](Row &now, Row &next) {
        const bool more = r - threadIdx.x / G + ahead < rows;
        if (more) load(next, r + ahead);
        now.x.settle(t, d);
        if constexpr (RES) {
            now.res.settle(t, d);
#pragma unroll
            for (int i = 0; i < E; ++i) now.x.set(i, now.x[i] + now.res[i]);
            if (r < rows) now.x.store((T *)o.sum + r * o.ld_sum, t, d);
        }
        float s = 0.0f, most = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            s = fmaf(now.x[i], now.x[i], s);
            most = fmaxf(most, fabsf(now.x[i] * w[i]));
        }
        group_sum_max<G>(s, most, lds, turns);
        float rstd = 1.0f / sqrtf(s / (float)d + eps), of_row = rstd;
        if (TINY && __syncthreads_or(s < RMS_TINY)) {  // (all groups of the workgroup)
            double s64 = 0.0;
            float up = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                s64 += (double)now.x[i] * (double)now.x[i];
                up = fmaxf(up, fabsf(now.x[i] * RMS_UP * w[i]));
            }
            s64 = group_sum64<G>(s64, lds64);
            float none = 0.0f;
            group_sum_max<G>(none, up, lds, turns);
            if (s < RMS_TINY) {
                const double one = 1.0 / sqrt(s64 / (double)d + (double)eps);
                of_row = (float)one;
                rstd = (float)(one / RMS_UP);
                most = up;
#pragma unroll
                for (int i = 0; i < E; ++i) now.x.set(i, now.x[i] * RMS_UP);
            }
        }
        if (r < rows) {
            if (o.bytes) {
                float scale;
                const float f = to_8bit(most * rstd, scale);
#pragma unroll
                for (int u = 0; u < P::P; ++u) {
                    float y[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) y[e] = now.x[u * N + e] * rstd * w[u * N + e] * f;
                    store_8bit<N>(y, (uint8_t *)o.y + r * d, (u * G + t) * N, d);
                }
                if (t == 0) o.scale[r] = scale;
            } else {
                P out;
#pragma unroll
                for (int i = 0; i < E; ++i) out.set(i, now.x[i] * rstd * w[i]);
                out.store((T *)o.y + r * d, t, d);
            }
            if (t == 0 && o.rstd) o.rstd[r] = of_row;
        }
        r += ahead;
        return more;
    };
    while (turn(one, two) && turn(two, one)) {
    }
}

struct RmsBack {
    const void *dy, *h, *dsum;  // dsum: null without
    int64_t ld_dy, ld_h, ld_dsum;
    const float *rstd;
    void *dx;      // [rows][d], or null
    float *parts;  // [workgroup][d], or null
};

// dx of the workgroup's rows and, where `parts` is set, their share of the weight's gradient.
template <typename T, int G, int E, int THREADS, bool AHEAD, bool SUM>
__global__ __launch_bounds__(THREADS) void rms_back_kernel(RmsBack b, const void *__restrict__ weight, bool wide, int64_t rows, int d)
{
    typedef Part<T, G, E> P;
    __shared__ float lds[2 * (1024 / WAVE)];
    constexpr int R = THREADS / G;
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    int64_t r = (int64_t)blockIdx.x * R + group;
    const int64_t ahead = (int64_t)gridDim.x * R;
    struct Row {
        P h, dy, sum;
        float rstd;
    } one, two;
    const auto load = [&](Row &row, int64_t at) {
        at = min(at, rows - 1);
        row.h.load((const T *)b.h + at * b.ld_h, t, d);
        row.dy.load((const T *)b.dy + at * b.ld_dy, t, d);
        if constexpr (SUM) row.sum.load((const T *)b.dsum + at * b.ld_dsum, t, d);
        row.rstd = b.rstd[at];
    };
    if (AHEAD) load(one, r);
    float w[E], dw[E];
    load_weights_of<T, G, E>(weight, wide, t, d, w);
#pragma unroll
    for (int i = 0; i < E; ++i) dw[i] = 0.0f;
    int turns = 0;
    // a row, while the next one comes in; false behind the last (all groups of a workgroup go round together)
    const auto turn = [&](Row &now, Row &next) {
        const bool more = r - group + ahead < rows;
        if (!AHEAD) load(now, r);
        else if (more) load(next, r + ahead);
        now.h.settle(t, d);
        now.dy.settle(t, d);
        if constexpr (SUM) now.sum.settle(t, d);
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < E; ++i) s[0] = fmaf(now.dy[i] * w[i], now.h[i] * now.rstd, s[0]);
        group_sums<G, 1>(s, lds, turns);
        if (r < rows) {
            const float a = s[0] / (float)d, rs = now.rstd;
            P out;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float dyi = now.dy[i], n = now.h[i] * rs;
                dw[i] = fmaf(dyi, n, dw[i]);
                const float g = fmaf(dyi, w[i], -n * a);
                if constexpr (SUM) out.set(i, fmaf(rs, g, now.sum[i]));
                else out.set(i, rs * g);
            }
            if (b.dx) out.store((T *)b.dx + r * d, t, d);
        }
        r += ahead;
        return more;
    };
    if constexpr (AHEAD) {
        while (turn(one, two) && turn(two, one)) {
        }
    } else {
        while (turn(one, one)) {
        }
    }
    if (!b.parts) return;
    if constexpr (R > 1) {  // the groups' sums, in their order
        __shared__ float both[G * E];
        for (int g = 0; g < R; ++g) {
            __syncthreads();
            if (group == g)
#pragma unroll
                for (int i = 0; i < E; ++i) both[i * G + t] = g ? both[i * G + t] + dw[i] : dw[i];
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int i = 0; i < E; ++i) dw[i] = both[i * G + t];
    }
    float *mine = b.parts + (size_t)blockIdx.x * d;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int c = P::column(i, t);
        if (c < d) mine[c] = dw[i];
    }
}

// The sum of `count` parts [count][d], 64 columns a workgroup, a sixteenth of the parts each wavefront.
__global__ __launch_bounds__(1024) void rms_join_kernel(const float *__restrict__ parts, int count, int d, float *__restrict__ dweight)
{
    __shared__ float lds[16][WAVE];
    const int wave = threadIdx.x >> 6, lane = lane_id();
    const int64_t c = workgroup() * WAVE + lane;
    float s = 0.0f;
    if (c < d) {
#pragma unroll 16
        for (int p = wave; p < count; p += 16) s += parts[(size_t)p * d + c];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave || c >= d) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += lds[w][lane];
    dweight[c] = s;
}

// Rows beyond 16384 elements, a workgroup each, a pack of each thread at a time.

// N elements of a row from column c on, zeros behind its end.
template <typename T>
__device__ __forceinline__ typename Pack<T>::V load_pack(const T *row, int64_t c, int d)
{
    constexpr int N = Pack<T>::N;
    if (c + N <= d) return *reinterpret_cast<const typename Pack<T>::V *>(row + c);
    typename Pack<T>::V v = (T)0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (c + e < d) v[e] = row[c + e];
    return v;
}
template <typename T>
__device__ __forceinline__ void store_pack(typename Pack<T>::V v, T *row, int64_t c, int d)
{
    constexpr int N = Pack<T>::N;
    if (c + N <= d) {
        *reinterpret_cast<typename Pack<T>::V *>(row + c) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (c + e < d) row[c + e] = v[e];
}
template <int N, typename T>
__device__ __forceinline__ void weight_pack(const void *w, bool wide, int64_t c, int d, float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e)
        v[e] = !w || c + e >= d ? 1.0f : wide ? ((const float *)w)[c + e] : (float)((const T *)w)[c + e];
}

template <typename T, bool TINY>
__global__ __launch_bounds__(RMS_WG) void rms_long_kernel(const T *x, int64_t ldx, const T *res, int64_t ldr, const void *weight,
                                                          bool wide, int64_t rows, int d, float eps, RmsOut o)
{
    constexpr int N = Pack<T>::N;
    __shared__ float lds[4 * (1024 / WAVE)];
    __shared__ double lds64[1024 / WAVE];
    int turns = 0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + r * ldx;
        T *sum = res ? (T *)o.sum + r * o.ld_sum : nullptr;
        float s = 0.0f, most = 0.0f;
        for (int64_t c = (int64_t)threadIdx.x * N; c < d; c += RMS_WG * N) {
            typename Pack<T>::V v = load_pack(xr, c, d);
            float w[N];
            weight_pack<N, T>(weight, wide, c, d, w);
            if (res) {
                const typename Pack<T>::V a = load_pack(res + r * ldr, c, d);
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = (T)((float)v[e] + (float)a[e]);
                store_pack(v, sum, c, d);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                s = fmaf((float)v[e], (float)v[e], s);
                most = fmaxf(most, fabsf((float)v[e] * w[e]));
            }
        }
        group_sum_max<RMS_WG>(s, most, lds, turns);
        float rstd = 1.0f / sqrtf(s / (float)d + eps), of_row = rstd, up = 1.0f;
        const T *from = res ? sum : xr;  // (each thread reads what it wrote itself)
        if (TINY && s < RMS_TINY) {  // (the same in all threads)
            double s64 = 0.0;
            most = 0.0f;
            for (int64_t c = (int64_t)threadIdx.x * N; c < d; c += RMS_WG * N) {
                const typename Pack<T>::V v = load_pack(from, c, d);
                float w[N];
                weight_pack<N, T>(weight, wide, c, d, w);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    s64 += (double)v[e] * (double)v[e];
                    most = fmaxf(most, fabsf((float)v[e] * RMS_UP * w[e]));
                }
            }
            s64 = group_sum64<RMS_WG>(s64, lds64);
            float none = 0.0f;
            group_sum_max<RMS_WG>(none, most, lds, turns);
            const double one = 1.0 / sqrt(s64 / (double)d + (double)eps);
            of_row = (float)one;
            rstd = (float)(one / RMS_UP);
            up = RMS_UP;
        }
        float scale = 0.0f;
        const float f = o.bytes ? to_8bit(most * rstd, scale) : 1.0f;
        for (int64_t c = (int64_t)threadIdx.x * N; c < d; c += RMS_WG * N) {
            typename Pack<T>::V v = load_pack(from, c, d);
            float w[N], y[N];
            weight_pack<N, T>(weight, wide, c, d, w);
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = (TINY ? (float)v[e] * up : (float)v[e]) * rstd * w[e];
            if (o.bytes) {
#pragma unroll
                for (int e = 0; e < N; ++e) y[e] *= f;
                store_8bit<N>(y, (uint8_t *)o.y + r * d, (int)c, d);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = (T)y[e];
                store_pack(v, (T *)o.y + r * d, c, d);
            }
        }
        if (threadIdx.x == 0) {
            if (o.bytes) o.scale[r] = scale;
            if (o.rstd) o.rstd[r] = of_row;
        }
    }
}

// The weight's gradient of a stretch of rows: a thread per column.  Before dx, which may take the place of what is read here.
template <typename T>
__global__ __launch_bounds__(NORM_WG) void rms_weights_kernel(RmsBack b, int64_t rows, int d, int64_t stretch)
{
    const int c = blockIdx.x * NORM_WG + threadIdx.x;
    if (c >= d) return;
    const int64_t r0 = (int64_t)blockIdx.y * stretch, r1 = min(r0 + stretch, rows);
    float s = 0.0f;
    for (int64_t r = r0; r < r1; ++r)
        s = fmaf((float)((const T *)b.dy)[r * b.ld_dy + c], (float)((const T *)b.h)[r * b.ld_h + c] * b.rstd[r], s);
    b.parts[(size_t)blockIdx.y * d + c] = s;
}

template <typename T>
__global__ __launch_bounds__(RMS_WG) void rms_dx_kernel(RmsBack b, const void *weight, bool wide, int64_t rows, int d)
{
    constexpr int N = Pack<T>::N;
    __shared__ float lds[2 * (1024 / WAVE)];
    int turns = 0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *dy = (const T *)b.dy + r * b.ld_dy, *h = (const T *)b.h + r * b.ld_h;
        const float rs = b.rstd[r];
        float s[1] = {0.0f};
        for (int64_t c = (int64_t)threadIdx.x * N; c < d; c += RMS_WG * N) {
            const typename Pack<T>::V g = load_pack(dy, c, d), v = load_pack(h, c, d);
            float w[N];
            weight_pack<N, T>(weight, wide, c, d, w);
#pragma unroll
            for (int e = 0; e < N; ++e) s[0] = fmaf((float)g[e] * w[e], (float)v[e] * rs, s[0]);
        }
        group_sums<RMS_WG, 1>(s, lds, turns);
        const float a = s[0] / (float)d;
        for (int64_t c = (int64_t)threadIdx.x * N; c < d; c += RMS_WG * N) {
            const typename Pack<T>::V g = load_pack(dy, c, d), v = load_pack(h, c, d);
            typename Pack<T>::V more = (T)0.0f, out;
            if (b.dsum) more = load_pack((const T *)b.dsum + r * b.ld_dsum, c, d);
            float w[N];
            weight_pack<N, T>(weight, wide, c, d, w);
#pragma unroll
            for (int e = 0; e < N; ++e)
                out[e] = (T)fmaf(rs, fmaf((float)g[e], w[e], -((float)v[e] * rs) * a), (float)more[e]);
            store_pack(out, (T *)b.dx + r * d, c, d);
        }
    }
}

int rms_back_rows(int d) { return d > NORM_LONG ? 16 : std::max(1, 512 / norm_group(d)); }  // rows of a workgroup at a time
// The most workgroups, each of which leaves a row of sums: two a compute unit, or one of 1024 threads.  bfloat16 16384 x 4096 91 us, 97 with
// one; float32 8000 x 1500 42 and 44, 16384 x 4096 179 and 172; of 1024 threads bfloat16 8192 x 8192 92, 97 with two.
int rms_back_most(int d) { return d <= NORM_LONG && norm_group(d) > 512 ? 256 : 512; }
int rms_back_wgs(int64_t rows, int d) { return norm_wgs(rows, rms_back_rows(d), rms_back_most(d)); }

int rms_check(const char *who, int type, int wtype, int64_t rows, int d)
{
    if (!type_ok(type)) return fail(QADC_EINVAL, "%s: unknown type %d", who, type);
    if (wtype != QADC_TYPE_F32 && wtype != type)
        return fail(QADC_EINVAL, "%s: wtype %d is neither QADC_TYPE_F32 nor the rows' type", who, wtype);
    if (rows < 0 || d < 1 || d > INT32_MAX - 16384) return fail(QADC_EINVAL, "%s: rows=%lld d=%d", who, (long long)rows, d);
    return QADC_OK;
}

}  // namespace

// Enough for these rows and for any fewer.
size_t rms_norm_workspace(int64_t rows, int d)
{
    if (rows < 0 || d < 1 || d > INT32_MAX - 16384) return 0;
    const int64_t alone = std::min<int64_t>(rows, rms_back_rows(d) * (int64_t)rms_back_most(d));  // the most rows done in one turn
    return (size_t)rms_back_wgs(alone, d) * (size_t)d * sizeof(float);
}

template <typename T, int G, int E, bool TINY>
static void rms_launch_rows(const T *x, int64_t ldx, const T *res, int64_t ldr, const void *weight, bool wide, int64_t rows, int d,
                            float eps, const RmsOut &o, hipStream_t st)
{
    constexpr int THREADS = G > 256 ? G : 256;
    // As many threads as fit a compute unit with their registers: float32 16384 x 4096 190 us, 203 with 1536 threads, 193 with 1024; of sixteen
    // elements 4096 x 16384 234, 240 with 2048.
    constexpr int most = 256 * std::max(1, (E == 16 ? 1024 : 2048) / THREADS);
    const unsigned grid = (unsigned)norm_wgs(rows, THREADS / G, most);
    if (res)
        launch(QADC_PROF_RMS, rms_rows_kernel<T, G, E, THREADS, true, TINY>, dim3(grid), dim3(THREADS), 0, st, x, ldx, res, ldr, weight,
               wide, rows, d, eps, o);
    else
        launch(QADC_PROF_RMS, rms_rows_kernel<T, G, E, THREADS, false, TINY>, dim3(grid), dim3(THREADS), 0, st, x, ldx, res, ldr, weight,
               wide, rows, d, eps, o);
}

// f(threads of a row, elements a thread), as constants, for rows of d elements in registers.
template <typename F>
static void by_group(int d, F f)
{
    const auto eight = std::integral_constant<int, 8>();
    switch (norm_group(d)) {
    case 16: f(std::integral_constant<int, 16>(), eight); break;
    case 32: f(std::integral_constant<int, 32>(), eight); break;
    case 64: f(std::integral_constant<int, 64>(), eight); break;
    case 128: f(std::integral_constant<int, 128>(), eight); break;
    case 256: f(std::integral_constant<int, 256>(), eight); break;
    case 512: f(std::integral_constant<int, 512>(), eight); break;
    default:
        if (d <= 8192) f(std::integral_constant<int, 1024>(), eight);
        else f(std::integral_constant<int, 1024>(), std::integral_constant<int, 16>());
        break;
    }
}

int rms_norm(const void *x, int64_t ldx, const void *res, int64_t ldr, int type, const void *weight, int wtype, int64_t rows, int d,
             float eps, void *sum, int64_t ld_sum, void *y, int ytype, float *scale, float *rstd, hipStream_t st)
{
    const char *who = "qadc_rms_norm";
    if (const int rc = rms_check(who, type, wtype, rows, d)) return rc;
    if (ytype != type && ytype != QADC_TYPE_E4M3)
        return fail(QADC_EINVAL, "%s: ytype %d is neither QADC_TYPE_E4M3 nor the rows' type", who, ytype);
    if (ldx < d || (res && (ldr < d || ld_sum < d))) return fail(QADC_EINVAL, "%s: rows of %d elements overlap", who, d);
    if (!(eps >= 0.0f)) return fail(QADC_EINVAL, "%s: eps=%g", who, (double)eps);
    if (rows == 0) return QADC_OK;
    const bool bytes = ytype == QADC_TYPE_E4M3;
    if (!x || !y || (res && !sum) || (bytes && !scale)) return fail(QADC_EINVAL, "%s: null pointer", who);
    if ((sum == x && res && ld_sum != ldx) || (sum == res && res && ld_sum != ldr))
        return fail(QADC_EINVAL, "%s: in place needs equal row distances", who);
    if (y == sum && res) return fail(QADC_EINVAL, "%s: y and sum in one place", who);
    if (((y == x && ldx != d) || (y == res && res && ldr != d)) && !bytes)
        return fail(QADC_EINVAL, "%s: in place needs dense rows", who);
    if (bytes && (y == x || (y == res && res))) return fail(QADC_EINVAL, "%s: 8 bits in place of wider rows", who);
    const RmsOut o = {sum, ld_sum, y, scale, rstd, bytes};
    const bool wide = wtype == QADC_TYPE_F32;
    QADC_BY_TYPE(type, {
        const T *xt = (const T *)x, *rt = (const T *)res;
        const auto run = [&](auto tiny) {
            constexpr bool TINY = decltype(tiny)::value;
            if (d > NORM_LONG) {
                launch(QADC_PROF_RMS, rms_long_kernel<T, TINY>, dim3(norm_grid(rows)), dim3(RMS_WG), 0, st, xt, ldx, rt, ldr, weight, wide,
                       rows, d, eps, o);
            } else {
                by_group(d, [&](auto g, auto e) {
                    rms_launch_rows<T, g.value, e.value, TINY>(xt, ldx, rt, ldr, weight, wide, rows, d, eps, o, st);
                });
            }
        };
        if constexpr (!std::is_same<T, _Float16>::value) {  // (which has no squares below 2^-48)
            if (eps < RMS_EPS_TINY) run(std::true_type());
            else run(std::false_type());
        } else {
            run(std::false_type());
        }
    });
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

template <typename T, int G, int E>
static void rms_launch_back(const RmsBack &b, const void *weight, bool wide, int64_t rows, int d, unsigned grid, hipStream_t st)
{
    constexpr int THREADS = G > 512 ? G : 512;
    constexpr bool AHEAD = E == 8;  // (sixteen elements a thread leave no registers for the next row's)
    if (b.dsum)
        launch(QADC_PROF_RMS, rms_back_kernel<T, G, E, THREADS, AHEAD, true>, dim3(grid), dim3(THREADS), 0, st, b, weight, wide, rows, d);
    else
        launch(QADC_PROF_RMS, rms_back_kernel<T, G, E, THREADS, AHEAD, false>, dim3(grid), dim3(THREADS), 0, st, b, weight, wide, rows, d);
}

int rms_norm_backward(const void *dy, int64_t lddy, const void *dsum, int64_t ldds, const void *h, int64_t ldh, int type,
                      const void *weight, int wtype, const float *rstd, int64_t rows, int d, void *dx, float *dweight, void *workspace,
                      size_t workspace_bytes, hipStream_t st)
{
    const char *who = "qadc_rms_norm_backward";
    if (const int rc = rms_check(who, type, wtype, rows, d)) return rc;
    if (lddy < d || ldh < d || (dsum && ldds < d)) return fail(QADC_EINVAL, "%s: rows of %d elements overlap", who, d);
    if (rows > 0 && (!dy || !h || !rstd)) return fail(QADC_EINVAL, "%s: null pointer", who);
    if (dx && ((dx == dy && lddy != d) || (dx == h && ldh != d) || (dx == dsum && ldds != d)))
        return fail(QADC_EINVAL, "%s: in place needs dense rows", who);
    const int count = rows > 0 ? rms_back_wgs(rows, d) : 0;  // without rows the sum of no parts is written
    if (dweight) {
        const size_t need = (size_t)count * (size_t)d * sizeof(float);
        if (rows > 0 && (!workspace || workspace_bytes < need))
            return fail(QADC_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, need);
        if ((uintptr_t)workspace % 16) return fail(QADC_EINVAL, "%s: workspace is not aligned to 16 bytes", who);
    }
    const RmsBack b = {dy, h, dsum, lddy, ldh, ldds, rstd, dx, dweight ? (float *)workspace : nullptr};
    const bool wide = wtype == QADC_TYPE_F32;
    if (rows > 0 && (dx || dweight)) {
        QADC_BY_TYPE(type, {
            if (d <= NORM_LONG) {
                by_group(d, [&](auto g, auto e) { rms_launch_back<T, g.value, e.value>(b, weight, wide, rows, d, (unsigned)count, st); });
            } else {
                if (dweight)
                    launch(QADC_PROF_RMS, rms_weights_kernel<T>, dim3((unsigned)ceil_div(d, NORM_WG), (unsigned)count), dim3(NORM_WG),
                           0, st, b, rows, d, ceil_div(rows, count));
                if (dx)
                    launch(QADC_PROF_RMS, rms_dx_kernel<T>, dim3(norm_grid(rows)), dim3(RMS_WG), 0, st, b, weight, wide, rows, d);
            }
        });
    }
    if (dweight)
        launch(QADC_PROF_RMS, rms_join_kernel, grid_of(ceil_div(d, WAVE), 1024), dim3(1024), 0, st, (const float *)b.parts, count, d,
               dweight);
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
