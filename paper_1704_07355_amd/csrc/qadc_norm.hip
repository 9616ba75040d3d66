// Layer norm and its backward pass on gfx950.
//
// Forward: mean = sum x / d, then the squared differences to that mean (two passes over the row: no difference of large sums),
// y = (x - mean) rstd w + b.  Backward: with h = (x - mean) rstd and g = dy w, dx = rstd (g - sum g / d - h sum(g h) / d); the
// weight's gradients are sums over the rows, added in a fixed order: each workgroup its stretch of rows, then the stretches.
//
// A row of up to 16384 elements stays in the registers of its group of threads, 8 or 16 a thread; the group goes on to further
// rows with the weights (and the sums of the weight's gradients) in registers, the next row's elements already on their way.
// Longer rows are read again for every pass.
//
// Bound by memory: 16384 x 4096 bfloat16 backward 79 us (402 MB at 5.1 TB/s) and 5 us for the join of the sums; 2049 x 1111
// float32 13 + 4.4, where three turns a workgroup leave each load and barrier exposed; five rows of 4096 bfloat16 forward 3.4 us, a
// launch's latency.  (These are kernels' times by the profiler; figures elsewhere in this file are calls one after the other: 86,
// 15.8 and 10 us.)  Rows beyond 16384 elements, an element a load and three reads of the row: 1000 x 20000 bfloat16 79 us
// forward, 93 backward, 4096 x 32768 332 and 545, a third of what the memory would give.

#include <algorithm>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int NORM_WG = 256;

// Sums over a group of G threads, in every one of them; `turn` alternates between calls (a buffer is written again only
// behind the barrier of the call in between).
template <int G, int NS>
__device__ __forceinline__ void group_sums(float (&v)[NS], float *lds, int &turn)
{
#pragma unroll
    for (int i = 0; i < NS; ++i) v[i] = lanes_sum<G < WAVE ? G : WAVE>(v[i]);
    if constexpr (G > WAVE) {
        constexpr int W = G / WAVE;
        float *buf = lds + (turn & 1) * (1024 / WAVE) * NS;
        ++turn;
        const int wave = threadIdx.x >> 6, first = wave / W * W;
        if (lane_id() == 0)
#pragma unroll
            for (int i = 0; i < NS; ++i) buf[wave * NS + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) v[i] += buf[(first + w) * NS + i];
        }
    }
}

// The elements of a row that thread t of a group of G holds: E / N packs, those of the group side by side.
template <typename T, int G, int E>
struct Part {
    static constexpr int N = Pack<T>::N, P = E / N;
    typedef typename Pack<T>::V V;
    V raw[P];

    // A pack across the row's end is loaded from N elements before it, and put in its place, zeros behind it, by settle(): the
    // row stays on its way, without a branch around a load, until it is needed.  (65536 x 768 bfloat16 with an element at a time
    // there: forward 48 us, backward 97.)
    __device__ __forceinline__ void load(const T *row, int t, int d)
    {
#pragma unroll
        for (int u = 0; u < P; ++u) {
            if (d < N) {
#pragma unroll
                for (int e = 0; e < N; ++e) raw[u][e] = (u * G + t) * N + e < d ? row[(u * G + t) * N + e] : (T)0.0f;
                continue;
            }
            // Every row is read once: past the caches it comes faster (16384 x 4096 float32: forward 97 -> 81 us, backward
            // 154 -> 131; bfloat16 backward 88 -> 82), but for rows so short that they share lines (200000 x 100: 20 -> 26).
            const V *from = reinterpret_cast<const V *>(row + min((u * G + t) * N, d - N));
            raw[u] = G > 16 ? __builtin_nontemporal_load(from) : *from;
        }
    }
    __device__ __forceinline__ void settle(int t, int d)
    {
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int beyond = (u * G + t) * N - (d - N);  // elements
            if (beyond <= 0 || d < N) continue;
            const V zero = (T)0.0f;
            if (beyond >= N) raw[u] = zero;
            else
#pragma unroll 1
                for (int e = 0; e < beyond; ++e) {
                    if constexpr (N == 8) raw[u] = __builtin_shufflevector(raw[u], zero, 1, 2, 3, 4, 5, 6, 7, 8);
                    else raw[u] = __builtin_shufflevector(raw[u], zero, 1, 2, 3, 4);
                }
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return (float)raw[i / N][i % N]; }
    __device__ static __forceinline__ int column(int i, int t) { return (i / N * G + t) * N + i % N; }
    __device__ __forceinline__ void set(int i, float v) { raw[i / N][i % N] = (T)v; }
    __device__ __forceinline__ void store(T *row, int t, int d) const
    {
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int c = (u * G + t) * N;
            if (c + N <= d) {
                *reinterpret_cast<V *>(row + c) = raw[u];
            } else if (c < d) {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (c + e < d) row[c + e] = raw[u][e];
            }
        }
    }
};

template <typename T, int G, int E, typename W>
__device__ __forceinline__ void load_weights(const W *w, float none, int t, int d, float (&v)[E])
{
    constexpr int N = Pack<T>::N;
    typedef W Wide __attribute__((ext_vector_type(N), aligned(sizeof(W))));
#pragma unroll
    for (int u = 0; u < E / N; ++u) {
        const int c = (u * G + t) * N;
        if (w && c + N <= d) {
            const Wide p = *reinterpret_cast<const Wide *>(w + c);
#pragma unroll
            for (int e = 0; e < N; ++e) v[u * N + e] = (float)p[e];
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[u * N + e] = w && c + e < d ? (float)w[c + e] : none;
        }
    }
}

// A group of G threads per row, THREADS / G rows of a workgroup at a time.
template <typename T, typename W, int G, int E, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_rows_kernel(const T *x, int64_t ldx, const W *__restrict__ weight,
                                                            const W *__restrict__ bias, int64_t rows, int d, float eps, T *y,
                                                            float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    __shared__ float lds[2 * (1024 / WAVE)];
    constexpr int R = THREADS / G;
    const int t = threadIdx.x % G;
    int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / G;
    const int64_t ahead = (int64_t)gridDim.x * R;
    Part<T, G, E> one, two;
    one.load(x + min(r, rows - 1) * ldx, t, d);
    float w[E], b[E];
    load_weights<T, G, E>(weight, 1.0f, t, d, w);
    load_weights<T, G, E>(bias, 0.0f, t, d, b);
    int turns = 0;
    // a row, while the next one comes in; false behind the last (all groups of a workgroup go round together)
    const auto turn = [&](Part<T, G, E> &now, Part<T, G, E> &next) {
        const bool more = r - threadIdx.x / G + ahead < rows;
        if (more) next.load(x + min(r + ahead, rows - 1) * ldx, t, d);
        now.settle(t, d);
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < E; ++i) s[0] += now[i];
        group_sums<G, 1>(s, lds, turns);
        const float mean = s[0] / (float)d;
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float h = Part<T, G, E>::column(i, t) < d ? now[i] - mean : 0.0f;
            s[0] = fmaf(h, h, s[0]);
        }
        group_sums<G, 1>(s, lds, turns);
        const float rstd = 1.0f / sqrtf(s[0] / (float)d + eps);
        if (r < rows) {
            Part<T, G, E> out;
#pragma unroll
            for (int i = 0; i < E; ++i) out.set(i, fmaf((now[i] - mean) * rstd, w[i], b[i]));
            out.store(y + r * d, t, d);
            if (t == 0) {
                if (mean_out) mean_out[r] = mean;
                if (rstd_out) rstd_out[r] = rstd;
            }
        }
        r += ahead;
        return more;
    };
    while (turn(one, two) && turn(two, one)) {
    }
}

// dx of the workgroup's rows and, where `parts` is set, their share of the weight's gradients: parts [workgroup][2][d].
template <typename T, typename W, int G, int E, int THREADS, bool AHEAD>
__global__ __launch_bounds__(THREADS) void norm_back_kernel(const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                            const W *__restrict__ weight, const float *__restrict__ mean,
                                                            const float *__restrict__ rstd, int64_t rows, int d, T *dx,
                                                            float *__restrict__ parts)
{
    __shared__ float lds[4 * (1024 / WAVE)];
    constexpr int R = THREADS / G;
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    int64_t r = (int64_t)blockIdx.x * R + group;
    const int64_t ahead = (int64_t)gridDim.x * R;
    typedef Part<T, G, E> P;
    struct Row {
        P x, dy;
        float mean, rstd;
    } one, two;
    const auto load = [&](Row &row, int64_t at) {
        at = min(at, rows - 1);
        row.x.load(x + at * ldx, t, d);
        row.dy.load(dy + at * lddy, t, d);
        row.mean = mean[at];
        row.rstd = rstd[at];
    };
    if (AHEAD) load(one, r);
    float w[E], dw[E], db[E];
    load_weights<T, G, E>(weight, 1.0f, t, d, w);
#pragma unroll
    for (int i = 0; i < E; ++i) dw[i] = db[i] = 0.0f;
    int turns = 0;
    // a row, while the next one comes in; false behind the last (all groups of a workgroup go round together)
    const auto turn = [&](Row &now, Row &next) {
        const bool more = r - group + ahead < rows;
        if (!AHEAD) load(now, r);
        else if (more) load(next, r + ahead);
        now.x.settle(t, d);
        now.dy.settle(t, d);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float g = now.dy[i] * w[i];
            s[0] += g;
            s[1] = fmaf(g, (now.x[i] - now.mean) * now.rstd, s[1]);
        }
        group_sums<G, 2>(s, lds, turns);
        if (r < rows) {
            const float a = s[0] / (float)d, b = s[1] / (float)d, rs = now.rstd;
            float mu = now.mean;
            asm volatile("" : "+v"(mu));  // (h is cheaper computed again than kept across the barrier)
            P out;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float dyi = now.dy[i], h = (now.x[i] - mu) * rs;
                dw[i] = fmaf(dyi, h, dw[i]);
                db[i] += dyi;
                out.set(i, rs * (fmaf(dyi, w[i], -a) - h * b));
            }
            if (dx) out.store(dx + r * d, t, d);
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
    if (!parts) return;
    if constexpr (R > 1) {  // the groups' sums, in their order
        __shared__ float both[2 * G * E];
        for (int g = 0; g < R; ++g) {
            __syncthreads();
            if (group == g)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float *p = both + 2 * (i * G + t);
                    p[0] = g ? p[0] + dw[i] : dw[i];
                    p[1] = g ? p[1] + db[i] : db[i];
                }
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            dw[i] = both[2 * (i * G + t)];
            db[i] = both[2 * (i * G + t) + 1];
        }
    }
    float *mine = parts + (size_t)blockIdx.x * 2 * d;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int c = P::column(i, t);
        if (c < d) {
            mine[c] = dw[i];
            mine[d + c] = db[i];
        }
    }
}

// The sums of `count` parts [count][2][d], 64 columns a workgroup, a sixteenth of the parts each wavefront.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float *__restrict__ parts, int count, int d,
                                                         float *__restrict__ dweight, float *__restrict__ dbias)
{
    __shared__ float lds[16][WAVE];
    const int wave = threadIdx.x >> 6, lane = lane_id();
    const int64_t c = (int64_t)blockIdx.x * WAVE + lane;
    float s = 0.0f;
    if (c < 2 * (int64_t)d) {
#pragma unroll 16
        for (int p = wave; p < count; p += 16) s += parts[(size_t)p * 2 * d + c];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave || c >= 2 * (int64_t)d) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += lds[w][lane];
    if (c < d) {
        if (dweight) dweight[c] = s;
    } else if (dbias) {
        dbias[c - d] = s;
    }
}

// Rows beyond 16384 elements.

// Sum over the workgroup, in every thread.
__device__ __forceinline__ float group_sum(float v, float *lds)
{
    v = wave_sum(v);
    __syncthreads();  // (the sum before has been read)
    if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < NORM_WG / WAVE; ++w) s += lds[w];
    return s;
}

// A workgroup per row.
template <typename T, typename W>
__global__ __launch_bounds__(NORM_WG) void norm_kernel(const T *x, int64_t ldx, const W *__restrict__ weight,
                                                       const W *__restrict__ bias, int64_t rows, int d, float eps, T *y,
                                                       float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    __shared__ float lds[NORM_WG / WAVE];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + r * ldx;
        T *yr = y + r * d;
        float s = 0.0f;
        for (int c = threadIdx.x; c < d; c += NORM_WG) s += (float)xr[c];
        const float mean = group_sum(s, lds) / (float)d;
        s = 0.0f;
        for (int c = threadIdx.x; c < d; c += NORM_WG) {
            const float h = (float)xr[c] - mean;
            s = fmaf(h, h, s);
        }
        const float rstd = 1.0f / sqrtf(group_sum(s, lds) / (float)d + eps);
        for (int c = threadIdx.x; c < d; c += NORM_WG) {
            const float w = weight ? (float)weight[c] : 1.0f, b = bias ? (float)bias[c] : 0.0f;
            yr[c] = (T)fmaf(((float)xr[c] - mean) * rstd, w, b);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[r] = mean;
            if (rstd_out) rstd_out[r] = rstd;
        }
    }
}

// The weight's gradients of a stretch of rows: a thread per column.  Before dx, which may take dy's or x's place.
template <typename T>
__global__ __launch_bounds__(NORM_WG) void norm_weights_kernel(const T *__restrict__ dy, int64_t lddy, const T *__restrict__ x,
                                                               int64_t ldx, const float *__restrict__ mean,
                                                               const float *__restrict__ rstd, int64_t rows, int d,
                                                               int64_t stretch, float *__restrict__ parts)
{
    const int c = blockIdx.x * NORM_WG + threadIdx.x;
    if (c >= d) return;
    const int64_t r0 = (int64_t)blockIdx.y * stretch, r1 = min(r0 + stretch, rows);
    float sw = 0.0f, sb = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float g = (float)dy[r * lddy + c];
        sw = fmaf(g, ((float)x[r * ldx + c] - mean[r]) * rstd[r], sw);
        sb += g;
    }
    parts[((size_t)blockIdx.y * 2) * d + c] = sw;
    parts[((size_t)blockIdx.y * 2 + 1) * d + c] = sb;
}

// dx, a workgroup per row.
template <typename T, typename W>
__global__ __launch_bounds__(NORM_WG) void norm_dx_kernel(const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                          const W *__restrict__ weight, const float *__restrict__ mean,
                                                          const float *__restrict__ rstd, int64_t rows, int d, T *dx)
{
    __shared__ float lds[NORM_WG / WAVE];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *gr = dy + r * lddy, *xr = x + r * ldx;
        const float mu = mean[r], rs = rstd[r];
        float a = 0.0f, b = 0.0f;
        for (int c = threadIdx.x; c < d; c += NORM_WG) {
            const float g = (float)gr[c] * (weight ? (float)weight[c] : 1.0f);
            a += g;
            b = fmaf(g, ((float)xr[c] - mu) * rs, b);
        }
        a = group_sum(a, lds) / (float)d;
        b = group_sum(b, lds) / (float)d;
        for (int c = threadIdx.x; c < d; c += NORM_WG) {
            const float g = (float)gr[c] * (weight ? (float)weight[c] : 1.0f);
            const float h = ((float)xr[c] - mu) * rs;
            dx[r * d + c] = (T)(rs * (g - a - h * b));
        }
    }
}

constexpr int NORM_LONG = 16384;  // longest rows that stay in registers

// Threads that share a row: eight elements each up to 8192, sixteen beyond.
int norm_group(int d) { return d <= 128 ? 16 : d <= 256 ? 32 : d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024; }

// Workgroups for `rows`, `at_once` of them at a time in each: at most `most`, and all with the same number of turns.
int norm_wgs(int64_t rows, int at_once, int most)
{
    const int64_t turns = std::max<int64_t>(1, ceil_div(rows, (int64_t)at_once * most));
    return (int)std::max<int64_t>(1, ceil_div(rows, at_once * turns));
}

// Workgroups of the backward pass, each with its own sums of the weight's gradients (8 d bytes written and read again): two of
// 512 threads a compute unit, one of 1024.  With 512 of the latter 665 x 5702 bfloat16 took 31 us, a third of it for the sums.
int back_rows(int d) { return d > NORM_LONG ? 16 : std::max(1, 512 / norm_group(d)); }  // rows of a workgroup at a time
int back_most(int d) { return d <= NORM_LONG && norm_group(d) > 512 ? 256 : 512; }
int back_wgs(int64_t rows, int d) { return norm_wgs(rows, back_rows(d), back_most(d)); }

unsigned norm_grid(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }

}  // namespace

static size_t back_bytes(int wgs, int d) { return (size_t)wgs * 2 * (size_t)d * sizeof(float); }

// Enough for these rows and for any fewer, of which up to twice as many workgroups can be made (4096 columns: 257 for 513 rows, 512
// for 512).  The call itself asks for its own rows' share only.
size_t layer_norm_workspace(int64_t rows, int d)
{
    if (rows < 0 || d < 1 || d > INT32_MAX - 1024) return 0;
    const int64_t alone = std::min<int64_t>(rows, back_rows(d) * (int64_t)back_most(d));  // the most rows that are done in one turn
    return back_bytes(back_wgs(alone, d), d);
}

static int norm_check(const char *who, int type, int wtype, int64_t rows, int d, int64_t ldx, int64_t ldy)
{
    if (!type_ok(type)) return fail(QADC_EINVAL, "%s: unknown type %d", who, type);
    if (wtype != QADC_TYPE_F32 && wtype != type)
        return fail(QADC_EINVAL, "%s: wtype %d is neither QADC_TYPE_F32 nor the rows' type", who, wtype);
    // (columns are counted in an int, a workgroup's width past the last one)
    if (rows < 0 || d < 1 || d > INT32_MAX - 1024) return fail(QADC_EINVAL, "%s: rows=%lld d=%d", who, (long long)rows, d);
    if (ldx < d || ldy < d) return fail(QADC_EINVAL, "%s: rows of %d elements, a row distance of %lld", who, d,
                                        (long long)std::min(ldx, ldy));
    return QADC_OK;
}

template <typename T, typename W, int G, int E>
static void norm_launch_rows(const void *x, int64_t ldx, const void *weight, const void *bias, int64_t rows, int d, float eps,
                             void *y, float *mean, float *rstd, hipStream_t st)
{
    constexpr int THREADS = G > 256 ? G : 256;
    // As many workgroups as the registers let a compute unit hold at once (a few more would be a round of their own): 65536 x 768
    // float32 76 us with 2048 workgroups of 256, 67 with 1536; 16384 x 4096 bfloat16 55 with 1024 of 512, 62 with 768.
    constexpr int most = 256 * std::max(1, (E == 16 ? 1024 : sizeof(T) == 2 ? 2048 : 1536) / THREADS);
    const unsigned grid = (unsigned)norm_wgs(rows, THREADS / G, most);
    launch(QADC_PROF_NORM, norm_rows_kernel<T, W, G, E, THREADS>, dim3(grid), dim3(THREADS), 0, st, (const T *)x, ldx,
           (const W *)weight, (const W *)bias, rows, d, eps, (T *)y, mean, rstd);
}

template <typename T, typename W>
static void norm_launch(const void *x, int64_t ldx, const void *weight, const void *bias, int64_t rows, int d, float eps,
                        void *y, float *mean, float *rstd, hipStream_t st)
{
#define ROWS(G_, E_) norm_launch_rows<T, W, G_, E_>(x, ldx, weight, bias, rows, d, eps, y, mean, rstd, st)
    if (d > NORM_LONG) {
        launch(QADC_PROF_NORM, norm_kernel<T, W>, dim3(norm_grid(rows)), dim3(NORM_WG), 0, st, (const T *)x, ldx,
               (const W *)weight, (const W *)bias, rows, d, eps, (T *)y, mean, rstd);
        return;
    }
    switch (norm_group(d)) {
    case 16: ROWS(16, 8); break;
    case 32: ROWS(32, 8); break;
    case 64: ROWS(64, 8); break;
    case 128: ROWS(128, 8); break;
    case 256: ROWS(256, 8); break;
    case 512: ROWS(512, 8); break;
    default:
        if (d <= 8192) ROWS(1024, 8);
        else ROWS(1024, 16);
        break;
    }
#undef ROWS
}

int layer_norm(const void *x, int64_t ldx, int type, const void *weight, const void *bias, int wtype, int64_t rows, int d,
               float eps, void *y, float *mean, float *rstd, hipStream_t st)
{
    if (const int rc = norm_check("qadc_layer_norm", type, wtype, rows, d, ldx, ldx)) return rc;
    if (!(eps >= 0.0f)) return fail(QADC_EINVAL, "qadc_layer_norm: eps=%g", (double)eps);
    if (rows == 0) return QADC_OK;
    if (!x || !y) return fail(QADC_EINVAL, "qadc_layer_norm: null pointer");
    if (x == y && ldx != d) return fail(QADC_EINVAL, "qadc_layer_norm: in place needs dense rows");
    if (wtype == type) {
        QADC_BY_TYPE(type, (norm_launch<T, T>(x, ldx, weight, bias, rows, d, eps, y, mean, rstd, st)));
    } else {
        QADC_BY_TYPE(type, (norm_launch<T, float>(x, ldx, weight, bias, rows, d, eps, y, mean, rstd, st)));
    }
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

template <typename T, typename W, int G, int E>
static void norm_launch_back(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *weight, const float *mean,
                             const float *rstd, int64_t rows, int d, void *dx, float *parts, hipStream_t st)
{
    constexpr int THREADS = G > 512 ? G : 512;
    constexpr bool AHEAD = E == 8;  // (sixteen elements a thread leave no registers for the next row's)
    const unsigned grid = (unsigned)back_wgs(rows, d);
    launch(QADC_PROF_NORM, norm_back_kernel<T, W, G, E, THREADS, AHEAD>, dim3(grid), dim3(THREADS), 0, st, (const T *)dy, lddy,
           (const T *)x, ldx, (const W *)weight, mean, rstd, rows, d, (T *)dx, parts);
}

template <typename T, typename W>
static void norm_backward_launch(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *weight,
                                 const float *mean, const float *rstd, int64_t rows, int d, void *dx, float *dweight,
                                 float *dbias, float *parts, hipStream_t st)
{
    const bool sums = dweight || dbias;
    int count = 0;  // without rows the sums of no parts are written
    if (rows > 0 && d <= NORM_LONG) {
        count = back_wgs(rows, d);
#define BACK(G_, E_) norm_launch_back<T, W, G_, E_>(dy, lddy, x, ldx, weight, mean, rstd, rows, d, dx, sums ? parts : nullptr, st)
        switch (norm_group(d)) {
        case 16: BACK(16, 8); break;
        case 32: BACK(32, 8); break;
        case 64: BACK(64, 8); break;
        case 128: BACK(128, 8); break;
        case 256: BACK(256, 8); break;
        case 512: BACK(512, 8); break;
        default:
            if (d <= 8192) BACK(1024, 8);
            else BACK(1024, 16);
            break;
        }
#undef BACK
    } else if (rows > 0 && sums) {
        count = back_wgs(rows, d);
        launch(QADC_PROF_NORM, norm_weights_kernel<T>, dim3((unsigned)ceil_div(d, NORM_WG), (unsigned)count), dim3(NORM_WG), 0,
               st, (const T *)dy, lddy, (const T *)x, ldx, mean, rstd, rows, d, ceil_div(rows, count), parts);
    }
    if (sums)
        launch(QADC_PROF_NORM, norm_join_kernel, dim3((unsigned)ceil_div(2 * (int64_t)d, WAVE)), dim3(1024), 0, st, parts, count,
               d, dweight, dbias);
    if (dx && rows > 0 && d > NORM_LONG)
        launch(QADC_PROF_NORM, norm_dx_kernel<T, W>, dim3(norm_grid(rows)), dim3(NORM_WG), 0, st, (const T *)dy, lddy,
               (const T *)x, ldx, (const W *)weight, mean, rstd, rows, d, (T *)dx);
}

int layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, int type, const void *weight, int wtype,
                        const float *mean, const float *rstd, int64_t rows, int d, void *dx, float *dweight, float *dbias,
                        void *workspace, size_t workspace_bytes, hipStream_t st)
{
    if (const int rc = norm_check("qadc_layer_norm_backward", type, wtype, rows, d, ldx, lddy)) return rc;
    if (rows > 0 && (!dy || !x || !mean || !rstd)) return fail(QADC_EINVAL, "qadc_layer_norm_backward: null pointer");
    if ((dx == dy && dx && lddy != d) || (dx == x && dx && ldx != d))
        return fail(QADC_EINVAL, "qadc_layer_norm_backward: in place needs dense rows");
    if (dweight || dbias) {
        const size_t need = back_bytes(back_wgs(rows, d), d);
        if (!workspace || workspace_bytes < need)
            return fail(QADC_ENOMEM, "qadc_layer_norm_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    }
    if (wtype == type) {
        QADC_BY_TYPE(type, (norm_backward_launch<T, T>(dy, lddy, x, ldx, weight, mean, rstd, rows, d, dx, dweight, dbias,
                                                       (float *)workspace, st)));
    } else {
        QADC_BY_TYPE(type, (norm_backward_launch<T, float>(dy, lddy, x, ldx, weight, mean, rstd, rows, d, dx, dweight, dbias,
                                                           (float *)workspace, st)));
    }
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
