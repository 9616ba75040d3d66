// Layer norm and its backward pass on gfx950.
//
// Forward: mean = sum x / d, then the squared differences to that mean (two passes over the row: no difference of large sums),
// y = (x - mean) rstd w + b.  Backward: with h = (x - mean) rstd and g = dy w, dx = rstd (g - sum g / d - h sum(g h) / d); the
// weight's gradients are sums over the rows, added in a fixed order: each workgroup its stretch of rows, then the stretches.

#include <algorithm>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int NORM_WG = 256;

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

// The sums of `count` parts [count][2][d].
__global__ __launch_bounds__(NORM_WG) void norm_join_kernel(const float *__restrict__ parts, int count, int d,
                                                            float *__restrict__ dweight, float *__restrict__ dbias)
{
    const int c = blockIdx.x * NORM_WG + threadIdx.x;
    if (c >= d) return;
    float sw = 0.0f, sb = 0.0f;
    for (int p = 0; p < count; ++p) {
        sw += parts[((size_t)p * 2) * d + c];
        sb += parts[((size_t)p * 2 + 1) * d + c];
    }
    if (dweight) dweight[c] = sw;
    if (dbias) dbias[c] = sb;
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

constexpr int NORM_PARTS = 256;  // stretches of rows whose weight gradients are summed apart

int norm_parts(int64_t rows) { return (int)std::min<int64_t>(NORM_PARTS, std::max<int64_t>(1, ceil_div(rows, 16))); }

unsigned norm_grid(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }

}  // namespace

size_t layer_norm_workspace(int64_t rows, int d)
{
    if (rows < 0 || d < 1) return 0;
    return (size_t)norm_parts(rows) * 2 * (size_t)d * sizeof(float);
}

static int norm_check(const char *who, int type, int wtype, int64_t rows, int d, int64_t ldx, int64_t ldy)
{
    if (!type_ok(type)) return fail(QADC_EINVAL, "%s: unknown type %d", who, type);
    if (wtype != QADC_TYPE_F32 && wtype != type)
        return fail(QADC_EINVAL, "%s: wtype %d is neither QADC_TYPE_F32 nor the rows' type", who, wtype);
    if (rows < 0 || d < 1) return fail(QADC_EINVAL, "%s: rows=%lld d=%d", who, (long long)rows, d);
    if (ldx < d || ldy < d) return fail(QADC_EINVAL, "%s: rows of %d elements, a row distance of %lld", who, d,
                                        (long long)std::min(ldx, ldy));
    return QADC_OK;
}

template <typename T, typename W>
static void norm_launch(const void *x, int64_t ldx, const void *weight, const void *bias, int64_t rows, int d, float eps,
                        void *y, float *mean, float *rstd, hipStream_t st)
{
    launch(QADC_PROF_NORM, norm_kernel<T, W>, dim3(norm_grid(rows)), dim3(NORM_WG), 0, st, (const T *)x, ldx,
           (const W *)weight, (const W *)bias, rows, d, eps, (T *)y, mean, rstd);
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

template <typename T, typename W>
static void norm_backward_launch(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *weight,
                                 const float *mean, const float *rstd, int64_t rows, int d, void *dx, float *dweight,
                                 float *dbias, float *parts, hipStream_t st)
{
    if (dweight || dbias) {
        const int count = norm_parts(rows);
        const int64_t stretch = ceil_div(rows, count);
        launch(QADC_PROF_NORM, norm_weights_kernel<T>, dim3((unsigned)ceil_div(d, NORM_WG), (unsigned)count), dim3(NORM_WG), 0,
               st, (const T *)dy, lddy, (const T *)x, ldx, mean, rstd, rows, d, stretch, parts);
        launch(QADC_PROF_NORM, norm_join_kernel, dim3((unsigned)ceil_div(d, NORM_WG)), dim3(NORM_WG), 0, st, parts, count, d,
               dweight, dbias);
    }
    if (dx && rows > 0)
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
        const size_t need = layer_norm_workspace(rows, d);
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
