// The tokens of the nearest stored states mixed into a model's log probabilities, on gfx950.
//
// A row's neighbours have v_i = -beta (d_i - min d), so the largest is 0 and Z = sum exp v_i is at least 1.  For a token, with
// a = the largest v_i among its votes: log P = a + log(sum of its exp(v_i - a)) - log Z, and
// mix = logaddexp(lm + log(1 - lambda), log P + log lambda); nothing leaves the logarithm, so no weight is too small.

#include <algorithm>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int MIX_WG = 256;

__device__ __forceinline__ float log_add(float a, float b)
{
    const float hi = fmaxf(a, b);
    return hi == -INFINITY || a != a || b != b ? a + b : hi + log1pf(expf(fminf(a, b) - hi));
}

template <typename F>
__device__ __forceinline__ float group_join(float v, float *lds, F f)
{
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) v = f(v, __shfl_xor(v, s));
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < MIX_WG / WAVE; ++w) v = f(v, lds[w]);
    return v;
}

// A workgroup per row, a thread per token.
template <typename D>
__global__ __launch_bounds__(MIX_WG) void mix_kernel(const uint32_t *__restrict__ ids, const D *__restrict__ dist,
                                                     const float *__restrict__ step, int64_t rows, int R,
                                                     const int32_t *__restrict__ values, int64_t n, float beta,
                                                     const int32_t *__restrict__ tokens, int T, const float *__restrict__ lm,
                                                     float log_keep, float log_lambda, float *__restrict__ mix,
                                                     float *__restrict__ knn)
{
    __shared__ float lds[MIX_WG / WAVE];
    __shared__ int value[QADC_MAX_R];
    __shared__ float vs[QADC_MAX_R];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float b = step ? beta * step[r] : beta;
        float near = INFINITY;
        __syncthreads();
        for (int i = threadIdx.x; i < R; i += MIX_WG) {
            const uint32_t id = ids[r * R + i];
            const float d = (float)dist[r * R + i];
            const bool used = (int64_t)id < n && fabsf(d) < INFINITY;
            value[i] = used ? values[id] : -1;
            vs[i] = used ? d : INFINITY;
            near = fminf(near, vs[i]);
        }
        near = group_join(near, lds, [](float p, float q) { return fminf(p, q); });
        float z = 0.0f;
        for (int i = threadIdx.x; i < R; i += MIX_WG) {
            vs[i] = vs[i] < INFINITY ? -b * (vs[i] - near) : -INFINITY;
            z += expf(vs[i]);
        }
        const float log_z = logf(group_join(z, lds, [](float p, float q) { return p + q; }));
        const bool any = near < INFINITY;
        for (int t = threadIdx.x; t < T; t += MIX_WG) {
            const int tok = tokens[r * T + t];
            float a = -INFINITY, s = 0.0f;
            for (int i = 0; i < R; ++i)
                if (value[i] == tok) a = fmaxf(a, vs[i]);
            if (a > -INFINITY)
                for (int i = 0; i < R; ++i)
                    if (value[i] == tok) s += expf(vs[i] - a);
            const float log_p = a > -INFINITY ? a + logf(s) - log_z : -INFINITY;
            const float l = lm[r * T + t];
            const float out = !any ? l : log_add(l + log_keep, log_p + log_lambda);
            mix[r * T + t] = tok >= 0 ? out : 0.0f;
            if (knn) knn[r * T + t] = tok >= 0 ? log_p : 0.0f;
        }
    }
}

}  // namespace

int neighbour_mix(const uint32_t *ids, const void *dist, int dist_bytes, const float *step, int64_t rows, int R,
                  const int32_t *values, int64_t n, float beta, const int32_t *tokens, int T, const float *lm_logp,
                  float lambda, float *mix, float *knn, hipStream_t st)
{
    if (rows < 0 || R < 1 || R > QADC_MAX_R || n < 0 || T < 0)
        return fail(QADC_EINVAL, "qadc_neighbour_mix: rows=%lld R=%d n=%lld T=%d", (long long)rows, R, (long long)n, T);
    if (dist_bytes != 1 && dist_bytes != 4) return fail(QADC_EINVAL, "qadc_neighbour_mix: dist_bytes=%d", dist_bytes);
    if (!(beta >= 0.0f) || beta == INFINITY || !(lambda >= 0.0f && lambda <= 1.0f))
        return fail(QADC_EINVAL, "qadc_neighbour_mix: beta=%g lambda=%g", (double)beta, (double)lambda);
    if (rows == 0 || T == 0) return QADC_OK;
    if (!ids || !dist || (n > 0 && !values) || !tokens || !lm_logp || !mix)
        return fail(QADC_EINVAL, "qadc_neighbour_mix: null pointer");
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 20));
    const float log_keep = log1pf(-lambda), log_lambda = logf(lambda);
    if (dist_bytes == 1)
        launch(QADC_PROF_MIX, mix_kernel<uint8_t>, grid, dim3(MIX_WG), 0, st, ids, (const uint8_t *)dist, step, rows, R, values, n,
               beta, tokens, T, lm_logp, log_keep, log_lambda, mix, knn);
    else
        launch(QADC_PROF_MIX, mix_kernel<float>, grid, dim3(MIX_WG), 0, st, ids, (const float *)dist, step, rows, R, values, n,
               beta, tokens, T, lm_logp, log_keep, log_lambda, mix, knn);
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
