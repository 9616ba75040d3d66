// The tokens of the nearest stored states mixed into a model's log probabilities, on gfx950.
//
// A row's neighbours have v_i = -beta (d_i - min d), so the largest is 0 and Z = sum exp v_i is at least 1.  For a token, with
// a = the largest v_i among its votes: log P = a + log(sum of its exp(v_i - a)) - log Z, and
// mix = logaddexp(lm + log(1 - lambda), log P + log lambda); nothing leaves the logarithm, so no weight is too small.
//
// A workgroup per row.  What costs most is the trip to values[ids[i]]: one for all neighbours of a row at once.  They then lie in
// LDS as (token, exp v), and a thread adds up what its token has among its share of them, three instructions a neighbour and no
// branch; P parts of a row's neighbours where there are fewer tokens than threads.  A token whose votes are all too small for
// that (below e^-69) is added up again relative to its own largest.
//
// Bound by the gathers: 2048 rows of 1024 neighbours from 10 M values 47 us, 2 M reads of 4 bytes, each a line (246 MB fetched);
// one row of 100 neighbours 5.4 us, three dependent round trips (kernel by the profiler; the call takes 10.8).

#include <algorithm>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

__device__ __forceinline__ float log_add(float a, float b)
{
    const float hi = fmaxf(a, b);
    return hi == -INFINITY || a != a || b != b ? a + b : hi + log1pf(expf(fminf(a, b) - hi));
}

template <int THREADS, typename F>
__device__ __forceinline__ float group_join(float v, float *lds, F f)
{
    if constexpr (THREADS == WAVE) return v;
    if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < THREADS / WAVE; ++w) v = f(v, lds[w]);
    return v;
}

template <typename D, int THREADS>
__global__ __launch_bounds__(THREADS) void mix_kernel(const uint32_t *__restrict__ ids, const D *__restrict__ dist,
                                                      const float *__restrict__ step, int64_t rows, int R,
                                                      const int32_t *__restrict__ values, int64_t n, float beta,
                                                      const int32_t *__restrict__ tokens, int T, int tokens_at_once,
                                                      const float *__restrict__ lm, float log_keep, float log_lambda,
                                                      float *__restrict__ mix, float *__restrict__ knn)
{
    constexpr int MINE = QADC_MAX_R / THREADS < 4 ? QADC_MAX_R / THREADS : 4;  // neighbours a thread, THREADS apart
    __shared__ float lds[2][THREADS / WAVE];
    __shared__ int4 pairs[THREADS * MINE / 2];  // (token, exp v), two neighbours in 16 bytes
    int2 *const votes = reinterpret_cast<int2 *>(pairs);
    static_assert(alignof(decltype(pairs)) == 16, "two neighbours are read at once");
    __shared__ float far[THREADS * MINE];   // v
    __shared__ float2 sums[THREADS];        // of a part: (sum of exp v, 1 if there is a vote)
    const int t_mine = threadIdx.x % tokens_at_once, part = threadIdx.x / tokens_at_once, parts = THREADS / tokens_at_once;
    const int padded = (R + 7) / 8 * 8;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float step_of = step ? step[r] : 1.0f, b = beta * step_of;
        int tok = t_mine < T ? tokens[r * T + t_mine] : -1;  // on their way with the neighbours
        float l = t_mine < T ? lm[r * T + t_mine] : 0.0f;
        uint32_t id[MINE];
        float d[MINE];
        int val[MINE];
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int at = i * THREADS + threadIdx.x;
            id[i] = at < R ? ids[r * R + at] : 0xFFFFFFFFu;
            d[i] = at < R ? (float)dist[r * R + at] : INFINITY;
        }
        float near = INFINITY;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const bool used = (int64_t)id[i] < n && fabsf(d[i]) < INFINITY;
            val[i] = used ? values[id[i]] : -1;
            d[i] = used ? d[i] : INFINITY;
            near = fminf(near, d[i]);
        }
        near = group_join<THREADS>(-wave_max(-near), lds[0], [](float p, float q) { return fminf(p, q); });
        const bool any = near < INFINITY;
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int at = i * THREADS + threadIdx.x;
            float v = -INFINITY;
            if (d[i] < INFINITY) {
                const float away = d[i] - near;
                if (b < INFINITY && away < INFINITY) v = -b * away;
                else v = (float)(-(double)beta * step_of * ((double)d[i] - near));  // (a float does not hold a part of it; no 0 times inf)
            }
            const float e = expf(v);
            z += e;
            if (at < padded) {
                votes[at] = make_int2(val[i], __float_as_int(e));
                far[at] = v;
            }
        }
        const float log_z = logf(group_join<THREADS>(wave_sum(z), lds[1], [](float p, float q) { return p + q; }));
        if constexpr (THREADS == WAVE) __syncthreads();
        for (int t0 = 0; t0 < T; t0 += tokens_at_once) {
            const int t = t0 + t_mine;
            if (t0) {
                tok = t < T ? tokens[r * T + t] : -1;
                l = t < T ? lm[r * T + t] : 0.0f;
            }
            float s[2] = {0.0f, 0.0f};
            bool vote = false;
#pragma unroll 4
            for (int i = 2 * part; i < padded; i += 2 * parts) {
                const int4 two = pairs[i / 2];
                s[0] += two.x == tok ? __int_as_float(two.y) : 0.0f;
                s[1] += two.z == tok ? __int_as_float(two.w) : 0.0f;
                vote |= two.x == tok || two.z == tok;
            }
            sums[threadIdx.x] = make_float2(s[0] + s[1], vote ? 1.0f : 0.0f);
            __syncthreads();
            if (part == 0 && t < T) {
                float sum = 0.0f, votes_of = 0.0f;
                for (int p = 0; p < parts; ++p) {
                    const float2 v = sums[p * tokens_at_once + t_mine];
                    sum += v.x;
                    votes_of += v.y;
                }
                float log_p = -INFINITY;
                if (votes_of > 0.0f && any && tok >= 0) {
                    log_p = logf(sum) - log_z;
                    if (sum < 1e-30f) {
                        float a = -INFINITY, own = 0.0f;
                        for (int i = 0; i < R; ++i) a = fmaxf(a, votes[i].x == tok ? far[i] : -INFINITY);
                        for (int i = 0; i < R; ++i) own += votes[i].x == tok ? expf(far[i] - a) : 0.0f;
                        log_p = a == -INFINITY ? a : a + logf(own) - log_z;
                    }
                }
                const float out = !any ? l : log_add(l + log_keep, log_p + log_lambda);
                mix[r * T + t] = tok >= 0 ? out : 0.0f;
                if (knn) knn[r * T + t] = tok >= 0 ? log_p : 0.0f;
            }
            __syncthreads();
        }
    }
}

}  // namespace

int neighbour_mix(const uint32_t *ids, const void *dist, int dist_bytes, const float *step, int64_t rows, int R,
                  const int32_t *values, int64_t n, float beta, const int32_t *tokens, int T, const float *lm_logp,
                  float lambda, float *mix, float *knn, hipStream_t st)
{
    // (tokens are counted in an int, up to 256 past the last one)
    if (rows < 0 || R < 1 || R > QADC_MAX_R || n < 0 || T < 0 || T > INT32_MAX - 1024)
        return fail(QADC_EINVAL, "qadc_neighbour_mix: rows=%lld R=%d n=%lld T=%d", (long long)rows, R, (long long)n, T);
    if (dist_bytes != 1 && dist_bytes != 4) return fail(QADC_EINVAL, "qadc_neighbour_mix: dist_bytes=%d", dist_bytes);
    if (!(beta >= 0.0f) || beta == INFINITY || !(lambda >= 0.0f && lambda <= 1.0f))
        return fail(QADC_EINVAL, "qadc_neighbour_mix: beta=%g lambda=%g", (double)beta, (double)lambda);
    if (rows == 0 || T == 0) return QADC_OK;
    if (!ids || !dist || (n > 0 && !values) || !tokens || !lm_logp || !mix)
        return fail(QADC_EINVAL, "qadc_neighbour_mix: null pointer");
    n = std::min<int64_t>(n, 0xFFFFFFFF);  // (the padding is no id)
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 20));
    const float log_keep = log1pf(-lambda), log_lambda = logf(lambda);
    // Rows of few neighbours and tokens have a wavefront each, where there are enough of them: 2048 rows of 128 neighbours and 32 tokens
    // 7.7 us (9.1 with a workgroup of 256 each), 4096 of 100 and 20 8.7 (14.7), of 256 and 64 20.1 (20.6); but 2048 of 256 and 64
    // 16.4 (12.9), 3000 of 200 and 40 15.4 (14.6), and 1024 of 128 and 32 6.7 (6.0); calls replayed from a graph.
    const int threads = R <= 256 && T <= 64 && rows >= (R > 128 && T > 16 ? 4096 : 2048) ? WAVE : 256;
    int at_once = 1;
    while (at_once < T && at_once < threads) at_once *= 2;
#define MIX(D_, THREADS_)                                                                                                       \
    launch(QADC_PROF_MIX, mix_kernel<D_, THREADS_>, grid, dim3(THREADS_), 0, st, ids, (const D_ *)dist, step, rows, R, values, n, \
           beta, tokens, T, at_once, lm_logp, log_keep, log_lambda, mix, knn)
    if (threads == WAVE) {
        if (dist_bytes == 1) MIX(uint8_t, WAVE);
        else MIX(float, WAVE);
    } else {
        if (dist_bytes == 1) MIX(uint8_t, 256);
        else MIX(float, 256);
    }
#undef MIX
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
