// Log probabilities of given tokens with the entropy and the likeliest alternatives, and their gradient, on gfx950.
//
// With x = scale logits, m = max x and e = exp(x - m): lse = m + log sum e, entropy = log sum e - sum e (x - m) / sum e.  The
// alternatives are the k largest under one 64-bit key: the logit's bits made monotone above, the complement of the token below.

#include <algorithm>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int LP_WG = 256;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// (logit descending, token ascending) as one number, larger first; 0 is below every key.
__device__ __forceinline__ uint64_t alt_key(float logit, uint32_t token)
{
    uint32_t u = __float_as_uint(logit + 0.0f);  // (-0 and +0 are equal)
    if (logit != logit) u = 0x7fffffffu;
    u = (int32_t)u < 0 ? ~u : u | 0x80000000u;
    return (uint64_t)u << 32 | (uint32_t)~token;
}
__device__ __forceinline__ float alt_logit(uint64_t key)
{
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float((int32_t)u < 0 ? u & 0x7fffffffu : ~u);
}

template <typename V, typename F>
__device__ __forceinline__ V group_join(V v, V *lds, F f)
{
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) v = f(v, (V)__shfl_xor(v, s));
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < LP_WG / WAVE; ++w) v = f(v, lds[w]);
    return v;
}

// A workgroup per row.
template <typename T>
__global__ __launch_bounds__(LP_WG) void logprobs_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int V, float scale,
                                                         const int32_t *__restrict__ tokens, int nt, int k,
                                                         float *__restrict__ logp, float *__restrict__ lse_out,
                                                         float *__restrict__ entropy_out, uint32_t *__restrict__ top_idx,
                                                         float *__restrict__ top_logp)
{
    __shared__ float lds[LP_WG / WAVE];
    __shared__ uint64_t keys[LP_WG / WAVE];
    const auto add = [](float a, float b) { return a + b; };
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = logits + r * ld;
        float m = -INFINITY;
        for (int v = threadIdx.x; v < V; v += LP_WG) m = fmaxf(m, scale * (float)row[v]);
        m = group_join(m, lds, [](float a, float b) { return fmaxf(a, b); });
        const float m0 = m == -INFINITY ? 0.0f : m;
        float s = 0.0f, w = 0.0f;
        for (int v = threadIdx.x; v < V; v += LP_WG) {
            const float t = scale * (float)row[v] - m0;
            const float e = expf(t);
            s += e;
            if (e > 0.0f) w = fmaf(e, t, w);
        }
        s = group_join(s, lds, add);
        w = group_join(w, lds, add);
        const float lse = m0 + logf(s);
        if (threadIdx.x == 0) {
            if (lse_out) lse_out[r] = lse;
            if (entropy_out) entropy_out[r] = s == 0.0f ? 0.0f : logf(s) - w / s;
        }
        const auto log_prob = [&](float logit) { return s == 0.0f ? -INFINITY : scale * logit - lse; };
        for (int t = threadIdx.x; t < nt; t += LP_WG) {
            const int tok = tokens[r * nt + t];
            logp[r * nt + t] = tok >= 0 && tok < V ? log_prob((float)row[tok]) : 0.0f;
        }
        uint64_t last = ~0ull;
        for (int i = 0; i < k; ++i) {
            uint64_t best = 0;
            for (int v = threadIdx.x; v < V; v += LP_WG) {
                const uint64_t key = alt_key((float)row[v], (uint32_t)v);
                if (key < last && key > best) best = key;
            }
            best = group_join(best, keys, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
            if (threadIdx.x == 0) {
                top_idx[r * k + i] = best ? ~(uint32_t)best : 0xFFFFFFFFu;
                top_logp[r * k + i] = best ? log_prob(alt_logit(best)) : -INFINITY;
            }
            last = best;
        }
    }
}

// A workgroup per row: first every logit's own share, then the given tokens', each once.
template <typename T>
__global__ __launch_bounds__(LP_WG) void logprobs_grad_kernel(const T *logits, int64_t ld, int64_t rows, int V, float scale,
                                                              const int32_t *__restrict__ tokens, int nt,
                                                              const float *__restrict__ lse, const float *__restrict__ entropy,
                                                              const float *__restrict__ dlogp,
                                                              const float *__restrict__ dentropy, T *dlogits, int64_t ldd)
{
    __shared__ float lds[LP_WG / WAVE];
    __shared__ int tok[QADC_MAX_R];
    __shared__ float at[QADC_MAX_R], dl[QADC_MAX_R];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = logits + r * ld;
        T *out = dlogits + r * ldd;
        const float l = lse[r], dh = dentropy ? dentropy[r] : 0.0f, h = dentropy ? entropy[r] : 0.0f;
        const bool none = l == -INFINITY;
        float total = 0.0f;
        for (int t = threadIdx.x; t < nt; t += LP_WG) {
            const int v = tokens[r * nt + t];
            const bool used = v >= 0 && v < V;
            tok[t] = used ? v : -1;
            at[t] = used ? (float)row[v] : 0.0f;
            dl[t] = used ? dlogp[r * nt + t] : 0.0f;
            total += dl[t];
        }
        total = group_join(total, lds, [](float a, float b) { return a + b; });
        const auto share = [&](float logit) {
            const float lp = scale * logit - l, p = expf(lp);
            return p > 0.0f || p != p ? -p * fmaf(dh, lp + h, total) : 0.0f;
        };
        for (int v = threadIdx.x; v < V; v += LP_WG) out[v] = (T)(none ? 0.0f : scale * share((float)row[v]));
        __syncthreads();
        for (int t = threadIdx.x; t < nt; t += LP_WG) {
            if (tok[t] < 0 || none) continue;
            float own = 0.0f;
            bool first = true;
            for (int u = 0; u < nt; ++u)
                if (tok[u] == tok[t]) {
                    first = first && u >= t;
                    own += dl[u];
                }
            if (first) out[tok[t]] = (T)(scale * (own + share(at[t])));
        }
        __syncthreads();
    }
}

int check_logits(const char *who, int type, int64_t ld, int64_t rows, int V, float scale, const int32_t *tokens, int T)
{
    if (!type_ok(type)) return fail(QADC_EINVAL, "%s: unknown type %d", who, type);
    if (rows < 0 || V < 1 || ld < V) return fail(QADC_EINVAL, "%s: rows=%lld V=%d ld=%lld", who, (long long)rows, V, (long long)ld);
    if (!(scale > 0.0f) || scale == INFINITY) return fail(QADC_EINVAL, "%s: scale=%g", who, (double)scale);
    if (T < 0 || T > QADC_MAX_R) return fail(QADC_EINVAL, "%s: T=%d", who, T);
    if (T > 0 && rows > 0 && !tokens) return fail(QADC_EINVAL, "%s: null pointer", who);
    return QADC_OK;
}

}  // namespace

size_t token_logprobs_workspace(int64_t rows, int V, int k)
{
    if (rows < 1 || V < 1 || k < 0 || k > QADC_MAX_ALTERNATIVES) return 0;
    return 256;
}

int token_logprobs(const void *logits, int64_t ld, int type, int64_t rows, int V, float scale, const int32_t *tokens, int T,
                   int k, float *logp, float *lse, float *entropy, uint32_t *top_idx, float *top_logp, void *workspace,
                   size_t workspace_bytes, hipStream_t st)
{
    if (const int rc = check_logits("qadc_token_logprobs", type, ld, rows, V, scale, tokens, T)) return rc;
    if (k < 0 || k > QADC_MAX_ALTERNATIVES) return fail(QADC_EINVAL, "qadc_token_logprobs: k=%d", k);
    if (rows == 0) return QADC_OK;
    if (!logits || (T > 0 && !logp) || (k > 0 && (!top_idx || !top_logp)))
        return fail(QADC_EINVAL, "qadc_token_logprobs: null pointer");
    const size_t need = token_logprobs_workspace(rows, V, k);
    if (!workspace || workspace_bytes < need)
        return fail(QADC_ENOMEM, "qadc_token_logprobs: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 20));
    const int nt = T;
    QADC_BY_TYPE(type, (launch(QADC_PROF_LOGPROBS, logprobs_kernel<T>, grid, dim3(LP_WG), 0, st, (const T *)logits, ld, rows, V,
                               scale, tokens, nt, k, logp, lse, entropy, top_idx, top_logp)));
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

int token_logprobs_backward(const void *logits, int64_t ld, int type, int64_t rows, int V, float scale, const int32_t *tokens,
                            int T, const float *lse, const float *entropy, const float *dlogp, const float *dentropy,
                            void *dlogits, int64_t ldd, hipStream_t st)
{
    if (const int rc = check_logits("qadc_token_logprobs_backward", type, ld, rows, V, scale, tokens, T)) return rc;
    if (ldd < V) return fail(QADC_EINVAL, "qadc_token_logprobs_backward: ldd=%lld", (long long)ldd);
    if (rows == 0) return QADC_OK;
    if (!logits || !lse || !dlogits || (T > 0 && !dlogp) || (dentropy && !entropy))
        return fail(QADC_EINVAL, "qadc_token_logprobs_backward: null pointer");
    if (logits == dlogits && ld != ldd)
        return fail(QADC_EINVAL, "qadc_token_logprobs_backward: in place needs equal row distances");
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 20));
    const int nt = T;
    QADC_BY_TYPE(type, (launch(QADC_PROF_LOGPROBS, logprobs_grad_kernel<T>, grid, dim3(LP_WG), 0, st, (const T *)logits, ld, rows,
                               V, scale, tokens, nt, lse, entropy, dlogp, dentropy, (T *)dlogits, ldd)));
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
