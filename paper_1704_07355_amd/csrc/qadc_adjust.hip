// Penalties for repeated tokens, biases and grammar masks on logits, on gfx950.
//
// A workgroup takes a stretch of a row's tokens.  It goes over the row's history twice: first every token that falls into the
// stretch marks its bit and clears its counter, then it is counted; so the counters need not be cleared as a whole.  Biases go the
// same way.  Then the stretch streams by, and only marked tokens look at their counter.  Tokens of a pack that a mask
// forbids altogether are not read.
#include <algorithm>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int ADJ_WG = 256;
constexpr unsigned ADJ_PROMPT = 1u << 31;   // a counter's mark of a token in the prompt; below, how often it was said since

struct Rules {
    const int32_t *history, *lengths, *prompt;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_tokens;
    const float *bias;
    const uint32_t *masks;
    const int32_t *mask_of;
    int64_t mask_ld;
    int H, B, states;
};

// The four 32-bit numbers from p on, as many of them as there are; -1 behind.
typedef int32_t Tokens4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ Tokens4 tokens4(const int32_t *p, int i, int n)
{
    if (i + 4 <= n) return *reinterpret_cast<const Tokens4 *>(p + i);
    Tokens4 t = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < n) t[e] = p[i + e];
    return t;
}

// PACKS packs of each thread: the stretch is ADJ_WG * PACKS * N tokens.
template <typename T, int PACKS>
__global__ __launch_bounds__(ADJ_WG) void adjust_kernel(const T *logits, int64_t ld, int64_t rows, int V, int stretches, Rules q, T *out,
                                                        int64_t ldo)
{
    constexpr int N = Pack<T>::N, SPAN = ADJ_WG * PACKS * N;
    typedef typename Pack<T>::V P;
    __shared__ uint32_t marks[SPAN / 32], twice[SPAN / 32];
    __shared__ uint32_t any_twice;
    extern __shared__ uint32_t counts[];                    // [SPAN] where there is a history, then
    float *sums = (float *)(counts + (q.H > 0 ? SPAN : 0));  // [SPAN] where there are biases
    const bool here = logits == out;
    for (int64_t i = blockIdx.x; i < rows * stretches; i += gridDim.x) {
        const int64_t r = i / stretches;
        const int v0 = (int)(i % stretches) * SPAN, span = min(SPAN, V - v0);
        const T *row = logits + r * ld + v0;
        T *to = out + r * ldo + v0;
        // the pack's tokens that the mask allows
        const uint32_t *mask = nullptr;
        if (q.masks) {
            const int64_t state = q.mask_of ? q.mask_of[r] : r;
            if (state >= 0 && state < q.states) mask = q.masks + state * q.mask_ld + v0 / 32;
        }
        unsigned allowed[PACKS];
#pragma unroll
        for (int u = 0; u < PACKS; ++u) {
            const int c = (u * ADJ_WG + threadIdx.x) * N;
            allowed[u] = (1u << N) - 1;
            if (mask && c < span) allowed[u] &= mask[c / 32] >> (c % 32);
        }
        P p[PACKS];
        if (!here) {
#pragma unroll
            for (int u = 0; u < PACKS; ++u) {
                const int c = (u * ADJ_WG + threadIdx.x) * N;
                if (c + N <= span && allowed[u]) p[u] = *reinterpret_cast<const P *>(row + c);
            }
        }
        for (int w = threadIdx.x; w < SPAN / 32; w += ADJ_WG) marks[w] = twice[w] = 0;
        if (threadIdx.x == 0) any_twice = 0;
        const int length = q.H > 0 ? q.lengths ? min(max(q.lengths[r], 0), q.H) : q.H : 0;
        const int prompt = q.prompt && q.H > 0 ? q.prompt[r] : 0;
        const int32_t *history = q.history + r * q.H;
        __syncthreads();
        for (int j = threadIdx.x * 4; j < length; j += ADJ_WG * 4) {
            const Tokens4 t = tokens4(history, j, length);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned c = (unsigned)t[e] - (unsigned)v0;
                if (c >= (unsigned)span || t[e] < 0) continue;
                counts[c] = 0;
                if (q.B > 0) sums[c] = 0.0f;
                atomicOr(&marks[c / 32], 1u << (c % 32));
            }
        }
        for (int j = threadIdx.x; j < q.B; j += ADJ_WG) {
            const int t = q.bias_tokens[r * q.B + j];
            const unsigned c = (unsigned)t - (unsigned)v0;
            if (c >= (unsigned)span || t < 0) continue;
            if (q.H > 0) counts[c] = 0;
            sums[c] = 0.0f;
            atomicOr(&marks[c / 32], 1u << (c % 32));
            if (atomicOr(&twice[c / 32], 1u << (c % 32)) >> (c % 32) & 1) any_twice = 1;
        }
        __syncthreads();
        for (int j = threadIdx.x * 4; j < length; j += ADJ_WG * 4) {
            const Tokens4 t = tokens4(history, j, length);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned c = (unsigned)t[e] - (unsigned)v0;
                if (c >= (unsigned)span || t[e] < 0) continue;
                if (j + e < prompt) atomicOr(&counts[c], ADJ_PROMPT);
                else atomicAdd(&counts[c], 1u);
            }
        }
        for (int j = threadIdx.x; j < q.B; j += ADJ_WG) {
            const int32_t *tokens = q.bias_tokens + r * q.B;
            const float *bias = q.bias + r * q.B;
            const int t = tokens[j];
            const unsigned c = (unsigned)t - (unsigned)v0;
            if (c >= (unsigned)span || t < 0) continue;
            float s = bias[j];
            if (any_twice) {  // a token's biases are added in their order, by its first one
                bool first = true;
                for (int k = 0; k < j; ++k) first = first && tokens[k] != t;
                if (!first) continue;
                for (int k = j + 1; k < q.B; ++k)
                    if (tokens[k] == t) s += bias[k];
            }
            sums[c] = s;
        }
        __syncthreads();
        const float rep = q.repetition && q.H > 0 ? q.repetition[r] : 1.0f;
        const float pres = q.presence && q.H > 0 ? q.presence[r] : 0.0f, freq = q.frequency && q.H > 0 ? q.frequency[r] : 0.0f;
        const auto adjusted = [&](float x, int c) {
            const unsigned n = q.H > 0 ? counts[c] : 0u, said = n & ~ADJ_PROMPT;
            if (n) x = x > 0.0f ? x / rep : x * rep;
            if (said) x -= freq * (float)said + pres;
            return q.B > 0 ? x + sums[c] : x;
        };
#pragma unroll
        for (int u = 0; u < PACKS; ++u) {
            const int c = (u * ADJ_WG + threadIdx.x) * N;
            if (c >= span) continue;
            const unsigned all = (1u << N) - 1, ok = allowed[u] & all;
            const unsigned marked = marks[c / 32] >> (c % 32) & ok;
            if (here && !marked && ok == all) continue;
            if (c + N <= span) {
                P v = p[u];
                if (here && ok) v = *reinterpret_cast<const P *>(row + c);
                if (marked || ok != all) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        if (marked >> e & 1) v[e] = (T)adjusted((float)v[e], c + e);
                        if (!(ok >> e & 1)) v[e] = (T)-INFINITY;
                    }
                }
                *reinterpret_cast<P *>(to + c) = v;
            } else {
#pragma unroll 1
                for (int e = 0; c + e < span; ++e) {
                    T v = row[c + e];
                    if (marked >> e & 1) v = (T)adjusted((float)v, c + e);
                    if (!(ok >> e & 1)) v = (T)-INFINITY;
                    to[c + e] = v;
                }
            }
        }
        __syncthreads();  // the counters are used again
    }
}

template <typename T, int PACKS>
void adjust_launch(const void *logits, int64_t ld, int64_t rows, int V, const Rules &q, void *out, int64_t ldo, hipStream_t st)
{
    constexpr int SPAN = ADJ_WG * PACKS * Pack<T>::N;
    const int stretches = (int)ceil_div(V, SPAN);
    const size_t lds = (size_t)SPAN * sizeof(uint32_t) * ((q.H > 0) + (q.B > 0));
    launch(QADC_PROF_ADJUST, adjust_kernel<T, PACKS>, dim3((unsigned)std::min<int64_t>(rows * stretches, 1 << 22)), dim3(ADJ_WG), lds, st,
           (const T *)logits, ld, rows, V, stretches, q, (T *)out, ldo);
}

}  // namespace

int adjust_logits(const void *logits, int64_t ld, int type, int64_t rows, int V, const int32_t *history, int H, const int32_t *lengths,
                  const int32_t *prompt, const float *repetition, const float *presence, const float *frequency,
                  const int32_t *bias_tokens, const float *bias, int B, const uint32_t *masks, int64_t mask_ld, int states,
                  const int32_t *mask_of, void *out, int64_t ldo, hipStream_t st)
{
    const char *who = "qadc_adjust_logits";
    if (!type_ok(type)) return fail(QADC_EINVAL, "%s: unknown type %d", who, type);
    // (tokens are counted in an int, a stretch past the last one)
    if (rows < 0 || V < 1 || V > INT32_MAX - 65536 || ld < V || ldo < V)
        return fail(QADC_EINVAL, "%s: rows=%lld V=%d ld=%lld ldo=%lld", who, (long long)rows, V, (long long)ld, (long long)ldo);
    if (H < 0 || H > QADC_MAX_HISTORY || B < 0 || B > QADC_MAX_R) return fail(QADC_EINVAL, "%s: H=%d B=%d", who, H, B);
    if (rows == 0) return QADC_OK;
    if (!logits || !out || (H > 0 && !history) || (B > 0 && (!bias_tokens || !bias)))
        return fail(QADC_EINVAL, "%s: null pointer", who);
    if (masks && (states < 1 || mask_ld < ceil_div(V, 32) || (!mask_of && states < rows)))
        return fail(QADC_EINVAL, "%s: %d masks of %lld words for %lld rows of %d tokens", who, states, (long long)mask_ld,
                    (long long)rows, V);
    if (logits == out && ld != ldo) return fail(QADC_EINVAL, "%s: in place needs equal row distances", who);
    const Rules q = {history, lengths, prompt, repetition, presence, frequency, bias_tokens, bias, masks, mask_of, mask_ld, H, B, states};
    QADC_BY_TYPE(type, (adjust_launch<T, 1>(logits, ld, rows, V, q, out, ldo, st)));
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
