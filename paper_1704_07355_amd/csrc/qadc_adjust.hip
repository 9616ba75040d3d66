// Penalties for repeated tokens, biases and grammar masks on logits, on gfx950.
//
// A workgroup takes a stretch of a row's tokens, with a counter each in LDS: it goes over the row's history once and counts what falls
// into the stretch, then the stretch streams by with its counters.  Tokens with biases are few: their counters are marked, and their
// places in the list of the stretch's biases lie beside.  In a pack of tokens those with a counter are taken one by one, which is
// a loop of one or two turns: all eight of a pack in line took 60 us where this takes 48.
//
// Bound by memory where histories are short (256 x 128001 binary16 28 us with a history of one token, 131 MB at 4.7 TB/s); every
// stretch reads the history again, from the L2 of the XCD that the row's stretches share (4099 tokens: 43 us; from all L2s in turn
// 52), and a mask, 32 biases a row and what they change take 5 us more.
#include <algorithm>
#include <type_traits>

#include "qadc_lm.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

// A counter: how often a token was said behind the prompt, and the marks of a token in the prompt, of one with a bias, and of one with
// several.
constexpr unsigned ADJ_PROMPT = 1u << 31, ADJ_BIASED = 1u << 30, ADJ_TWICE = 1u << 29, ADJ_SAID = ADJ_TWICE - 1;
static_assert(QADC_MAX_HISTORY <= (int)ADJ_SAID && QADC_MAX_R <= 1 << 16, "a history's length fits a counter, a bias's place 16 bits");

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

typedef int32_t Tokens4 __attribute__((ext_vector_type(4), aligned(4)));

// A pack without the tokens whose bit in `ok` is 0: two elements of 16 bits in four instructions, where a test of each took twenty-five.
template <typename T>
__device__ __forceinline__ typename Pack<T>::V masked(typename Pack<T>::V v, unsigned ok)
{
    typedef unsigned Words __attribute__((ext_vector_type(4)));
    Words w = __builtin_bit_cast(Words, v);
    const auto bit = [&](int e) { return (unsigned)((int)(ok << (31 - e)) >> 31); };  // all ones where it is set
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned keep, low;
        if constexpr (sizeof(T) == 2) {
            keep = (bit(2 * i) & 0xffffu) | (bit(2 * i + 1) & ~0xffffu);
            low = __builtin_bit_cast(unsigned short, (T)-INFINITY) * 0x10001u;
        } else {
            keep = bit(i);
            low = __float_as_uint(-INFINITY);
        }
        w[i] = (w[i] & keep) | (low & ~keep);
    }
    return __builtin_bit_cast(typename Pack<T>::V, w);
}

// Element e of a pack, which differs between the lanes.
typedef unsigned PackWords __attribute__((ext_vector_type(4)));
__device__ __forceinline__ float get(Pack<float>::V v, int e) { return e & 2 ? e & 1 ? v[3] : v[2] : e & 1 ? v[1] : v[0]; }
__device__ __forceinline__ void set(Pack<float>::V &v, int e, float x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = e == i ? x : v[i];
}
template <typename V>
__device__ __forceinline__ float get(V v, int e)
{
    const PackWords w = __builtin_bit_cast(PackWords, v);
    const unsigned two = e & 4 ? e & 2 ? w[3] : w[2] : e & 2 ? w[1] : w[0];
    return (float)__builtin_bit_cast(std::remove_reference_t<decltype(v[0])>, (unsigned short)(e & 1 ? two >> 16 : two));
}
template <typename V>
__device__ __forceinline__ void set(V &v, int e, float x)
{
    PackWords w = __builtin_bit_cast(PackWords, v);
    const unsigned short bits = __builtin_bit_cast(unsigned short, (std::remove_reference_t<decltype(v[0])>)x);
    const unsigned keep = e & 1 ? 0xffffu : 0xffff0000u, put = (unsigned)bits << (e & 1 ? 16 : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = e / 2 == i ? (w[i] & keep) | put : w[i];
    v = __builtin_bit_cast(V, w);
}

struct Bias {
    int at;  // in the stretch
    float by;
};

template <typename T, int SPAN, int WG>
__global__ __launch_bounds__(WG) void adjust_kernel(const T *logits, int64_t ld, int64_t rows, int V, int stretches, Rules q, T *out,
                                                    int64_t ldo)
{
    constexpr int N = Pack<T>::N, PACKS = SPAN / WG / N;
    typedef typename Pack<T>::V P;
    __shared__ __attribute__((aligned(16))) uint32_t counts[SPAN];
    __shared__ int biases;
    extern __shared__ __attribute__((aligned(16))) Bias biased[];  // up to B, then, where there are any,
    uint16_t *place = (uint16_t *)(biased + q.B);                  // [SPAN] of a biased token in that list
    const bool here = logits == out;
    const int tid = threadIdx.x;
    // Workgroups go round the eight XCDs in turn: those of one of them take stretches that follow each other, and find the row's history in
    // their L2.
    const int64_t units = rows * stretches, share = (units + 7) / 8;
    for (int64_t k = blockIdx.x; k < share * 8; k += gridDim.x) {
        const int64_t i = k % 8 * share + k / 8;
        if (i >= units) continue;
        const int64_t r = i / stretches;
        const int v0 = (int)(i % stretches) * SPAN, span = min(SPAN, V - v0);
        const T *row = logits + r * ld + v0;
        T *to = out + r * ldo + v0;
        // the stretch and the beginning of the history first, then what takes several steps to reach
        P p[PACKS];
        if (!here) {
#pragma unroll
            for (int u = 0; u < PACKS; ++u) {
                const int c = (u * WG + tid) * N;
                if (c + N <= span) p[u] = __builtin_nontemporal_load(reinterpret_cast<const P *>(row + c));
            }
        }
        const int32_t *history = q.history + r * q.H;
        const uint32_t *mask = nullptr;
        if (q.masks) {
            const int64_t state = q.mask_of ? q.mask_of[r] : r;
            if (state >= 0 && state < q.states) mask = q.masks + state * q.mask_ld + v0 / 32;
        }
        unsigned allowed[PACKS];  // the pack's tokens that the mask allows
#pragma unroll
        for (int u = 0; u < PACKS; ++u) {
            const int c = (u * WG + tid) * N;
            allowed[u] = ~0u;
            if (mask && c < span) allowed[u] = mask[c / 32];
        }
        const int length = q.H > 0 ? q.lengths ? min(max(q.lengths[r], 0), q.H) : q.H : 0;
        const int prompt = q.prompt && q.H > 0 ? q.prompt[r] : 0;
        const float rep = q.repetition && q.H > 0 ? q.repetition[r] : 1.0f;
        const float pres = q.presence && q.H > 0 ? q.presence[r] : 0.0f, freq = q.frequency && q.H > 0 ? q.frequency[r] : 0.0f;
        if (q.B > 0 && tid < WAVE) {
            int n = 0;
            for (int j = tid; j - tid < q.B; j += WAVE) {
                const int t = j < q.B ? q.bias_tokens[r * q.B + j] : -1;
                const float by = j < q.B ? q.bias[r * q.B + j] : 0.0f;
                const bool in = t >= v0 && t < v0 + span;
                const unsigned long long m = __ballot(in);
                if (in) biased[n + (int)rank_in_mask(m)] = {t - v0, by};
                n += __popcll(m);
            }
            if (tid == 0) biases = n;
        }
        for (int w = tid; w < SPAN / 4; w += WG) reinterpret_cast<uint4 *>(counts)[w] = uint4{0, 0, 0, 0};
        __syncthreads();
        const int marked = q.B > 0 ? biases : 0;
        for (int j = tid; j < marked; j += WG) {
            atomicOr(&counts[biased[j].at], ADJ_BIASED);
            place[biased[j].at] = (uint16_t)j;
        }
        // (a negative token is beyond the stretch as an unsigned number too)
        const auto see = [&](int token) {
            const unsigned c = (unsigned)token - (unsigned)v0;
            if (c < (unsigned)span) atomicOr(&counts[c], ADJ_PROMPT);
        };
        const auto say = [&](int token) {
            const unsigned c = (unsigned)token - (unsigned)v0;
            if (c < (unsigned)span) atomicAdd(&counts[c], 1u);
        };
        const auto four = [&](const Tokens4 &t, int j) {
            if (j >= prompt) {
#pragma unroll
                for (int e = 0; e < 4; ++e) say(t[e]);
            } else if (j + 4 <= prompt) {
#pragma unroll
                for (int e = 0; e < 4; ++e) see(t[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (j + e < prompt) see(t[e]);
                    else say(t[e]);
                }
            }
        };
#pragma unroll 2
        for (int j = tid * 4; j + 4 <= length; j += WG * 4) four(*reinterpret_cast<const Tokens4 *>(history + j), j);
        if (tid < length % 4) {
            const int j = length - 1 - tid;
            if (j < prompt) see(history[j]);
            else say(history[j]);
        }
        __syncthreads();
        if (marked > 0) {  // (the same in all threads)
            for (int j = tid; j < marked; j += WG)
                if (place[biased[j].at] != j) atomicOr(&counts[biased[j].at], ADJ_TWICE);
            __syncthreads();
        }
        const float inverse = 1.0f / rep;
        // (the quotient as the product with the inverse and what that leaves: the row's penalty is the same for all)
        const auto adjusted = [&](float x, unsigned n) {
            const unsigned said = n & ADJ_SAID;
            const float q0 = x * inverse, q1 = fmaf(fmaf(-q0, rep, x), inverse, q0);
            const float quotient = fabsf(q1) < INFINITY ? q1 : q0;
            x = !(n & ~(ADJ_BIASED | ADJ_TWICE)) ? x : x > 0.0f ? quotient : x * rep;
            return said ? x - fmaf(freq, (float)said, pres) : x;
        };
        const auto bias_of = [&](int c, bool twice) {
            float s = biased[place[c]].by;
            if (twice) {  // its biases in their order
                bool some = false;
                for (int j = 0; j < marked; ++j)
                    if (biased[j].at == c) {
                        s = some ? s + biased[j].by : biased[j].by;
                        some = true;
                    }
            }
            return s;
        };
        const auto value = [&](float x, unsigned n, int c) {
            x = adjusted(x, n);
            return n & ADJ_BIASED ? x + bias_of(c, n & ADJ_TWICE) : x;
        };
        const auto pack = [&](auto whole, int u) {
            constexpr bool WHOLE = decltype(whole)::value;  // the stretch is a whole one
            const int c = (u * WG + tid) * N;
            if (!WHOLE && c >= span) return;
            uint32_t n[N], any = 0;
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const uint4 four = *reinterpret_cast<const uint4 *>(&counts[c + e]);
                n[e] = four.x, n[e + 1] = four.y, n[e + 2] = four.z, n[e + 3] = four.w;
                any |= four.x | four.y | four.z | four.w;
            }
            const unsigned all = (1u << N) - 1, ok = allowed[u] >> (c % 32) & all;
            if (WHOLE || c + N <= span) {
                P v = p[u];
                if (here) {
                    if (!any && (!mask || ok == all)) return;
                    v = *reinterpret_cast<const P *>(row + c);
                }
                if (any) {  // token by token: in a pack they are few
                    unsigned left = 0;
#pragma unroll
                    for (int e = 0; e < N; ++e) left |= min(n[e], 1u) << e;
                    for (; left; left &= left - 1) {
                        const int e = __builtin_ctz(left);
                        set(v, e, value(get(v, e), counts[c + e], c + e));
                    }
                }
                if (mask) v = masked<T>(v, ok);
                if (here) *reinterpret_cast<P *>(to + c) = v;
                else __builtin_nontemporal_store(v, reinterpret_cast<P *>(to + c));
            } else {
#pragma unroll 1
                for (int e = 0; c + e < span; ++e) {
                    T v = row[c + e];
                    if (counts[c + e]) v = (T)value((float)v, counts[c + e], c + e);
                    if (mask && !(ok >> e & 1)) v = (T)-INFINITY;
                    to[c + e] = v;
                }
            }
        };
        if (span == SPAN) {
#pragma unroll
            for (int u = 0; u < PACKS; ++u) pack(std::true_type(), u);
        } else {
#pragma unroll
            for (int u = 0; u < PACKS; ++u) pack(std::false_type(), u);
        }
        __syncthreads();  // (the counters are used again)
    }
}

template <typename T, int SPAN, int WG>
void adjust_launch(const void *logits, int64_t ld, int64_t rows, int V, const Rules &q, void *out, int64_t ldo, hipStream_t st)
{
    const int stretches = (int)ceil_div(V, SPAN);
    launch(QADC_PROF_ADJUST, adjust_kernel<T, SPAN, WG>, dim3((unsigned)std::min<int64_t>(ceil_div(rows * stretches, 8) * 8, 1 << 22)), dim3(WG),
           q.B > 0 ? (size_t)q.B * sizeof(Bias) + SPAN * sizeof(uint16_t) : 0, st, (const T *)logits, ld, rows, V, stretches, q, (T *)out, ldo);
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
    // Every stretch goes over the row's whole history: of long ones longer stretches with more threads (256 x 131072 bfloat16 with a history of
    // 32768 73 us for 95, one row 10.2 for 12.5), of short ones shorter, of which a compute unit holds more (1024 x 32768 with 1000 42
    // for 45, 845 x 25461 with 934 32 for 39).
    QADC_BY_TYPE(type, {
        if (H >= 4096) adjust_launch<T, 8192, 512>(logits, ld, rows, V, q, out, ldo, st);
        else adjust_launch<T, 4096, 256>(logits, ld, rows, V, q, out, ldo, st);
    });
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
