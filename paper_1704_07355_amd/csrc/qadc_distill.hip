// Distillation from a teacher's likeliest tokens: the loss of every row, its gradient, and both in one call, on gfx950.
//
// With x = scale logits, m = max x, e = exp(x - m) over the row, own = sum of e over the stored tokens and others = sum over all
// others: log q_t = x_t - m - log(own + others), and the student's probability of everything that was not stored is
// Q = others / (own + others), log Q = -log(1 + own / others).  The stored tokens are left out of the running sum by a bit each in
// LDS, so that neither others nor log Q is a difference of nearly equal numbers.  What is computed once a row, the teacher's
// probabilities and the loss itself (a difference of logarithms that are nearly equal), is held in 64 bits.
//
// Gradient: with T the teacher's whole probability and r what it has outside the stored tokens,
// dx_v = scale w ((T - r / Q [v not stored]) q_v - p_v [v stored]): every token but the stored ones gets one factor times q_v.
//
// Bound by memory in large calls: 4096 x 65536 bfloat16, loss and gradient in one call, 228 us, 4.7 TB/s read and written (the row lies
// in registers between them, so that a compute unit loads or stores at a time, not both); 512 x 128001 74 us, two
// rounds of one workgroup a compute unit; the gradient alone, 1111 x 32003 float32, 57 us, 5.0 TB/s, in calls one after the other that share their
// output, 70 us, 4.1 TB/s, with a new one in every call.  Small calls are bound by the host and the launches: 48 x 50021 binary16, loss alone,
// 14 us, parts 5.2 and join 6.4.  Tails below 2^-80 of every row are summed twice: 4096 x 65536 261 us in one call, and in two as others.
#include <algorithm>

#include "qadc_logits.h"
#include "qadc_profile.h"

namespace qadc {

namespace {

constexpr int DS_MARKED = 16;  // chunks whose stored tokens are marked at a time: 131072 tokens, 16 KB of LDS
constexpr int DS_WAVES = QADC_MAX_ALTERNATIVES / WAVE;  // wavefronts with stored tokens, one a thread
static_assert(QADC_MAX_ALTERNATIVES % WAVE == 0 && QADC_MAX_ALTERNATIVES <= LP_WG, "a thread per stored token");

struct Teacher {
    const uint32_t *idx;  // [rows][k]
    const float *logp;    // [rows][k]
    int k;
    bool tail;
};

// A part of a row without its stored tokens: the largest logit and the sum of 2^(c (logit - m)).
struct Part2 {
    float m, s;
};
__device__ __forceinline__ void raise(Part2 &a, float to, float c)
{
    a.s *= exp2_fast(shift_of(a.m, to, c));
    a.m = to;
}
__device__ __forceinline__ Part2 join(Part2 a, Part2 b, float c)
{
    const float m = fmaxf(a.m, b.m);
    raise(a, m, c);
    raise(b, m, c);
    return {m, a.s + b.s};
}
__device__ __forceinline__ void add_block(Part2 &a, const float (&x)[LP_BLOCK], float c)
{
    float v = x[0];
#pragma unroll
    for (int e = 1; e < LP_BLOCK; ++e) v = fmaxf(v, x[e]);
    const float m = fmaxf(a.m, v), m0 = m == -INFINITY ? 0.0f : m;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < LP_BLOCK; ++i) s[i & 1] += exp2_fast(c * (x[i] - m0));
    raise(a, m, c);
    a.s += s[0] + s[1];
}

// A stored token as it is in the row.
struct Stored {
    int token;   // -1: none
    float logit, logp;
};
template <typename T>
__device__ __forceinline__ Stored stored_of(const T *row, int64_t r, int V, const Teacher &t, int at)
{
    Stored s = {-1, -INFINITY, -INFINITY};
    if (at < t.k) {
        const uint32_t i = t.idx[r * t.k + at];
        const float logp = t.logp[r * t.k + at];
        if (i < (uint32_t)V) {
            s.token = (int)i;
            s.logit = (float)row[i];
            s.logp = logp;
        }
    }
    return s;
}

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// The share of this thread's stored token in the row's loss; m: the row's largest logit, log_s: the logarithm of its sum.
__device__ __forceinline__ double loss_of(const Stored &st, double p, double P, bool tail, bool none, float scale, float m, double log_s)
{
    if (!(p > 0.0) && p == p) return 0.0;
    const double log_q = none ? -INFINITY : (double)scale * ((double)st.logit - (double)m) - log_s;
    return tail ? p * ((double)st.logp - log_q) : p / P * ((double)st.logp - log(P) - log_q);
}

// Whether none of the tokens before number `at` is `token`.
__device__ __forceinline__ bool first_of(const int *tokens, int token, int k, int at)
{
    bool first = true;
    for (int i = 0; i < k; i += 4) {
        const int4 v = *reinterpret_cast<const int4 *>(&tokens[i]);
        const int before = at - i;
        first = first && !((v.x == token && before > 0) || (v.y == token && before > 1) || (v.z == token && before > 2) ||
                           (v.w == token && before > 3));
    }
    return first;
}

// Of the teacher's probabilities p of a row: their sum, and with the tail what is left.
struct Mass {
    double P, rest;
};
__device__ __forceinline__ Mass mass_of(double P, bool tail) { return {P, tail && P < 1.0 ? 1.0 - P : 0.0}; }
// The gradient's factors, where log Q is `log_tail`: T, the teacher's whole probability; and of a token that was not stored, with
// T q - r q / Q = (T Q - r) q / Q, the factor of q / Q, which does not grow where Q is small, and log Q (1, and 0, without a tail).
struct Factors {
    float total, other, log_tail;
};
__device__ __forceinline__ Factors factors(const Mass &a, bool tail, double log_tail)
{
    const double rest = log_tail == -INFINITY ? 0.0 : a.rest;  // (nothing is left to the student there)
    const double T = tail ? a.P + rest : a.P > 0.0 ? 1.0 : 0.0;
    if (rest == 0.0) return {(float)T, (float)T, 0.0f};
    return {(float)T, (float)(T * exp(log_tail) - rest), (float)log_tail};
}
constexpr double DS_NOTHING = 1e-37;  // what the other tokens have, of what the stored ones have, that counts as nothing
// Below this they are taken in 64 bits: as float32 they run out of the exponent.  (Above it, of a row of 2^17 exponentials each of which is there
// down to 2^-126, no more than 2^-29 of the sum is missing.)
constexpr float DS_DEEP = 0x1p-80f;

struct Loss {
    float *loss, *lse, *log_tail;  // lse and log_tail nullable
};

// The stored tokens of a wavefront's row, a few a lane.
struct WaveStored {
    Stored at[DS_WAVES];
};
template <typename T>
__device__ __forceinline__ WaveStored wave_stored(const T *row, int64_t r, int V, const Teacher &t)
{
    WaveStored s;
#pragma unroll
    for (int i = 0; i < DS_WAVES; ++i) s.at[i] = stored_of(row, r, V, t, i * WAVE + lane_id());
    return s;
}

// The row's loss from what its other tokens have, by one wavefront.  tokens: a place for the row's stored tokens.
__device__ __forceinline__ void finish_row(Part2 others, const WaveStored &st, int64_t r, float scale, const Teacher &t, const Loss &o,
                                           int *tokens)
{
    const float c = scale * LOG2E;
    double p[DS_WAVES], P = 0.0;
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < DS_WAVES; ++i) {
        tokens[i * WAVE + lane_id()] = st.at[i].token;
        p[i] = st.at[i].token < 0 ? 0.0 : exp((double)st.at[i].logp);
        P += p[i];
        most = fmaxf(most, st.at[i].logit);
    }
    __builtin_amdgcn_wave_barrier();
    const Mass mass = mass_of(wave_sum64(P), t.tail);
    const float m = fmaxf(others.m, wave_max(most)), m0 = m == -INFINITY ? 0.0f : m;
    float own = 0.0f;
#pragma unroll
    for (int i = 0; i < DS_WAVES; ++i) {  // a token that is stored twice counts once for the student
        const bool first = st.at[i].token >= 0 && first_of(tokens, st.at[i].token, t.k, i * WAVE + lane_id());
        own += first ? exp2_fast(c * (st.at[i].logit - m0)) : 0.0f;
    }
    own = wave_sum(own);
    double rest = others.s * exp2_fast(shift_of(others.m, m, c));
    if (rest < (double)own * DS_DEEP) rest = (double)others.s * exp((double)scale * ((double)others.m - (double)m));
    const bool none = m == -INFINITY && (double)own + rest == 0.0;  // (NaN where there is one among the masked)
    if (rest < (double)own * DS_NOTHING) rest = 0.0;
    const double log_s = log((double)own + rest);
    const double log_tail = rest == 0.0 ? -INFINITY : -log1p((double)own / rest);
    double l = 0.0;
#pragma unroll
    for (int i = 0; i < DS_WAVES; ++i) l += loss_of(st.at[i], p[i], mass.P, t.tail, none, scale, m, log_s);
    l = wave_sum64(l);
    if (lane_id() == 0) {
        if (mass.rest > 0.0 && log_tail != -INFINITY) l += mass.rest * (log(mass.rest) - log_tail);
        o.loss[r] = log_s == log_s ? (float)l : NAN;  // (a broken row is one to an empty teacher too)
        if (o.lse) {
            const float lse = (float)((double)scale * (double)m + log_s);  // (no float holds it: NaN)
            o.lse[r] = none ? -INFINITY : fabsf(lse) < INFINITY ? lse : NAN;
        }
        if (o.log_tail) o.log_tail[r] = (float)log_tail;
    }
}

// The stored token of this thread, -1: none.
__device__ __forceinline__ int token_of(int64_t r, int V, const Teacher &t)
{
    const uint32_t v = (int)threadIdx.x < t.k ? t.idx[r * t.k + threadIdx.x] : ~0u;
    return v < (uint32_t)V ? (int)v : -1;
}

// Marks the stored token if it lies in chunks j0 .. j1 - 1 of the row, whose first token is at `lead`; a barrier before and behind.
__device__ __forceinline__ void mark(uint32_t *marks, int token, int64_t j0, int64_t j1, int lead, int threads)
{
    __syncthreads();
    for (int64_t w = threadIdx.x; w < (j1 - j0) * (LP_CHUNK / 32); w += threads) marks[w] = 0;
    __syncthreads();
    const int64_t at = (int64_t)token + lead - j0 * LP_CHUNK;
    if (token >= 0 && at >= 0 && at < (j1 - j0) * LP_CHUNK) atomicOr(&marks[at / 32], 1u << (at % 32));
    __syncthreads();
}
// The marks of the N tokens from position `at` on, a multiple of N.
template <int N>
__device__ __forceinline__ unsigned marks_at(const uint32_t *marks, int at)
{
    const unsigned b = reinterpret_cast<const uint8_t *>(marks)[at / 8];
    return N == 8 ? b : b >> (at % 8) & 15u;
}

// What chunks j0 .. j1 - 1 of a row have, joined over the workgroup.
template <typename T>
__device__ __forceinline__ Part2 chunks_part(const T *row, int64_t j0, int64_t j1, int V, int lead, float c, int token,
                                             uint32_t *marks, Part2 *waves)
{
    constexpr int N = Pack<T>::N;
    Part2 a = {-INFINITY, 0.0f};
    for (int64_t j = j0; j < j1; ++j) {
        const int at = (int)((j - j0) % DS_MARKED);
        float x[LP_BLOCK];
        load_block(row, j, V, lead, x);
        if (at == 0) mark(marks, token, j, min(j + DS_MARKED, j1), lead, LP_WG);
#pragma unroll
        for (int u = 0; u < LP_BLOCK / N; ++u) {
            const unsigned b = marks_at<N>(marks, at * LP_CHUNK + (u * LP_WG + (int)threadIdx.x) * N);
            if (b)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (b >> e & 1) x[u * N + e] = -INFINITY;
        }
        add_block(a, x, c);
    }
    const float m = wave_max(a.m);
    raise(a, m, c);
    a.s = wave_sum(a.s);
    __syncthreads();
    if (lane_id() == 0) waves[threadIdx.x >> 6] = a;
    __syncthreads();
    a = waves[0];
#pragma unroll
    for (int w = 1; w < LP_WG / WAVE; ++w) a = join(a, waves[w], c);
    return a;
}

// A workgroup per row.
template <typename T>
__global__ __launch_bounds__(LP_WG) void distill_row_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int V, float scale,
                                                            Teacher t, Loss o)
{
    __shared__ uint32_t marks[DS_MARKED * LP_CHUNK / 32];
    __shared__ Part2 waves[LP_WG / WAVE];
    __shared__ __attribute__((aligned(16))) int tokens[QADC_MAX_ALTERNATIVES];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = logits + r * ld;
        const int lead = lead_of(row);
        const int token = token_of(r, V, t);
        const Part2 a = chunks_part(row, 0, chunks_of(V, lead), V, lead, scale * LOG2E, token, marks, waves);
        if (threadIdx.x < WAVE) finish_row(a, wave_stored(row, r, V, t), r, scale, t, o, tokens);
    }
}

// A workgroup per `per` chunks of a row, into the workspace.
template <typename T>
__global__ __launch_bounds__(LP_WG) void distill_part_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int V, float scale,
                                                             Teacher t, int parts, int per, Part2 *__restrict__ stats)
{
    __shared__ uint32_t marks[DS_MARKED * LP_CHUNK / 32];
    __shared__ Part2 waves[LP_WG / WAVE];
    for (int64_t i = blockIdx.x; i < rows * parts; i += gridDim.x) {
        const int64_t r = i / parts, j0 = i % parts * per;
        const T *row = logits + r * ld;
        const int lead = lead_of(row);
        const Part2 a = chunks_part(row, j0, min(j0 + per, chunks_of(V, lead)), V, lead, scale * LOG2E, token_of(r, V, t), marks, waves);
        if (threadIdx.x == 0) stats[i] = a;
    }
}
// A wavefront per row: no barriers.
template <typename T>
__global__ __launch_bounds__(LP_WG) void distill_join_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int V, float scale,
                                                             Teacher t, int parts, const Part2 *__restrict__ stats, Loss o)
{
    __shared__ __attribute__((aligned(16))) int tokens[LP_WG / WAVE][QADC_MAX_ALTERNATIVES];
    const float c = scale * LOG2E;
    const int wave = threadIdx.x >> 6;
    for (int64_t r = (int64_t)blockIdx.x * (LP_WG / WAVE) + wave; r < rows; r += (int64_t)gridDim.x * (LP_WG / WAVE)) {
        const WaveStored st = wave_stored(logits + r * ld, r, V, t);
        Part2 a = {-INFINITY, 0.0f};
        for (int p = lane_id(); p < parts; p += WAVE) a = join(a, stats[r * parts + p], c);
        const float m = wave_max(a.m);
        raise(a, m, c);
        a.s = wave_sum(a.s);
        a.m = m;
        finish_row(a, st, r, scale, t, o, tokens[wave]);
    }
}

// The stored tokens' gradients, each token once: value(logit) is what a stored token has from the student, own the teacher's share.
struct GradLds {
    __attribute__((aligned(16))) int tokens[QADC_MAX_ALTERNATIVES];
    float p[QADC_MAX_ALTERNATIVES];
};
template <typename T, typename F>
__device__ __forceinline__ void write_stored(T *out, const Stored &st, int k, const GradLds &lds, F value)
{
    if (st.token < 0) return;
    float p = 0.0f;
    bool first = true;
    for (int i = 0; i < k; ++i)
        if (lds.tokens[i] == st.token) {
            first = first && i >= (int)threadIdx.x;
            p += lds.p[i];
        }
    if (first) out[st.token] = (T)value(st.logit, p);
}

// A workgroup per `per` chunks of a row: first every token's share as if it was not stored, then the stored tokens.  STREAM: stores past
// the caches.
template <typename T, bool STREAM>
__global__ __launch_bounds__(LP_WG) void distill_grad_kernel(const T *logits, int64_t ld, int64_t rows, int V, float scale, Teacher t,
                                                             int parts, int per, const float *__restrict__ lse,
                                                             const float *__restrict__ log_tail, const float *__restrict__ dloss,
                                                             T *dlogits, int64_t ldd)
{
    constexpr int N = Pack<T>::N, PACKS = LP_BLOCK / N;
    __shared__ double masses[DS_WAVES];
    __shared__ GradLds grad;
    for (int64_t i = blockIdx.x; i < rows * parts; i += gridDim.x) {
        const int64_t r = i / parts;
        const T *row = logits + r * ld;
        T *out = dlogits + r * ldd;
        const int lead = lead_of(out);
        const int64_t j0 = i % parts * per, j1 = min(j0 + per, chunks_of(V, lead));
        const int64_t v0 = max((int64_t)0, j0 * LP_CHUNK - lead), v1 = min(j1 * LP_CHUNK - lead, (int64_t)V);
        const float l = lse[r], w = scale * dloss[r];
        const bool zero = w == 0.0f || l == -INFINITY;  // (a row without a share of the loss is not read)
        Stored st = {-1, -INFINITY, -INFINITY};
        double p = 0.0;
        if ((int)threadIdx.x < t.k && !zero) {
            const uint32_t v = t.idx[r * t.k + threadIdx.x];
            if (v < (uint32_t)V) {
                p = exp((double)t.logp[r * t.k + threadIdx.x]);
                if ((int64_t)v >= v0 && (int64_t)v < v1) {
                    st.token = (int)v;
                    st.logit = (float)row[v];
                }
            }
        }
        if (threadIdx.x < QADC_MAX_ALTERNATIVES) {
            const double P = wave_sum64(p);
            if (lane_id() == 0) masses[threadIdx.x >> 6] = P;
        }
        __syncthreads();
        double P = 0.0;
#pragma unroll
        for (int w = 0; w < DS_WAVES; ++w) P += masses[w];
        const Mass mass = mass_of(P, t.tail);
        const Factors by = factors(mass, t.tail, (double)log_tail[r]);
        if ((int)threadIdx.x < t.k) {
            grad.tokens[threadIdx.x] = st.token;
            grad.p[threadIdx.x] = (float)(t.tail ? p : mass.P > 0.0 ? p / mass.P : 0.0);
        }
        const float f = w * by.other;
        const auto value = [&](float logit) { return zero ? 0.0f : f * exp_of<T>(fmaf(scale, logit, -l) - by.log_tail); };
        for (int64_t j = j0; j < j1; ++j) {
            typename Pack<T>::V q[PACKS];
            if ((j > 0 || lead == 0) && (j + 1) * LP_CHUNK - lead <= v1) {
                if (!zero)
#pragma unroll
                    for (int u = 0; u < PACKS; ++u)
                        q[u] = __builtin_nontemporal_load(reinterpret_cast<const typename Pack<T>::V *>(row + pack_at<T>(j, u, lead)));
#pragma unroll
                for (int u = 0; u < PACKS; ++u) {
#pragma unroll
                    for (int e = 0; e < N; ++e) q[u][e] = (T)value((float)q[u][e]);
                    auto *const to = reinterpret_cast<typename Pack<T>::V *>(out + pack_at<T>(j, u, lead));
                    if constexpr (STREAM) __builtin_nontemporal_store(q[u], to);
                    else *to = q[u];
                }
            } else {
#pragma unroll
                for (int u = 0; u < PACKS; ++u) q[u] = load_edge(row, pack_at<T>(j, u, lead), v1, 0.0f);
#pragma unroll
                for (int u = 0; u < PACKS; ++u) {
                    const int64_t at = pack_at<T>(j, u, lead);
                    if (at >= v1) continue;
#pragma unroll
                    for (int e = 0; e < N; ++e) q[u][e] = (T)value((float)q[u][e]);
                    if (at >= 0 && at + N <= v1) {
                        *reinterpret_cast<typename Pack<T>::V *>(out + at) = q[u];
                    } else {
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (at + e >= 0 && at + e < v1) out[at + e] = q[u][e];
                    }
                }
            }
        }
        __syncthreads();
        write_stored(out, st, t.k, grad, [&](float logit, float own) { return w * fmaf(by.total, exp_of<T>(fmaf(scale, logit, -l)), -own); });
        __syncthreads();
    }
}

struct StepLds {
    double mass[DS_WAVES], loss[DS_WAVES];
    float most[16], others[16], own[DS_WAVES];
    GradLds grad;
};

// Loss and gradient of a row whose logits stay in the registers of its workgroup: PACKS packs a thread, read and written once, and the
// logits before the first line of 128 bytes and behind the last pack of 16 one a thread.  What the gradient needs (the largest logit, the two
// sums, the teacher's mass) comes first, the loss after the stores.  128 registers: half of them hold the row.
// Stores past the caches: 2048 x 128001 bfloat16 222 us and 240 through them, 512 x 32768 20.5 and 23.8 (2048 x 32768 alone 59 and 58).
template <typename T, int THREADS, int PACKS>
__global__ __launch_bounds__(THREADS, 4) void distill_step_kernel(const T *logits, int64_t ld, int V, float scale, Teacher t,
                                                                  const float *__restrict__ weight, float *__restrict__ loss, T *dlogits,
                                                                  int64_t ldd)
{
    constexpr int N = Pack<T>::N, W = THREADS / WAVE;
    typedef typename Pack<T>::V P;
    constexpr int LINE = 128 / (int)sizeof(T), MARKS = (THREADS * PACKS * N + LINE) / 32 + 1;
    __shared__ uint32_t marks[MARKS];  // from the beginning of the row's first line on
    __shared__ StepLds lds;
    const int64_t r = blockIdx.x;
    const T *row = logits + r * ld;
    T *out = dlogits + r * ldd;
    const int lead = (int)((uintptr_t)row % 128 / sizeof(T)), wave = threadIdx.x >> 6, tid = threadIdx.x;
    const float c = scale * LOG2E;
    const Stored st = stored_of(row, r, V, t, tid);
    // whole packs begin .. end - 1 from the line that holds the row's first logit on, the first of them where a line begins; this thread's
    // at begin + u THREADS + tid
    const int begin = lead ? LINE / N : 0, end = (V + lead) / N, here = end - begin - tid;  // (u THREADS < here: there is one)
    const int head = lead ? min(LINE - lead, V) : 0, tail = max(end * N - lead, head);
    const int edge = tid < head ? tid : tail + tid - head;  // < V: this thread's logit at an end
    const T *from = row + (begin + tid) * N - lead;
    T *to = out + (begin + tid) * N - lead;
    P x[PACKS];
#pragma unroll
    for (int u = 0; u < PACKS; ++u) {
        x[u] = (T)-INFINITY;
        if (u * THREADS < here) x[u] = __builtin_nontemporal_load(reinterpret_cast<const P *>(from + u * THREADS * N));
    }
    const float at_edge = edge < V ? (float)row[edge] : -INFINITY;
    // the teacher, while the row comes in
    for (int i = threadIdx.x; i < MARKS; i += THREADS) marks[i] = 0;
    double p = 0.0;
    if (wave < DS_WAVES) {
        p = st.token < 0 ? 0.0 : exp((double)st.logp);
        const double mass = wave_sum64(p);
        if (lane_id() == 0) lds.mass[wave] = mass;
        lds.grad.tokens[threadIdx.x] = st.token;
    }
    __syncthreads();
    double P64 = 0.0;
#pragma unroll
    for (int w = 0; w < DS_WAVES; ++w) P64 += lds.mass[w];
    const Mass mass = mass_of(P64, t.tail);
    bool first = st.token >= 0;  // a token that is stored twice counts once for the student
    if (wave < DS_WAVES) {
        if (st.token >= 0) atomicOr(&marks[(st.token + lead) / 32], 1u << ((st.token + lead) % 32));
        first = first && first_of(lds.grad.tokens, st.token, t.k, tid);
        lds.grad.p[threadIdx.x] = (float)(t.tail ? p : mass.P > 0.0 ? p / mass.P : 0.0);
    }
    float m = at_edge;
#pragma unroll
    for (int u = 0; u < PACKS; ++u) {
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, (float)x[u][e]);
        asm volatile("" : "+v"(m));  // (pack after pack: otherwise all are held as float32 at once, beyond 128 registers)
    }
    m = wave_max(m);
    if (lane_id() == 0) lds.most[wave] = m;
    __syncthreads();
    m = lds.most[0];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, lds.most[w]);
    const float m0 = m == -INFINITY ? 0.0f : m;
    const bool marked_edge = edge < V && (marks[(edge + lead) / 32] >> ((edge + lead) % 32) & 1);
    float s = edge < V && !marked_edge ? exp2_fast(c * (at_edge - m0)) : 0.0f;
#pragma unroll
    for (int u = 0; u < PACKS; ++u) {
        asm volatile("" : "+v"(x[u]));  // (converted again rather than kept)
        const unsigned b = u * THREADS < here ? marks_at<N>(marks, (begin + u * THREADS + tid) * N) : 0u;
        float e[N], part = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = exp2_fast(c * ((float)x[u][i] - m0));
        if (b)
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = b >> i & 1 ? 0.0f : e[i];
#pragma unroll
        for (int i = 0; i < N; ++i) part += e[i];
        s += part;
        asm volatile("" : "+v"(s));
    }
    s = wave_sum(s);
    if (lane_id() == 0) lds.others[wave] = s;
    if (wave < DS_WAVES) {
        const float own = wave_sum(first ? exp2_fast(c * (st.logit - m0)) : 0.0f);
        if (lane_id() == 0) lds.own[wave] = own;
    }
    __syncthreads();
    float others = 0.0f, own = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) others += lds.others[w];
#pragma unroll
    for (int w = 0; w < DS_WAVES; ++w) own += lds.own[w];
    // What the other tokens have, relative to the row's largest logit as float32: far below it their exponentials run out of the exponent
    // one by one, and are summed again, relative to the largest of their own.
    float base = m0;  // what `others` and the gradient's exponentials are relative to
    double left = others;  // `others` relative to m0
    if (mass.rest > 0.0 && others < own * DS_DEEP) {  // (the same in all threads)
        float v = edge < V && !marked_edge ? at_edge : -INFINITY;
#pragma unroll
        for (int u = 0; u < PACKS; ++u) {
            asm volatile("" : "+v"(x[u]));
            const unsigned b = u * THREADS < here ? marks_at<N>(marks, (begin + u * THREADS + tid) * N) : 0u;
#pragma unroll
            for (int i = 0; i < N; ++i) v = fmaxf(v, b >> i & 1 ? -INFINITY : (float)x[u][i]);
            asm volatile("" : "+v"(v));
        }
        v = wave_max(v);
        if (lane_id() == 0) lds.most[wave] = v;
        __syncthreads();
        v = lds.most[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = fmaxf(v, lds.most[w]);
        base = v == -INFINITY ? m0 : v;
        s = edge < V && !marked_edge ? exp2_fast(c * (at_edge - base)) : 0.0f;
#pragma unroll
        for (int u = 0; u < PACKS; ++u) {
            asm volatile("" : "+v"(x[u]));
            const unsigned b = u * THREADS < here ? marks_at<N>(marks, (begin + u * THREADS + tid) * N) : 0u;
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) part += b >> i & 1 ? 0.0f : exp2_fast(c * ((float)x[u][i] - base));
            s += part;
            asm volatile("" : "+v"(s));
        }
        s = wave_sum(s);
        if (lane_id() == 0) lds.others[wave] = s;
        __syncthreads();
        others = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) others += lds.others[w];
        left = (double)others * exp((double)scale * ((double)base - (double)m0));
        if (left < (double)own * DS_NOTHING) {
            left = 0.0;
            base = m0;
        }
    }
    const float sum = own + (float)left;
    const bool none = m == -INFINITY && sum == 0.0f;  // (NaN where there is one among the masked)
    const bool rest = mass.rest > 0.0 && left != 0.0;  // (left out where the student has nothing left)
    const double whole = t.tail ? mass.P + (rest ? mass.rest : 0.0) : mass.P > 0.0 ? 1.0 : 0.0;
    const float total = (float)whole;
    // of q: T - r / Q, as (T others / sum - r) / others of e
    const float share = rest ? (float)((whole * (left / (double)sum) - mass.rest) / (double)others) : total / sum;
    const float w = scale * weight[r];
    const bool zero = w == 0.0f || none;
    const float f = zero ? 0.0f : w * share;
    const auto value = [&](float logit) { return zero ? 0.0f : f * exp2_fast(c * (logit - base)); };
    if (edge < V) out[edge] = (T)value(at_edge);
#pragma unroll
    for (int u = 0; u < PACKS; ++u) {
        asm volatile("" : "+v"(x[u]));
        P g;
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = (T)value((float)x[u][e]);
        if (u * THREADS < here) __builtin_nontemporal_store(g, reinterpret_cast<P *>(to + u * THREADS * N));
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    if (wave < DS_WAVES) {
        if (!zero)
            write_stored(out, st, t.k, lds.grad,
                         [&](float logit, float p) { return w * fmaf(total, exp2_fast(c * (logit - m)) / sum, -p); });
        double l = loss_of(st, p, mass.P, t.tail, none, scale, m, log((double)own + left));
        if (tid == 0 && rest) l += mass.rest * (log(mass.rest) + log1p((double)own / left));
        l = wave_sum64(l);
        if (lane_id() == 0) lds.loss[wave] = l;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double l = 0.0;
#pragma unroll
        for (int v = 0; v < DS_WAVES; ++v) l += lds.loss[v];
        loss[r] = sum == sum ? (float)l : NAN;  // (a broken row is one to an empty teacher too)
    }
}

int check_distill(const char *who, int type, int64_t ld, int64_t rows, int V, float scale, const uint32_t *idx, const float *logp, int k)
{
    if (!type_ok(type)) return fail(QADC_EINVAL, "%s: unknown type %d", who, type);
    // (tokens are counted in an int, a chunk past the last one)
    if (rows < 0 || V < 1 || V > INT32_MAX - 65536 || ld < V)
        return fail(QADC_EINVAL, "%s: rows=%lld V=%d ld=%lld", who, (long long)rows, V, (long long)ld);
    if (!(scale > 0.0f) || !(scale * LOG2E < INFINITY)) return fail(QADC_EINVAL, "%s: scale=%g", who, (double)scale);
    if (k < 0 || k > QADC_MAX_ALTERNATIVES) return fail(QADC_EINVAL, "%s: k=%d", who, k);
    if (rows > 0 && k > 0 && (!idx || !logp)) return fail(QADC_EINVAL, "%s: null pointer", who);
    return QADC_OK;
}

// How the loss of a call is cut: a row per workgroup where the rows alone nearly fill the chip or are short, parts of rows otherwise.  A
// call of bfloat16 rows, whole and in parts: 400 x 131072 29.4 us and 26.9, 512 x 131072 30.3 and 31.7, 400 x 65536 18.4 and 18.6; 64 x 32000
// 11.7 and 14.4, 64 x 50000 15.0 and 14.6, 64 x 131072 26.4 and 14.7, 1 x 50000 12.9 and 14.3.
constexpr int64_t DS_WHOLE = 400, DS_SHORT = 5, DS_PARTS = 1024;  // rows; chunks of a row (some 40000 logits); workgroups
struct Cut {
    int parts, per;
};
Cut cut_of(int64_t rows, int V)
{
    const int64_t chunks = ceil_div((int64_t)V + 7, LP_CHUNK);  // (a row begins up to seven logits into its first pack)
    const int64_t want = rows >= DS_WHOLE || chunks <= DS_SHORT ? 1 : ceil_div(DS_PARTS, std::max<int64_t>(1, rows));
    const int per = (int)ceil_div(chunks, std::min(chunks, want));
    return {(int)ceil_div(chunks, per), per};
}

}  // namespace

// Parts of rows, then lse and log Q for a gradient that follows: enough for these rows and for any fewer, and for shorter ones.
static size_t part_bytes(int64_t rows, int V)
{
    const int64_t chunks = ceil_div((int64_t)V + 7, LP_CHUNK), few = std::min(rows, DS_WHOLE - 1);
    return align_up((size_t)std::min(few * chunks, DS_PARTS + few) * sizeof(Part2), 256);
}
size_t distill_workspace(int64_t rows, int V)
{
    if (rows < 1 || V < 1 || V > INT32_MAX - 65536) return 0;
    return part_bytes(rows, V) + 2 * align_up((size_t)rows * sizeof(float), 256);
}

template <typename T>
static void launch_loss(const void *logits, int64_t ld, int64_t rows, int V, float scale, const Teacher &t, const Loss &o, void *workspace,
                        hipStream_t st)
{
    const Cut p = cut_of(rows, V);
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 20));
    if (p.parts == 1) {
        launch(QADC_PROF_DISTILL, distill_row_kernel<T>, grid, dim3(LP_WG), 0, st, (const T *)logits, ld, rows, V, scale, t, o);
        return;
    }
    launch(QADC_PROF_DISTILL, distill_part_kernel<T>, dim3((unsigned)std::min<int64_t>(rows * p.parts, 1 << 20)), dim3(LP_WG), 0, st,
           (const T *)logits, ld, rows, V, scale, t, p.parts, p.per, (Part2 *)workspace);
    launch(QADC_PROF_DISTILL, distill_join_kernel<T>, dim3((unsigned)std::min<int64_t>(ceil_div(rows, LP_WG / WAVE), 1 << 20)), dim3(LP_WG), 0,
           st, (const T *)logits, ld, rows, V, scale, t, p.parts, (const Part2 *)workspace, o);
}

template <typename T>
static void launch_grad(const void *logits, int64_t ld, int64_t rows, int V, float scale, const Teacher &t, const float *lse,
                        const float *log_tail, const float *dloss, void *dlogits, int64_t ldd, hipStream_t st)
{
    // (where rows begin off 16 bytes, up to seven logits into their first pack)
    const bool even = (uintptr_t)dlogits % 16 == 0 && (size_t)ldd * sizeof(T) % 16 == 0;
    const int64_t chunks = ceil_div((int64_t)V + (even ? 0 : 7), LP_CHUNK);
    // Chunks a workgroup: more of them share the stored tokens and the factors, fewer fill the chip.  One and four: 32 x 128001 bfloat16 10.5 us
    // and 12.7, 128 x 128001 19.6 and 20.9, 512 x 128001 57.7 and 50.9.
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(4, chunks * rows / 2048));
    const int parts = (int)ceil_div(chunks, most), per = (int)ceil_div(chunks, parts);
    // A gradient beyond the last cache's size goes past it: with inputs that change 2048 x 128001 bfloat16 211 us and 226, 4096 x 65536 190 and 211,
    // 4096 x 50257 float32 351 and 363, 8192 x 128001 878 and 868; but 512 x 128001 59 and 51.  Between the products of a training step the
    // gradient itself is slower past the caches (2048 x 128001 236 and 207) and the product behind it faster: both 1220 and 1224 there, 4096 x
    // 65536 1001 and 1012, 8192 x 65536 1194 and 1261.
    const bool stream = (size_t)rows * V * sizeof(T) > ((size_t)384 << 20);
    const auto kernel = stream ? &distill_grad_kernel<T, true> : &distill_grad_kernel<T, false>;
    launch(QADC_PROF_DISTILL, kernel, dim3((unsigned)std::min<int64_t>(rows * parts, 1 << 22)), dim3(LP_WG), 0, st, (const T *)logits, ld,
           rows, V, scale, t, parts, per, lse, log_tail, dloss, (T *)dlogits, ldd);
}

int distill(const void *logits, int64_t ld, int type, int64_t rows, int V, float scale, const uint32_t *idx, const float *logp, int k,
            int tail, float *loss, float *lse, float *log_tail, void *workspace, size_t workspace_bytes, hipStream_t st)
{
    const char *who = "qadc_distill";
    if (const int rc = check_distill(who, type, ld, rows, V, scale, idx, logp, k)) return rc;
    if (rows == 0) return QADC_OK;
    if (!logits || !loss) return fail(QADC_EINVAL, "%s: null pointer", who);
    const Cut p = cut_of(rows, V);
    const size_t need = p.parts > 1 ? (size_t)rows * p.parts * sizeof(Part2) : 0;
    if (need && (!workspace || workspace_bytes < need))
        return fail(QADC_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, need);
    if (need && (uintptr_t)workspace % 16) return fail(QADC_EINVAL, "%s: workspace is not aligned to 16 bytes", who);
    const Teacher t = {idx, logp, k, tail != 0};
    QADC_BY_TYPE(type, (launch_loss<T>(logits, ld, rows, V, scale, t, {loss, lse, log_tail}, workspace, st)));
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

int distill_backward(const void *logits, int64_t ld, int type, int64_t rows, int V, float scale, const uint32_t *idx, const float *logp,
                     int k, int tail, const float *lse, const float *log_tail, const float *dloss, void *dlogits, int64_t ldd,
                     hipStream_t st)
{
    const char *who = "qadc_distill_backward";
    if (const int rc = check_distill(who, type, ld, rows, V, scale, idx, logp, k)) return rc;
    if (ldd < V) return fail(QADC_EINVAL, "%s: ldd=%lld", who, (long long)ldd);
    if (rows == 0) return QADC_OK;
    if (!logits || !lse || !log_tail || !dloss || !dlogits) return fail(QADC_EINVAL, "%s: null pointer", who);
    if (logits == dlogits && ld != ldd) return fail(QADC_EINVAL, "%s: in place needs equal row distances", who);
    const Teacher t = {idx, logp, k, tail != 0};
    QADC_BY_TYPE(type, (launch_grad<T>(logits, ld, rows, V, scale, t, lse, log_tail, dloss, dlogits, ldd, st)));
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

template <typename T, int THREADS, int PACKS>
static void launch_step(const void *logits, int64_t ld, int64_t rows, int V, float scale, const Teacher &t, const float *weight,
                        float *loss, void *dlogits, int64_t ldd, hipStream_t st)
{
    launch(QADC_PROF_DISTILL, distill_step_kernel<T, THREADS, PACKS>, dim3((unsigned)rows), dim3(THREADS), 0, st, (const T *)logits, ld, V,
           scale, t, weight, loss, (T *)dlogits, ldd);
}

int distill_step(const void *logits, int64_t ld, int type, int64_t rows, int V, float scale, const uint32_t *idx, const float *logp, int k,
                 int tail, const float *weight, float *loss, void *dlogits, int64_t ldd, void *workspace, size_t workspace_bytes,
                 hipStream_t st)
{
    const char *who = "qadc_distill_step";
    if (const int rc = check_distill(who, type, ld, rows, V, scale, idx, logp, k)) return rc;
    if (ldd < V) return fail(QADC_EINVAL, "%s: ldd=%lld", who, (long long)ldd);
    if (rows == 0) return QADC_OK;
    if (!logits || !weight || !loss || !dlogits) return fail(QADC_EINVAL, "%s: null pointer", who);
    if (logits == dlogits && ld != ldd) return fail(QADC_EINVAL, "%s: in place needs equal row distances", who);
    const Cut p = cut_of(rows, V);
    const size_t stats = align_up(p.parts > 1 ? (size_t)rows * p.parts * sizeof(Part2) : 0, 256), each = align_up((size_t)rows * 4, 256);
    if (!workspace || workspace_bytes < stats + 2 * each)
        return fail(QADC_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, stats + 2 * each);
    if ((uintptr_t)workspace % 16) return fail(QADC_EINVAL, "%s: workspace is not aligned to 16 bytes", who);
    const Teacher t = {idx, logp, k, tail != 0};
    float *lse = (float *)((char *)workspace + stats), *log_tail = (float *)((char *)workspace + stats + each);
    const size_t e = type_bytes(type);
    const size_t bytes = (size_t)V * e;
    // A row in a workgroup's registers: 16 x 16384 bfloat16 12 us, 17 in the two steps that other rows take, 256 x 65536 19 and 35, 1024 x
    // 131072 115 and 133; of rows beyond 128 KB, one a compute unit, from 64 on (32: 25 and 19; 128: 26 and 35).  A grid's threads are
    // counted in 32 bits.
    if ((bytes <= 131072 || rows >= 64) && rows <= 1 << 21 && bytes <= 262144) {
        QADC_BY_TYPE(type, {
            if (bytes <= 16384) launch_step<T, 256, 4>(logits, ld, rows, V, scale, t, weight, loss, dlogits, ldd, st);
            else if (bytes <= 32768) launch_step<T, 256, 8>(logits, ld, rows, V, scale, t, weight, loss, dlogits, ldd, st);
            else if (bytes <= 65536) launch_step<T, 256, 16>(logits, ld, rows, V, scale, t, weight, loss, dlogits, ldd, st);
            else if (bytes <= 131072) launch_step<T, 512, 16>(logits, ld, rows, V, scale, t, weight, loss, dlogits, ldd, st);
            else launch_step<T, 1024, 16>(logits, ld, rows, V, scale, t, weight, loss, dlogits, ldd, st);
        });
    } else {
        QADC_BY_TYPE(type, {
            launch_loss<T>(logits, ld, rows, V, scale, t, {loss, lse, log_tail}, workspace, st);
            launch_grad<T>(logits, ld, rows, V, scale, t, lse, log_tail, weight, dlogits, ldd, st);
        });
    }
    QADC_HIP_TRY(hipGetLastError());
    return QADC_OK;
}

}  // namespace qadc
