// Rows of logits in chunks of a workgroup, shared by the log probabilities and the distillation.
#pragma once

#include "qadc_lm.h"

namespace qadc {

namespace {

constexpr int LP_WG = 256;
constexpr int LP_BLOCK = 32;                  // logits of a thread whose largest is kept
constexpr int LP_CHUNK = LP_WG * LP_BLOCK;    // logits of a workgroup at a time
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// What a part whose largest logit is m has to be shifted by to be relative to `to` (>= m).
__device__ __forceinline__ float shift_of(float m, float to, float c)
{
    return m == to ? 0.0f : m == -INFINITY ? -INFINITY : c * (m - to);
}

// The logits of block (chunk, thread): LP_BLOCK / N packs, those of a wavefront side by side.  Packs lie at multiples of 16
// bytes in memory: a row that does not begin at one has its first pack begin `lead` logits before it (packs across those
// multiples took a quarter longer: 4096 rows of 50021 bfloat16 logits 92 us for 75).
template <typename T>
__device__ __forceinline__ int64_t pack_at(int64_t chunk, int u, int lead)
{
    return chunk * LP_CHUNK + ((int64_t)u * LP_WG + threadIdx.x) * Pack<T>::N - lead;
}
// A pack that may begin before the row or end behind it; `fill` there.
template <typename T>
__device__ __forceinline__ typename Pack<T>::V load_edge(const T *row, int64_t at, int64_t V, float fill)
{
    constexpr int N = Pack<T>::N;
    if (at >= 0 && at + N <= V) return *reinterpret_cast<const typename Pack<T>::V *>(row + at);
    typename Pack<T>::V p = (T)fill;
    if (at < V) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (at + e >= 0 && at + e < V) p[e] = row[at + e];
    }
    return p;
}
__device__ __forceinline__ int64_t chunks_of(int64_t V, int lead) { return (V + lead + LP_CHUNK - 1) / LP_CHUNK; }
template <typename T>
__device__ __forceinline__ void load_block(const T *row, int64_t chunk, int V, int lead, float (&x)[LP_BLOCK])
{
    constexpr int N = Pack<T>::N, PACKS = LP_BLOCK / N;
    typename Pack<T>::V p[PACKS];
    if ((chunk > 0 || lead == 0) && (chunk + 1) * LP_CHUNK - lead <= V) {  // (the same in all threads: loads without a wait)
#pragma unroll
        for (int u = 0; u < PACKS; ++u)
            p[u] = __builtin_nontemporal_load(reinterpret_cast<const typename Pack<T>::V *>(row + pack_at<T>(chunk, u, lead)));
    } else {
#pragma unroll
        for (int u = 0; u < PACKS; ++u) p[u] = load_edge(row, pack_at<T>(chunk, u, lead), V, -INFINITY);
    }
#pragma unroll
    for (int i = 0; i < LP_BLOCK; ++i) x[i] = (float)p[i / N][i % N];
}

// exp(t), t <= 0 or thereabouts.  A float32 gradient shows the rounding of t log2(e), |t| units in its last place of a p that
// has its own size (16-bit ones do not): there what the product leaves out is put back in.
template <typename T>
__device__ __forceinline__ float exp_of(float t)
{
    const float y = t * LOG2E;
    if constexpr (sizeof(T) == 2) return exp2_fast(y);
    const float rest = fmaf(t, LOG2E, -y) + t * 1.9259629911e-8f;  // log2(e) - LOG2E = 1.92596e-8
    const float p = exp2_fast(y);
    return y > -3000.0f ? fmaf(p, rest * LN2, p) : p;  // (an infinite t: no infinity less infinity)
}

}  // namespace

}  // namespace qadc
