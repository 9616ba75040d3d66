// Rows of states in the registers of a group of threads, shared by the layer norm and the root-mean-square norm.
#pragma once

#include <algorithm>

#include "qadc_lm.h"

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

constexpr int NORM_LONG = 16384;  // longest rows that stay in registers

// Threads that share a row: eight elements each up to 8192, sixteen beyond.
inline int norm_group(int d) { return d <= 128 ? 16 : d <= 256 ? 32 : d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024; }

// Workgroups for `rows`, `at_once` of them at a time in each: at most `most`, and all with the same number of turns.
inline int norm_wgs(int64_t rows, int at_once, int most)
{
    const int64_t turns = std::max<int64_t>(1, ceil_div(rows, (int64_t)at_once * most));
    return (int)std::max<int64_t>(1, ceil_div(rows, at_once * turns));
}

inline unsigned norm_grid(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }

}  // namespace

}  // namespace qadc
