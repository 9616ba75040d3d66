// Element types and row access shared by the language-model operators (layer norm, 4-bit products, log probabilities).
#pragma once

#include "qadc_common.h"

namespace qadc {

inline size_t type_bytes(int type) { return type == QADC_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == QADC_TYPE_F32 || type == QADC_TYPE_F16 || type == QADC_TYPE_BF16; }

// Sixteen bytes of a row.  Rows start at multiples of their element's size only; the memory unit takes wide loads and
// stores at any such address, so no variant is kept for aligned rows.
template <typename T>
struct Pack {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// Elements c .. c + N - 1 of a row of d, `fill` beyond its end.
template <typename T>
__device__ __forceinline__ void load_pack(const T *row, int64_t c, int64_t d, float fill, float (&v)[Pack<T>::N])
{
    constexpr int N = Pack<T>::N;
    if (c + N <= d) {
        const typename Pack<T>::V p = *reinterpret_cast<const typename Pack<T>::V *>(row + c);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)p[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = c + e < d ? (float)row[c + e] : fill;
    }
}

template <typename T>
__device__ __forceinline__ void store_pack(T *row, int64_t c, int64_t d, const float (&v)[Pack<T>::N])
{
    constexpr int N = Pack<T>::N;
    if (c + N <= d) {
        typename Pack<T>::V p;
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = (T)v[e];
        *reinterpret_cast<typename Pack<T>::V *>(row + c) = p;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < d) row[c + e] = (T)v[e];
    }
}

// Float joined over the wavefront without a trip through LDS, in every lane: lanes of 16, then rows, then the last lane's value.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_or(float old, float v)
{
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp((int)__float_as_uint(old), (int)__float_as_uint(v), CTRL, ROWS,
                                                                 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp_or<0x111, 0xf>(0.0f, v);
    v += dpp_or<0x112, 0xf>(0.0f, v);
    v += dpp_or<0x114, 0xf>(0.0f, v);
    v += dpp_or<0x118, 0xf>(0.0f, v);
    v += dpp_or<0x142, 0xa>(0.0f, v);
    v += dpp_or<0x143, 0xc>(0.0f, v);
    return __uint_as_float(lane_value(__float_as_uint(v), 63));
}
// Sum over groups of 16, 32 or 64 lanes, in every lane: a row of 16 turned by 8, 4, 2 and 1, then the rows.
template <int G>
__device__ __forceinline__ float lanes_sum(float v)
{
    if constexpr (G == WAVE) return wave_sum(v);
    v += dpp_or<0x128, 0xf>(0.0f, v);
    v += dpp_or<0x124, 0xf>(0.0f, v);
    v += dpp_or<0x122, 0xf>(0.0f, v);
    v += dpp_or<0x121, 0xf>(0.0f, v);
    if constexpr (G == 32) v += __shfl_xor(v, 16);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, dpp_or<0x111, 0xf>(v, v));
    v = fmaxf(v, dpp_or<0x112, 0xf>(v, v));
    v = fmaxf(v, dpp_or<0x114, 0xf>(v, v));
    v = fmaxf(v, dpp_or<0x118, 0xf>(v, v));
    v = fmaxf(v, dpp_or<0x142, 0xa>(v, v));
    v = fmaxf(v, dpp_or<0x143, 0xc>(v, v));
    return __uint_as_float(lane_value(__float_as_uint(v), 63));
}

// Runs `call` with T = float, _Float16 or __bf16 by the element type.
#define QADC_BY_TYPE(type, ...)                                     \
    switch (type) {                                                 \
    case QADC_TYPE_F32: { using T = float; __VA_ARGS__; } break;    \
    case QADC_TYPE_F16: { using T = _Float16; __VA_ARGS__; } break; \
    default: { using T = __bf16; __VA_ARGS__; } break;              \
    }

}  // namespace qadc
