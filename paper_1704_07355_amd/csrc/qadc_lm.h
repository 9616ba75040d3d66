// Element types and row access shared by the language-model operators (layer norm, 4-bit products, log probabilities).
#pragma once

#include "qadc_common.h"

namespace qadc {

inline size_t type_bytes(int type) { return type == QADC_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == QADC_TYPE_F32 || type == QADC_TYPE_F16 || type == QADC_TYPE_BF16; }

// Sixteen bytes of a row.  Rows begin at multiples of their element's size only; the memory unit takes wide loads and stores at
// any such address, if more slowly.
template <typename T>
struct Pack {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// How many elements before a row the 16 bytes that hold its first one begin.
template <typename T>
__device__ __forceinline__ int lead_of(const T *row)
{
    return (int)((uintptr_t)row % 16 / sizeof(T));
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
