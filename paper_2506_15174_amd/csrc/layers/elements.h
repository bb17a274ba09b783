// Elements of activations (internal, device code): f32, f16 and bf16 as fp32 and back.
#ifndef SPMM_ELEMENTS_H
#define SPMM_ELEMENTS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace layers {

template <int TYPE> struct element;  // SPMM_F32, SPMM_F16, SPMM_BF16
template <> struct element<0> { typedef float type; };
template <> struct element<1> { typedef _Float16 type; };
template <> struct element<2> { typedef __bf16 type; };

// fp32 -> bf16 and f16 round to nearest, ties to even (one rounding, where a result is written).
__device__ inline void store_as(char *data, int64_t at, int32_t type, float v)
{
    if (type == 0) reinterpret_cast<float *>(data)[at] = v;
    else if (type == 1) reinterpret_cast<_Float16 *>(data)[at] = (_Float16)v;
    else reinterpret_cast<__bf16 *>(data)[at] = (__bf16)v;
}

__device__ inline float load_as(const char *data, int64_t at, int32_t type)
{
    if (type == 0) return reinterpret_cast<const float *>(data)[at];
    if (type == 1) return (float)reinterpret_cast<const _Float16 *>(data)[at];
    return (float)reinterpret_cast<const __bf16 *>(data)[at];
}

}  // namespace layers

#endif
