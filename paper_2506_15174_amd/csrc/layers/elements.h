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

// Neighbouring elements in one access: the hardware takes wide loads and stores at any alignment, so rows of odd
// length and views that begin anywhere need no other path.
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) neighbours {
    T v[N];
};

// N elements from `at` on, of which `there` exist (the others are 0).
template <typename T, int N> __device__ inline void load_row(const char *data, int64_t at, int there, float (&v)[N])
{
    const T *p = reinterpret_cast<const T *>(data) + at;
    if (there >= N) {
        const neighbours<T, N> n = *reinterpret_cast<const neighbours<T, N> *>(p);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (float)n.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = j < there ? (float)p[j] : 0.0f;
    }
}

template <typename T, int N> __device__ inline void store_row(char *data, int64_t at, int there, const float (&v)[N])
{
    T *p = reinterpret_cast<T *>(data) + at;
    if (there >= N) {
        neighbours<T, N> n;
#pragma unroll
        for (int j = 0; j < N; ++j) n.v[j] = (T)v[j];
        *reinterpret_cast<neighbours<T, N> *>(p) = n;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < there) p[j] = (T)v[j];
    }
}

// The same where the type is known at run time only (it is the same for all lanes).
template <int N> __device__ inline void load_row_as(const char *data, int64_t at, int there, int32_t type, float (&v)[N])
{
    if (type == 0) load_row<float>(data, at, there, v);
    else if (type == 1) load_row<_Float16>(data, at, there, v);
    else load_row<__bf16>(data, at, there, v);
}

template <int N> __device__ inline void store_row_as(char *data, int64_t at, int there, int32_t type, const float (&v)[N])
{
    if (type == 0) store_row<float>(data, at, there, v);
    else if (type == 1) store_row<_Float16>(data, at, there, v);
    else store_row<__bf16>(data, at, there, v);
}

}  // namespace layers

#endif
