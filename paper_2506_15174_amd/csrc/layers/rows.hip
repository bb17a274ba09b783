// What stands between two products (gfx950): the root-mean-square norm with the residual's addition, and the gated
// activation, both with floating output or in 8-bit codes with a scale a token.
//
// A workgroup has all features of its tokens: a first pass makes the sum of squares and the largest magnitude (of
// values without the token's common factor, so that codes do not wait for it), a second one the output.
#include <hip/hip_runtime.h>

#include "../../../include/spmm_layers.h"
#include "../spmm_launch.h"
#include "elements.h"
#include "layers.h"

namespace layers {
namespace {

constexpr int THREADS = 256;

__device__ inline float act_of(float x, int32_t act)
{
    if (act == SPMM_ACT_SILU) return x / (1.0f + expf(-x));
    if (act == SPMM_ACT_GELU) return x / (1.0f + expf(-1.5957691216057308f * (x + 0.044715f * x * x * x)));  // 1 + tanh(u) = 2 / (1 + exp(-2 u)), which does not cancel
    return x < 0.0f ? 0.0f : x;
}

// The larger magnitude; an infinity or a NaN stays one.
__device__ inline float larger(float most, float v)
{
    const float m = fabsf(v);
    return m <= most ? most : m != m ? __builtin_inff() : m;
}

template <bool NORM, int TYPE> __device__ inline float value_of(const rows_args &a, int64_t at, int64_t k)
{
    const float x = load_as(a.x.data, at, TYPE);
    if constexpr (NORM) {
        if (!a.y.data) return x;
        typename element<TYPE>::type t = (typename element<TYPE>::type)(x + load_as(a.y.data, at, TYPE));
        return (float)t;
    } else {
        return act_of(x, a.act) * (a.y.data ? load_as(a.y.data, at, TYPE) : 1.0f);
    }
}

// TOKENS tokens a workgroup, THREADS / TOKENS threads each.
template <bool NORM, int TYPE, int TOKENS> __global__ __launch_bounds__(THREADS) void rows_kernel(rows_args a)
{
    constexpr int EACH = THREADS / TOKENS;
    __shared__ float squares[EACH][TOKENS], mosts[EACH][TOKENS];
    const int token = threadIdx.x % TOKENS, part = threadIdx.x / TOKENS;
    const int64_t n = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * TOKENS + token;
    const bool there = n < a.tokens;
    auto at = [&](const tensor &t, int64_t k) { return t.by_token ? n * t.ld + k : k * t.ld + n; };
    float square = 0.0f, most = 0.0f;
    if (there) {
        for (int64_t k = part; k < a.features; k += EACH) {
            float v = value_of<NORM, TYPE>(a, at(a.x, k), k);
            if constexpr (NORM) {
                if (a.total.data) store_as(a.total.data, at(a.total, k), TYPE, v);
                square += v * v;
                v *= load_as(a.weight, k, a.weight_type);
            }
            most = larger(most, v);
        }
    }
    squares[part][token] = square;
    mosts[part][token] = most;
    __syncthreads();
    square = most = 0.0f;
    for (int p = 0; p < EACH; ++p) {
        square += squares[p][token];
        most = larger(most, mosts[p][token]);
    }
    if (!there) return;
    const float factor = NORM ? 1.0f / sqrtf(square / (float)a.features + a.eps) : 1.0f;
    const bool codes = a.out.type == SPMM_I8;
    // 127 / most overflows for the smallest values: those are made larger first
    const float up = most < 0x1p-100f ? 0x1p100f : 1.0f;
    const float steps = most > 0.0f && most < __builtin_inff() ? 127.0f / (most * up) : 0.0f;
    if (codes && part == 0) a.scales[n] = most < __builtin_inff() ? most * factor / 127.0f : __builtin_nanf("");
    for (int64_t k = part; k < a.features; k += EACH) {
        float v = NORM && a.total.data ? load_as(a.total.data, at(a.total, k), TYPE) : value_of<NORM, TYPE>(a, at(a.x, k), k);
        const float w = NORM ? load_as(a.weight, k, a.weight_type) : 1.0f;
        if (codes) reinterpret_cast<int8_t *>(a.out.data)[at(a.out, k)] = steps == 0.0f ? 0 : (int8_t)rintf(v * w * up * steps);
        else store_as(a.out.data, at(a.out, k), a.out.type, v * factor * w);
    }
}

// A launch has less than 2^32 threads along an axis.
dim3 grid_of(int64_t blocks)
{
    const int64_t x = blocks < 1 << 20 ? blocks : 1 << 20;
    return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

template <bool NORM> hipError_t launch(const rows_args &a, hipStream_t stream)
{
    auto run = [&](auto type) {
        constexpr int TYPE = decltype(type)::value;
        if (a.x.by_token) return launch_kernel(rows_kernel<NORM, TYPE, 1>, grid_of(a.tokens), THREADS, 0, stream, a);
        return launch_kernel(rows_kernel<NORM, TYPE, 16>, grid_of((a.tokens + 15) / 16), THREADS, 0, stream, a);
    };
    switch (a.x.type) {
    case SPMM_F32: return run(std::integral_constant<int, SPMM_F32>());
    case SPMM_F16: return run(std::integral_constant<int, SPMM_F16>());
    default: return run(std::integral_constant<int, SPMM_BF16>());
    }
}

}  // namespace

int64_t rows_workspace(const rows_args &, bool) { return 0; }

hipError_t rows_launch(const rows_args &a, bool norm, char *, hipStream_t stream)
{
    return norm ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace layers
