// The product with 4-bit weights on the matrix cores (gfx950): C = W x B.
//
//   W[m, k] = scale[m, g] (code[m, k] - zero[m, g]),   C[m, n] = sum_g scale[m, g] sum_{k in g} (code - zero)[m, k] B[k, n]
//
// The inner sums are matrix instructions on whole numbers: code - zero lies in -15..15, which bf16, f16 and int8 hold
// exactly, so no weight is rounded; the outer sum is one fp32 multiply-add per element and group.  B is the first operand
// (its 16 tokens are the rows of an instruction), W the second: a lane then holds four tokens of one row of W and
// needs one scale a group.
//
// pack_kernel lays B out as the instructions take it; product_kernel gives a tile of 16 rows and up to 128 tokens to a workgroup, whose waves share K.
#include <hip/hip_runtime.h>

#include "../../../include/spmm_layers.h"
#include "../spmm_launch.h"
#include "elements.h"
#include "layers.h"

namespace layers {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Parts of B: fp32 is held in three bf16 parts that add up to it.
template <int BT> constexpr int PARTS = BT == SPMM_F32 ? 3 : 1;
// Bytes of one part of 16 tokens x 32 columns.
template <int BT> constexpr int STEP_BYTES = BT == SPMM_I8 ? 512 : 1024;

constexpr int WAVES = 8;

// ---- B as the instructions take it ---------------------------------------------------------------------------
//
// [token tile of 16][block of 128 columns][step of 32][part][lane][8 columns], 16 bytes a lane for 16-bit elements;
// codes hold two steps in the 16 bytes of a lane: [token tile][block][pair of steps][lane][step][8 columns].
// Lane 16 q + t holds token t, columns 32 s + 8 q + j.  Tokens and columns that do not exist are zeros.

template <int BT> __global__ __launch_bounds__(256) void pack_kernel(tensor B, int64_t K, int64_t N, int32_t blocks, char *out)
{
    const int lane = threadIdx.x & 63, s = threadIdx.x >> 6, t = lane & 15, q = lane >> 4;
    const int64_t block = blockIdx.x, tile = blockIdx.y, n = tile * 16 + t, k0 = block * BLOCK_COLS + 32 * s + 8 * q;
    const int64_t stride = B.by_token ? 1 : B.ld, at = B.by_token ? n * B.ld + k0 : k0 * B.ld + n;
    const int there = n < N ? (int)min((int64_t)8, K - k0) : 0;
    char *block_out = out + (tile * blocks + block) * (4 * PARTS<BT> * STEP_BYTES<BT>);
    if constexpr (BT == SPMM_I8) {
        // the order in which the weights' nibbles become bytes
        constexpr int order[8] = {0, 4, 1, 5, 2, 6, 3, 7};
        int8_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < there ? reinterpret_cast<const int8_t *>(B.data)[at + j * stride] : 0;
        u32x2 word = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) word[j / 4] |= (uint32_t)(uint8_t)v[order[j]] << (8 * (j % 4));
        *reinterpret_cast<u32x2 *>(block_out + (s >> 1) * 1024 + lane * 16 + (s & 1) * 8) = word;
    } else if constexpr (BT == SPMM_F32) {
        u32x4 parts[3];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // Each part is the upper half of what is left: cut off, not rounded, so that large values stay finite.  An infinity or a NaN
            // is the first part's alone.
            const float v = j < there ? reinterpret_cast<const float *>(B.data)[at + j * stride] : 0.0f;
            float left = v;
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                uint32_t bits = __builtin_bit_cast(uint32_t, left) & 0xffff0000u;
                if (p == 0 && v != v) bits = 0x7fc00000u;
                parts[p][j / 2] = (j & 1) ? parts[p][j / 2] | bits : bits >> 16;
                left = __builtin_isfinite(v) ? left - __builtin_bit_cast(float, bits) : 0.0f;
            }
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4 *>(block_out + (s * 3 + p) * 1024 + lane * 16) = parts[p];
    } else {
        u32x4 word = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t v = j < there ? reinterpret_cast<const uint16_t *>(B.data)[at + j * stride] : 0;
            word[j / 2] |= v << (16 * (j & 1));
        }
        *reinterpret_cast<u32x4 *>(block_out + s * 1024 + lane * 16) = word;
    }
}

// ---- weights as the instructions take them -------------------------------------------------------------------

// code - zero of eight columns in f16: 1024 + code is a mask away (its last bit is worth 1), the difference is exact.
__device__ inline f16x8 weights_f16(uint32_t w, int zero)
{
    const _Float16 z = (_Float16)(float)(1024 + zero);
    const f16x2 base = {z, z};
    f16x2 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(f16x2, ((w >> (4 * i)) & 0x000f000fu) | 0x64006400u) - base;
    return __builtin_bit_cast(f16x8, *reinterpret_cast<u32x4 *>(v));
}

// The same in bf16, by way of fp32: 2^23 + code and 128 + code are a mask away, the upper half of the exact difference is its bf16.
__device__ inline bf16x8 weights_bf16(uint32_t w, int zero)
{
    const float low_base = 8388608.0f + (float)zero, high_base = 128.0f + (float)zero;
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t t = w >> (4 * i);
        const float low = __builtin_bit_cast(float, (t & 0xfu) | 0x4b000000u) - low_base;
        const float high = __builtin_bit_cast(float, (t & 0xf0000u) | 0x43000000u) - high_base;
        v[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, high), __builtin_bit_cast(uint32_t, low), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, v);
}

// The same in bytes, columns in the order 0 4 1 5, 2 6 3 7: no borrow leaves a byte that has 128 added.
__device__ inline u32x2 weights_i8(uint32_t w, uint32_t zero4)
{
    u32x2 v;
    v[0] = (((w & 0x0f0f0f0fu) | 0x80808080u) - zero4) ^ 0x80808080u;
    v[1] = ((((w >> 4) & 0x0f0f0f0fu) | 0x80808080u) - zero4) ^ 0x80808080u;
    return v;
}

// ---- the product ---------------------------------------------------------------------------------------------

template <int BT, int NT> __global__ __launch_bounds__(64 * WAVES) void product_kernel(quant_matrix W, const char *B, const float *B_scales, int64_t N, tensor C)
{
    __shared__ float sums[WAVES][NT][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15;
    const int64_t row_tile = blockIdx.x, token_tiles = (N + 15) / 16, tile0 = (int64_t)blockIdx.y * NT;
    const int per_group = W.group < BLOCK_COLS ? (int)W.group / 32 : 4;   // steps behind which a group's sum is full
    const int group_blocks = W.group < BLOCK_COLS ? 1 : (int)(W.group / BLOCK_COLS), groups_block = W.group < BLOCK_COLS ? BLOCK_COLS / (int)W.group : 1;
    constexpr int BLOCK_BYTES = 4 * PARTS<BT> * STEP_BYTES<BT>;
    const char *tiles[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) tiles[t] = B + min(tile0 + t, token_tiles - 1) * W.blocks * BLOCK_BYTES + lane * 16;
    const uint32_t *codes = W.codes + row_tile * W.blocks * BLOCK_WORDS + lane * 4;
    const float *scales = W.scales + row_tile * W.groups * TILE_ROWS + r;
    const uint8_t *zeros = W.zeros ? W.zeros + row_tile * W.groups * TILE_ROWS + r : nullptr;

    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0, 0, 0, 0};
    const int first = (int)((int64_t)W.blocks * wave / WAVES), last = (int)((int64_t)W.blocks * (wave + 1) / WAVES);
    for (int b = first; b < last; ++b) {
        const u32x4 word = *reinterpret_cast<const u32x4 *>(codes + (int64_t)b * BLOCK_WORDS);
        const int64_t at = (int64_t)b * BLOCK_BYTES;
        auto group_of = [&](int s) { return min(W.groups - 1, groups_block > 1 ? b * groups_block + s / per_group : b / group_blocks); };
        if constexpr (BT == SPMM_I8) {
            i32x4 part[NT];
            auto flush = [&](int s) {
                const float scale = scales[group_of(s) * TILE_ROWS];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][i] += scale * (float)part[t][i];
            };
#pragma unroll
            for (int s = 0; s < 4; s += 2) {
                i32x4 a[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) a[t] = *reinterpret_cast<const i32x4 *>(tiles[t] + at + (s / 2) * 1024);
                const uint32_t zero0 = (zeros ? zeros[group_of(s) * TILE_ROWS] : 8) * 0x01010101u;
                const uint32_t zero1 = (zeros ? zeros[group_of(s + 1) * TILE_ROWS] : 8) * 0x01010101u;
                const u32x2 w0 = weights_i8(word[s], zero0), w1 = weights_i8(word[s + 1], zero1);
                if (per_group == 1) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const long w = __builtin_bit_cast(long, h ? w1 : w0);
#pragma unroll
                        for (int t = 0; t < NT; ++t)
                            part[t] = __builtin_amdgcn_mfma_i32_16x16x32_i8((long)(uint32_t)a[t][2 * h] | ((long)a[t][2 * h + 1] << 32), w, i32x4{0, 0, 0, 0}, 0, 0, 0);
                        flush(s + h);
                    }
                } else {
                    const i32x4 w = {(int)w0[0], (int)w0[1], (int)w1[0], (int)w1[1]};
                    const bool begins = s == 0 || per_group == 2;
#pragma unroll
                    for (int t = 0; t < NT; ++t) part[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[t], w, begins ? i32x4{0, 0, 0, 0} : part[t], 0, 0, 0);
                    if (s == 2 || per_group == 2) flush(s);
                }
            }
        } else {
            f32x4 part[NT];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int group = group_of(s);
                const int zero = zeros ? zeros[group * TILE_ROWS] : 8;
                const bool begins = s % per_group == 0;
                if (begins)
#pragma unroll
                    for (int t = 0; t < NT; ++t) part[t] = f32x4{0, 0, 0, 0};
                if constexpr (BT == SPMM_F16) {
                    const f16x8 w = weights_f16(word[s], zero);
#pragma unroll
                    for (int t = 0; t < NT; ++t) part[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8 *>(tiles[t] + at + s * 1024), w, part[t], 0, 0, 0);
                } else {
                    const bf16x8 w = weights_bf16(word[s], zero);
#pragma unroll
                    for (int p = PARTS<BT> - 1; p >= 0; --p)
#pragma unroll
                        for (int t = 0; t < NT; ++t)
                            part[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8 *>(tiles[t] + at + (s * PARTS<BT> + p) * 1024), w, part[t], 0, 0, 0);
                }
                if (s % per_group == per_group - 1) {
                    const float scale = scales[group * TILE_ROWS];
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[t][i] += scale * part[t][i];
                }
            }
        }
    }

    // The waves' sums meet in LDS, in wave order.
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(&sums[wave][t][lane * 4]) = acc[t];
    __syncthreads();
    for (int e = threadIdx.x; e < NT * 256; e += 64 * WAVES) {
        const int m = C.by_token ? e % 16 : e / (16 * NT), t = C.by_token ? e / 16 : e % (16 * NT);
        const int64_t row = row_tile * TILE_ROWS + m, n = tile0 * 16 + t;
        if (row >= W.M || n >= N) continue;
        const int at = ((t & 15) >> 2) * 64 + m * 4 + (t & 3);
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[w][t >> 4][at];
        if (BT == SPMM_I8) v *= B_scales[n];
        store_as(C.data, C.by_token ? n * C.ld + row : row * C.ld + n, C.type, v);
    }
}

template <int BT> hipError_t execute(const quant_matrix &w, const tensor &B, const float *B_scales, int64_t N, const tensor &C, char *workspace, hipStream_t stream)
{
    const int64_t token_tiles = (N + 15) / 16;
    // a launch of each for 2^16 - 1 tiles of tokens at a time
    constexpr int64_t MOST = 65535 / 8 * 8;
    for (int64_t t0 = 0; t0 < token_tiles; t0 += MOST) {
        const int64_t tiles = token_tiles - t0 < MOST ? token_tiles - t0 : MOST, n0 = t0 * 16, n = N - n0 < tiles * 16 ? N - n0 : tiles * 16;
        const int64_t size = BT == SPMM_I8 ? 1 : BT == SPMM_F32 ? 4 : 2, c_size = C.type == SPMM_F32 ? 4 : 2;
        tensor b = B, c = C;
        b.data += n0 * (B.by_token ? B.ld : 1) * size;
        c.data += n0 * (C.by_token ? C.ld : 1) * c_size;
        const float *scales = B_scales ? B_scales + n0 : nullptr;
        hipError_t e = hipSuccess;
        if (w.blocks > 0) e = launch_kernel(pack_kernel<BT>, dim3((unsigned)w.blocks, (unsigned)tiles), 256, 0, stream, b, w.K, n, w.blocks, workspace);
        if (e != hipSuccess) return e;
        auto product = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            return launch_kernel(product_kernel<BT, NT>, dim3((unsigned)w.tiles, (unsigned)((tiles + NT - 1) / NT)), 64 * WAVES, 0, stream, w, (const char *)workspace, scales, n, c);
        };
        if (tiles == 1) e = product(std::integral_constant<int, 1>());
        else if (tiles == 2) e = product(std::integral_constant<int, 2>());
        else if (tiles <= 4) e = product(std::integral_constant<int, 4>());
        else e = product(std::integral_constant<int, 8>());
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t quant_workspace(const quant_matrix &w, int32_t type, int64_t N)
{
    const int64_t step = type == SPMM_F32 ? 3 * 1024 : type == SPMM_I8 ? 512 : 1024, tiles = (N + 15) / 16;
    const int64_t most = 65535 / 8 * 8;
    return (tiles < most ? tiles : most) * w.blocks * 4 * step;
}

hipError_t quant_execute(const quant_matrix &w, const tensor &B, const float *B_scales, int64_t N, const tensor &C, char *workspace, hipStream_t stream)
{
    switch (B.type) {
    case SPMM_F32: return execute<SPMM_F32>(w, B, B_scales, N, C, workspace, stream);
    case SPMM_F16: return execute<SPMM_F16>(w, B, B_scales, N, C, workspace, stream);
    case SPMM_BF16: return execute<SPMM_BF16>(w, B, B_scales, N, C, workspace, stream);
    default: return execute<SPMM_I8>(w, B, B_scales, N, C, workspace, stream);
    }
}

}  // namespace layers
