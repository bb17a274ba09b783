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

#include <type_traits>

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

// Eight columns of a token as operands: a part each; codes are eight bytes.
template <int BT> struct operands {
    u32x4 part[PARTS<BT>];
};
template <> struct operands<SPMM_I8> {
    u32x2 part[1];
};

// fp32: each part is the upper half of what is left, cut off, not rounded, so that large values stay finite.  An infinity or a NaN is the first
// part's alone.
__device__ inline void split(const float (&v)[8], operands<SPMM_F32> &o)
{
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        uint32_t bits[2][3];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float x = v[j + h];
            const bool finite = __builtin_isfinite(x);
            const uint32_t b0 = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
            const float left1 = x - __builtin_bit_cast(float, b0);
            const uint32_t b1 = __builtin_bit_cast(uint32_t, left1) & 0xffff0000u;
            const float left2 = left1 - __builtin_bit_cast(float, b1);
            bits[h][0] = x != x ? 0x7fc00000u : b0;
            bits[h][1] = finite ? b1 : 0;
            bits[h][2] = finite ? __builtin_bit_cast(uint32_t, left2) : 0;
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) o.part[p][j / 2] = __builtin_amdgcn_perm(bits[1][p], bits[0][p], 0x07060302u);
    }
}

// Columns k0 .. k0 + 7 of token n, of which `there` exist (the others are 0).
template <int BT> __device__ inline void fetch(const tensor &B, int64_t n, int64_t k0, int there, operands<BT> &o)
{
    const int64_t stride = B.by_token ? 1 : B.ld, at = B.by_token ? n * B.ld + k0 : k0 * B.ld + n;
    if constexpr (BT == SPMM_I8) {
        u32x2 raw = {0, 0};  // (codes lie one token a row)
        if (there >= 8) {
            raw = __builtin_bit_cast(u32x2, *reinterpret_cast<const neighbours<int8_t, 8> *>(B.data + at));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < there) raw[j / 4] |= (uint32_t) reinterpret_cast<const uint8_t *>(B.data)[at + j] << (8 * (j % 4));
        }
        // the order in which the weights' nibbles become bytes: 0 4 1 5, 2 6 3 7
        o.part[0] = u32x2{__builtin_amdgcn_perm(raw[1], raw[0], 0x05010400u), __builtin_amdgcn_perm(raw[1], raw[0], 0x07030602u)};
    } else if constexpr (BT == SPMM_F32) {
        float v[8];
        if (B.by_token) {
            load_row<float>(B.data, at, there, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < there ? reinterpret_cast<const float *>(B.data)[at + j * stride] : 0.0f;
        }
        split(v, o);
    } else {
        if (B.by_token && there >= 8) {
            o.part[0] = __builtin_bit_cast(u32x4, *reinterpret_cast<const neighbours<uint16_t, 8> *>(B.data + 2 * at));
        } else {
            u32x4 word = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t v = j < there ? reinterpret_cast<const uint16_t *>(B.data)[at + j * stride] : 0;
                word[j / 2] |= v << (16 * (j & 1));
            }
            o.part[0] = word;
        }
    }
}

template <int BT> __global__ __launch_bounds__(256) void pack_kernel(tensor B, int64_t K, int64_t N, int32_t blocks, char *out)
{
    const int lane = threadIdx.x & 63, s = threadIdx.x >> 6, t = lane & 15, q = lane >> 4;
    const int64_t block = blockIdx.x, tile = blockIdx.y, n = tile * 16 + t, k0 = block * BLOCK_COLS + 32 * s + 8 * q;
    char *block_out = out + (tile * blocks + block) * (4 * PARTS<BT> * STEP_BYTES<BT>);
    operands<BT> o;
    fetch<BT>(B, n, k0, n < N ? (int)min((int64_t)8, K - k0) : 0, o);
    if constexpr (BT == SPMM_I8) {
        *reinterpret_cast<u32x2 *>(block_out + (s >> 1) * 1024 + lane * 16 + (s & 1) * 8) = o.part[0];
    } else {
#pragma unroll
        for (int p = 0; p < PARTS<BT>; ++p) *reinterpret_cast<u32x4 *>(block_out + (s * PARTS<BT> + p) * 1024 + lane * 16) = o.part[p];
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

// ---- few tokens ------------------------------------------------------------------------------------------------
//
// Up to 16 tokens are one tile, and a product is over in the time of a few memory accesses: one launch, in which every wave reads its columns of
// B as it reads its weights and makes operands of them itself.  Lanes of tokens that do not exist read the last one's (an access the
// wave makes anyway); their results are not stored.  Weights, scales and B of AHEAD blocks are asked for before the first is used.
// PER_GROUP: steps of 32 columns behind which a group's sum is full (4, 2 or 1).

template <int BT, int PER_GROUP, int KWAVES> __global__ __launch_bounds__(64 * KWAVES) void few_kernel(quant_matrix W, tensor B, const float *B_scales, int32_t N, tensor C)
{
    __shared__ float sums[KWAVES][256];
    constexpr int AHEAD = BT == SPMM_F32 ? 1 : 2, SUMS = 4 / PER_GROUP;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4, n = min(r, N - 1);
    const int64_t row_tile = blockIdx.x;
    const int group_blocks = PER_GROUP < 4 ? 1 : (int)(W.group / BLOCK_COLS);
    const uint32_t *codes = W.codes + row_tile * W.blocks * BLOCK_WORDS + lane * 4;
    const float *scales = W.scales + row_tile * W.groups * TILE_ROWS + r;
    const uint8_t *zeros = W.zeros ? W.zeros + row_tile * W.groups * TILE_ROWS + r : nullptr;
    const int first = (int)((int64_t)W.blocks * wave / KWAVES), last = (int)((int64_t)W.blocks * (wave + 1) / KWAVES);
    struct asked {
        u32x4 word;
        float scale[SUMS];
        int zero[SUMS];
        operands<BT> b[4];
    };
    auto ask = [&](int b, asked &a) {
        a.word = *reinterpret_cast<const u32x4 *>(codes + (int64_t)b * BLOCK_WORDS);
#pragma unroll
        for (int g = 0; g < SUMS; ++g) {
            const int group = PER_GROUP < 4 ? min(W.groups - 1, b * SUMS + g) : b / group_blocks;
            a.scale[g] = scales[group * TILE_ROWS];
            a.zero[g] = zeros ? zeros[group * TILE_ROWS] : 8;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int64_t k0 = (int64_t)b * BLOCK_COLS + 32 * s + 8 * q;
            fetch<BT>(B, n, k0, (int)min((int64_t)8, W.K - k0), a.b[s]);
        }
    };
    f32x4 acc = {0, 0, 0, 0};
    auto use = [&](const asked &a) {
        if constexpr (BT == SPMM_I8) {
            u32x2 w[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) w[s] = weights_i8(a.word[s], a.zero[s / PER_GROUP] * 0x01010101u);
            i32x4 part;
#pragma unroll
            for (int s = 0; s < 4; s += PER_GROUP == 1 ? 1 : 2) {
                const bool begins = s % PER_GROUP == 0;
                if constexpr (PER_GROUP == 1) {
                    part = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a.b[s].part[0]), __builtin_bit_cast(long, w[s]), i32x4{0, 0, 0, 0}, 0, 0, 0);
                } else {
                    const i32x4 x = {(int)a.b[s].part[0][0], (int)a.b[s].part[0][1], (int)a.b[s + 1].part[0][0], (int)a.b[s + 1].part[0][1]};
                    const i32x4 y = {(int)w[s][0], (int)w[s][1], (int)w[s + 1][0], (int)w[s + 1][1]};
                    part = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, begins ? i32x4{0, 0, 0, 0} : part, 0, 0, 0);
                }
                if (PER_GROUP < 4 || s == 2) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] += a.scale[s / PER_GROUP] * (float)part[i];
                }
            }
        } else {
            f32x4 part;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s % PER_GROUP == 0) part = f32x4{0, 0, 0, 0};
                if constexpr (BT == SPMM_F16) {
                    part = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.b[s].part[0]), weights_f16(a.word[s], a.zero[s / PER_GROUP]), part, 0, 0, 0);
                } else {
                    const bf16x8 w = weights_bf16(a.word[s], a.zero[s / PER_GROUP]);
#pragma unroll
                    for (int p = PARTS<BT> - 1; p >= 0; --p) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.b[s].part[p]), w, part, 0, 0, 0);
                }
                if (s % PER_GROUP == PER_GROUP - 1) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] += a.scale[s / PER_GROUP] * part[i];
                }
            }
        }
    };
    asked ring[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (first + i < last) ask(first + i, ring[i]);
    for (int b = first; b < last; b += AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (b + i >= last) break;
            use(ring[i]);
            if (b + i + AHEAD < last) ask(b + i + AHEAD, ring[i]);
        }
    }
    *reinterpret_cast<f32x4 *>(&sums[wave][lane * 4]) = acc;
    __syncthreads();
    // the waves' sums, in wave order: a thread an element of C
    if (threadIdx.x >= 256) return;
    const int e = threadIdx.x, m = C.by_token ? e % 16 : e / 16, t = C.by_token ? e / 16 : e % 16;
    const int64_t row = row_tile * TILE_ROWS + m;
    if (row >= W.M || t >= N) return;
    const int at = (t >> 2) * 64 + m * 4 + (t & 3);
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < KWAVES; ++w) v += sums[w][at];
    if (BT == SPMM_I8) v *= B_scales[t];
    store_as(C.data, C.by_token ? t * C.ld + row : row * C.ld + t, C.type, v);
}

template <int BT> hipError_t execute_few(const quant_matrix &w, const tensor &B, const float *B_scales, int64_t N, const tensor &C, hipStream_t stream)
{
    auto run = [&](auto per_group) {
        constexpr int PER_GROUP = decltype(per_group)::value;
        return launch_kernel(few_kernel<BT, PER_GROUP, 8>, dim3((unsigned)w.tiles), 512, 0, stream, w, B, B_scales, (int32_t)N, C);
    };
    if (w.group == 32) return run(std::integral_constant<int, 1>());
    if (w.group == 64) return run(std::integral_constant<int, 2>());
    return run(std::integral_constant<int, 4>());
}

template <int BT> hipError_t execute(const quant_matrix &w, const tensor &B, const float *B_scales, int64_t N, const tensor &C, char *workspace, hipStream_t stream)
{
    if (N <= 16) return execute_few<BT>(w, B, B_scales, N, C, stream);
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
        if (tiles <= 2) e = product(std::integral_constant<int, 2>());
        else if (tiles <= 4) e = product(std::integral_constant<int, 4>());
        else e = product(std::integral_constant<int, 8>());
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t quant_workspace(const quant_matrix &w, int32_t type, int64_t N)
{
    if (N <= 16) return 0;
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
