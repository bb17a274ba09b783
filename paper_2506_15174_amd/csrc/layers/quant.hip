// The product with 4-bit weights on the matrix cores (gfx950): C = W x B.
//
//   W[m, k] = scale[m, g] (code[m, k] - zero[m, g]),   C[m, n] = sum_g scale[m, g] sum_{k in g} (code - zero)[m, k] B[k, n]
//
// The inner sums are matrix instructions on whole numbers: code - zero lies in -15..15, which bf16, f16 and int8 hold
// exactly, so no weight is rounded; the outer sum is one fp32 multiply-add per element and group.  B is the first operand
// (its 16 tokens are the rows of an instruction), W the second: a lane then holds four tokens of one row of W and
// needs one scale a group.
//
// Up to 16 tokens, and somewhat more on short rows, go in one launch (direct_kernel): bound by a launch's few memory accesses, then by the weights' bytes.  More take two: pack_kernel
// lays B out as the instructions take it, then many_kernel, half of whose time B's way through the vector L1 takes, or, on prompts of all but fp32, wide_kernel, bound by the matrix cores and by
// the instructions that make operands of weights.
#include <algorithm>
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

// A launch has at most 65535 workgroups along its second axis, of four tiles of tokens or fewer.
constexpr int64_t MOST_TOKEN_TILES = 65535 / 8 * 8;

// ---- B as the instructions take it ---------------------------------------------------------------------------
//
// [token tile of 16][block of 128 columns][step of 32][part][lane][8 columns], 16 bytes a lane for 16-bit elements;
// codes hold two steps in the 16 bytes of a lane: [token tile][block][pair of steps][lane][step][8 columns].
// Lane 16 q + t holds token t, columns 32 s + 8 q + j.  Columns that do not exist are zeros.

// Eight columns of a token, as they are read.
template <int BT> struct raw {
    u32x4 v;
};
template <> struct raw<SPMM_F32> {
    float v[8];
};
template <> struct raw<SPMM_I8> {
    u32x2 v;
};

template <int BT> struct stored {
    typedef uint16_t type;
};
template <> struct stored<SPMM_F32> {
    typedef float type;
};
template <> struct stored<SPMM_I8> {
    typedef uint8_t type;
};

// Columns k0 .. k0 + 7 of a token whose column 0 lies at `base`; `ld` bytes from one column to the next where a row of memory is a feature.
// TAIL: of columns 0 .. `left` - 1 only; the others are 0 (and read at the last one's place).
template <int BT, bool BY_TOKEN, bool TAIL> __device__ inline raw<BT> fetch(const char *base, int64_t ld, int k0, int left)
{
    typedef typename stored<BT>::type T;
    raw<BT> o;
    T x[8];
    if constexpr (BY_TOKEN && !TAIL) {
        const neighbours<T, 8> n = *reinterpret_cast<const neighbours<T, 8> *>(base + k0 * (int)sizeof(T));
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = n.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = TAIL ? min(k0 + j, left - 1) : k0 + j;
            x[j] = *reinterpret_cast<const T *>(base + k * (BY_TOKEN ? (int64_t)sizeof(T) : ld));
            if (TAIL && k0 + j >= left) x[j] = 0;
        }
    }
    if constexpr (BT == SPMM_F32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j] = x[j];
    } else {
        constexpr int EACH = 4 / (int)sizeof(T);
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j / EACH] = (j % EACH ? o.v[j / EACH] : 0u) | (uint32_t)x[j] << (32 / EACH * (j % EACH));
    }
    return o;
}

// The same as operands of matrix instructions, a part each; codes are eight bytes.
template <int BT> struct operands {
    u32x4 part[PARTS<BT>];
};
template <> struct operands<SPMM_I8> {
    u32x2 part[1];
};

// A value in a register of its own.  Without this the compiler (ROCm 7.2) gave operands made of a wide load's words the load's own registers and wrote the first
// before it read the last: v18 = perm(v39, v38), then v20 = perm(v19, v18), where v18 to v21 held the words 4 to 7.  (That was an earlier form of the callers; the assembly of the
// present ones has no such place with it or without.  It costs some moves, 2 % of all instructions here; the cause is not known.)
__device__ inline uint32_t apart(uint32_t v)
{
    asm("" : "+v"(v));
    return v;
}

// What lanes of a wave have written to LDS is there for its other lanes: the hardware takes a wave's accesses to LDS in order, so this only keeps the compiler from changing it.  (Accesses to
// other memory may pass.)
__device__ inline void lanes_in_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

template <int BT> __device__ inline operands<BT> operands_of(const raw<BT> &x)
{
    operands<BT> o;
    if constexpr (BT == SPMM_I8) {
        // the order in which the weights' nibbles become bytes: 0 4 1 5, 2 6 3 7
        const uint32_t low = apart(x.v[0]), high = apart(x.v[1]);
        o.part[0] = u32x2{__builtin_amdgcn_perm(high, low, 0x05010400u), __builtin_amdgcn_perm(high, low, 0x07030602u)};
    } else if constexpr (BT == SPMM_F32) {
        // Each part is the upper half of what is left: cut off, not rounded, so that large values stay finite.
        uint32_t first[8], second[8], third[8], largest = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            first[j] = apart(__builtin_bit_cast(uint32_t, x.v[j]));
            largest = max(largest, first[j] & 0x7fffffffu);
            const float left = x.v[j] - __builtin_bit_cast(float, first[j] & 0xffff0000u);
            second[j] = __builtin_bit_cast(uint32_t, left);
            third[j] = __builtin_bit_cast(uint32_t, left - __builtin_bit_cast(float, second[j] & 0xffff0000u));
        }
        if (largest >= 0x7f800000u) {  // an infinity or a NaN is the first part's alone
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t magnitude = first[j] & 0x7fffffffu;
                first[j] = magnitude > 0x7f800000u ? 0x7fc00000u : first[j];
                second[j] = magnitude >= 0x7f800000u ? 0 : second[j];
                third[j] = magnitude >= 0x7f800000u ? 0 : third[j];
            }
        }
        auto upper = [](const uint32_t (&v)[8]) {
            constexpr uint32_t HALVES = 0x07060302u;
            return u32x4{__builtin_amdgcn_perm(v[1], v[0], HALVES), __builtin_amdgcn_perm(v[3], v[2], HALVES), __builtin_amdgcn_perm(v[5], v[4], HALVES),
                         __builtin_amdgcn_perm(v[7], v[6], HALVES)};
        };
        o.part[0] = upper(first), o.part[1] = upper(second), o.part[2] = upper(third);
    } else {
        o.part[0] = x.v;
    }
    return o;
}

template <int BT, bool BY_TOKEN> __global__ __launch_bounds__(256) void pack_kernel(tensor B, int64_t K, int64_t N, int32_t blocks, char *out)
{
    constexpr int64_t SIZE = sizeof(typename stored<BT>::type);
    const int lane = threadIdx.x & 63, s = threadIdx.x >> 6, t = lane & 15, q = lane >> 4;
    const int64_t block = blockIdx.x, tile = blockIdx.y, n = tile * 16 + t;
    char *block_out = out + (tile * blocks + block) * (4 * PARTS<BT> * STEP_BYTES<BT>);
    const int left = (int)min((int64_t)BLOCK_COLS, K - block * BLOCK_COLS);
    // tokens that do not exist: the last one's (what they give is not stored)
    const char *base = B.data + (min(n, N - 1) * (BY_TOKEN ? B.ld : 1) + block * BLOCK_COLS * (BY_TOKEN ? 1 : B.ld)) * SIZE;
    const operands<BT> o = operands_of<BT>(left == BLOCK_COLS ? fetch<BT, BY_TOKEN, false>(base, B.ld * SIZE, 32 * s + 8 * q, left) :
                                                                fetch<BT, BY_TOKEN, true>(base, B.ld * SIZE, 32 * s + 8 * q, left));
    if constexpr (BT == SPMM_I8) {
        *reinterpret_cast<u32x2 *>(block_out + (s >> 1) * 1024 + lane * 16 + (s & 1) * 8) = o.part[0];
    } else {
#pragma unroll
        for (int p = 0; p < PARTS<BT>; ++p) *reinterpret_cast<u32x4 *>(block_out + (s * PARTS<BT> + p) * 1024 + lane * 16) = o.part[p];
    }
}

// ---- weights as the instructions take them -------------------------------------------------------------------

// A nibble is code - 8 in two's complement: `zero` is the zero point.

// code - zero of eight columns in f16: 1024 + code is a mask away (its last bit is worth 1), the difference is exact.
__device__ inline f16x8 weights_f16(uint32_t w, int zero)
{
    const _Float16 z = (_Float16)(float)(1024 + zero);
    const f16x2 base = {z, z};
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, ((w >> (4 * i)) & 0x000f000fu) ^ 0x64086408u) - base);
    return __builtin_bit_cast(f16x8, u32x4{v[0], v[1], v[2], v[3]});
}

// (code - 8) / 16 of the low nibble of byte I, which the hardware has an instruction for.
template <int I> __device__ inline float sixteenths(uint32_t w)
{
    float f;
    if constexpr (I == 0) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(w));
    if constexpr (I == 1) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(w));
    if constexpr (I == 2) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(w));
    if constexpr (I == 3) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(w));
    return f;
}

// (code - zero) / 16 of eight columns in fp32 (WEIGHT_UNIT makes up for the 16).  ZEROS: the plan has zero points, else they are 8.
template <bool ZEROS> __device__ inline void weights_f32(uint32_t w, int zero, float (&v)[8])
{
    const uint32_t odd = w >> 4;  // nibbles 0 2 4 6 are columns 0 4 1 5, the others 2 6 3 7
    v[0] = sixteenths<0>(w), v[4] = sixteenths<1>(w), v[1] = sixteenths<2>(w), v[5] = sixteenths<3>(w);
    v[2] = sixteenths<0>(odd), v[6] = sixteenths<1>(odd), v[3] = sixteenths<2>(odd), v[7] = sixteenths<3>(odd);
    if constexpr (ZEROS) {
        const float less = (float)(zero - 8) * 0.0625f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] -= less;
    }
}

// The same in bf16: the upper half of the fp32, which holds it exactly.
template <bool ZEROS> __device__ inline bf16x8 weights_bf16(uint32_t w, int zero)
{
    float v[8];
    weights_f32<ZEROS>(w, zero, v);
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[2 * i + 1]), __builtin_bit_cast(uint32_t, v[2 * i]), 0x07060302u);
    return __builtin_bit_cast(bf16x8, u32x4{o[0], o[1], o[2], o[3]});
}

// code - zero in bytes, columns in the order 0 4 1 5, 2 6 3 7: no borrow leaves a byte that has 128 added.
__device__ inline u32x2 weights_i8(uint32_t w, uint32_t zero4)
{
    u32x2 v;
    v[0] = (((w & 0x0f0f0f0fu) ^ 0x88888888u) - zero4) ^ 0x80808080u;
    v[1] = ((((w >> 4) & 0x0f0f0f0fu) ^ 0x88888888u) - zero4) ^ 0x80808080u;
    return v;
}

// What a lane's row has in a span of K: a scale and a zero point for each group.
template <int GROUPS, bool ZEROS> struct span_values {
    float scale[GROUPS];
    uint32_t zeros;  // a byte each
    __device__ int zero(int g) const { return ZEROS ? (int)(zeros >> (8 * g) & 15u) : 8; }
};

// Of row r of a tile of rows, at the span that holds `block`.
template <int GROUPS, bool ZEROS> __device__ inline span_values<GROUPS, ZEROS> span_of(const quant_matrix &W, int64_t tile, int block, int r)
{
    const int span = GROUPS > 1 || W.group == BLOCK_COLS ? block : block / (int)(W.group / BLOCK_COLS);
    const int64_t at = (tile * W.spans + span) * (TILE_ROWS * GROUPS);
    span_values<GROUPS, ZEROS> v;
    const neighbours<float, GROUPS> s = reinterpret_cast<const neighbours<float, GROUPS> *>(W.scales + at)[r];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) v.scale[g] = s.v[g];
    v.zeros = 0;
    if constexpr (ZEROS) {
        typedef std::conditional_t<GROUPS == 4, uint32_t, std::conditional_t<GROUPS == 2, uint16_t, uint8_t>> packed;
        v.zeros = reinterpret_cast<const packed *>(W.zeros + at)[r];
    }
    return v;
}

// What a whole number of the products' second operand stands for.
template <int BT> constexpr float WEIGHT_UNIT = BT == SPMM_F32 || BT == SPMM_BF16 ? 16.0f : 1.0f;

// ---- many tokens -----------------------------------------------------------------------------------------------
//
// A wave has RT tiles of rows and NT tiles of tokens, a workgroup KWAVES such waves that share K; their sums meet in LDS.  Weights become operands once a block and
// are used for all of its tokens, B (laid out by pack_kernel) comes a tile of tokens at a time, the next one while one is multiplied.  With the layout of B: 4096 x 4096, 128 tokens
// in bf16 14.0 us, 307 TF; 8192 x 8192, 512 in fp32 220 us, 312 TF (three products of bf16 for each).  8192 x 8192, 128 in bf16, 37 us: of 94 k clocks the address unit before the vector L1 is busy 50 k, vector
// instructions issue for 44 k, matrix instructions take 16 k; waves wait for memory half of their time.

template <int BT, int NT, int RT, int KWAVES, int STEPS, bool ZEROS> __global__ __launch_bounds__(64 * KWAVES) void many_kernel(quant_matrix W, const char *B, const float *B_scales, int64_t N,
                                                                                                                          tensor C)
{
    // K goes by pieces of STEPS steps of 32 columns, which lie in one group.
    extern __shared__ float sums[];  // [KWAVES][RT][NT][256]
    constexpr int PIECES = 4 / STEPS, P = PARTS<BT>, BLOCK_BYTES = 4 * P * STEP_BYTES<BT>, LOADS = BT == SPMM_I8 ? (STEPS + 1) / 2 : STEPS * P;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int64_t token_tiles = (N + 15) / 16, token0 = (int64_t)blockIdx.y * NT, tile0 = (int64_t)blockIdx.x * RT;
    const int pieces = W.blocks * PIECES;
    const int first = (int)((int64_t)pieces * wave / KWAVES), last = (int)((int64_t)pieces * (wave + 1) / KWAVES);
    const uint32_t *const codes = W.codes + tile0 * W.blocks * BLOCK_WORDS;
    struct asked {
        uint32_t word[RT][STEPS];
        float scale[RT];
        int zero[RT];
    };
    auto ask = [&](int piece, asked &a) {
        const int block = piece / PIECES, of_block = piece % PIECES, span = PIECES > 1 || W.group == BLOCK_COLS ? block : block / (int)(W.group / BLOCK_COLS);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const uint32_t *at = codes + ((int64_t)i * W.blocks + block) * BLOCK_WORDS + of_block * STEPS + lane * 4;
            if constexpr (STEPS == 4) {
                const u32x4 v = *reinterpret_cast<const u32x4 *>(at);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) a.word[i][s] = v[s];
            } else if constexpr (STEPS == 2) {
                const u32x2 v = *reinterpret_cast<const u32x2 *>(at);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) a.word[i][s] = v[s];
            } else {
                a.word[i][0] = *at;
            }
            const int64_t values = ((tile0 + i) * W.spans + span) * (TILE_ROWS * PIECES) + of_block;
            a.scale[i] = (W.scales + values)[r * PIECES] * WEIGHT_UNIT<BT>;
            a.zero[i] = ZEROS ? (W.zeros + values)[r * PIECES] : 8;
        }
    };
    // Tiles of tokens past the last: the last one again (not stored).  Codes of one step are half of a lane's 16 bytes.
    auto ask_tokens = [&](int piece, int t, u32x4(&x)[LOADS]) {
        const char *at = B + (min(token0 + t, token_tiles - 1) * W.blocks + piece / PIECES) * BLOCK_BYTES;
        if constexpr (BT == SPMM_I8 && STEPS == 1) {
            const u32x2 v = *reinterpret_cast<const u32x2 *>(at + piece % PIECES / 2 * 1024 + lane * 16 + piece % 2 * 8);
            x[0][0] = v[0], x[0][1] = v[1];
        } else {
            at += piece % PIECES * (STEPS * P * STEP_BYTES<BT>);
#pragma unroll
            for (int l = 0; l < LOADS; ++l) x[l] = reinterpret_cast<const u32x4 *>(at + l * 1024)[lane];
        }
    };
    f32x4 acc[RT][NT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0, 0, 0, 0};
    asked now, next;
    // B of AHEAD tiles of tokens is on its way while one is multiplied: what the registers hold
    constexpr int AHEAD = 2;
    static_assert(NT % AHEAD == 0);
    u32x4 x[AHEAD][LOADS];
    if (first < last) {
        ask(first, now);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) ask_tokens(first, t, x[t]);
    }
    for (int piece = first; piece < last; ++piece) {
        if (piece + 1 < last) ask(piece + 1, next);
        // W as operands: four words of a step, of two steps for codes
        u32x4 w[RT][STEPS];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                if constexpr (BT == SPMM_I8) {
                    const u32x2 v = weights_i8(now.word[i][s], (uint32_t)now.zero[i] * 0x01010101u);
                    w[i][s / 2][2 * (s % 2)] = v[0], w[i][s / 2][2 * (s % 2) + 1] = v[1];
                } else if constexpr (BT == SPMM_F16) {
                    w[i][s] = __builtin_bit_cast(u32x4, weights_f16(now.word[i][s], now.zero[i]));
                } else {
                    w[i][s] = __builtin_bit_cast(u32x4, weights_bf16<ZEROS>(now.word[i][s], now.zero[i]));
                }
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            u32x4(&a)[LOADS] = x[t % AHEAD];
            if constexpr (BT == SPMM_I8) {
                i32x4 part[RT];
                if constexpr (STEPS == 1) {
#pragma unroll
                    for (int i = 0; i < RT; ++i)
                        part[i] = __builtin_amdgcn_mfma_i32_16x16x32_i8((long)((uint64_t)a[0][0] | (uint64_t)a[0][1] << 32), (long)((uint64_t)w[i][0][0] | (uint64_t)w[i][0][1] << 32),
                                                                        i32x4{0, 0, 0, 0}, 0, 0, 0);
                } else {
#pragma unroll
                    for (int s = 0; s < STEPS / 2; ++s)
#pragma unroll
                        for (int i = 0; i < RT; ++i)
                            part[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a[s]), __builtin_bit_cast(i32x4, w[i][s]), s == 0 ? i32x4{0, 0, 0, 0} : part[i], 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][t][e] += now.scale[i] * (float)part[i][e];
            } else {
                f32x4 part[RT];
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            const f32x4 from = s == 0 && p == P - 1 ? f32x4{0, 0, 0, 0} : part[i];
                            if constexpr (BT == SPMM_F16) part[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a[s]), __builtin_bit_cast(f16x8, w[i][s]), from, 0, 0, 0);
                            else part[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[s * P + p]), __builtin_bit_cast(bf16x8, w[i][s]), from, 0, 0, 0);
                        }
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][t][e] += now.scale[i] * part[i][e];
            }
            if (t + AHEAD < NT) ask_tokens(piece, t + AHEAD, x[t % AHEAD]);
            else if (piece + 1 < last) ask_tokens(piece + 1, t + AHEAD - NT, x[t % AHEAD]);
        }
        now = next;
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(sums + ((wave * RT + i) * NT + t) * 256 + lane * 4) = acc[i][t];
    __syncthreads();
    // the waves' sums, in wave order: a thread an element of C
    for (int e = threadIdx.x; e < RT * NT * 256; e += 64 * KWAVES) {
        const int m = C.by_token ? e % (16 * RT) : e / (16 * NT), t = C.by_token ? e / (16 * RT) : e % (16 * NT);
        const int64_t row = tile0 * TILE_ROWS + m, n = token0 * 16 + t;
        if (row >= W.M || n >= N) continue;
        const int at = ((m / 16) * NT + t / 16) * 256 + ((t & 15) >> 2) * 64 + (m % 16) * 4 + (t & 3);
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < KWAVES; ++w) v += sums[w * RT * NT * 256 + at];
        if (BT == SPMM_I8) v *= B_scales[n];
        store_as(C.data, C.by_token ? n * C.ld + row : row * C.ld + n, C.type, v);
    }
}

// ---- prompts -----------------------------------------------------------------------------------------------------
//
// A wave has 16 tiles of sums, NT of tokens beside 16 / NT of rows.  Of a workgroup's eight, teams of SHARE lie one below the other and share the tokens' B; K is split over the
// 8 / SHARE teams, whose sums meet in LDS at the end.  B goes through LDS, since without sharing it would take all of the vector L1's 64 bytes a clock; a block of 128 columns is on its
// way there while the block before is multiplied.  A team waits for its own waves only: with a barrier for the workgroup 8192 x 8192, 512 tokens, took 105 us, without 89 (teams of two;
// a second block on its way, with which waves of a team may be a block apart, gained nothing).  Weights are made operands by each wave for itself, 13 instructions for a tile of rows and
// 32 columns, which matrix instructions share with NT tiles of tokens: 128 tokens a wave instead of 64 take 81 us and 83, in teams of eight 142 and 150 on 1024 (LDS does not hold
// them for teams of two).  8192 x 8192, 512 in bf16: of 175 k clocks a SIMD's matrix instructions take 65 k (37 %), 15 k other vector instructions of 4 clocks 60 k; waves wait for memory or LDS 31 % of
// their time and to issue 31 %.  Putting the two kinds in turn by the program gained nothing (with 64 tokens a wave).
// 8192 x 8192 in bf16, with 6 us to lay out B for 512 tokens: 512 79 us, 870 TF; 4096 544, 1010 TF; in codes 512 57 us, 1210 TOPS, 2048 198 us, 1390 TOPS.

constexpr int WIDE_LDS = 128 * 1024;

template <int BT, int SHARE, int NT, int STEPS, bool ZEROS> __global__ __launch_bounds__(512) void wide_kernel(quant_matrix W, const char *B, const float *B_scales, int64_t N, tensor C)
{
    extern __shared__ __align__(16) char lds[];
    constexpr int TEAMS = 8 / SHARE, RT = 16 / NT, SUMS = 4 / STEPS, BLOCK_BYTES = 4 * STEP_BYTES<BT>, OF_TILE = BLOCK_BYTES / 1024, STAGE = NT * BLOCK_BYTES, EACH = STAGE / 1024 / SHARE;
    static_assert(BT != SPMM_F32 && EACH * SHARE == NT * OF_TILE && 2 * TEAMS * STAGE <= WIDE_LDS && 8 * RT * NT * 1024 == WIDE_LDS && RT <= TILES_OF);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int member = wave % SHARE, team = wave / SHARE;
    const int64_t token_tiles = (N + 15) / 16, token0 = (int64_t)blockIdx.y * NT, wg_tile0 = (int64_t)blockIdx.x * (SHARE * RT);
    // (a wave whose rows do not exist has the last ones)
    const int64_t tile0 = min(wg_tile0 + member * RT, ((int64_t)W.tiles - 1) / RT * RT);
    const int first = (int)((int64_t)W.blocks * team / TEAMS), last = (int)((int64_t)W.blocks * (team + 1) / TEAMS);
    __shared__ int arrived[8];  // blocks whose share of B a wave has brought
    if (threadIdx.x < 8) arrived[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t *const codes = W.codes + tile0 * W.blocks * BLOCK_WORDS;
    struct asked {
        u32x4 word[RT];
        span_values<SUMS, ZEROS> span[RT];
    };
    auto ask = [&](int b, asked &a) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            a.word[i] = reinterpret_cast<const u32x4 *>(codes + ((int64_t)i * W.blocks + b) * BLOCK_WORDS)[lane];
            a.span[i] = span_of<SUMS, ZEROS>(W, tile0 + i, b, r);
        }
    };
    // This wave's share of a block of B, straight to LDS: [place][team][tile of tokens][a block of it]
    auto place_of = [&](int place) { return lds + (place * TEAMS + team) * STAGE; };
    auto send = [&](int b, int place) {
#pragma unroll
        for (int l = 0; l < EACH; ++l) {
            const int at = member * EACH + l;
            const char *from = B + (min(token0 + at / OF_TILE, token_tiles - 1) * W.blocks + b) * BLOCK_BYTES + at % OF_TILE * 1024 + lane * 16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)(place_of(place) + at * 1024), 16, 0, 0);
        }
    };
    typedef std::conditional_t<BT == SPMM_I8, i32x4, f32x4> sum;
    f32x4 acc[RT][NT];
    sum part[RT][NT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0, 0, 0, 0};
    asked now, next;
    constexpr int AT_ONCE = BT == SPMM_I8 && STEPS > 1 ? 2 : 1;  // steps that go into one instruction
    if (first < last) {
        send(first, 0);
        ask(first, now);
    }
    for (int b = first; b < last; ++b) {
        const int round = b - first;
        // This wave's share of the block is there (and what it asked for besides), then the team's; all of them have read the block before.
        // (The wait ends: a workgroup's waves are all on the compute unit, have as many blocks as their team, and say that they arrived before they wait.)
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __hip_atomic_store(&arrived[wave], round + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        if (b + 1 < last) ask(b + 1, next);
        while (!__all(__hip_atomic_load(&arrived[team * SHARE + lane % SHARE], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) > round)) {}
        asm volatile("" ::: "memory");
        if (b + 1 < last) send(b + 1, (round + 1) & 1);
        const char *const from = place_of(round & 1) + lane * 16;
#pragma unroll
        for (int s = 0; s < 4; s += AT_ONCE) {
            // (scales of several groups, zero points in f16: no registers for two steps at a time)
            if (STEPS < 4 || (BT == SPMM_F16 && ZEROS)) __builtin_amdgcn_sched_barrier(0);
            if constexpr (BT == SPMM_I8) {
                i32x4 x[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) x[t] = *reinterpret_cast<const i32x4 *>(from + t * BLOCK_BYTES + s / 2 * 1024);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const u32x2 w0 = weights_i8(now.word[i][s], (uint32_t)now.span[i].zero(s / STEPS) * 0x01010101u);
                    if constexpr (STEPS == 1) {
#pragma unroll
                        for (int t = 0; t < NT; ++t)
                            part[i][t] = __builtin_amdgcn_mfma_i32_16x16x32_i8((long)((uint64_t)(uint32_t)x[t][2 * (s % 2)] | (uint64_t)(uint32_t)x[t][2 * (s % 2) + 1] << 32),
                                                                               __builtin_bit_cast(long, w0), sum{0, 0, 0, 0}, 0, 0, 0);
                    } else {
                        const u32x2 w1 = weights_i8(now.word[i][s + 1], (uint32_t)now.span[i].zero(s / STEPS) * 0x01010101u);
                        const i32x4 w = {(int)w0[0], (int)w0[1], (int)w1[0], (int)w1[1]};
#pragma unroll
                        for (int t = 0; t < NT; ++t) part[i][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[t], w, s % STEPS == 0 ? sum{0, 0, 0, 0} : part[i][t], 0, 0, 0);
                    }
                }
            } else {
                u32x4 w[RT], x[NT];
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    if constexpr (BT == SPMM_F16) w[i] = __builtin_bit_cast(u32x4, weights_f16(now.word[i][s], now.span[i].zero(s / STEPS)));
                    else w[i] = __builtin_bit_cast(u32x4, weights_bf16<ZEROS>(now.word[i][s], now.span[i].zero(s / STEPS)));
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) x[t] = *reinterpret_cast<const u32x4 *>(from + t * BLOCK_BYTES + s * 1024);
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const sum c = s % STEPS == 0 ? sum{0, 0, 0, 0} : part[i][t];
                        if constexpr (BT == SPMM_F16) part[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x[t]), __builtin_bit_cast(f16x8, w[i]), c, 0, 0, 0);
                        else part[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[t]), __builtin_bit_cast(bf16x8, w[i]), c, 0, 0, 0);
                    }
            }
            if ((s + AT_ONCE) % STEPS == 0) {
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][t][e] += now.span[i].scale[s / STEPS] * WEIGHT_UNIT<BT> * (float)part[i][t][e];
            }
        }
        now = next;
    }
    // The teams' sums meet in LDS: [team][tile of rows][tile of tokens][256]
    __syncthreads();
    float *const sums = reinterpret_cast<float *>(lds);
    constexpr int ROW_TILES = SHARE * RT;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(sums + ((team * ROW_TILES + member * RT + i) * NT + t) * 256 + lane * 4) = acc[i][t];
    __syncthreads();
    for (int e = threadIdx.x; e < ROW_TILES * NT * 256; e += 512) {
        const int m = C.by_token ? e % (16 * ROW_TILES) : e / (16 * NT), t = C.by_token ? e / (16 * ROW_TILES) : e % (16 * NT);
        const int64_t row = wg_tile0 * TILE_ROWS + m, n = token0 * 16 + t;
        if (row >= W.M || n >= N) continue;
        const int at = ((m / 16) * NT + t / 16) * 256 + ((t & 15) >> 2) * 64 + (m % 16) * 4 + (t & 3);
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < TEAMS; ++k) v += sums[k * ROW_TILES * NT * 256 + at];
        if (BT == SPMM_I8) v *= B_scales[n];
        store_as(C.data, C.by_token ? n * C.ld + row : row * C.ld + n, C.type, v);
    }
}

template <int V> using constant = std::integral_constant<int, V>;

// ---- in one launch ---------------------------------------------------------------------------------------------
//
// A product of few tokens is over in the time of a few memory accesses, of which a launch is two or three: every wave reads its columns of
// B as it reads its weights and makes operands of them itself.  In bf16, one token, weights from memory: 4096 x 4096 4.9 us, 1.8 TB/s of weights and scales; 8192 x 8192 10.9 us, 3.3 TB/s; 16384 x 16384
// 37 us, 3.9 TB/s, where a large copy reaches 5.1 (from the Infinity Cache 3.5 and 9.1 us).  Lanes of tokens that do not exist read the last one's (an access the
// wave makes anyway); their results are not stored.  Weights, scales and B of AHEAD blocks are asked for before the first is used.
//   PER_GROUP  steps of 32 columns behind which a group's sum is full (4, 2 or 1)
//   RT, NT     tiles of rows and of tokens of a wave
//   FMA        one token in fp32 is multiplied by ordinary instructions, a lane a row and a quarter of the columns: making three parts of a value
//              takes six
//   KWAVES     waves of a workgroup, which share K

template <int BT, bool BY_TOKEN, int PER_GROUP, int RT, int NT, int KWAVES, int AHEAD, bool FMA, bool STAGED, bool ZEROS> __global__ __launch_bounds__(64 * KWAVES) void direct_kernel(quant_matrix W, tensor B, const float *B_scales, int64_t N, tensor C)
{
    __shared__ float sums[KWAVES][RT][NT][256], token_scales[BT == SPMM_I8 ? 16 * NT : 1];
    constexpr int SUMS = 4 / PER_GROUP;
    constexpr int64_t SIZE = sizeof(typename stored<BT>::type);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int first = (int)((int64_t)W.blocks * wave / KWAVES), last = (int)((int64_t)W.blocks * (wave + 1) / KWAVES);
    // (the plan's memory has whole fours of row tiles)
    const int64_t tile0 = (int64_t)blockIdx.x * RT;
    const uint32_t *const codes = W.codes + tile0 * W.blocks * BLOCK_WORDS;
    const int64_t column = (BY_TOKEN ? 1 : B.ld) * SIZE;  // bytes from one to the next
    const int64_t n0 = (int64_t)blockIdx.y * (16 * NT);
    const char *token[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) token[t] = B.data + (FMA ? 0 : min(n0 + 16 * t + r, N - 1)) * (BY_TOKEN ? B.ld : 1) * SIZE;
    if (BT == SPMM_I8 && threadIdx.x < 16 * NT) token_scales[threadIdx.x] = B_scales[min(n0 + (int64_t)threadIdx.x, N - 1)];
    // STAGED, for one tile of tokens, one a row of memory: a load of operands touches all 16 rows for 8 to 32 bytes each, and the vector L1 takes 3 clocks a row.  So
    // lanes read along the rows instead, 16 bytes each, and operands change places in LDS.  (Rows that do not exist are read as the last one and cost nothing.)
    static_assert(!STAGED || (BY_TOKEN && NT == 1 && !FMA));
    constexpr int ROW_LANES = 8 * (int)SIZE, ROWS_AT_ONCE = 64 / ROW_LANES, PIECES = 16 / ROWS_AT_ONCE, PART_SIZE = BT == SPMM_I8 ? 1 : 2, PITCH = BLOCK_COLS * PART_SIZE + 16;
    __shared__ __align__(16) char staged[STAGED ? KWAVES * PARTS<BT> * 16 * PITCH : 16];
    struct asked {
        u32x4 word[RT];
        span_values<SUMS, ZEROS> span[RT];
        raw<BT> b[NT][4];       // operands as they are read
        u32x4 piece[PIECES];    // STAGED: pieces of rows
    };
    auto ask = [&](int b, asked &a, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if constexpr (STAGED && !TAIL) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int row = min(p * ROWS_AT_ONCE + lane / ROW_LANES, (int)N - 1);
                a.piece[p] = __builtin_bit_cast(u32x4, *reinterpret_cast<const neighbours<typename stored<BT>::type, 16 / SIZE> *>(B.data + row * B.ld * SIZE + (int64_t)b * (BLOCK_COLS * SIZE) + lane % ROW_LANES * 16));
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) a.word[i] = reinterpret_cast<const u32x4 *>(codes + ((int64_t)i * W.blocks + b) * BLOCK_WORDS)[lane];
        const int left = (int)(W.K - (int64_t)b * BLOCK_COLS);
        if constexpr (!STAGED || TAIL)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < 4; ++s) a.b[t][s] = fetch<BT, BY_TOKEN, TAIL>(token[t] + (b * BLOCK_COLS + (TAIL ? 0 : 8 * q)) * column, column, 32 * s + (TAIL ? 8 * q : 0), left);
#pragma unroll
        for (int i = 0; i < RT; ++i) a.span[i] = span_of<SUMS, ZEROS>(W, tile0 + i, b, r);
    };
    f32x4 acc[RT][NT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0, 0, 0, 0};
    auto use = [&](const asked &a, auto tail) {
        operands<BT> o[NT][4];
        if constexpr (STAGED && !decltype(tail)::value) {
            char *const mine = staged + wave * (PARTS<BT> * 16 * PITCH);
            lanes_in_lds();  // (the lanes' reads of the block before)
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                char *const to = mine + (p * ROWS_AT_ONCE + lane / ROW_LANES) * PITCH + lane % ROW_LANES * (16 / SIZE * PART_SIZE);
                if constexpr (BT == SPMM_F32) {
                    raw<BT> x = {};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t bits = a.piece[p][j];  // (a bit cast of a vector's element itself is one of its first)
                        x.v[j] = __builtin_bit_cast(float, bits);
                    }
                    const operands<BT> parts = operands_of<BT>(x);
#pragma unroll
                    for (int part = 0; part < 3; ++part) *reinterpret_cast<u32x2 *>(to + part * 16 * PITCH) = u32x2{parts.part[part][0], parts.part[part][1]};
                } else {
                    *reinterpret_cast<u32x4 *>(to) = a.piece[p];
                }
            }
            lanes_in_lds();
            const char *const from = mine + r * PITCH + 8 * q * PART_SIZE;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if constexpr (BT == SPMM_I8) {
                    o[0][s] = operands_of<BT>(raw<BT>{*reinterpret_cast<const u32x2 *>(from + 32 * s)});
                } else {
#pragma unroll
                    for (int part = 0; part < PARTS<BT>; ++part) o[0][s].part[part] = *reinterpret_cast<const u32x4 *>(from + part * 16 * PITCH + 64 * s);
                }
            }
        }
        auto operand = [&](int t, int s) {
            if constexpr (STAGED && !decltype(tail)::value) return o[t][s];
            else return operands_of<BT>(a.b[t][s]);
        };
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            // (one tile's weights at a time: the registers do not hold all of them as operands)
            if (RT > 1) __builtin_amdgcn_sched_barrier(0);
            if constexpr (FMA) {
                float part = 0.0f;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    float w[8];
                    __builtin_amdgcn_sched_barrier(0);
                    weights_f32<ZEROS>(a.word[i][s], a.span[i].zero(s / PER_GROUP), w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) part = __builtin_fmaf(w[j], a.b[0][s].v[j], part);
                    if (s % PER_GROUP == PER_GROUP - 1) acc[i][0][0] += a.span[i].scale[s / PER_GROUP] * WEIGHT_UNIT<BT> * part, part = 0.0f;
                }
                continue;
            }
            u32x4 w[4];  // codes: two steps in one
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int zero = a.span[i].zero(s / PER_GROUP);
                if constexpr (BT == SPMM_I8) {
                    const u32x2 v = weights_i8(a.word[i][s], (uint32_t)zero * 0x01010101u);
                    w[s / 2][2 * (s % 2)] = v[0], w[s / 2][2 * (s % 2) + 1] = v[1];
                } else if constexpr (BT == SPMM_F16) {
                    w[s] = __builtin_bit_cast(u32x4, weights_f16(a.word[i][s], zero));
                } else {
                    w[s] = __builtin_bit_cast(u32x4, weights_bf16<ZEROS>(a.word[i][s], zero));
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (BT == SPMM_F32 && NT > 1) __builtin_amdgcn_sched_barrier(0);  // (nor three parts of two tiles of tokens)
                if constexpr (BT == SPMM_I8) {
                    i32x4 part;
#pragma unroll
                    for (int s = 0; s < 4; s += PER_GROUP == 1 ? 1 : 2) {
                        const u32x2 x0 = operand(t, s).part[0];
                        if constexpr (PER_GROUP == 1) {
                            const int h = 2 * (s % 2);
                            part = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, x0), (long)((uint64_t)w[s / 2][h] | (uint64_t)w[s / 2][h + 1] << 32), i32x4{0, 0, 0, 0}, 0, 0, 0);
                        } else {
                            const u32x2 x1 = operand(t, s + 1).part[0];
                            const i32x4 x = {(int)x0[0], (int)x0[1], (int)x1[0], (int)x1[1]};
                            part = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, __builtin_bit_cast(i32x4, w[s / 2]), s % PER_GROUP == 0 ? i32x4{0, 0, 0, 0} : part, 0, 0, 0);
                        }
                        if (PER_GROUP < 4 || s == 2) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][t][e] += a.span[i].scale[s / PER_GROUP] * (float)part[e];
                        }
                    }
                } else {
                    f32x4 part;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const operands<BT> x = operand(t, s);
                        if (s % PER_GROUP == 0) part = f32x4{0, 0, 0, 0};
#pragma unroll
                        for (int p = PARTS<BT> - 1; p >= 0; --p) {
                            if constexpr (BT == SPMM_F16) part = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x.part[p]), __builtin_bit_cast(f16x8, w[s]), part, 0, 0, 0);
                            else part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.part[p]), __builtin_bit_cast(bf16x8, w[s]), part, 0, 0, 0);
                        }
                        if (s % PER_GROUP == PER_GROUP - 1) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][t][e] += a.span[i].scale[s / PER_GROUP] * WEIGHT_UNIT<BT> * part[e];
                        }
                    }
                }
            }
        }
    };
    // The last block of a K that is no multiple of 128 comes by itself.
    const int whole = min(last, (int)(W.K / BLOCK_COLS));
    asked ring[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (first + i < whole) ask(first + i, ring[i], std::false_type());
    for (int b = first; b < whole; b += AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (b + i >= whole) break;
            use(ring[i], std::false_type());
            if (b + i + AHEAD < whole) ask(b + i + AHEAD, ring[i], std::false_type());
        }
    }
    if (whole < last) {
        ask(whole, ring[0], std::true_type());
        use(ring[0], std::true_type());
    }
    if constexpr (FMA) {  // the four quarters of the columns
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            acc[i][0][0] += __shfl_xor(acc[i][0][0], 16);
            acc[i][0][0] += __shfl_xor(acc[i][0][0], 32);
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(&sums[wave][i][t][lane * 4]) = acc[i][t];
    __syncthreads();
    // the waves' sums, in wave order: a thread an element of C
    for (int e = threadIdx.x; e < RT * NT * 256; e += 64 * KWAVES) {
        const int m = C.by_token ? e % (16 * RT) : e / (16 * NT), t = C.by_token ? e / (16 * RT) : e % (16 * NT);
        const int64_t row = tile0 * TILE_ROWS + m, n = n0 + t;
        if (row >= W.M || n >= N) continue;
        const int at = ((t & 15) >> 2) * 64 + (m % 16) * 4 + (t & 3);
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < KWAVES; ++w) v += sums[w][m / 16][t / 16][at];
        if (BT == SPMM_I8) v *= token_scales[t];
        store_as(C.data, C.by_token ? n * C.ld + row : row * C.ld + n, C.type, v);
    }
}

// Token by token of fp32 by multiply-adds, else on the matrix cores.  Tiles: a wave has more where workgroups are left over otherwise (256 compute units).
template <int BT, bool BY_TOKEN, bool FMA> hipError_t execute_direct(const quant_matrix &w, const tensor &B, const float *B_scales, int64_t N, const tensor &C, hipStream_t stream)
{
    auto shaped = [&](auto per_group, auto rt, auto nt, auto kwaves, auto ahead, auto staged) {
        constexpr int PER_GROUP = decltype(per_group)::value, RT = decltype(rt)::value, NT = decltype(nt)::value, KWAVES = decltype(kwaves)::value, AHEAD = decltype(ahead)::value;
        constexpr bool STAGED = decltype(staged)::value;
        const dim3 blocks((unsigned)((w.tiles + RT - 1) / RT), (unsigned)((N + 16 * NT - 1) / (16 * NT)));
        if (w.zeros) return launch_kernel(direct_kernel<BT, BY_TOKEN, PER_GROUP, RT, NT, KWAVES, AHEAD, FMA, STAGED, true>, blocks, 64 * KWAVES, 0, stream, w, B, B_scales, N, C);
        return launch_kernel(direct_kernel<BT, BY_TOKEN, PER_GROUP, RT, NT, KWAVES, AHEAD, FMA, STAGED, false>, blocks, 64 * KWAVES, 0, stream, w, B, B_scales, N, C);
    };
    auto run = [&](auto per_group) {
        constexpr int PER_GROUP = decltype(per_group)::value;
        constexpr std::false_type no = {};
        if constexpr (!FMA) {
            if (N > 16) return shaped(per_group, constant<1>(), constant<2>(), constant<8>(), constant<1>(), no);
        }
        // (what the registers hold)
        constexpr int AHEAD = BT == SPMM_F32 && !FMA ? 1 : 2, LESS = PER_GROUP < 4 || FMA ? 1 : AHEAD;
        constexpr int MOST = PER_GROUP == 1 || (BT == SPMM_F32 && !BY_TOKEN) ? 2 : 4;
        // STAGED or straight, us.  1024 x 4096: one token in codes 3.4 and 3.6, 16 3.6 and 6.2; in bf16 one 4.1 and 3.6, 4 4.1 and 4.2, 16 4.4 and 6.2.  8192 x 8192, two tiles of rows: 16 in codes
        // 10.3 and 12.3, in bf16 8 11.7 and 11.1, 16 12.3 and 13.0.  With four tiles a wave B is read less often: 16384 x 16384, one in codes 37.7 and 34.3, 16 34.8 and 34.9.  fp32, whose parts
        // are made once then: 3 on 1024 x 4096 8.8 and 7.7, on 8192 x 8192 21.5 and 24.7, on 16384 x 16384 54 and 90.  256 x 256, where all is one wait: 2.5 and 2.4, fp32 3.8 and 3.3.
        constexpr std::bool_constant<BY_TOKEN && !FMA> yes = {};
        constexpr std::bool_constant<yes() && BT == SPMM_F32> parts = {};
        constexpr bool SPLIT = BY_TOKEN && BT != SPMM_F32, HALF = SPLIT && BT != SPMM_I8;
        if (w.tiles >= 1024) return shaped(per_group, constant<MOST>(), constant<1>(), constant<8>(), constant<LESS>(), parts);
        if constexpr (HALF) {
            if (w.tiles >= 512 && N <= 8) return shaped(per_group, constant<2>(), constant<1>(), constant<8>(), constant<AHEAD>(), no);
            if (w.tiles < 512 && w.blocks > 8 && N <= 4) return shaped(per_group, constant<1>(), constant<1>(), constant<16>(), constant<LESS>(), no);
        }
        if (w.tiles >= 512) return shaped(per_group, constant<2>(), constant<1>(), constant<8>(), constant<AHEAD>(), yes);
        if constexpr (SPLIT) {
            if (w.blocks > 8) return shaped(per_group, constant<1>(), constant<1>(), constant<16>(), constant<LESS>(), yes);
        }
        return shaped(per_group, constant<1>(), constant<1>(), constant<8>(), constant<1>(), no);
    };
    if (w.group == 32) return run(constant<1>());
    if (w.group == 64) return run(constant<2>());
    return run(constant<4>());
}

template <int BT, int NT, int RT, int KWAVES> hipError_t launch_many(const quant_matrix &w, const char *B, const float *B_scales, int64_t N, const tensor &C, hipStream_t stream)
{
    const dim3 blocks((unsigned)((w.tiles + RT - 1) / RT), (unsigned)((N + 16 * NT - 1) / (16 * NT)));
    auto shaped = [&](auto per_group, auto zeros) {
        constexpr int PER_GROUP = decltype(per_group)::value;
        constexpr bool ZEROS = decltype(zeros)::value;
        constexpr unsigned LDS = KWAVES * RT * NT * 1024;
        return launch_kernel(many_kernel<BT, NT, RT, KWAVES, PER_GROUP, ZEROS>, blocks, 64 * KWAVES, LDS, stream, w, B, B_scales, N, C);
    };
    auto run = [&](auto per_group) { return w.zeros ? shaped(per_group, std::true_type()) : shaped(per_group, std::false_type()); };
    if (w.group == 32) return run(constant<1>());
    if (w.group == 64) return run(constant<2>());
    return run(constant<4>());
}

template <int BT, int SHARE, int NT> hipError_t launch_wide(const quant_matrix &w, const char *B, const float *B_scales, int64_t N, const tensor &C, hipStream_t stream)
{
    constexpr int ROWS = SHARE * (16 / NT);
    const dim3 blocks((unsigned)((w.tiles + ROWS - 1) / ROWS), (unsigned)((N + 16 * NT - 1) / (16 * NT)));
    auto run = [&](auto per_group) {
        constexpr int PER_GROUP = decltype(per_group)::value;
        if (w.zeros) return launch_kernel(wide_kernel<BT, SHARE, NT, PER_GROUP, true>, blocks, 512, WIDE_LDS, stream, w, B, B_scales, N, C);
        return launch_kernel(wide_kernel<BT, SHARE, NT, PER_GROUP, false>, blocks, 512, WIDE_LDS, stream, w, B, B_scales, N, C);
    };
    if (w.group == 32) return run(constant<1>());
    if (w.group == 64) return run(constant<2>());
    return run(constant<4>());
}

// On B laid out by pack_kernel.  Small tiles while they leave no compute unit without a workgroup; then larger ones, which read B and make operands of weights less often.
// us, tiles of rows x of tokens of a wave (teams of two, four and eight waves: wide_kernel), bf16:
//   1024 x 4096, 128 tokens   1x2  9.4   2x2 10.8   2x4 13.2                        4096 x 4096, 128    1x2 17.0   2x2 14.7   2x4 14.0   two 25.3
//   16384 x 4096, 64          1x2 33     2x2 26     2x4 27     two 28               3001 x 2511, 200    1x2 15.5   2x2 14.7   2x4 18.8   two 20.4
//   8192 x 8192, 128          2x2 40     two 42     four 71                         8192 x 8192, 192    2x2 56     two 45     four 72
//   8192 x 8192, 320          2x2 90     two 81     four 74    eight 126            8192 x 8192, 2048   2x2 513    two 335    four 309   eight 275
//   16384 x 4096, 300         2x2 91     two 75     four 81    eight 74             1024 x 1024, 8192   2x2 57     two 59     four 52    eight 42
// in codes: 8192 x 8192, 128 2x2 30, two 34; 256 2x2 53, 4x4 42, two 37; 512 4x4 74, two 67, four 60, eight 96; 2048 4x4 260, two 246, four 210, eight 197;
//   2048 x 8192, 512 2x2 28, two 34; with groups of 32 and zero points 8192 x 8192, 512 4x4 235, four 101
// in fp32: 4096 x 4096, 128 2x2 26, 2x4 23, 4x4 34; 4096 x 4096, 256 2x2 47, 2x4 42, 4x4 36
template <int BT> hipError_t execute_many(const quant_matrix &w, const char *B, const float *B_scales, int64_t N, const tensor &C, hipStream_t stream)
{
    auto workgroups = [&](int64_t rows, int64_t tokens) { return (w.tiles + rows - 1) / rows * ((N + 16 * tokens - 1) / (16 * tokens)); };
    if (workgroups(1, 2) <= 256) return launch_many<BT, 2, 1, 8>(w, B, B_scales, N, C, stream);
    if constexpr (BT == SPMM_F32) {
        if (workgroups(4, 4) >= 180) return launch_many<BT, 4, 4, 4>(w, B, B_scales, N, C, stream);
        if (workgroups(2, 4) >= 180) return launch_many<BT, 4, 2, 8>(w, B, B_scales, N, C, stream);
    } else {
        // Rounds of 256 workgroups, by what one takes (of 8192 columns): the fewer rows a team has, the more often B is read.
        auto us = [&](int64_t rows, int64_t tokens, int64_t round) { return (workgroups(rows, tokens) + 255) / 256 * round; };
        constexpr bool CODES = BT == SPMM_I8;
        const int64_t small = us(2, 2, CODES ? 7 : 8), two = us(8, 4, CODES ? 32 : 41), four = us(8, 8, CODES ? 50 : 74), eight = us(16, 8, CODES ? 92 : 124);
        if (std::min({two, four, eight}) < small) {
            if (eight <= std::min(two, four)) return launch_wide<BT, 8, 8>(w, B, B_scales, N, C, stream);
            if (four <= two) return launch_wide<BT, 4, 8>(w, B, B_scales, N, C, stream);
            return launch_wide<BT, 2, 4>(w, B, B_scales, N, C, stream);
        }
    }
    return launch_many<BT, 2, 2, 8>(w, B, B_scales, N, C, stream);
}

// Whether a product goes in one launch.  Up to 16 tokens always.  With more, lanes read B in pieces of 16 bytes of as many rows of memory, which many_kernel reads from the laid out
// B in pieces of 1 KiB, and only what a launch costs speaks for it: where each wave has one block of columns and each compute unit one workgroup.
// us in one launch and in two, bf16: 4096 x 1024, 32 tokens 4.2 and 5.0; 4096 x 2048 6.4 and 6.5; 4096 x 4096 10.0 and 8.5; 16384 x 1024 14 and 7.6.
// fp32 by features: 4096 x 1024, 32 tokens 6.7 and 7.2; 4096 x 2048 9.9 and 9.5.
bool is_direct(const quant_matrix &w, int64_t N)
{
    return N <= 16 || (N <= 128 && w.blocks <= 8 && w.tiles * ((N + 31) / 32) <= 256);
}

template <int BT> hipError_t execute(const quant_matrix &w, const tensor &B, const float *B_scales, int64_t N, const tensor &C, char *workspace, hipStream_t stream)
{
    if (is_direct(w, N)) {
        if constexpr (BT == SPMM_F32)
            if (B.by_token && N == 1) return execute_direct<BT, true, true>(w, B, B_scales, N, C, stream);
        if (B.by_token) return execute_direct<BT, true, false>(w, B, B_scales, N, C, stream);
        if constexpr (BT != SPMM_I8) return execute_direct<BT, false, false>(w, B, B_scales, N, C, stream);
    }
    // a launch of each for 2^16 - 1 tiles of tokens at a time
    const int64_t token_tiles = (N + 15) / 16;
    for (int64_t t0 = 0; t0 < token_tiles; t0 += MOST_TOKEN_TILES) {
        const int64_t tiles = token_tiles - t0 < MOST_TOKEN_TILES ? token_tiles - t0 : MOST_TOKEN_TILES, n0 = t0 * 16, n = N - n0 < tiles * 16 ? N - n0 : tiles * 16;
        const int64_t size = BT == SPMM_I8 ? 1 : BT == SPMM_F32 ? 4 : 2, c_size = C.type == SPMM_F32 ? 4 : 2;
        tensor b = B, c = C;
        b.data += n0 * (B.by_token ? B.ld : 1) * size;
        c.data += n0 * (C.by_token ? C.ld : 1) * c_size;
        const float *scales = B_scales ? B_scales + n0 : nullptr;
        hipError_t e = hipSuccess;
        const dim3 grid((unsigned)w.blocks, (unsigned)tiles);
        if (w.blocks > 0 && b.by_token) e = launch_kernel(pack_kernel<BT, true>, grid, 256, 0, stream, b, w.K, n, w.blocks, workspace);
        else if (w.blocks > 0) e = launch_kernel(pack_kernel<BT, false>, grid, 256, 0, stream, b, w.K, n, w.blocks, workspace);
        if (e != hipSuccess) return e;
        e = execute_many<BT>(w, workspace, scales, n, c, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t quant_workspace(const quant_matrix &w, const tensor &B, int64_t N)
{
    if (is_direct(w, N)) return 0;
    const int64_t step = B.type == SPMM_F32 ? 3 * 1024 : B.type == SPMM_I8 ? 512 : 1024, tiles = (N + 15) / 16;
    return (tiles < MOST_TOKEN_TILES ? tiles : MOST_TOKEN_TILES) * w.blocks * 4 * step;
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
