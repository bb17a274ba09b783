// What stands between two products (gfx950): the root-mean-square norm with the residual's addition, and the gated
// activation, both with floating output or in 8-bit codes with a scale a token.
//
//   norm  t = x + r, rounded;  p = t w;    f = 1 / sqrt(mean t^2 + eps)
//   gate                       p = act(a) b;  f = 1
//   out = p f (norm: t f w), or code = rint(p (127 / max |p|)), scale = max |p| f / 127
//
// Squares are added up in fp32 by a thread, over up to 32 of them, and by the lanes of a wave, from there on in 64 bits: what a few waves or tiles leave costs nothing to add up, and the mean is right to
// its rounding (in fp32 throughout, 15 waves' sums could vanish beside one).
// Codes do not wait for f: they depend on p alone, so one look at the token gives both statistics.  All of it is bound by
// memory, or by the latency of one launch: elements are read once and held in registers between the statistics
// and the output where registers hold them.  With the residual's addition, us (of which a launch is 2.4): one token of 4096 in bf16 3.1; 2048 tokens of 8192 in bf16 29, 4.6 TB/s, in codes 30;
// where a row of memory is a feature, fp32, 128 tokens of 1024 6.7, 2048 tokens of 4096 46, 2.9 TB/s (3.6 with the sum's second reading).  The gate: 16 tokens of 4096 in f16 2.3; 2048 of
// 16384 in bf16 37, 5.4 TB/s, 2048 of 8192 to codes 21 (by features 50, where values are read and made twice).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../../include/spmm_layers.h"
#include "../spmm_launch.h"
#include "elements.h"
#include "layers.h"

namespace layers {
namespace {

// x / (1 + exp(-u)): silu for u = x; gelu for u = 2 sqrt(2 / pi) (x + 0.044715 x^3), since (1 + tanh(u / 2)) / 2 = 1 / (1 + exp(-u)), which does not
// cancel for negative x.  The exponential by its base-2 instruction, the quotient by the reciprocal's: both are right to a unit of the last place.  The exponential's argument -u log2(e) is
// a product whose rounding is worth |u| 2^-24 of the result, and exp(-u) has no reciprocal that the instruction gives from u = -87 on, where the result is 0 instead of 88 2^-126.
// WHOLE, for results that go out in fp32: e = exp(-|u|), which is at most 1, in x e / (1 + e) for negative u and x / (1 + e) for others, right as long as e is a normal number; what the
// product's rounding left, exactly a multiply-add, comes in as a factor 1 + left ln(2) (left is below 2^-16, its square below a rounding).  Fp32 of 4096 x 2048 takes 18.6 us with and without; in
// 16 bits and codes, whose own rounding is 2^-12 of a value and more, it would be 38.5 us for 37.5 and, 8192 x 2048 to codes, 22.2 for 20.6.
template <bool WHOLE> __device__ inline float act_of(float x, int32_t act)
{
    if (act == SPMM_ACT_RELU) return x < 0.0f ? 0.0f : x;
    constexpr float LOG2_E = 1.4426950408889634f, LOG2_E_LEFT = 1.4426950408889634 - (double)LOG2_E, LN_2 = 0.6931471805599453f;
    const float u = act == SPMM_ACT_SILU ? x : 1.5957691216057308f * (x + 0.044715f * x * x * x);
    if constexpr (WHOLE) {
        const float m = -fminf(fabsf(u), 128.0f);  // (e is 0 there)
        const float whole = m * LOG2_E, left = __builtin_fmaf(m, LOG2_E_LEFT, __builtin_fmaf(m, LOG2_E, -whole));
        const float e0 = __builtin_amdgcn_exp2f(whole), e = __builtin_fmaf(e0, left * LN_2, e0);
        return (u < 0.0f ? x * e : x) * __builtin_amdgcn_rcpf(1.0f + e);
    }
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2_E * u));
}

// The larger magnitude; an infinity or a NaN counts as an infinity.
__device__ inline float larger(float most, float v)
{
    const float m = fabsf(v);
    return m <= most ? most : m != m ? __builtin_inff() : m;
}

// What a token's codes and values are made with.
struct token_factors {
    float factor;     // f
    float up, steps;  // code = rint(p * up * steps); up keeps 127 / max |p| finite for the smallest values
    float scale;
    __device__ token_factors(bool norm, double square, float most, const rows_args &a)
    {
        factor = norm ? 1.0f / sqrtf((float)(square * a.per_feature + a.eps)) : 1.0f;
        up = most < 0x1p-100f ? 0x1p100f : 1.0f;
        steps = most > 0.0f && most < __builtin_inff() ? 127.0f / (most * up) : 0.0f;
        // (f is infinite where all of a token's squares vanish and eps is 0)
        scale = most == 0.0f ? 0.0f : most < __builtin_inff() ? most * factor / 127.0f : __builtin_nanf("");
    }
    __device__ int8_t code(float p) const { return steps == 0.0f ? (int8_t)0 : (int8_t)rintf(p * up * steps); }
};

// Elements from `at` on of x and, where there is one, of its companion: t (norm, rounded to x's type) or p (gate).
template <bool NORM, int TYPE, bool WHOLE = false, int N> __device__ inline void values_at(const rows_args &a, int64_t x_at, int64_t y_at, int there, float (&v)[N])
{
    typedef typename element<TYPE>::type T;
    float y[N];
    load_row<T>(a.x.data, x_at, there, v);
    if (a.y.data) load_row<T>(a.y.data, y_at, there, y);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if constexpr (NORM) {
            if (a.y.data) v[j] = (float)(T)(v[j] + y[j]);
        } else {
            v[j] = act_of<WHOLE>(v[j], a.act) * (a.y.data ? y[j] : 1.0f);
        }
    }
}

template <bool SQUARE, bool MOST> __device__ inline void reduce_lanes(float &square, float &most, int from)
{
    for (int d = from; d < 64; d *= 2) {
        if constexpr (SQUARE) square += __shfl_xor(square, d);
        if constexpr (MOST) most = fmaxf(most, __shfl_xor(most, d));
    }
}

// ---- a token a row of memory -----------------------------------------------------------------------------------

constexpr int UNIT = 8;  // neighbouring elements of a thread: 16 bytes of 16-bit elements

// T threads a token, TOKENS tokens a workgroup; every thread holds R units.
template <bool NORM, bool CODES, int TYPE, int T, int R, int TOKENS> __global__ __launch_bounds__(T *TOKENS) void rows_kernel(rows_args a)
{
    typedef typename element<TYPE>::type E;
    constexpr int WAVES = T / 64;
    constexpr bool KEEP_WEIGHTS = NORM && !CODES && R <= 2;  // (with codes p is kept in t's place; longer ones read the weights again)
    __shared__ float squares[WAVES * TOKENS], mosts[WAVES * TOKENS];
    const int t = threadIdx.x % T;
    const int64_t n = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * TOKENS + threadIdx.x / T;
    if (n >= a.tokens) return;  // (a workgroup of several waves has one token)
    auto unit = [&](int i) { return ((int64_t)i * T + t) * UNIT; };
    auto there = [&](int i) { return (int)min((int64_t)UNIT, max((int64_t)0, a.features - unit(i))); };
    float v[R][UNIT], w[R][UNIT];
#pragma unroll
    for (int i = 0; i < R; ++i) values_at<NORM, TYPE>(a, n * a.x.ld + unit(i), n * a.y.ld + unit(i), there(i), v[i]);
    if constexpr (NORM && (CODES || KEEP_WEIGHTS)) {
#pragma unroll
        for (int i = 0; i < R; ++i) load_row_as(a.weight, unit(i), there(i), a.weight_type, w[i]);
    }
    float square = 0.0f, most = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if constexpr (NORM)
            if (a.total.data) store_row<E>(a.total.data, n * a.total.ld + unit(i), there(i), v[i]);
#pragma unroll
        for (int j = 0; j < UNIT; ++j) {
            if constexpr (NORM) square += v[i][j] * v[i][j];
            if constexpr (NORM && CODES) v[i][j] *= w[i][j];
            if constexpr (CODES) most = larger(most, v[i][j]);
        }
    }
    reduce_lanes<NORM, CODES>(square, most, 1);
    double sum = square;
    if constexpr (WAVES > 1) {
        if ((t & 63) == 0) squares[t / 64] = square, mosts[t / 64] = most;
        __syncthreads();
        sum = squares[0], most = mosts[0];
#pragma unroll
        for (int wave = 1; wave < WAVES; ++wave) sum += squares[wave], most = fmaxf(most, mosts[wave]);
    }
    const token_factors f(NORM, sum, most, a);
    if (CODES && t == 0) a.scales[n] = f.scale;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if constexpr (CODES) {
#pragma unroll
            for (int j = 0; j < UNIT; ++j) v[i][j] = (float)f.code(v[i][j]);
            store_row<int8_t>(a.out.data, n * a.out.ld + unit(i), there(i), v[i]);
        } else {
            if constexpr (!KEEP_WEIGHTS) load_row_as(a.weight, unit(i), there(i), a.weight_type, w[i]);
#pragma unroll
            for (int j = 0; j < UNIT; ++j) v[i][j] = v[i][j] * f.factor * w[i][j];
            store_row_as(a.out.data, n * a.out.ld + unit(i), there(i), a.out.type, v[i]);
        }
    }
}

// Tokens longer than a workgroup holds: read twice (the second time the sum, where it was written: it may be x's own memory).
template <bool NORM, bool CODES, int TYPE> __global__ __launch_bounds__(1024) void long_rows_kernel(rows_args a)
{
    typedef typename element<TYPE>::type E;
    __shared__ float squares[16], mosts[16];
    const int t = threadIdx.x;
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= a.tokens) return;
    double of_thread = 0.0;
    float most = 0.0f;
    for (int64_t k = t * UNIT; k < a.features; k += 1024 * UNIT) {
        const int there = (int)min((int64_t)UNIT, a.features - k);
        float v[UNIT], w[UNIT];
        values_at<NORM, TYPE>(a, n * a.x.ld + k, n * a.y.ld + k, there, v);
        if constexpr (NORM)
            if (a.total.data) store_row<E>(a.total.data, n * a.total.ld + k, there, v);
        if constexpr (NORM && CODES) load_row_as(a.weight, k, there, a.weight_type, w);
        float square = 0.0f;
#pragma unroll
        for (int j = 0; j < UNIT; ++j) {
            if constexpr (NORM) square += v[j] * v[j];
            if constexpr (CODES) most = larger(most, NORM ? v[j] * w[j] : v[j]);
        }
        of_thread += square;
    }
    float square = (float)of_thread;
    reduce_lanes<NORM, CODES>(square, most, 1);
    if ((t & 63) == 0) squares[t / 64] = square, mosts[t / 64] = most;
    __syncthreads();
    double sum = squares[0];
    most = mosts[0];
    for (int wave = 1; wave < 16; ++wave) sum += squares[wave], most = fmaxf(most, mosts[wave]);
    const token_factors f(NORM, sum, most, a);
    if (CODES && t == 0) a.scales[n] = f.scale;
    for (int64_t k = t * UNIT; k < a.features; k += 1024 * UNIT) {
        const int there = (int)min((int64_t)UNIT, a.features - k);
        float v[UNIT], w[UNIT];
        if (NORM && a.total.data) load_row<E>(a.total.data, n * a.total.ld + k, there, v);
        else values_at<NORM, TYPE>(a, n * a.x.ld + k, n * a.y.ld + k, there, v);
        if constexpr (NORM) load_row_as(a.weight, k, there, a.weight_type, w);
#pragma unroll
        for (int j = 0; j < UNIT; ++j) v[j] = CODES ? (float)f.code(NORM ? v[j] * w[j] : v[j]) : v[j] * f.factor * w[j];
        if constexpr (CODES) store_row<int8_t>(a.out.data, n * a.out.ld + k, there, v);
        else store_row_as(a.out.data, n * a.out.ld + k, there, a.out.type, v);
    }
}

// ---- a feature a row of memory ---------------------------------------------------------------------------------

// Few tokens of not too many features: a workgroup has all features of some tokens.  A thread reads 16 bytes of a row, COLS threads lie side by side, HELD rows stay in
// a thread's registers.
template <int TYPE> constexpr int COLUMN_UNIT = TYPE == SPMM_F32 ? 4 : 8;
constexpr int COLUMN_THREADS = 1024;

template <bool NORM, bool CODES, int TYPE, int COLS, int HELD> __global__ __launch_bounds__(COLUMN_THREADS) void columns_kernel(rows_args a)
{
    typedef typename element<TYPE>::type E;
    constexpr int U = COLUMN_UNIT<TYPE>, TOKENS = COLS * U, ROWS = COLUMN_THREADS / COLS, WAVES = COLUMN_THREADS / 64;
    __shared__ float squares[WAVES][TOKENS], mosts[WAVES][TOKENS], factors[2][TOKENS];
    __shared__ int8_t turned[CODES ? 2 : 1][CODES ? TOKENS : 1][ROWS + 4];
    const int col = threadIdx.x % COLS, row = threadIdx.x / COLS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * TOKENS, n = n0 + col * U;
    if (n0 >= a.tokens) return;
    const int wide = (int)min((int64_t)U, max((int64_t)0, a.tokens - n));
    float square[U], most[U], held[HELD][U];
#pragma unroll
    for (int j = 0; j < U; ++j) square[j] = most[j] = 0.0f;
    float w[HELD][1];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int64_t k = (int64_t)i * ROWS + row;
        values_at<NORM, TYPE>(a, k * a.x.ld + n, k * a.y.ld + n, k < a.features ? wide : 0, held[i]);
        if constexpr (NORM) load_row_as(a.weight, k, k < a.features, a.weight_type, w[i]);
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int64_t k = (int64_t)i * ROWS + row;
        if constexpr (NORM)
            if (a.total.data && k < a.features) store_row<E>(a.total.data, k * a.total.ld + n, wide, held[i]);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if constexpr (NORM) square[j] += held[i][j] * held[i][j];
            if constexpr (NORM && CODES) held[i][j] *= w[i][0];  // p in t's place
            if constexpr (CODES) most[j] = larger(most[j], held[i][j]);
        }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) reduce_lanes<NORM, CODES>(square[j], most[j], COLS);
    if (lane < COLS) {
#pragma unroll
        for (int j = 0; j < U; ++j) squares[wave][lane * U + j] = square[j], mosts[wave][lane * U + j] = most[j];
    }
    __syncthreads();
    if (threadIdx.x < TOKENS && n0 + threadIdx.x < a.tokens) {  // a thread a token
        double s = squares[0][threadIdx.x];
        float m = mosts[0][threadIdx.x];
        for (int w = 1; w < WAVES; ++w) s += squares[w][threadIdx.x], m = fmaxf(m, mosts[w][threadIdx.x]);
        const token_factors f(NORM, s, m, a);
        if (CODES) a.scales[n0 + threadIdx.x] = f.scale;
        factors[0][threadIdx.x] = CODES ? f.up : f.factor;
        factors[1][threadIdx.x] = f.steps;
    }
    __syncthreads();
    float first[U], second[U];  // f, or the two factors of codes
#pragma unroll
    for (int j = 0; j < U; ++j) first[j] = factors[0][col * U + j], second[j] = factors[1][col * U + j];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int64_t k0 = (int64_t)i * ROWS, k = k0 + row;
        if constexpr (!CODES) {
#pragma unroll
            for (int j = 0; j < U; ++j) held[i][j] = held[i][j] * first[j] * w[i][0];
            if (k < a.features) store_row_as(a.out.data, k * a.out.ld + n, wide, a.out.type, held[i]);
        } else {
            // codes change places through LDS: a row of memory is a token there.  Two places in turn, so that one barrier a step is enough.
            int8_t(&tile)[TOKENS][ROWS + 4] = turned[i & 1];
#pragma unroll
            for (int j = 0; j < U; ++j) tile[col * U + j][row] = second[j] == 0.0f ? (int8_t)0 : (int8_t)rintf(held[i][j] * first[j] * second[j]);
            __syncthreads();
            constexpr int EACH = TOKENS * ROWS / COLUMN_THREADS;  // 4 or 8 codes of a token
            const int token = threadIdx.x / (ROWS / EACH), r = threadIdx.x % (ROWS / EACH) * EACH;
            const int there = (int)min((int64_t)EACH, max((int64_t)0, a.features - k0 - r));
            if (n0 + token < a.tokens) {
                int8_t *to = reinterpret_cast<int8_t *>(a.out.data) + (n0 + token) * a.out.ld + k0 + r;
                if (there == EACH) {
                    *reinterpret_cast<neighbours<int8_t, EACH> *>(to) = *reinterpret_cast<const neighbours<int8_t, EACH> *>(&tile[token][r]);
                } else {
                    for (int j = 0; j < there; ++j) to[j] = tile[token][r + j];
                }
            }
        }
    }
}

// Otherwise two launches.  A workgroup has a tile of whole pieces of rows: `side` threads of 16 bytes lie side by side (a power of two), 256 / side rows are read at a time.  The
// first launch leaves every tile's statistics of its tokens, and the sum where it is asked for; in the second every tile adds up those of its tokens, in order, and reads its values again.
struct column_tiles {
    int32_t side_bits, rows;  // log2 of side; rows of a tile
    int64_t across;           // tiles side by side; tiles of a column are gridDim.y
    float *partial;           // [tile of a column][square, most][tokens]
};

// (128 bytes of a row side by side; a thread asks for AT_ONCE rows before it looks at the first)
constexpr int TILE_THREADS = 256, MOST_SIDE_BITS = 3, PIECE_ROWS = 64, AT_ONCE = 4;

// The first token of a tile `wide` tokens across: the tiles side by side go along the first and the third axis (a launch has less than 2^32 threads along one).
__device__ inline int64_t first_token(int wide) { return ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * wide; }

template <bool NORM, bool CODES, int TYPE> __global__ __launch_bounds__(TILE_THREADS) void column_stats_kernel(rows_args a, column_tiles tiles)
{
    typedef typename element<TYPE>::type E;
    constexpr int U = COLUMN_UNIT<TYPE>;
    __shared__ float squares[4][U << MOST_SIDE_BITS], mosts[4][U << MOST_SIDE_BITS];
    const int side = 1 << tiles.side_bits, col = threadIdx.x & (side - 1), row = threadIdx.x >> tiles.side_bits, step = TILE_THREADS >> tiles.side_bits;
    const int64_t n0 = first_token(side * U), n = n0 + col * U, k0 = (int64_t)blockIdx.y * tiles.rows, k1 = min(k0 + tiles.rows, a.features);
    if (n0 >= a.tokens) return;
    const int wide = (int)min((int64_t)U, max((int64_t)0, a.tokens - n));
    double of_thread[U];
    float square[U], most[U];
#pragma unroll
    for (int j = 0; j < U; ++j) of_thread[j] = 0.0, most[j] = 0.0f;
    for (int64_t k = k0 + row; k < k1; k += AT_ONCE * step) {
        float v[AT_ONCE][U];
#pragma unroll
        for (int j = 0; j < U; ++j) square[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int64_t at = k + i * step;
            values_at<NORM, TYPE>(a, at * a.x.ld + n, at * a.y.ld + n, at < k1 ? wide : 0, v[i]);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int64_t at = k + i * step;
            float w[1] = {1.0f};
            if (at >= k1) break;
            if constexpr (NORM)
                if (a.total.data) store_row<E>(a.total.data, at * a.total.ld + n, wide, v[i]);
            if constexpr (NORM && CODES) load_row_as(a.weight, at, 1, a.weight_type, w);
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if constexpr (NORM) square[j] += v[i][j] * v[i][j];
                if constexpr (CODES) most[j] = larger(most[j], v[i][j] * w[0]);
            }
        }
        if constexpr (NORM) {
#pragma unroll
            for (int j = 0; j < U; ++j) of_thread[j] += square[j];
        }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) square[j] = (float)of_thread[j];
#pragma unroll
    for (int j = 0; j < U; ++j) reduce_lanes<NORM, CODES>(square[j], most[j], side);
    const int wave = threadIdx.x >> 6;
    if ((int)(threadIdx.x & 63) < side) {
#pragma unroll
        for (int j = 0; j < U; ++j) squares[wave][col * U + j] = square[j], mosts[wave][col * U + j] = most[j];
    }
    __syncthreads();
    for (int t = threadIdx.x; t < side * U; t += TILE_THREADS) {
        if (n0 + t >= a.tokens) continue;
        float *to = tiles.partial + (int64_t)blockIdx.y * 2 * a.tokens + n0 + t;
        if constexpr (NORM) to[0] = (float)((double)squares[0][t] + squares[1][t] + squares[2][t] + squares[3][t]);
        if constexpr (CODES) to[a.tokens] = fmaxf(fmaxf(mosts[0][t], mosts[1][t]), fmaxf(mosts[2][t], mosts[3][t]));
    }
}

template <bool NORM, bool CODES, int TYPE> __global__ __launch_bounds__(TILE_THREADS) void column_apply_kernel(rows_args a, column_tiles tiles)
{
    constexpr int U = COLUMN_UNIT<TYPE>, MOST_TOKENS = U << MOST_SIDE_BITS;
    __shared__ double sums[TILE_THREADS];
    __shared__ float mosts[TILE_THREADS], factors[2][MOST_TOKENS];
    extern __shared__ int8_t turned[];  // codes: [token][rows of a piece + 4]
    const int side = 1 << tiles.side_bits, col = threadIdx.x & (side - 1), row = threadIdx.x >> tiles.side_bits, step = TILE_THREADS >> tiles.side_bits, tokens = side * U;
    const int64_t n0 = first_token(tokens), n = n0 + col * U, k0 = (int64_t)blockIdx.y * tiles.rows, k1 = min(k0 + tiles.rows, a.features);
    if (n0 >= a.tokens) return;
    const int wide = (int)min((int64_t)U, max((int64_t)0, a.tokens - n));
    // The statistics of this tile's tokens: TILE_THREADS / tokens threads each (tokens is at most TILE_THREADS).
    {
        const int t = threadIdx.x & (tokens - 1), token_bits = tiles.side_bits + (U == 4 ? 2 : 3), part = threadIdx.x >> token_bits, parts = TILE_THREADS >> token_bits;
        double s = 0.0;
        float m = 0.0f;
        if (n0 + t < a.tokens) {
            for (int c = part; c < (int)gridDim.y; c += parts) {
                const float *from = tiles.partial + (int64_t)c * 2 * a.tokens + n0 + t;
                if constexpr (NORM) s += from[0];
                if constexpr (CODES) m = fmaxf(m, from[a.tokens]);
            }
        }
        sums[threadIdx.x] = s, mosts[threadIdx.x] = m;
        __syncthreads();
        if (part == 0) {
            for (int p = 1; p < parts; ++p) s += sums[p * tokens + t], m = fmaxf(m, mosts[p * tokens + t]);
            const token_factors f(NORM, s, m, a);
            if (CODES && blockIdx.y == 0 && n0 + t < a.tokens) a.scales[n0 + t] = f.scale;
            factors[0][t] = CODES ? f.up : f.factor;
            factors[1][t] = f.steps;
        }
        __syncthreads();
    }
    float first[U], second[U];  // f, or the two factors of codes
#pragma unroll
    for (int j = 0; j < U; ++j) first[j] = factors[0][col * U + j], second[j] = factors[1][col * U + j];
    auto value = [&](int64_t k, float (&v)[U], float &w) {
        float weight[1] = {1.0f};
        values_at<NORM, TYPE>(a, k * a.x.ld + n, k * a.y.ld + n, k < k1 ? wide : 0, v);
        if constexpr (NORM) load_row_as(a.weight, k, k < k1, a.weight_type, weight);
        w = weight[0];
    };
    if constexpr (!CODES) {
        for (int64_t k = k0 + row; k < k1; k += AT_ONCE * step) {
            float v[AT_ONCE][U], w[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) value(k + i * step, v[i], w[i]);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
#pragma unroll
                for (int j = 0; j < U; ++j) v[i][j] = v[i][j] * first[j] * w[i];
                if (k + i * step < k1) store_row_as(a.out.data, (k + i * step) * a.out.ld + n, wide, a.out.type, v[i]);
            }
        }
    } else {
        // codes change places through LDS, a piece of rows at a time: a row of memory is a token there
        const int piece = max(step, PIECE_ROWS), pitch = piece + 4;
        for (int64_t p0 = k0; p0 < k1; p0 += piece) {
            for (int q = row; q < piece; q += step) {
                if (p0 + q >= k1) break;
                float v[U], w;
                value(p0 + q, v, w);
#pragma unroll
                for (int j = 0; j < U; ++j) turned[(col * U + j) * pitch + q] = second[j] == 0.0f ? (int8_t)0 : (int8_t)rintf(v[j] * w * first[j] * second[j]);
            }
            __syncthreads();
            // four codes of a token a thread; pieces are powers of two
            const int unit_bits = __builtin_ctz(piece) - 2;
            for (int e = threadIdx.x; e < tokens << unit_bits; e += TILE_THREADS) {
                const int t = e >> unit_bits, q = (e & ((1 << unit_bits) - 1)) * 4, there = (int)min((int64_t)4, k1 - p0 - q);
                if (n0 + t >= a.tokens || there <= 0) continue;
                int8_t *to = reinterpret_cast<int8_t *>(a.out.data) + (n0 + t) * a.out.ld + p0 + q;
                if (there == 4) {
                    *reinterpret_cast<neighbours<int8_t, 4> *>(to) = *reinterpret_cast<const neighbours<int8_t, 4> *>(turned + t * pitch + q);
                } else {
                    for (int j = 0; j < there; ++j) to[j] = turned[t * pitch + q + j];
                }
            }
            __syncthreads();
        }
    }
}

// ---- the gate with floating output: element by element ---------------------------------------------------------

// `rows` rows of memory of `units` units each; short rows without gaps have been made one long row by the launch.
template <int TYPE> __global__ __launch_bounds__(256) void elements_kernel(rows_args a, int64_t rows, int64_t length, uint32_t units)
{
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    int64_t row, unit;
    if (rows == 1) {
        row = 0, unit = at;
    } else {
        row = at >> 32 ? at / units : (int64_t)((uint32_t)at / units);
        unit = at - row * units;
    }
    if (row >= rows || unit * UNIT >= length) return;
    const int64_t k = unit * UNIT;
    const int there = (int)min((int64_t)UNIT, length - k);
    float v[UNIT];
    if (a.out.type == SPMM_F32) values_at<false, TYPE, true>(a, row * a.x.ld + k, row * a.y.ld + k, there, v);
    else values_at<false, TYPE>(a, row * a.x.ld + k, row * a.y.ld + k, there, v);
    store_row_as(a.out.data, row * a.out.ld + k, there, a.out.type, v);
}

// A launch has less than 2^32 threads along an axis.
dim3 grid_of(int64_t blocks)
{
    const int64_t x = blocks < 1 << 20 ? blocks : 1 << 20;
    return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

template <int TYPE> hipError_t launch_elements(const rows_args &a, hipStream_t stream)
{
    int64_t rows = a.x.by_token ? a.tokens : a.features, length = a.x.by_token ? a.features : a.tokens;
    if (rows == 1 || (a.x.ld == length && a.out.ld == length && (!a.y.data || a.y.ld == length))) length *= rows, rows = 1;
    const int64_t units = (length + UNIT - 1) / UNIT;
    return launch_kernel(elements_kernel<TYPE>, grid_of((rows * units + 255) / 256), 256, 0, stream, a, rows, length, (uint32_t)units);
}

// One launch, whose workgroups have all features of their tokens, or two, as far as a workgroup's registers hold its tokens and few workgroups read the same lines: 0, or the threads side by side.
// us of one thread, 64 bytes side by side and two launches, K x N in fp32: 1024 x 32 4.8, 6.8, 7.7; 1024 x 128 7.7, 6.9, 7.7; 1024 x 256 9.4, 10.1, 8.7; 300 x 1000 7.4, 6.6, 10.2;
// 4096 x 8 7.6, -, 8.7; 4096 x 16 13.7, -, 8.3; 4096 x 256 34, -, 10.5.  bf16: 1024 x 64 6.5, 7.2, 9.9; 1024 x 256 10.0, 9.9, 10.0; 2048 x 32 8.0, -, 10.6; 4096 x 16 8.1, -, 11.1; 4096 x 64 18, -, 10.7.
int in_one_launch(int64_t K, int64_t N, int unit)
{
    if (K <= 4 * COLUMN_THREADS && K * N <= 8192 * unit) return 1;
    return K <= COLUMN_THREADS && N <= (K <= 512 ? 1024 : 32 * unit) ? 16 / unit : 0;
}

// Tiles of AT_ONCE steps of rows, or as many as leave 64 in a column; whole pieces of codes.
column_tiles tiles_of(int64_t K, int64_t N, int unit)
{
    column_tiles t = {};
    while (t.side_bits < MOST_SIDE_BITS && (int64_t)unit << t.side_bits < N) ++t.side_bits;
    const int64_t wide = (int64_t)unit << t.side_bits, step = TILE_THREADS >> t.side_bits, rows = (K + 63) / 64;
    t.across = (N + wide - 1) / wide;
    t.rows = (int32_t)((rows + AT_ONCE * step - 1) / (AT_ONCE * step) * (AT_ONCE * step));
    return t;
}

template <bool NORM, bool CODES, int TYPE> hipError_t launch(const rows_args &a, char *workspace, hipStream_t stream)
{
    const int64_t K = a.features, N = a.tokens;
    if (!a.x.by_token) {
        auto at_once = [&](auto cols) {
            constexpr int COLS = decltype(cols)::value, TOKENS = COLS * COLUMN_UNIT<TYPE>, ROWS = COLUMN_THREADS / COLS;
            const dim3 grid = grid_of((N + TOKENS - 1) / TOKENS);
            if (K <= ROWS) return launch_kernel(columns_kernel<NORM, CODES, TYPE, COLS, 1>, grid, COLUMN_THREADS, 0, stream, a);
            return launch_kernel(columns_kernel<NORM, CODES, TYPE, COLS, 4>, grid, COLUMN_THREADS, 0, stream, a);
        };
        const int cols = in_one_launch(K, N, COLUMN_UNIT<TYPE>);
        if (cols == 1) return at_once(std::integral_constant<int, 1>());
        if (cols > 1) return at_once(std::integral_constant<int, 16 / COLUMN_UNIT<TYPE>>());
        column_tiles tiles = tiles_of(K, N, COLUMN_UNIT<TYPE>);
        tiles.partial = reinterpret_cast<float *>(workspace);
        const dim3 across = grid_of(tiles.across), grid(across.x, (unsigned)((K + tiles.rows - 1) / tiles.rows), across.y);
        const hipError_t e = launch_kernel(column_stats_kernel<NORM, CODES, TYPE>, grid, TILE_THREADS, 0, stream, a, tiles);
        if (e != hipSuccess) return e;
        const int step = TILE_THREADS >> tiles.side_bits, piece = step > PIECE_ROWS ? step : PIECE_ROWS;
        rows_args written = a;  // the sum, where it was written: it may be x's own memory
        if (a.total.data) written.x = a.total, written.y.data = nullptr;
        return launch_kernel(column_apply_kernel<NORM, CODES, TYPE>, grid, TILE_THREADS, CODES ? (unsigned)((COLUMN_UNIT<TYPE> << tiles.side_bits) * (piece + 4)) : 0u, stream, written, tiles);
    }
    const int64_t units = (K + UNIT - 1) / UNIT;
    if (units <= 64) return launch_kernel(rows_kernel<NORM, CODES, TYPE, 64, 1, 4>, grid_of((N + 3) / 4), 256, 0, stream, a);
    if (units <= 256) return launch_kernel(rows_kernel<NORM, CODES, TYPE, 256, 1, 1>, grid_of(N), 256, 0, stream, a);
    // Few tokens are over when their slowest is: more threads each.  Many are a matter of bandwidth, which smaller workgroups, of which a compute unit has
    // several in different phases, come nearer to.  us with 1024 threads and with 256, bf16: 8192 x 16 3.5 and 5.2, x 512 8.8 and 9.9, x 1024 16.2 and 14.9; 4096 x 4096 34 and 27.
    const bool few = N <= 512;
    if (units <= 512 && !few) return launch_kernel(rows_kernel<NORM, CODES, TYPE, 256, 2, 1>, grid_of(N), 256, 0, stream, a);
    if (units <= 1024 && !few) return launch_kernel(rows_kernel<NORM, CODES, TYPE, 256, 4, 1>, grid_of(N), 256, 0, stream, a);
    if (units <= 1024) return launch_kernel(rows_kernel<NORM, CODES, TYPE, 1024, 1, 1>, grid_of(N), 1024, 0, stream, a);
    if (units <= 2048) return launch_kernel(rows_kernel<NORM, CODES, TYPE, 1024, 2, 1>, grid_of(N), 1024, 0, stream, a);
    if (units <= 4096) return launch_kernel(rows_kernel<NORM, CODES, TYPE, 1024, 4, 1>, grid_of(N), 1024, 0, stream, a);
    return launch_kernel(long_rows_kernel<NORM, CODES, TYPE>, grid_of(N), 1024, 0, stream, a);
}

template <int TYPE> hipError_t launch_type(const rows_args &a, bool norm, char *workspace, hipStream_t stream)
{
    const bool codes = a.out.type == SPMM_I8;
    if (norm) return codes ? launch<true, true, TYPE>(a, workspace, stream) : launch<true, false, TYPE>(a, workspace, stream);
    return codes ? launch<false, true, TYPE>(a, workspace, stream) : launch_elements<TYPE>(a, stream);
}

}  // namespace

int64_t rows_workspace(const rows_args &a, bool norm)
{
    if (a.x.by_token || (!norm && a.out.type != SPMM_I8)) return 0;
    const int unit = a.x.type == SPMM_F32 ? COLUMN_UNIT<SPMM_F32> : COLUMN_UNIT<SPMM_F16>;
    if (in_one_launch(a.features, a.tokens, unit)) return 0;
    const column_tiles t = tiles_of(a.features, a.tokens, unit);
    return (a.features + t.rows - 1) / t.rows * 2 * a.tokens * (int64_t)sizeof(float);
}

hipError_t rows_launch(const rows_args &a, bool norm, char *workspace, hipStream_t stream)
{
    switch (a.x.type) {
    case SPMM_F32: return launch_type<SPMM_F32>(a, norm, workspace, stream);
    case SPMM_F16: return launch_type<SPMM_F16>(a, norm, workspace, stream);
    default: return launch_type<SPMM_BF16>(a, norm, workspace, stream);
    }
}

}  // namespace layers
