// What the operators beside the sparse product share (internal): the layout of 4-bit weights, the shapes that the
// host hands to the kernels and the launchers.
#ifndef SPMM_LAYERS_H
#define SPMM_LAYERS_H

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace layers {

// ---- 4-bit weights -------------------------------------------------------------------------------------------
//
// Rows come in tiles of TILE_ROWS (the columns of one matrix instruction), columns in blocks of BLOCK_COLS.  The
// codes of a (tile, block) are 1 KiB in one piece, which a wave reads as 16 bytes a lane: lane 16 q + r holds the
// codes of row r, word s of its four those of columns 32 s + 8 q + j, j = 0..7, of the block.  So one word is what a
// lane hands to a matrix instruction of 32 columns, and the four words of a lane lie in one group of 128 columns, in
// one of 64 two by two, in one of 32 each.  Inside a word nibble i holds j = NIBBLE_COLUMN[i]: a shift by 4 i and one mask give
// the neighbours 2 i and 2 i + 1 in the low halves of a 32-bit word, as 16-bit operands are held.  A nibble is code - 8 in two's complement.
//
// Scales and zero points are [tile][span][TILE_ROWS][groups of a span]: a span is a group, or the groups of a block where they are
// shorter, which a lane reads at once.  Rows past M and groups past K have scale 0 and zero point 8, columns past K the code of
// their group's zero point, so that they are whole numbers of 0.  Memory is there for whole TILES_OF tiles, rows past M as above: a wave may have
// that many.
constexpr int TILE_ROWS = 16, BLOCK_COLS = 128, BLOCK_WORDS = TILE_ROWS * BLOCK_COLS / 8, TILES_OF = 4;
constexpr int NIBBLE_COLUMN[8] = {0, 2, 4, 6, 1, 3, 5, 7};

struct quant_matrix {
    int64_t M, K, group;
    int32_t tiles, blocks, groups;  // ceil(M / 16), ceil(K / 128), ceil(K / group)
    int32_t spans, span_groups;     // spans of K, groups of one
    const uint32_t *codes;          // DEVICE
    const float *scales;
    const uint8_t *zeros;           // NULL: 8 everywhere
};

// A tensor as the kernels see it: `ld` elements from one row of memory to the next.
struct tensor {
    char *data;
    int64_t ld;
    int32_t type;  // SPMM_F32 ...
    bool by_token; // a row of memory is a token (else a feature)
};

// Bytes of B laid out for the product, and the launches.
int64_t quant_workspace(const quant_matrix &w, const tensor &B, int64_t N);
hipError_t quant_execute(const quant_matrix &w, const tensor &B, const float *B_scales, int64_t N, const tensor &C, char *workspace, hipStream_t stream);

// ---- norm and gate -------------------------------------------------------------------------------------------
struct rows_args {
    int64_t features, tokens;
    tensor x, y;      // norm: x and the residual; gate: a and b (data NULL: none)
    tensor total;     // norm: where the sum goes (data NULL: nowhere)
    tensor out;
    float *scales;
    const char *weight;
    int32_t weight_type;
    float eps;
    int32_t act;
    double per_feature;  // 1 / features
};

int64_t rows_workspace(const rows_args &a, bool norm);
hipError_t rows_launch(const rows_args &a, bool norm, char *workspace, hipStream_t stream);

}  // namespace layers

#endif
