/*
 * spmm_layers.h -- C ABI of the operators that stand beside the sparse product (spmm.h) in a layer with compressed
 * weights: the product with 4-bit weights, the root-mean-square norm that makes its operand and the gated
 * activation between two products.
 *
 * Activations are 2-D, features x tokens, as B and C of spmm_execute, and lie in memory in either order
 * (spmm_tensor_t).  Sizes, statuses, streams and devices are treated as in spmm.h: no call aborts or throws, every
 * failure is a status code; a call that computes is asynchronous, allocates nothing, does not synchronise, and every
 * buffer that it uses, its workspace too, belongs to its caller.  So any number of calls may be in flight on any
 * streams, and every call may be captured into a graph; two that overlap in time need workspaces of their own, as
 * they need outputs of their own.  Results are bit-identical from run to run.
 */
#ifndef SPMM_LAYERS_CDNA4_H
#define SPMM_LAYERS_CDNA4_H

#include "spmm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of activations. */
enum { SPMM_F32 = 0, SPMM_F16 = 1, SPMM_BF16 = 2, SPMM_I8 = 3 };

/*
 * A 2-D tensor in DEVICE memory, features x tokens: element (i, n) is at data[i * feature_stride + n * token_stride]
 * (strides in elements).  One of the two strides is 1:
 *   token_stride 1    one row of memory a feature, as B and C of spmm_execute; feature_stride >= tokens
 *   feature_stride 1  one row of memory a token; token_stride >= features
 * A stride along an extent of one element is not looked at.  Two tensors overlap where an element of one lies in one of
 * the other: rows of memory may lie between those of another tensor that are as far apart (in bytes; rows that are not as
 * far apart, of which some lie between the other's first and last, count as overlapping).  data is aligned to its element; it may be NULL where
 * the tensor is optional (the other fields are then not looked at) and where it has no element.
 */
typedef struct {
    void *data;
    int64_t feature_stride, token_stride;
    int32_t type; /* SPMM_F32, SPMM_F16, SPMM_BF16 or SPMM_I8 */
} spmm_tensor_t;

/* ---- the product with 4-bit weights ------------------------------------------------------------------------- */

typedef struct spmm_quant spmm_quant_t; /* opaque */

/*
 * Lays a matrix of 4-bit weights (M x K) out for the kernels and uploads it:
 *   W[m, k] = scale[m, k / group] * (code[m, k] - zero[m, k / group])
 *
 *   plan    HOST  out; set to NULL on failure
 *   M, K    rows / columns of W; 0 is legal; more than 2^26 / 2^30 is SPMM_ERR_UNSUPPORTED
 *   group   columns that share a scale: 32, 64 or a multiple of 128 (else SPMM_ERR_UNSUPPORTED); the last group of
 *           a row is shorter where K is not a multiple
 *   codes   HOST  uint8[M * ceil(K / 2)]: two codes of 0..15 a byte, that of the even column in the low half; rows
 *                 start at a byte, the high half of a row's last byte is not looked at where K is odd
 *   scales  HOST  float[M * ceil(K / group)], magnitudes up to 2^120 (else SPMM_ERR_INVALID_ARG)
 *   zeros   HOST  uint8[M * ceil(K / group)], each in 0..15 (else SPMM_ERR_INVALID_ARG), or NULL: 8 everywhere
 *
 * The arrays are only read during the call.  The plan owns its device memory on the device that is current at the
 * time of the call.  Uploads are ordered behind the work of the default stream; when the call returns, every stream
 * may use the plan.  A plan is never written again.
 */
spmm_status_t spmm_quant_create(spmm_quant_t **plan, int64_t M, int64_t K, int64_t group, const uint8_t *codes,
                                const float *scales, const uint8_t *zeros);

/* Frees the plan and its device memory.  NULL is a no-op returning SPMM_OK. */
spmm_status_t spmm_quant_destroy(spmm_quant_t *plan);

/* Read-only facts of a plan; any of the pointers may be NULL. */
spmm_status_t spmm_quant_describe(const spmm_quant_t *plan, int64_t *M, int64_t *K, int64_t *group,
                                  int64_t *device_bytes);

/*
 * Bytes of DEVICE memory that spmm_quant_execute needs as its workspace for N columns of a B of this type and
 * memory order (data is not read); 0: none, as always up to 16 columns.
 */
spmm_status_t spmm_quant_workspace(const spmm_quant_t *plan, const spmm_tensor_t *B, int64_t N, size_t *bytes);

/*
 * C <- W x B.
 *   B        K x N, any type.  Floating values may be infinite or NaN: they reach the elements of C that the sum
 *            says (an absent tail of a group adds nothing).  Codes (SPMM_I8) stand for code * B_scales[n] and lie
 *            one token a row (feature_stride 1, else SPMM_ERR_UNSUPPORTED)
 *   B_scales DEVICE  float[N] where B is SPMM_I8; else not looked at
 *   N        columns of B and C, 1 .. 2^31 - 1
 *   C        M x N, SPMM_F32, SPMM_F16 or SPMM_BF16; every element is overwritten; must not overlap B and B_scales
 *   workspace DEVICE, 16-byte aligned, of spmm_quant_workspace bytes or more (else SPMM_ERR_INVALID_ARG); its
 *            content before the call does not matter
 * Sums are held in 32 bits: weights enter as whole numbers (code - zero), a sum of up to 128 of them, or of a group
 * if that is smaller, is exact in whole numbers for codes and accumulated in fp32 for floating B (fp32 B in three
 * bf16 parts that add up to it), then multiplied by the group's scale in fp32.  Values of B below 2^-100 may count as
 * zero.
 */
spmm_status_t spmm_quant_execute(const spmm_quant_t *plan, const spmm_tensor_t *B, const float *B_scales, int64_t N,
                                 const spmm_tensor_t *C, void *workspace, size_t workspace_bytes, void *stream);

/* ---- between products ---------------------------------------------------------------------------------------- */

/*
 * 8-bit output (SPMM_I8): one row of memory a token (feature_stride 1), codes in -127..127 and a scale a token, so
 * that code * scale stands for the value.  With p the values before a token's common factor f and P = max |p| over
 * the token, in fp32: code = rint(p * (127 / P)), ties to even; scale = P * f / 127.  A token whose P is 0 has codes
 * and scale 0; one with an infinite or NaN value has codes 0 and scale NaN.
 */

typedef struct {
    spmm_tensor_t x;        /* K x N; SPMM_F32, SPMM_F16 or SPMM_BF16 */
    spmm_tensor_t residual; /* optional (data NULL): added to x; x's type and memory order */
    spmm_tensor_t total;    /* optional: where t = x + residual (x without one), rounded to x's type, is written; x's
                               type and memory order; may be x's or residual's own memory, with the same strides */
    const void *weight;     /* DEVICE [K] */
    int32_t weight_type;    /* SPMM_F32, SPMM_F16 or SPMM_BF16 */
    float eps;              /* >= 0 */
    spmm_tensor_t out;      /* K x N; any type; floating types in x's memory order */
    float *scales;          /* DEVICE [N] where out is SPMM_I8; else not looked at */
} spmm_norm_t;

/*
 * Root-mean-square norm over the features of every token, with the residual's addition:
 *   t = x + residual in fp32, rounded to x's type;  r = 1 / sqrt(mean_k t^2 + eps), in fp32;  out = t * r * weight
 * (8-bit output: p = t * weight, f = r).  Squares of values beyond 2^63 overflow and those of values
 * below 2^-75 are 0, as in fp32 arithmetic.
 *   K  features, 1 .. 2^31 - 1;  N  tokens, 1 .. 2^31 - 1
 *   workspace  DEVICE, 16-byte aligned, of spmm_norm_workspace bytes or more (0: may be NULL)
 * out and total must not overlap each other, nor x, residual, weight and scales but as said above.
 */
spmm_status_t spmm_norm_workspace(int64_t K, int64_t N, const spmm_norm_t *args, size_t *bytes);
spmm_status_t spmm_norm(int64_t K, int64_t N, const spmm_norm_t *args, void *workspace, size_t workspace_bytes,
                        void *stream);

enum {
    SPMM_ACT_SILU = 0, /* x / (1 + exp(-x)) */
    SPMM_ACT_GELU = 1, /* x / 2 * (1 + tanh(sqrt(2 / pi) * (x + 0.044715 x^3))) */
    SPMM_ACT_RELU = 2  /* max(x, 0), NaN stays NaN */
};

typedef struct {
    spmm_tensor_t a;   /* F x N; SPMM_F32, SPMM_F16 or SPMM_BF16 */
    spmm_tensor_t b;   /* optional (data NULL: 1 everywhere); a's type and memory order */
    spmm_tensor_t out; /* F x N; any type; floating types in a's memory order */
    float *scales;     /* DEVICE [N] where out is SPMM_I8; else not looked at */
    int32_t act;       /* SPMM_ACT_* */
} spmm_gate_t;

/*
 * Gated activation: out = act(a) * b, in fp32 (8-bit output: p = act(a) * b, f = 1).  silu and gelu are right to 2^-20 of
 * their value, u = a and u = 2 sqrt(2 / pi) (a + 0.044715 a^3) taken as they come out in fp32 and values below 2^-119 counting as 0 or not;
 * where out is not SPMM_F32, before its rounding, to (2 |u| + 16) 2^-24.  F, N and the workspace as for
 * spmm_norm.  out must not overlap a, b and scales.
 */
spmm_status_t spmm_gate_workspace(int64_t F, int64_t N, const spmm_gate_t *args, size_t *bytes);
spmm_status_t spmm_gate(int64_t F, int64_t N, const spmm_gate_t *args, void *workspace, size_t workspace_bytes,
                        void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPMM_LAYERS_CDNA4_H */
