/*
 * razer_step.h -- what a serving step needs beside the linear layers (razer.h) and the cache
 * (razer_cache.h) of the MI355X (gfx950) RaZeR library:
 *
 *   razer_norm          root-mean-square norm of the hidden states with the residual's addition; the
 *                       output in bf16 or fp32, or as the 4-bit activations that razer_linear reads
 *   razer_moe_route     the experts of each token: the router's product and the choice of top_k
 *   razer_moe_experts   the chosen experts' products on 4-bit weights, summed with the routing weights
 *   razer_sample        one token per row of logits: temperature, top-k, top-p, min-p
 *
 * Like razer.h: device pointers, the caller's stream, status codes, no allocation, no
 * synchronisation, nothing kept from one call to the next.  Values that steer memory accesses on the
 * device (expert ids) are checked there.  Every result is the same for the same inputs and sizes.
 * razer_moe_experts has kernels with more than 64 KiB of LDS: as for razer_linear, a caller that captures a
 * stream into a HIP graph makes one ordinary call of each shape first.
 */
#ifndef RAZER_STEP_H
#define RAZER_STEP_H

#include "razer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* y = h / sqrt(mean(h^2) + eps) * (weight_offset + weight) over each row, h = x + residual.
 * h is one fp32 addition, its mean of squares and the root are formed in 64 bits, and
 * y = (h * r) * w with r and w = weight_offset + weight in fp32, each operation rounded once.  y is
 * rounded to the type of `out`, or encoded as razer_quantize does with fp32 elements and
 * RAZER_GIVEN_TENSOR_SCALE (codes and scale bytes are then the ones that it would write), or both.
 * sum: h in the residual's type.  A row with an infinity or a NaN gives what the formula gives;
 * codes of such a row are unspecified.
 * out may be x itself and sum may be residual itself (same type and leading dimension); otherwise
 * nothing written may overlap what is read. */
typedef struct {
    const void *x;             /* [rows][ld_x] of x_dtype, cols used                        */
    int64_t ld_x;
    const void *residual;      /* [rows][ld_residual] of residual_dtype, or NULL            */
    int64_t ld_residual;
    void *sum;                 /* [rows][ld_sum] of residual_dtype, or NULL                 */
    int64_t ld_sum;
    const void *weight;        /* [cols] of weight_dtype                                    */
    void *out;                 /* [rows][ld_out] of out_dtype, or NULL                      */
    int64_t ld_out;
    uint8_t *codes;            /* [rows][cols/2] and                                        */
    uint8_t *scales;           /* [rows][cols/block], dense, 16-byte aligned; or NULL       */
    const float *tensor_scale; /* device float: with codes                                  */
    razer_config cfg;          /* with codes: RAZER_FMT_ACT, as for razer_quantize          */
    int64_t rows, cols;        /* rows < 2^22; cols <= 32768, with codes a multiple of max(32, block) */
    int32_t x_dtype, residual_dtype, weight_dtype, out_dtype;      /* RAZER_F32, RAZER_BF16 */
    float eps, weight_offset;
} razer_norm_args;

/* Pointers aligned to their elements; rows of 16-byte aligned memory whose leading dimensions are multiples
 * of 16 bytes (weight: 16-byte aligned; cols % 8 == 0) go eight elements at a time, all others one by one;
 * with codes the former is required (RAZER_ERR_ALIGN).                                                  */
razer_status razer_norm(const razer_norm_args *args, void *hip_stream);

/* The top_k experts of each token, best first, and the weights of their outputs.
 *   l[t][e]   = sum_k x[t][k] router[e][k]                       (or logits[t][e], given)
 *   score     = l (RAZER_SOFTMAX) or 1 / (1 + exp(-l)) (RAZER_SIGMOID);  order by score + bias[e] -- with RAZER_SOFTMAX the
 *               bias is added to the product itself, not to its share exp(l) / sum exp(l) --
 *               equal ones by the lower index; a NaN stands behind everything (one among the products weighs 0),
 *               +infinity counts as the largest finite number
 *   weight    = exp(l) / sum_e exp(l) over all experts, or 1 / (1 + exp(-l)); without the bias
 *   renormalize: divided by the sum of the token's top_k weights;  then multiplied by scale
 * Products of bf16 operands are summed over 32 at a time in fp32 and from there on in 64 bits; scores, their
 * order and the weights are formed in 64 bits and the weights rounded to fp32 once.  */
enum { RAZER_SOFTMAX = 0, RAZER_SIGMOID = 1 };
typedef struct {
    const void *x;             /* bf16 [tokens][ld_x], hidden used; NULL: logits are given  */
    int64_t ld_x;
    const void *router;        /* bf16 [experts][hidden]                                    */
    const void *logits;        /* [tokens][ld_logits] of logits_dtype, where x is NULL      */
    int64_t ld_logits;
    const float *bias;         /* [experts] or NULL                                         */
    int32_t *ids;              /* [tokens][top_k]                                           */
    float *weights;            /* [tokens][top_k]                                           */
    int64_t tokens;            /* <= 2^20                                                   */
    int32_t hidden;            /* a multiple of 32                                          */
    int32_t experts;           /* 1 .. 512                                                  */
    int32_t top_k;             /* 1 .. min(experts, 32)                                     */
    int32_t score;             /* RAZER_SOFTMAX or RAZER_SIGMOID                            */
    int32_t renormalize;
    int32_t logits_dtype;
    float scale;
} razer_moe_route_args;

/* workspace: device, 16-byte aligned, >= razer_moe_route_workspace_bytes(args) bytes (0 with given logits);
 * calls that overlap in time need their own.  x and router 16-byte aligned, ld_x a multiple of 8. */
size_t razer_moe_route_workspace_bytes(const razer_moe_route_args *args);
razer_status razer_moe_route(const razer_moe_route_args *args, void *workspace, size_t workspace_bytes,
                             void *hip_stream);

/* The weights of one projection of all experts: RAZER_FMT_WEIGHT tensors of equal shape, one behind the
 * other (codes [experts][rows][cols/2], scales [experts][rows][cols/block], 16-byte aligned), each with its
 * own tensor scale. */
typedef struct {
    const uint8_t *codes;
    const uint8_t *scales;
    const float *tensor_scales;    /* [experts] */
    int64_t rows, cols;
    int32_t experts;
    razer_config cfg;
} razer_experts;

/* y[t] = sum_j weights[t][j] * down_e( act(gate_e(x[t])) * up_e(x[t]) ), e = ids[t][j]
 * act: z / (1 + exp(-z)) (RAZER_SILU), 0.5 z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) (RAZER_GELU) or
 * max(z, 0) (RAZER_RELU); without `up` the activation alone.  Products of bf16 activations and exactly decoded
 * weights (but for special values of 9.5: 9.5 times a block scale whose significand is 15 / 8 has 9 bits and is rounded to
 * the 8 of a bf16, by 1 / 285 of itself) are accumulated in fp32; what stands between the two products is kept to 16 bits (two bf16 numbers, the operand
 * type of the second product); the sum over j is formed in fp32 and rounded to bf16 once.
 * An id outside 0 .. experts-1 counts as no expert: a token without experts gets 0.  A token may name an expert
 * more than once.
 * Made for a serving step's few tokens, where the experts' weights are what has to be read: each expert that
 * some token chose is read once for up to 32 of its tokens.  Any number of tokens is right. */
enum { RAZER_SILU = 0, RAZER_GELU = 1, RAZER_RELU = 2 };
typedef struct {
    const void *x;                 /* bf16 [tokens][ld_x]: gate->cols used                   */
    int64_t ld_x;
    const int32_t *ids;            /* [tokens][top_k]                                        */
    const float *weights;          /* [tokens][top_k]                                        */
    void *y;                       /* bf16 [tokens][ld_y]: down->rows used                   */
    int64_t ld_y;
    int64_t tokens;                /* tokens * top_k <= 2^20; tokens * ld_x and tokens *     */
                                   /* top_k * gate->rows < 2^31                              */
    int32_t top_k;                 /* 1 .. 32                                                */
    int32_t act;
    const razer_experts *gate;     /* [experts][inter][hidden]                               */
    const razer_experts *up;       /* the same, or NULL                                      */
    const razer_experts *down;     /* [experts][hidden_out][inter]                           */
} razer_moe_args;

/* workspace: device, 16-byte aligned, >= razer_moe_workspace_bytes(args) bytes, which depends on the sizes
 * alone and is no smaller for more tokens; calls that overlap in time need their own.  At most 1024 experts;
 * gate and up in the same format; x and y 16-byte aligned, ld_x and ld_y multiples of 8; every rows a multiple
 * of 32, cols as in razer.h and at most 2^20. */
size_t razer_moe_workspace_bytes(const razer_moe_args *args);
razer_status razer_moe_experts(const razer_moe_args *args, void *workspace, size_t workspace_bytes, void *hip_stream);

/* One token of each row.  The tokens of a row stand in the order of their logits, largest first, equal ones by the lower
 * index, each with the weight exp((logit - largest) / temperature).  Of them stay
 *   the first top_k (<= 0: all);
 *   of these the fewest first ones whose weights reach top_p of theirs together, at least one (>= 1: all);
 *   of these the ones with a weight of at least min_p (<= 0: all; the largest is 1), at least one.
 * The row's token is the first of the order whose running sum of weights exceeds uniform times the sum over what stays
 * (uniform below 0 counts as 0; 1 and more give the last token that stays), and logprob the logarithm of its share of it.
 * temperature <= 0: the first of the order, logprob 0; an infinite one counts as the largest finite number.  A logit of
 * -infinity or NaN is no token, +infinity counts as the largest finite number of its type; a row without any token
 * gives -1 and -infinity.  A setting that is NaN counts as absent (temperature: as 0, uniform: as 0).
 * Weights are formed in 64 bits; their sums are the same in any order and right to 2^-27 of themselves.  Tokens that weigh
 * less than 2^-57 of the largest may count as weightless. */
typedef struct {
    const void *logits;            /* [rows][ld] of dtype, vocab used                        */
    int64_t ld;
    const float *uniform;          /* [rows], in [0, 1)                                      */
    const float *temperature;      /* [rows] or NULL: 1                                      */
    const int32_t *top_k;          /* [rows] or NULL                                         */
    const float *top_p;            /* [rows] or NULL                                         */
    const float *min_p;            /* [rows] or NULL                                         */
    int32_t *tokens;               /* [rows]                                                 */
    float *logprobs;               /* [rows] or NULL                                         */
    int64_t rows, vocab;           /* rows < 2^22, 1 <= vocab <= 2^24                        */
    int32_t dtype;                 /* RAZER_F32 or RAZER_BF16                                */
} razer_sample_args;

/* workspace: device, 16-byte aligned, >= razer_sample_workspace_bytes(args) bytes (0: may be NULL); calls that
 * overlap in time need their own.  Pointers aligned to their elements. */
size_t razer_sample_workspace_bytes(const razer_sample_args *args);
razer_status razer_sample(const razer_sample_args *args, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RAZER_STEP_H */
