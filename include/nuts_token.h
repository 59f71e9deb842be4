/*
 * nuts_token.h -- C ABI of the operators of a token model's potential
 * (MI355X, gfx950), part of the library declared in nuts.h: handles, status
 * codes and messages are the ones declared there.
 *
 * U of a model whose covariates are tokens, whose mean is a network and whose
 * outcome is one of V classes is made of four operators and their gradients:
 * nuts_embedding, nuts_linear, nuts_gated, nuts_categorical.
 *
 * Conventions of these entry points:
 *   - Everything is memory of the handle's device (NUTS_EINVAL otherwise).  A
 *     call only enqueues kernels on `hip_stream` (NULL: the device's default
 *     stream) and returns: it allocates nothing, copies nothing and does not
 *     wait, so it can be captured into a HIP graph.  Inputs and workspace must
 *     stay until the stream has passed the call.
 *   - dtype is NUTS_F32 or NUTS_BF16 (else NUTS_EINVAL) and holds for every
 *     pointer declared void*.  Matrices are row-major with a row stride ld in
 *     elements, ld >= the row's length; any alignment of the element type is
 *     taken (bf16 rows of a whole multiple of 8 elements on 16-byte boundaries
 *     are the fast case).  Sizes are >= 0 and below 2^31; strides of the linear
 *     layer's and the gated block's matrices below 2^23, and of any two of the three
 *     sizes of a product, (one / 64) (other / 32) below 2^24 (NUTS_EUNSUPPORTED);
 *     nothing is done where an output is empty, and an empty sum is zero.
 *   - A scale is taken in fp32: zero, or a magnitude of 2^-126 to the largest fp32
 *     value (NUTS_EINVAL otherwise).
 *   - Outputs do not overlap inputs, except where stated.
 *   - Arithmetic is fp32 or wider, rounded once on output.  bf16 matrix
 *     products run on the bf16 matrix cores with fp32 sums; fp32 ones either on
 *     the fp32 matrix cores (forward, few rows of x) or as three bf16 parts a factor
 *     (products of relative size 2^-22 and below left out; a factor to multiples
 *     of 2^-133, so below 2^-110 it has fewer digits and below 2^-133 it is zero).
 *     Infinities and NaN come out as in fp32 products of these factors.
 *   - Where a function nuts_..._workspace exists, the call needs that many
 *     bytes of device memory, 16-byte aligned, in `workspace` (NUTS_EINVAL if
 *     fewer are given); the size is a function of the arguments alone, zero in
 *     many cases, and negative (a NUTS_ code) for arguments that the call
 *     refuses.  Two calls that may run at the same time need workspaces of
 *     their own.
 *   - Results do not depend on what else runs: sums are taken in a fixed
 *     order, without floating-point atomics. */
#ifndef NUTS_TOKEN_H
#define NUTS_TOKEN_H

#include "nuts.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { NUTS_BF16 = 2 };  /* beside NUTS_F32: the types of these operators */

enum {
    NUTS_ACT_NONE = 0,
    NUTS_ACT_RELU = 1,     /* max(z, 0), slope 0 at 0 */
    NUTS_ACT_SIGMOID = 2,  /* 1 / (1 + exp(-z)) */
    NUTS_ACT_SILU = 3,     /* z sigmoid(z) */
    NUTS_ACT_GELU = 4      /* z Phi(z), Phi the normal distribution function */
};

/* Added to `act` of a gradient's arguments: for bf16, dz (dg and du) is rounded
 * to bf16 for the matrix products, which halves them.  Without it two bf16 parts
 * hold 16 of its bits, so that the rounding of the outputs is all that shows. */
enum { NUTS_ROUND_DZ = 256 };

/* Embedding of tokens: out[i] = scale table[ids[i]], i < N, rows of D
 * elements; a row of zeros where ids[i] lies outside [0, V) (a position
 * without a token). */
typedef struct {
    int32_t dtype;
    int32_t _reserved;
    int64_t N, V, D;
    const int64_t* ids;  /* [N] */
    const void* table;   /* [V][D], row stride ld_table */
    int64_t ld_table;
    double scale;
    void* out;           /* [N][D], row stride ld_out */
    int64_t ld_out;
} nuts_embedding_args;
int nuts_embedding(nuts_handle* h, const nuts_embedding_args* a, void* hip_stream);

/* Gradient of the table: dtable[v] = scale sum over {i: ids[i] = v} of
 * dout[i] for every v < V (zeros where no position holds v; ids outside
 * [0, V) are skipped).  The positions are sorted by token (stable, on the
 * device), and each token's rows are summed in fp32 in that order.
 * N <= 2^26, V <= 2^30 - 1. */
typedef struct {
    int32_t dtype;
    int32_t _reserved;
    int64_t N, V, D;
    const int64_t* ids;  /* [N] */
    const void* dout;    /* [N][D], row stride ld_dout */
    int64_t ld_dout;
    double scale;
    void* dtable;        /* [V][D], row stride ld_dtable */
    int64_t ld_dtable;
} nuts_embedding_grad_args;
int64_t nuts_embedding_grad_workspace(const nuts_embedding_grad_args* a);
int nuts_embedding_grad(nuts_handle* h, const nuts_embedding_grad_args* a, void* workspace, int64_t workspace_bytes,
    void* hip_stream);

/* Linear layer: y = act(z) + residual, z = x w^T + bias.  residual may be y
 * itself (same stride).  pre, if given, receives z in fp32 for the gradient. */
typedef struct {
    int32_t dtype;
    int32_t act;           /* NUTS_ACT_ */
    int64_t M, N, K;
    const void* x;         /* [M][K], row stride ldx */
    int64_t ldx;
    const void* w;         /* [N][K], row stride ldw */
    int64_t ldw;
    const void* bias;      /* [N], or NULL */
    const void* residual;  /* [M][N], row stride ldr, or NULL */
    int64_t ldr;
    void* y;               /* [M][N], row stride ldy */
    int64_t ldy;
    float* pre;            /* [M][N], or NULL */
} nuts_linear_args;
int64_t nuts_linear_workspace(const nuts_linear_args* a);
int nuts_linear(nuts_handle* h, const nuts_linear_args* a, void* workspace, int64_t workspace_bytes,
    void* hip_stream);

/* Its gradients for dy: dz = dy act'(z); dx = dz w, dw = dz^T x, dbias =
 * sum over the rows of dz (residual's gradient is dy).  Each output may be
 * NULL; pre may be NULL with NUTS_ACT_NONE.  For bf16 with an activation the two
 * products (not dbias) take dz in two bf16 parts, in one with NUTS_ROUND_DZ. */
typedef struct {
    int32_t dtype;
    int32_t act;           /* NUTS_ACT_, + NUTS_ROUND_DZ */
    int64_t M, N, K;
    const void* dy;    /* [M][N], row stride lddy */
    int64_t lddy;
    const void* x;     /* [M][K], row stride ldx (NULL without dw) */
    int64_t ldx;
    const void* w;     /* [N][K], row stride ldw (NULL without dx) */
    int64_t ldw;
    const float* pre;  /* [M][N] */
    void* dx;          /* [M][K], row stride lddx, or NULL */
    int64_t lddx;
    void* dw;          /* [N][K], row stride lddw, or NULL */
    int64_t lddw;
    void* dbias;       /* [N], or NULL */
} nuts_linear_grad_args;
int64_t nuts_linear_grad_workspace(const nuts_linear_grad_args* a);
int nuts_linear_grad(nuts_handle* h, const nuts_linear_grad_args* a, void* workspace, int64_t workspace_bytes,
    void* hip_stream);

/* Gated block: y = act(g) u, g = x wg^T, u = x wu^T, both products in one
 * kernel.  pre, if given, receives g and u in fp32 for the gradient. */
typedef struct {
    int32_t dtype;
    int32_t act;
    int64_t M, F, K;
    const void* x;   /* [M][K], row stride ldx */
    int64_t ldx;
    const void* wg;  /* [F][K], row stride ldwg */
    int64_t ldwg;
    const void* wu;  /* [F][K], row stride ldwu */
    int64_t ldwu;
    void* y;         /* [M][F], row stride ldy */
    int64_t ldy;
    float* pre;      /* [2][M][F]: g, then u; or NULL */
} nuts_gated_args;
int64_t nuts_gated_workspace(const nuts_gated_args* a);
int nuts_gated(nuts_handle* h, const nuts_gated_args* a, void* workspace, int64_t workspace_bytes,
    void* hip_stream);

/* Its gradients for dy: dg = dy u act'(g), du = dy act(g); dx = dg wg +
 * du wu, dwg = dg^T x, dwu = du^T x.  dx may be NULL, and dwg and dwu both.
 * For bf16 the products take dg and du in two bf16 parts, in one with
 * NUTS_ROUND_DZ. */
typedef struct {
    int32_t dtype;
    int32_t act;       /* NUTS_ACT_, + NUTS_ROUND_DZ */
    int64_t M, F, K;
    const void* dy;    /* [M][F], row stride lddy */
    int64_t lddy;
    const void* x;     /* [M][K], row stride ldx (NULL without dwg) */
    int64_t ldx;
    const void* wg;    /* [F][K], row stride ldwg (NULL without dx) */
    int64_t ldwg;
    const void* wu;    /* [F][K], row stride ldwu (NULL without dx) */
    int64_t ldwu;
    const float* pre;  /* [2][M][F] */
    void* dx;          /* [M][K], row stride lddx, or NULL */
    int64_t lddx;
    void* dwg;         /* [F][K], row stride lddwg, or NULL */
    int64_t lddwg;
    void* dwu;         /* [F][K], row stride lddwu, or NULL */
    int64_t lddwu;
} nuts_gated_grad_args;
int64_t nuts_gated_grad_workspace(const nuts_gated_grad_args* a);
int nuts_gated_grad(nuts_handle* h, const nuts_gated_grad_args* a, void* workspace, int64_t workspace_bytes,
    void* hip_stream);

/* Categorical likelihood: nll[i] = log sum_j exp(logits[i][j]) -
 * logits[i][targets[i]] (fp32), total = sum of nll (fp64), dlogits[i][j] =
 * scale (softmax(logits[i])[j] - [j = targets[i]]).  A target outside [0, V)
 * marks a row without an observation: nll 0 and a zero gradient, whatever its
 * logits.  A logit of -infinity is a class that cannot occur (probability 0);
 * where the target's is, or every one is, nll is +infinity, and where every
 * one is the gradient is zero.  dlogits may be logits itself (same stride).
 * total and dlogits may be NULL. */
typedef struct {
    int32_t dtype;
    int32_t _reserved;
    int64_t M, V;
    const void* logits;      /* [M][V], row stride ld_logits */
    int64_t ld_logits;
    const int64_t* targets;  /* [M] */
    double scale;
    float* nll;              /* [M] */
    double* total;           /* [1], or NULL */
    void* dlogits;           /* [M][V], row stride ld_dlogits, or NULL */
    int64_t ld_dlogits;
} nuts_categorical_args;
int nuts_categorical(nuts_handle* h, const nuts_categorical_args* a, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* NUTS_TOKEN_H */
