/*
 * cconv, operators of a gated feed-forward sub-block (row-major token matrices), NVIDIA B200.
 *
 * Part of libcconv.so (see cconv.h for the convolution).  T tokens, D channels, F hidden channels:
 *
 *   feed-forward    y = (act(x Wg^T) * (x Wu^T)) Wd^T                     and its gradients
 *   residual norm   r' = scale r + gate * norm(y) * w_post,  x = norm(r') * w_pre   and its gradients
 *                   norm(v) = v / sqrt(mean(v^2) + eps), over the D channels of a token
 *   8-bit product   C[m,n] = sum_kb (sa[m,kb] sb[n/128,kb]) sum_{k in block kb} A[m,k] B[n,k]
 *   quantisation    8-bit values (e4m3) and a scale for each 1 x 128 or 128 x 128 block
 *   4-bit product   C[m,n] = sum_g s[n,g] sum_{k in group g} (q[n,k] - z[n,g]) X[m,k], and the quantiser of its weights
 *   mixture         y = sum_j p_j ffn_{e_j}(x) over the k of E experts that a router scores highest, for a few tokens
 *   clipping        norm over all elements of a list of gradients, and factor = min(1, max_norm / (norm + eps))
 *   norm in 8 bits  the residual norm whose x is written as 8-bit values and scales
 *
 * Matrices are given by the address of element (0,0) and two strides in elements.  Strides of inputs
 * are any non-negative numbers (0 repeats a row or column); the elements of an output are distinct.
 * Addresses are aligned to the element.  Rows of unit column stride whose address and row pitch are
 * multiples of 16 bytes are read in place; other operands of the products are first copied into the
 * workspace in that layout.
 *
 * Everything is computed from values in 32 bits: products accumulate, norms and sums of gradients are
 * held in fp32, and each output is rounded once to its type.  The hidden activations h = act(g) * u
 * and the gradients of the pre-activations, which are operands of the tensor cores, are rounded to
 * the type in between (fp16: infinite beyond 65504); forward calls of up to 4 tokens whose operands are
 * read in place keep what the rounding of h left.  The last bits of a token's result may so depend on
 * how many tokens share its call.  They do not depend on timing: no sum is formed by atomics.
 *
 * Ownership: all pointers are DEVICE pointers of the current device, owned by the caller; a NULL
 * `data` stands for an absent matrix where the text allows one.  The workspace is device memory,
 * 256-byte aligned, of at least the size that the matching *_workspace function gives for the same
 * arguments; its contents do not matter before or after a call, and calls that may run at the same
 * time need workspaces of their own.  Outputs must not overlap inputs, each other or the workspace,
 * but for the two cases named below, where an output may be one input itself (address and strides).
 * (Slices of one array, and columns that lie in it in turn, are told from overlaps by pitch and strides;
 * operands that interleave in other ways are refused.)
 * Calls are asynchronous on `cuda_stream`, ordered with the stream's other work like any kernel,
 * allocate nothing, and may be captured in a CUDA graph.
 *
 * Errors: CCONV_OK (0) or a negative code as in cconv.h; nothing throws, aborts or traps.  Lengths
 * may be zero (the result is then empty, gradients of weights are zero).
 */
#ifndef CCONV_BLOCK_H_
#define CCONV_BLOCK_H_

#include "cconv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define CCONV_TYPE_BF16 0
#define CCONV_TYPE_FP16 1
#define CCONV_TYPE_FP32 2

/* Activations of the gate: g/(1+exp(-g)), g Phi(g), its tanh form, max(g,0). */
#define CCONV_ACT_SILU 0
#define CCONV_ACT_GELU 1
#define CCONV_ACT_GELU_TANH 2
#define CCONV_ACT_RELU 3

typedef struct {
  void* data; /* element (0,0) */
  int64_t row_stride, col_stride;
} cconv_matrix;

/* ---- gated feed-forward block ------------------------------------------------------------------ */
typedef struct {
  int64_t T, D, F;
  int32_t dtype; /* CCONV_TYPE_BF16 or _FP16, of every matrix */
  int32_t act;
  cconv_matrix x;            /* [T][D] */
  cconv_matrix w_gate, w_up; /* [F][D] */
  cconv_matrix w_down;       /* [D][F] */
  cconv_matrix gate_pre, up_pre; /* [T][F]: x Wg^T and x Wu^T.  Forward: written if given (both or
                                    neither); backward: read */
  cconv_matrix out;          /* forward only: y [T][D] */
  cconv_matrix dout, dx;     /* backward only: dL/dy in, dL/dx out, [T][D] */
  cconv_matrix dw_gate, dw_up, dw_down; /* backward only, out: shaped like the weights */
  void* workspace;
  uint64_t workspace_bytes;
} cconv_ffn_args;

/* Bytes of workspace that the call with these arguments needs (>= 0), or a negative code.  Only the
 * sizes, types, strides and alignment of the addresses matter (NULL is aligned, but for gate_pre and
 * up_pre of the forward call, which it makes absent); nothing is dereferenced. */
int64_t cconv_ffn_forward_workspace(const cconv_ffn_args* args);
int64_t cconv_ffn_backward_workspace(const cconv_ffn_args* args);
int cconv_ffn_forward(const cconv_ffn_args* args, void* cuda_stream);
/* Every gradient is written.  h is formed again from gate_pre and up_pre. */
int cconv_ffn_backward(const cconv_ffn_args* args, void* cuda_stream);

/* ---- norms before and after a block, with its gate and residual scale -------------------------- */
typedef struct {
  int64_t T, D;
  int32_t dtype;         /* CCONV_TYPE_*, of every array */
  float scale, eps;      /* eps > 0 */
  int64_t rows_per_gate; /* token t uses gate row t / rows_per_gate; 0: all tokens use row 0 */
  cconv_matrix resid;     /* forward in: r [T][D] */
  cconv_matrix block;     /* in: y [T][D]; absent: r' = scale r */
  cconv_matrix gate;      /* in: [ceil(T / rows_per_gate)][D]; absent: 1 */
  const void* w_post;     /* in: [D]; absent: y is not normed */
  const void* w_pre;      /* in: [D]; absent: 1 */
  cconv_matrix resid_out; /* r' [T][D]: forward out, may be `resid` itself; backward in */
  cconv_matrix norm_out;  /* forward out: x [T][D]; absent: no second norm */
  /* backward: */
  cconv_matrix dresid_out; /* in: dL/dr' by its direct uses; absent: 0 */
  cconv_matrix dnorm_out;  /* in: dL/dx; absent: 0 */
  cconv_matrix dresid;     /* out, may be `dresid_out` itself */
  cconv_matrix dblock;     /* out; given exactly when `block` is */
  cconv_matrix dgate;      /* out; given exactly when `gate` is */
  void* dw_post;           /* out; given exactly when `w_post` is */
  void* dw_pre;            /* out; given exactly when `w_pre` and `dnorm_out` are */
  void* workspace;         /* backward only */
  uint64_t workspace_bytes;
} cconv_residual_norm_args;
/* Column strides are 1; row strides any. */

int64_t cconv_residual_norm_backward_workspace(const cconv_residual_norm_args* args);
int cconv_residual_norm_forward(const cconv_residual_norm_args* args, void* cuda_stream);
int cconv_residual_norm_backward(const cconv_residual_norm_args* args, void* cuda_stream);

/* The forward call with x in 8 bits, a scale for each 128 channels of a token, as cconv_quantize_blocks gives
 * them for x before its rounding to `dtype`: scale = max|x| / 448, q = x / scale.  norm.norm_out (x rounded to
 * `dtype`) may be given too; resid_out as in the forward call. */
typedef struct {
  cconv_residual_norm_args norm; /* its forward operands; the others and the workspace are not looked at */
  cconv_matrix q;                /* out: [T][D] e4m3, column stride 1 */
  cconv_matrix q_scale;          /* out: [T][ceil(D/128)] fp32, any strides */
} cconv_residual_norm_quantize_args;

int cconv_residual_norm_quantize(const cconv_residual_norm_quantize_args* args, void* cuda_stream);

/* ---- product in 8-bit floating point with a scale for each block of 128 ------------------------ */
typedef struct {
  int64_t M, N, K;
  int32_t dtype;        /* CCONV_TYPE_*, of C */
  int32_t reserved;     /* 0 */
  cconv_matrix a;       /* [M][K] e4m3 */
  cconv_matrix b;       /* [N][K] e4m3 */
  cconv_matrix a_scale; /* [M][ceil(K/128)] fp32 */
  cconv_matrix b_scale; /* [ceil(N/128)][ceil(K/128)] fp32 */
  cconv_matrix c;       /* out: [M][N] */
  void* workspace;
  uint64_t workspace_bytes;
} cconv_fp8_product_args;

int64_t cconv_fp8_product_workspace(const cconv_fp8_product_args* args);
int cconv_fp8_product(const cconv_fp8_product_args* args, void* cuda_stream);

/* ---- quantisation in blocks ---------------------------------------------------------------------
 * scale = max|x| over the block / 448 (the largest e4m3 value), q = x / scale rounded to nearest,
 * ties to even; a block of zeros has scale 0 and q = 0; a block that holds a NaN has scale NaN, one
 * that holds an infinity scale infinity (and q = NaN where x is infinite, 0 elsewhere). */
typedef struct {
  int64_t T, D;
  int32_t dtype;      /* CCONV_TYPE_*, of x */
  int32_t block_rows; /* 1 or 128 */
  cconv_matrix x;     /* in: [T][D] */
  cconv_matrix q;     /* out: [T][D] e4m3 */
  cconv_matrix scale; /* out: [ceil(T/block_rows)][ceil(D/128)] fp32 */
} cconv_quantize_args;

int cconv_quantize_blocks(const cconv_quantize_args* args, void* cuda_stream);

/* ---- product with 4-bit weights and a scale for each group of a row --------------------------------
 *   C[m,n] = sum_g scale[n,g] sum_{k in group g} (q[n,k] - zero[n,g]) X[m,k],   group g: k / group = g
 * Element 2j of a row of q is the low half of byte j, element 2j + 1 its high half; what lies behind K in the last
 * byte does not matter.  A token that holds an infinity or a NaN gives infinities or NaN.
 * Up to 64 tokens, sums are of q and X as they are, in fp32, and scaled in fp32 (of one or two tokens, and up to 8 of small
 * matrices, as sums of (16 + q) X less (16 + zero) times that of X: fp32's rounding is then of these); with more, the weights
 * scale (q - zero) are rounded to the precision of `dtype` first, as operands of the tensor cores (fp16: not to its range;
 * a row's groups whose scale is below 2^-24 of its largest lose bits, 2^-31 of that one at most). */
typedef struct {
  int64_t M, N, K;
  int32_t dtype;       /* CCONV_TYPE_BF16 or _FP16, of X and C */
  int32_t scale_dtype; /* CCONV_TYPE_*, of the scales */
  int32_t group;       /* 32, 64 or 128 */
  int32_t reserved;    /* 0 */
  cconv_matrix x;      /* [M][K] */
  cconv_matrix q;      /* [N][ceil(K/2)] bytes */
  cconv_matrix scale;  /* [N][ceil(K/group)] */
  cconv_matrix zero;   /* [N][ceil(K/group)] bytes, 0 to 15 in their low halves; absent: 8 */
  cconv_matrix c;      /* out: [M][N] */
  void* workspace;
  uint64_t workspace_bytes;
} cconv_int4_product_args;

int64_t cconv_int4_product_workspace(const cconv_int4_product_args* args);
int cconv_int4_product(const cconv_int4_product_args* args, void* cuda_stream);

/* Weights in 4 bits, in fp32 up to the last rounding; s' = s rounded to scale_dtype, quotients nearest, ties to even:
 *   zero absent  s = max|w| / 7 over the group,          q = 8 + clamp(rint(w / s'), -8, 7)
 *   zero given   s = (max(w, 0) - min(w, 0)) / 15,       zero = clamp(rint(-min(w, 0) / s'), 0, 15),
 *                                                        q = clamp(rint(w / s') + zero, 0, 15)
 * Where s' is 0 or not finite, q and zero are 8 throughout; a group that holds an infinity or a NaN has scale NaN.
 * The half byte behind an odd K is 0. */
typedef struct {
  int64_t N, K;
  int32_t dtype; /* CCONV_TYPE_*, of w */
  int32_t scale_dtype, group;
  int32_t reserved;   /* 0 */
  cconv_matrix w;     /* in: [N][K] */
  cconv_matrix q;     /* out: [N][ceil(K/2)] bytes */
  cconv_matrix scale; /* out: [N][ceil(K/group)] */
  cconv_matrix zero;  /* out: [N][ceil(K/group)] bytes; absent: see above */
} cconv_quantize_groups_args;

int cconv_quantize_groups(const cconv_quantize_groups_args* args, void* cuda_stream);

/* ---- mixture of experts, for a few tokens --------------------------------------------------------
 * logits = x Wr^T; token t goes through the top_k experts of the largest logits, in falling order (of equal ones the
 * lower number first; a NaN counts as the lowest), with weights p = softmax over them (normalize 1) or over all
 * experts (normalize 0):   out[t] = sum_j p_j (act(x Wg_e^T) * (x Wu_e^T)) Wd_e^T,  e = ids[t][j].
 * Without a router ids and weights are read instead; numbers that are no expert's add nothing (those of other
 * ranks, say), and an expert that a token names twice counts with both weights.
 * h = act(x Wg_e^T) * (x Wu_e^T) is held as the sum of two numbers of `dtype`: twice its precision, and its range.
 * The weights of each expert in use are read once for 64 tokens; calls of more run 64 at a time. */
typedef struct {
  int64_t T, D, F, E;  /* E at most 1024, T at most 2^20, D and F at most 2^29 */
  int32_t dtype;       /* CCONV_TYPE_BF16 or _FP16, of x, the weights' matrices and out */
  int32_t act, top_k;  /* top_k: 1 to 32, at most E where there is a router */
  int32_t normalize;   /* 0 or 1 */
  cconv_matrix x;      /* [T][D] */
  cconv_matrix router; /* [E][D]; absent: see above */
  cconv_matrix w_gate, w_up; /* [F][D] of expert 0 */
  cconv_matrix w_down;       /* [D][F] of expert 0 */
  int64_t gate_stride, up_stride, down_stride; /* elements from an expert's matrix to the next one's */
  cconv_matrix ids;    /* [T][top_k] int32; out with a router, in without */
  cconv_matrix weights; /* [T][top_k] fp32; out with a router, in without */
  cconv_matrix out;    /* out: [T][D] */
  void* workspace;
  uint64_t workspace_bytes;
} cconv_moe_args;

int64_t cconv_moe_workspace(const cconv_moe_args* args); /* (a router of NULL is absent) */
int cconv_moe_forward(const cconv_moe_args* args, void* cuda_stream);

/* ---- the norm of a list of gradients, and clipping -------------------------------------------------
 * norm = sqrt(sum of squares over all elements), the sum in 64 bits (but for up to 66 neighbours' in fp32, where that holds
 * them), rounded to fp32; every element times
 * min(1, max_norm / (norm + eps)), in fp32, rounded to its type.  A norm that is infinite makes the factor 0, one that is
 * NaN, or as infinite as max_norm, makes every element NaN.  Tensors of more than two dimensions are lists of rows where their strides allow. */
typedef struct {
  void* data;
  int64_t rows, cols, row_stride, col_stride; /* strides in elements */
  int32_t dtype;                              /* CCONV_TYPE_* */
  int32_t reserved;                           /* 0 */
} cconv_tensor;

typedef struct {
  int64_t count;
  const cconv_tensor* grads; /* HOST array of `count`, read during the call */
  const cconv_tensor* outs;  /* HOST array: where results go, rows, cols and types as in grads; NULL: in place.  Every
                                out is apart from all gradients, or all of its own one */
  float max_norm, eps;       /* max_norm >= 0, eps >= 0, not both 0 */
  int32_t norm_given;        /* 1: `norm` holds the norm (of this list and others, say) and is read, not written */
  int32_t reserved;          /* 0 */
  void* norm;                /* fp32, one element */
  void* workspace;           /* none needed where the norm is given */
  uint64_t workspace_bytes;
} cconv_clip_args;

int64_t cconv_clip_workspace(const cconv_clip_args* args);
int cconv_gradient_norm(const cconv_clip_args* args, void* cuda_stream); /* writes `norm`; reads grads and workspace only */
int cconv_clip_gradients(const cconv_clip_args* args, void* cuda_stream);

/* Synchronises `cuda_stream`, reads the status word that the product kernels of the current device
 * share and clears it: CCONV_OK, CCONV_EDEVICE_TIMEOUT (a bounded wait on the device ran out; the
 * bits of *detail_out say which) or CCONV_ECUDA. */
int cconv_block_status(void* cuda_stream, int* detail_out);

#ifdef __cplusplus
}
#endif
#endif /* CCONV_BLOCK_H_ */
