/*
 * attn_layer.h -- C ABI of what stands around the attention forward (attn.h) in a layer on MI355X (gfx950):
 * its backward pass, and the norm and position rotation of queries and keys in front of it with its gradient.
 *
 * All pointers are DEVICE pointers owned by the caller.  The library allocates nothing, never synchronises and never
 * throws; calls only enqueue work on `stream` (a hipStream_t, or NULL for the default stream), on the current device.
 * Every argument is checked on the host before the device is touched; the return value is ATTN_OK or one of the
 * negative codes of attn.h (texts: attn_strerror).  Outputs must not overlap inputs, workspaces or each other.  Calls
 * can be recorded into a HIP graph (kernel nodes only) once one ordinary call has been made on the device, and replay
 * correctly; calls that may run at the same time need workspaces of their own.  The same inputs give the same bits.
 */
#ifndef PAPER_2603_24517_ATTN_LAYER_H
#define PAPER_2603_24517_ATTN_LAYER_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 * attn_bwd -- gradients of attn_fwd.
 *
 * With s_ij = scale * q_i . k_j, g = h / (Hq / Hkv) and valid(i, j) as in attn_fwd, for every batch entry and query head
 *     P_ij    = exp(s_ij - LSE_i) where valid, else 0; a row with LSE = -inf has P = 0
 *     delta_i = dO_i . O_i - dLSE_i
 *     dS_ij   = P_ij * (dO_i . V_j - delta_i)
 *     dQ_i = scale * sum_j dS_ij K_j        dK_j = scale * sum_{h in group, i} dS_ij Q_i
 *                                           dV_j = sum_{h in group, i} P_ij dO_i
 * O and LSE are those that attn_fwd returned for the same q, k, v, causal and scale.  Products run on BF16 matrix cores
 * with FP32 accumulation; the probabilities, delta and dS are FP32, and P and dS are rounded to BF16 (nearest even) before
 * they multiply; dQ, dK and dV are rounded to BF16 once.  Gradients of heads that share K and V are added in FP32.
 *
 *   dout      in   BF16 [B, Sq,  Hq,  D] contiguous
 *   dlse      in   FP32 [B, Hq, Sq] contiguous, or NULL if LSE was not used
 *   q, k, v, o, lse   as in attn_fwd, inputs here
 *   dq        out  BF16 [B, Sq,  Hq,  D] contiguous, fully overwritten
 *   dk, dv    out  BF16 [B, Skv, Hkv, D] contiguous, fully overwritten
 *   workspace      at least attn_bwd_workspace(...) bytes, 16-byte aligned; contents need not be set and are not kept
 *   B, Hq, Hkv, Sq, Skv, D, causal, scale   as in attn_fwd
 *
 * Masked pairs take no part, whatever they hold, but for one thing: a value that is not finite in row i of q or dout also makes the
 * gradients of keys NaN that are masked for it, but none from i + Skv - Sq + 160 on; and one in key j of k those of query rows that it is masked for, but none up
 * to j - (Skv - Sq) - 160.  (Sums run over whole tiles, with a probability of 0 where a pair is masked, and 0 times such a value is NaN.)
 * Size limits (ATTN_E_UNSUPPORTED): D, Sq + Skv, Hq and Hkv as in attn_fwd; B * Hkv * ceil(Skv / 128) and B * Hq / p * ceil(Sq * p / 128), p = 4, 2
 * or 1 the largest that divides Hq / Hkv, below 2^23.  ATTN_E_WORKSPACE if the workspace is too small.
 */
int attn_bwd(const void *dout, const float *dlse, const void *q, const void *k, const void *v, const void *o,
             const float *lse, void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes,
             int B, int Hq, int Hkv, int Sq, int Skv, int D, int causal, float scale, void *stream);

/* Bytes of workspace that attn_bwd needs for these sizes, or a negative code. */
long long attn_bwd_workspace(int B, int Hq, int Hkv, int Sq, int Skv, int D, int causal);

/*
 * A BF16 tensor [B, S, H, D] with its last dimension contiguous: strides in elements, each a multiple of 8 (16 bytes) unless
 * its dimension is 1, ptr 16-byte aligned.  Strides may be 0 or negative in inputs; outputs must not overlap themselves.
 */
typedef struct {
    void *ptr;
    long long batch, token, head;
} attn_heads;

enum { ATTN_ROPE_HALVES = 0, ATTN_ROPE_ADJACENT = 1 };
enum { ATTN_BF16 = 0, ATTN_FP32 = 1 };
enum { ATTN_INT32 = 0, ATTN_INT64 = 1 };

/* What the norm and the rotation have in common for both directions. */
typedef struct {
    int B, S, Hq, Hkv, D;       /* sizes, all > 0; D must be 128 (here Hq need not be a multiple of Hkv) */
    const void *q_weight;       /* [D] contiguous, or NULL: 1.  Both or neither */
    const void *k_weight;
    int weight_type;            /* ATTN_BF16 or ATTN_FP32 */
    const float *cos, *sin;     /* FP32 [places, rotated / 2] contiguous, 16-byte aligned */
    long long places;           /* > 0 */
    int rotated;                /* leading elements of a head that are rotated: a multiple of 16, 16 .. D */
    int pairing;                /* ATTN_ROPE_HALVES: (i, i + rotated / 2); ATTN_ROPE_ADJACENT: (2 i, 2 i + 1) */
    const void *positions;      /* [B, S] contiguous: the table row of each token; NULL: token s takes row s (S <= places) */
    int position_type;          /* ATTN_INT32 or ATTN_INT64 */
    float eps;                  /* >= 0, finite */
} attn_rope;

/*
 * attn_qk_norm_rope -- the norm of each head of q and k with the position rotation.  For each head x of a token
 *     y = x / sqrt(mean(x^2) + eps) * weight;  each rotated pair (a, b) of y becomes (a cos - b sin, b cos + a sin)
 * with cos and sin of the token's table row; computed in FP32, rounded to BF16 once.  v, where given (v_in->ptr not NULL), is
 * copied, so that slices of one projection come out as the contiguous tensors that attn_fwd takes, in one pass.
 * A token whose place lies outside the table gets NaN in q and k.  The squares too are FP32: a head whose 2-norm is beyond 1.8e19 comes out as zeros
 * (and has no gradient), and one whose mean square and eps together are below 1.2e-38 loses precision.
 * Size limits (ATTN_E_UNSUPPORTED), for both directions: B * S * Hq and B * S * Hkv at most 2^31 - 2^16; here also the heads of all tokens,
 * B * S * (Hq + Hkv), or B * S * (Hq + 2 * Hkv) with v, below 2^29 - 96.
 */
int attn_qk_norm_rope(const attn_rope *r, const attn_heads *q_in, const attn_heads *k_in, const attn_heads *v_in,
                      const attn_heads *q_out, const attn_heads *k_out, const attn_heads *v_out, void *stream);

/*
 * attn_qk_norm_rope_bwd -- the gradient of attn_qk_norm_rope: from dq_out, dk_out (and dv_out, where given) and the inputs
 * q_in, k_in to dq_in, dk_in (and dv_in, a copy).  With z the rotated gradient turned back, xhat = x / sqrt(mean(x^2) + eps):
 *     dweight = sum over tokens and heads of z * xhat      dx = (z w - xhat * mean(z w xhat)) / sqrt(mean(x^2) + eps)
 * A token whose place lies outside the table, whose q and k were NaN whatever the inputs and weights, gets NaN in dq_in and dk_in and
 * is left out of the sums.  dq_weight and dk_weight: FP32 [D], fully overwritten; both NULL if they are not wanted.  The sums are FP32
 * in a fixed order.  workspace: attn_qk_norm_rope_bwd_workspace(r) bytes, 16-byte aligned, if dq_weight is given.
 */
int attn_qk_norm_rope_bwd(const attn_rope *r, const attn_heads *dq_out, const attn_heads *dk_out, const attn_heads *dv_out,
                          const attn_heads *q_in, const attn_heads *k_in, const attn_heads *dq_in, const attn_heads *dk_in,
                          const attn_heads *dv_in, float *dq_weight, float *dk_weight, void *workspace, size_t workspace_bytes,
                          void *stream);

long long attn_qk_norm_rope_bwd_workspace(const attn_rope *r);

#ifdef __cplusplus
}
#endif
#endif
