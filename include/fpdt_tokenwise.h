/*
 * fpdt_tokenwise.h -- C ABI of the token-wise chunked neighbours of the attention path
 * (Sec. 5.4, "Chunk Granularity"): operations whose cost is linear in the sequence length and
 * whose intermediate buffers, not their FLOPs, are the problem at long sequences.  They are
 * chunked along the sequence without offloading; the intermediates exist for one chunk at a
 * time.
 *
 *   fpdt_tw_loss_fwd_bwd   softmax cross-entropy over the vocabulary with its last linear
 *                          projection, forward and backward fused: the fp32 logits
 *                          [rows, vocab] exist for as many rows at a time as the workspace has
 *                          room for, one chunk and a half (Sec. 5.4 names the loss over a large
 *                          vocabulary as the place where memory peaks and suggests
 *                          vocab / hidden * 2 chunks).
 *   fpdt_tw_linear_*       the per-chunk QKV projection in front of the attention.
 *   fpdt_tw_ffn_*          the feed-forward block, chunked with twice the attention's chunk
 *                          count, forward and (recomputing) backward.
 *   fpdt_tw_rope_*         rotary positions and the split of the QKV product into Q, K, V.
 *   fpdt_tw_norm_*         residual add and RMS or layer normalisation.
 *   fpdt_tw_grad_norm, fpdt_tw_adamw_*   norm of all gradients, the optimizer's step.
 *
 * The dense products run on this library's own bf16 MFMA kernels (csrc/tw_gemm.hip: operands
 * read in place, output tiles of up to 256 x 256, fp32 accumulation); the row-wise softmax /
 * loss / gradient and the activations are HIP kernels of this library as well.  Built as a
 * separate shared library (libfpdt_tokenwise.so).
 *
 * Conventions as in fpdt.h: row-major contiguous tensors, device pointers, caller-owned
 * buffers, `stream` is a hipStream_t passed as void*, calls only enqueue, every function returns
 * an fpdt status code (0 = OK, 1 = invalid argument, 2 = unsupported, 3 = workspace, 4 = HIP
 * failure; text from fpdt_tw_last_error).  Besides the caller's workspace the library keeps one
 * device scratch pool per GPU for the running call: logit gradients of up to 2 hidden rows (of a
 * chunk, where that is more and the vocabulary is not a multiple of 8), fp32 sums of output tiles
 * that several workgroups share, copies of operands whose rows are not 16-byte aligned.  It grows on
 * demand with hipMalloc -- so the first call of a given size must not run under stream capture -- by
 * doubling from 256 MiB, and is kept until the process ends, as are the buffers it has outgrown (work
 * in flight may read them): up to four times what the largest call needs.  Calls that overlap in time
 * on one GPU (different streams or threads) would share that pool: keep the library's calls on one
 * stream.
 */
#ifndef FPDT_TOKENWISE_H
#define FPDT_TOKENWISE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device workspace fpdt_tw_loss_fwd_bwd needs: one chunk of fp32 logits and one chunk
 * of bf16 logit gradients, chunk = ceil(rows / n_chunks) rows; where the gradients are in the
 * library's scratch, or not asked for, all of it holds logits.  0 if the arguments are invalid. */
size_t fpdt_tw_loss_workspace_bytes(int64_t rows, int hidden, int vocab, int n_chunks);

/*
 * Chunked cross-entropy loss with its output projection (Sec. 5.4).  For every row r:
 *     logits_r = H_r W^T                      (bf16 x bf16 -> fp32)
 *     lse_r    = log sum_v exp(logits_r[v])   (fp32, max-subtracted)
 *     loss_r   = lse_r - logits_r[target_r]
 * and, when dH / dW are given, the gradient of sum_r grad_scale * loss_r:
 *     G_r  = grad_scale * (softmax(logits_r) - onehot(target_r))    (rounded to bf16)
 *     dH_r = G_r W                            (written, bf16)
 *     dW  += G^T H                            (ACCUMULATED into the caller's fp32 buffer)
 *   H [rows, hidden] bf16, W [vocab, hidden] bf16, target [rows] int32 in [0, vocab)   in
 *   loss, lse [rows] fp32                                                             out
 *   dH [rows, hidden] bf16 or NULL, dW [vocab, hidden] fp32 or NULL                   out / in-out
 *   workspace: device memory, 256-byte aligned, >= fpdt_tw_loss_workspace_bytes(...)
 * dW is summed in fp32 over groups of up to 2 hidden rows, of about the same size and in general not
 * whole chunks; the logit gradients of a group are gathered in the library's scratch, [rows, vocab rounded
 * up to 8], and the workspace holds logits only, of one and a half chunks.  Where a chunk has more than
 * hidden rows, dW is summed chunk by chunk, and if vocab is a multiple of 8 both the chunk's logits and its
 * gradients are in the workspace.  Status 4 if there is no memory for the scratch.
 * A target outside [0, vocab) is not detected (its row's loss is lse_r and its gradient the
 * plain softmax).
 */
int fpdt_tw_loss_fwd_bwd(const void *H, const void *W, const int32_t *target, float grad_scale,
                         float *loss, float *lse, void *dH, float *dW, int64_t rows, int hidden,
                         int vocab, int n_chunks, void *workspace, size_t workspace_bytes,
                         void *stream);

/*
 * Chunked linear projection (Sec. 4.1: every sequence chunk T_i is projected to q_i, k_i, v_i on
 * its own, so that chunk i's attention can start while chunk i+1 is still being projected).
 *     Y = X W^T          X [rows, n_in] bf16, W [n_out, n_in] bf16  ->  Y [rows, n_out] bf16
 * needs no workspace.  Backward:
 *     dX = dY W  (written, bf16; NULL to skip),   dW += dY^T X  (accumulated, fp32; NULL to skip)
 * dW is summed ceil(rows / n_chunks) rows at a time; Y and dX, whose rows are independent and which
 * have no intermediates, are computed over all rows at once, or chunk by chunk where X or dY has to be
 * copied first (rows that are not 16-byte aligned, or Y in the place of X, dX in that of dY: allowed).
 */
int fpdt_tw_linear_fwd(const void *X, const void *W, void *Y, int64_t rows, int n_in, int n_out,
                       int n_chunks, void *stream);
int fpdt_tw_linear_bwd(const void *X, const void *W, const void *dY, void *dX, float *dW,
                       int64_t rows, int n_in, int n_out, int n_chunks, void *stream);

/*
 * Chunked feed-forward block (Sec. 5.4: token-wise, its [rows, n_ffn] intermediates are what has
 * to be bounded; twice the attention's chunk count is enough, and nothing is offloaded).
 *   FPDT_TW_GELU    Y = gelu(X W1^T) W2^T                      (GPT; exact erf form)
 *   FPDT_TW_SWIGLU  Y = (silu(X W1^T) * (X W3^T)) W2^T         (Llama)
 *   X, Y, dX, dY [rows, n_model] bf16; W1, W3 [n_ffn, n_model] bf16; W2 [n_model, n_ffn] bf16
 *   (W3, dW3: SWIGLU only, NULL otherwise).  Intermediates are rounded to bf16 between GEMMs.
 * The backward recomputes the pre-activations of a chunk from X (the forward saves nothing),
 * writes dX and ACCUMULATES into the caller's fp32 dW1, dW3, dW2 (each may be NULL to skip).
 *   workspace: device memory, 256-byte aligned, >= fpdt_tw_ffn_workspace_bytes(..., is_bwd)
 */
enum { FPDT_TW_GELU = 0, FPDT_TW_SWIGLU = 1 };
size_t fpdt_tw_ffn_workspace_bytes(int64_t rows, int n_model, int n_ffn, int act, int n_chunks,
                                   int is_bwd);
int fpdt_tw_ffn_fwd(const void *X, const void *W1, const void *W3, const void *W2, void *Y,
                    int64_t rows, int n_model, int n_ffn, int act, int n_chunks, void *workspace,
                    size_t workspace_bytes, void *stream);
int fpdt_tw_ffn_bwd(const void *X, const void *W1, const void *W3, const void *W2, const void *dY,
                    void *dX, float *dW1, float *dW3, float *dW2, int64_t rows, int n_model,
                    int n_ffn, int act, int n_chunks, void *workspace, size_t workspace_bytes,
                    void *stream);

/*
 * What follows takes tensors of one dtype, and tensors of any alignment that its elements have.  Nothing of it uses
 * the library's scratch pool, copies from the host or allocates: calls may overlap in time, and may be captured (every
 * address, workspaces included, must then stay valid for every replay; two graphs that may run at once need workspaces of
 * their own).  A tensor that is written overlaps no other argument, but where a line says so.
 */
enum { FPDT_TW_F32 = 0, FPDT_TW_BF16 = 1 };

/*
 * Rotary positions (Sec. 4.1: q_i, k_i, v_i of a chunk, projected in one product), and the split of that product's rows
 * into the attention's contiguous Q, K, V.  The token in row r has the position positions[r] (int64, device; any order, any
 * value twice), or position0 + r where positions is NULL.  Pair i of the first `rot` channels of each head of Q and K
 * turns by t = position * freqs[i] (the product is formed in 64 bits, so that positions of millions keep their angle):
 *     (a, b)  ->  amplitude * (a cos t - b sin t,  b cos t + a sin t)
 *     FPDT_TW_ROPE_HALF         a, b = channels i and i + rot / 2
 *     FPDT_TW_ROPE_INTERLEAVED  a, b = channels 2 i and 2 i + 1
 * Channels from rot on, and V, are copied.  The backward is the transpose: t becomes -t.
 *   Q, K, V     [rows, Hq or Hkv, D] of `dtype`; the heads of a token are contiguous, tokens q_row, k_row, v_row elements
 *               apart (a slice of the QKV product: all (Hq + 2 Hkv) D).  K and V, or V alone, may be NULL (on both sides).
 *   Qo, Ko, Vo  the same, with distances of their own.  An output may be its own input (same address and distance: in place).
 *   freqs       rot / 2 radians per token, fp64, device;  even rot in [2, D], D <= 8192, at most 4096 heads and 2^31 - 1 rows, which are
 *               at most 2^28 elements apart
 * Arithmetic in fp32, rounded once.
 */
enum { FPDT_TW_ROPE_HALF = 0, FPDT_TW_ROPE_INTERLEAVED = 1 };
int fpdt_tw_rope_fwd(const void *Q, int64_t q_row, const void *K, int64_t k_row, const void *V, int64_t v_row,
                     void *Qo, int64_t qo_row, void *Ko, int64_t ko_row, void *Vo, int64_t vo_row,
                     const int64_t *positions, int64_t position0, const double *freqs, float amplitude,
                     int64_t rows, int Hq, int Hkv, int D, int rot, int layout, int dtype, void *stream);
int fpdt_tw_rope_bwd(const void *dQo, int64_t qo_row, const void *dKo, int64_t ko_row, const void *dVo, int64_t vo_row,
                     void *dQ, int64_t q_row, void *dK, int64_t k_row, void *dV, int64_t v_row,
                     const int64_t *positions, int64_t position0, const double *freqs, float amplitude,
                     int64_t rows, int Hq, int Hkv, int D, int rot, int layout, int dtype, void *stream);

/*
 * The rot / 2 frequencies for fpdt_tw_rope_*, written to HOST memory.  Host logic only: no device is touched.
 *   FPDT_TW_ROPE_PLAIN   f_i = base^(-2 i / rot)
 *   FPDT_TW_ROPE_LINEAR  f_i / factor (positions interpolated)
 *   FPDT_TW_ROPE_RAISED  base * factor^(rot / (rot - 2)) for base: the slowest pair is slowed by factor, the fastest kept
 *   FPDT_TW_ROPE_PARTS   by the turns n_i = context f_i / 2 pi that a pair makes over the trained context: f_i where
 *                        n_i >= high, f_i / factor where n_i <= low, in between mixed linearly in n_i
 * (factor is ignored by PLAIN; context, low and high by all but PARTS).
 */
enum { FPDT_TW_ROPE_PLAIN = 0, FPDT_TW_ROPE_LINEAR = 1, FPDT_TW_ROPE_RAISED = 2, FPDT_TW_ROPE_PARTS = 3 };
int fpdt_tw_rope_freqs(int rot, double base, int scaling, double factor, double context, double low, double high,
                       double *freqs);

/*
 * Normalisation of rows, with the residual add in front of it.
 *     S = X + R (rounded to dtype; R NULL: S = X, and the argument S is NULL)
 *     FPDT_TW_RMSNORM    Y = S rstd W                    rstd = 1 / sqrt(mean(S^2) + eps)
 *     FPDT_TW_LAYERNORM  Y = (S - mean) rstd W + B       rstd = 1 / sqrt(mean((S - mean)^2) + eps)
 *   X, R, S, Y [rows, hidden], W, B [hidden] of `dtype`;  B may be NULL, and is with RMSNORM;  hidden <= 16384
 *   S may be NULL although R is given.  S and Y may each be X or R (not both the same).
 *   stats       fp32, for the backward: rstd [rows]; LAYERNORM: mean [rows], then rstd [rows].  May be NULL.
 * The backward reads the S of the forward (X, where there was no R):
 *     H = dY W,  U = (S - mean) rstd,  dX = rstd (H - mean(H) - U mean(H U)) + dR     (RMSNORM: without mean and mean(H))
 *     dW += sum over rows of dY U,   dB += sum over rows of dY     (ACCUMULATED into the caller's fp32 buffers)
 *   dR [rows, hidden]: the gradient that reaches S by another way (the residual stream's), or NULL.  dX is the gradient
 *   of X and of R; it may be S, dY or dR itself.  dW and dB may be NULL to skip; without both no workspace is needed.
 *   workspace: device memory, 256-byte aligned, >= fpdt_tw_norm_bwd_workspace_bytes(...)
 * Arithmetic and sums in fp32 (a row whose sum of squares fp32 does not hold has rstd = 0), but for the quotients and root of the statistics and
 * the last sums of dW and dB, which are formed in fp64 and rounded once; the order of the sums depends on the arguments alone.
 */
enum { FPDT_TW_RMSNORM = 0, FPDT_TW_LAYERNORM = 1 };
int fpdt_tw_norm_fwd(const void *X, const void *R, const void *W, const void *B, void *S, void *Y, float *stats,
                     int64_t rows, int hidden, int kind, float eps, int dtype, void *stream);
size_t fpdt_tw_norm_bwd_workspace_bytes(int64_t rows, int hidden, int kind);
int fpdt_tw_norm_bwd(const void *S, const void *W, const float *stats, const void *dY, const void *dR, void *dX, float *dW,
                     float *dB, int64_t rows, int hidden, int kind, int dtype, void *workspace, size_t workspace_bytes,
                     void *stream);

/*
 * One tensor of the optimizer.  A list of them is an array in HOST memory that is read before the call returns; all
 * buffers are device memory of n elements (n = 0: nothing is read), and no two of a list overlap.
 *   g                 gradient, fp32 or bf16 (one type for the whole list)
 *   p, w              parameter in fp32; its copy in bf16 for the products, written by the step, or NULL
 *   m, v              moments: fp32, or 8-bit codes with one exponent byte for each 128 elements in m_exp, v_exp
 *                     [ceil(n / 128)] (zeros are the initial state; NULL with 32-bit states)
 *   m_value, v_value  bf16, written by fpdt_tw_adamw_unpack; NULL elsewhere
 */
typedef struct {
    int64_t n;
    void *g;
    float *p;
    void *w, *m, *v;
    uint8_t *m_exp, *v_exp;
    void *m_value, *v_value;
    double weight_decay;
} fpdt_tw_param;

/*
 * Norm of all gradients of a list, and the factor that brings it down to max_norm (infinity: 1):
 *     out[0] = sqrt(sum g^2),   out[1] = min(1, max_norm / (norm + 1e-6)), NaN where the norm is not finite
 * Squares and sums in fp64; their order depends on the list's lengths alone.
 *   out [2] fp32, device;  workspace: device memory, 256-byte aligned, >= fpdt_tw_grad_norm_workspace_bytes(count)
 */
size_t fpdt_tw_grad_norm_workspace_bytes(int count);
int fpdt_tw_grad_norm(const fpdt_tw_param *params, int count, int grad_dtype, double max_norm, float *out,
                      void *workspace, size_t workspace_bytes, void *stream);

/*
 * AdamW step over a list.  With g the gradient times *grad_scale (device, fp32; NULL: 1):
 *     m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *     p = p (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps),   w = bf16(p)
 * in fp32 (the factors in fp64, rounded to fp32; root and quotient to half a step with 32-bit states, to a step of 2^-23 each with
 * 8-bit states; in the root, a v that is no normal number counts as the smallest).  Where
 * *grad_scale is not finite nothing changes: a step whose gradients overflowed is passed over.  lr_dev (fp32) and step_dev
 * (int64, values below 1 count as 1) on the device replace lr and step where they are given: a captured step reads them at
 * every replay.
 *   FPDT_TW_ADAMW_ZERO_GRAD  the gradients are set to zero in the same pass (in a step that is passed over, too)
 *   state_bits 8             in a block of 128, E is the exponent field of the block's largest |value| rounded up to three
 *                            fraction bits (at least 40; 255: a value is not finite, and the whole block becomes NaN); a code c > 0
 *                            stands for the float of bits (E - D) 2^23 + c 2^20, D = 15 for m (bit 7 is the sign), 31 for
 *                            v; 0 for zero.  p takes the new moments before they are rounded.  They are rounded to codes at
 *                            random, up with the probability of what is cut off (v never to zero), by 16 bits each, m's the
 *                            lower ones, of
 *                                mix(i * 0x9E3779B1 ^ key),  key = mix(mix(mix(seed ^ 0x243F6A88) ^ step * 0x9E3779B1) ^ k * 0x85A308D3)
 *                                mix(x): x ^= x >> 15; x *= 0xB7E15163; x ^= x >> 13; x *= 0x93C467E3; x ^ x >> 16
 *                            for element i of tensor k of the list, mod 2^32 (where i / 2^32 = h > 0 the key is mix(key + h)).  Lists
 *                            that are stepped with one seed round with the same bits: give each list of a model a seed of its own.
 * fpdt_tw_adamw_unpack writes what the 8-bit states stand for into m_value and v_value (bf16 holds it exactly).
 */
enum { FPDT_TW_ADAMW_ZERO_GRAD = 1u << 0 };
int fpdt_tw_adamw_step(const fpdt_tw_param *params, int count, int grad_dtype, int state_bits, double lr, double beta1,
                       double beta2, double eps, int64_t step, const float *lr_dev, const int64_t *step_dev,
                       const float *grad_scale, unsigned seed, unsigned flags, void *stream);
int fpdt_tw_adamw_unpack(const fpdt_tw_param *params, int count, void *stream);

/* Text describing the calling thread's most recent error ("" if none). Never NULL. */
const char *fpdt_tw_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FPDT_TOKENWISE_H */
