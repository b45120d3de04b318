/*
 * wn_train.h -- C ABI of libwn's operators at the ends of a training step on an
 * AMD Instinct MI355X (gfx950): the loss of an output layer and its gradients,
 * log probabilities with entropies and alternatives and their gradients,
 * an embedding and its gradient, the clip of all gradients, and updates orthogonalised by
 * Newton-Schulz products.
 *
 * A voice's two ends (the embedding of the samples before, and the softmax over
 * the classes of the next one; Deep Voice, arXiv 1702.07825, Appendix A.1) run
 * forwards inside wn_generate and wn_teacher_force.  These calls are their forms
 * for scoring and training, for any vocabulary: the 256 mu-law classes, the
 * 65536 of 16-bit samples, or tokens of text.  wn_score (wn.h) takes the loss of
 * recorded speech from a model handle.
 *
 * Conventions:
 *  - All pointers are DEVICE pointers owned by the caller, all on one device, and
 *    arrays are dense and row-major.  They may start at any element; a workspace
 *    is 256-byte aligned.  No output overlaps an input or another output, except
 *    where wn_clip and wn_orthogonalize say so.
 *  - `dtype` (wn_dtype_t, WN_F32 or WN_BF16) is the type of the matrices: x, w,
 *    dx, dw, an embedding table and its rows.  Biases, losses, and upstream
 *    gradients of losses are fp32.  Every sum is in fp32 or wider.
 *  - There is no handle: a call runs on the device its arrays live on, makes that
 *    device current while it runs, and is asynchronous, ordered on `stream`, which
 *    must be a stream of that device (NULL: its default stream).  Nothing is
 *    allocated and the host waits for nothing, so every call can be captured in a
 *    graph.  Two calls that share a workspace must not overlap in time (nor may
 *    two graphs that captured it).  Results are the same, bit for bit, from run
 *    to run.
 *  - Return codes as in wn.h; nothing is launched when an argument check fails.
 */
#ifndef WN_TRAIN_H_
#define WN_TRAIN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The loss of N rows under an output layer of V classes, without keeping the logits:
 *   l[n][v] = b[v] + sum_k x[n][k] w[v][k],  lse[n] = log sum_v exp(l[n][v]),
 *   loss[n] = lse[n] - l[n][y[n]]
 *   x     [N][D]   w [V][D]   b fp32 [V] or NULL (no bias)
 *   y     int32 [N]; a row whose y is outside 0 .. V-1 has no target (padding): its loss is 0
 *         whatever x holds there
 *   loss  fp32 [N] out;  lse fp32 [N] out (wn_loss_backward takes it)
 * A class of bias -inf is masked: it has probability 0 (a row whose target is masked has loss +inf;
 * if every class is masked, or a logit is NaN or +inf, the loss is NaN or infinite).  An infinity in
 * x or w itself may leave a row that meets it NaN.
 * From 65 rows on fp32 products are taken as three products of fp16 parts that hold each value to 2^-22 of
 * itself (or to 2^-39 of the largest value of its row); fewer rows take them in fp32.  lse of a row
 * without a target is that of what x holds.
 * N 0 .. 2^20 (0: nothing to do), D 1 .. 2^16, V 1 .. 2^24.
 * Errors: WN_EINVAL (a size out of range, a null pointer, memory that is not on a device or on
 * different ones, a short or misaligned workspace); WN_EUNSUPPORTED (dtype WN_I8); WN_EHIP.
 */
int wn_loss(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* x, const void* w, const float* b,
            const int32_t* y, float* loss, float* lse, void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace wn_loss needs (0 for sizes out of range or N = 0). */
size_t wn_loss_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V);

/*
 * Gradients of sum_n g[n] loss[n] (the losses of wn_loss with the same x, w, b and y, whose lse this
 * takes), again without keeping the logits: they are computed anew for pieces of the vocabulary.
 *   q[n][v] = g[n] (exp(l[n][v] - lse[n]) - [v = y[n]]), 0 in rows without a target
 *   dx[n][k] = sum_v q[n][v] w[v][k],  dw[v][k] = sum_n q[n][v] x[n][k],  db[v] = sum_n q[n][v]
 *   g     fp32 [N] upstream gradients (1 / rows for a mean)
 *   dx    [N][D] out, or NULL if not wanted; 0 in rows without a target, whatever x, lse and g hold there
 *   dw    [V][D] out, or NULL;   db fp32 [V] out, or NULL (with b NULL it is the gradient at b = 0)
 * With dtype WN_BF16 q / g (dx) and q / max |g| (dw) enter the last two products rounded to bf16 (db sums q in
 * fp32); with WN_F32 as wn_loss takes its products, from 65 rows on with q / g in dw's held to 2^-22 of itself, to 2^-39
 * of its class's largest (of 1 if a row targets the class) or to 2^-105, in dx's to 2^-22 of itself or to 2^-39.  Sizes
 * and errors as wn_loss; all three outputs NULL is an error.  N = 0: dw and db are zeroed.
 */
int wn_loss_backward(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* x, const void* w, const float* b,
                     const int32_t* y, const float* lse, const float* g, void* dx, void* dw, float* db,
                     void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace wn_loss_backward needs, whichever outputs are wanted (0 for sizes out of range). */
size_t wn_loss_backward_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V);

/*
 * Log probabilities of given tokens under an output layer (l and lse as in wn_loss), the entropies of the rows'
 * distributions p[n][v] = exp(l[n][v] - lse[n]), and the `top` likeliest classes of each, without keeping the logits:
 *   logprob[n] = l[n][y[n]] - lse[n],  entropy[n] = lse[n] - sum_v p[n][v] l[n][v]
 *   y             int32 [N]; a row whose y is outside 0 .. V-1 has no token: its logprob is 0 (the rest is as of any row)
 *   logprob, entropy, lse   fp32 [N] out
 *   top_ids       int32 [N][top] out, the classes of the largest logits in falling order, of equal ones the lowest first;
 *   top_logprobs  fp32 [N][top] out, their log probabilities.  Both may be NULL where top is 0.
 * The alternatives' logits are summed in 64 bits, so classes closer to each other than the other logits' rounding (their
 * products' and their bias's addition's) are in order; one that that rounding moves behind more than two others (and one more for each 8 of top) in other groups of 8
 * classes may be missed (more than 64 rows of up to 1024 classes: in any groups).  A class of bias -inf is masked: it adds
 * nothing to the entropy and is an alternative (of log probability -inf) only where fewer than top are left.  If every class
 * is masked, or a logit is NaN or +inf, the row's logprob, entropy, lse and top_logprobs are NaN or infinite and its top_ids
 * any classes.
 * Sizes and errors as wn_loss; top 0 .. 32 and at most V.
 */
int wn_logprobs(int32_t dtype, int32_t N, int32_t D, int32_t V, int32_t top, const void* x, const void* w, const float* b,
                const int32_t* y, float* logprob, float* entropy, float* lse, int32_t* top_ids, float* top_logprobs,
                void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace wn_logprobs needs (0 for sizes out of range or N = 0). */
size_t wn_logprobs_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V, int32_t top);

/*
 * Gradients of sum_n g[n] logprob[n] + h[n] entropy[n] over the rows with a token (of wn_logprobs with the same x, w, b and
 * y, whose lse and entropy this takes):
 *   q[n][v] = g[n] ([v = y[n]] - p[n][v]) - h[n] p[n][v] (log p[n][v] + entropy[n]), 0 in rows without a token
 *   dx, dw, db  from q as in wn_loss_backward
 *   g, h        fp32 [N] upstream gradients; either may be NULL (all 0)
 * With c[n] = max(|g[n]|, |h[n]|), q / c enters the last two products as q / g does in wn_loss_backward, but for one bit:
 * its fp16 parts for dx are held to 2^-38.  Sizes, NULL outputs and errors as there.
 */
int wn_logprobs_backward(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* x, const void* w, const float* b,
                         const int32_t* y, const float* lse, const float* entropy, const float* g, const float* h, void* dx,
                         void* dw, float* db, void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace wn_logprobs_backward needs, whichever outputs are wanted (0 for sizes out of range). */
size_t wn_logprobs_backward_workspace_bytes(int32_t dtype, int32_t N, int32_t D, int32_t V);

/*
 * Embedding: out[n][k] = scale * table[t[n]][k], rounded once to dtype; a row whose token is outside
 * 0 .. V-1 (padding) is 0.
 *   table [V][D]   t int32 [N]   out [N][D]   scale finite
 * N 0 .. 2^27, D 1 .. 2^16, V 1 .. 2^24.  Errors as wn_loss.
 */
int wn_embed(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* table, const int32_t* t, float scale,
             void* out, void* stream);

/*
 * Its gradient: dtable[v][k] = scale * sum over the n with t[n] = v of dout[n][k], 0 where no token is v.
 * The tokens are sorted first (a stable sort), and each table row's sum goes over its rows in
 * that order, in fp32 pieces whose place depends on N alone.
 *   dout [N][D]   t int32 [N]   dtable [V][D] out
 * Sizes and errors as wn_embed.  N = 0: dtable is zeroed.
 */
int wn_embed_backward(int32_t dtype, int32_t N, int32_t D, int32_t V, const void* dout, const int32_t* t, float scale,
                      void* dtable, void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace wn_embed_backward needs (0 for sizes out of range or N = 0). */
size_t wn_embed_backward_workspace_bytes(int32_t N, int32_t D, int32_t V);

/* One array of wn_clip: n elements of dtype (WN_F32 or WN_BF16) at g; the clipped ones go to out, which
 * may be g itself.  Nothing else may overlap. */
typedef struct {
  const void* g;
  void* out;
  int64_t n;       /* 0 .. 2^40; 0: g and out are not looked at */
  int32_t dtype;
} wn_clip_array;

/*
 * The norm over all elements of n_arrays gradient arrays (`arrays` is a HOST array, read before the call
 * returns), and the arrays scaled so that the norm is at most max_norm:
 *   norm = sqrt(sum g^2)  (summed in fp64: fp32 gradients neither overflow nor vanish)
 *   out  = g * (max_norm / norm): the factor rounded to 24 bits, however small it is, then the product to fp32, and
 *          that to bf16 in arrays of bf16; a copy where norm <= max_norm
 *   norm     fp32 [1] device, out
 * Where the norm is not finite (an infinity or NaN among the gradients, or a norm beyond fp32),
 * out is a copy of g: the caller sees it in *norm and can skip the step.  max_norm >= 0 (inf:
 * only the norm counts).  n_arrays 0 .. 2^20.
 * Errors as wn_loss (of the arrays only the first one's memory is looked at), WN_EINVAL for a max_norm
 * that is negative or NaN and for arrays that overlap (the same one listed twice, say), and WN_ENOMEM.
 */
int wn_clip(int32_t n_arrays, const wn_clip_array* arrays, float max_norm, float* norm, void* workspace,
            size_t ws_bytes, void* stream);

/* Bytes of workspace wn_clip needs, whatever the arrays. */
size_t wn_clip_workspace_bytes(void);

/* One matrix of wn_orthogonalize: rows x cols elements of dtype (WN_F32 or WN_BF16) at g; the update goes to out, which may
 * be g itself.  Nothing else may overlap. */
typedef struct {
  const void* g;
  void* out;
  int32_t rows, cols;  /* 0 .. 2^18, their product at most 2^32; 0: g and out are not looked at */
  int32_t dtype;
  float scale;         /* finite */
} wn_ortho_array;

/*
 * Updates orthogonalised by Newton-Schulz products, as the Muon optimizer takes them: every matrix G of `arrays` (a HOST
 * array, read before the call returns) by itself
 *   X = G / (norm + eps), norm its Frobenius norm (summed in fp64), transposed if rows > cols;
 *   `steps` times, with (a, b, c) = coefficients[0], [1], [2] of the step:  A = X X',  X <- (a I + b A + c A A) X
 *   out = scale X, transposed back
 * coefficients is a HOST array [steps][3].  With (3.4445, -4.7750, 2.0315) five times the singular values of out / scale
 * lie about 1 (0.68 to 1.21, and the roundings) where those of X were above 0.002; any others may be given as long as no entry of a step's X, A or
 * a I + b A + c A A reaches 16, 16 or 64 in size (a matrix where one does ends up not finite).
 * A zero matrix gives zeros; an infinity or NaN in a matrix makes its update NaN, and no other's.
 * Products are summed in fp32: of WN_BF16 matrices X, A and a I + b A + c A A are rounded to fp16 between products (2^-11 of a value, and
 * 2^-37 to 2^-35), of WN_F32 ones held in two fp16 parts (2^-22) and three products of them taken for one.
 * n_arrays 0 .. 2^16, steps 1 .. 64, eps finite and >= 0.
 * Errors as wn_loss (of the arrays only the first one's memory is looked at), WN_EINVAL for arrays that overlap, and WN_ENOMEM.
 */
int wn_orthogonalize(int32_t n_arrays, const wn_ortho_array* arrays, int32_t steps, const float* coefficients, float eps,
                     void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace wn_orthogonalize needs for arrays of these sizes and dtypes (0 for sizes out of range): about six times
 * the arrays in 16 bits (fp32: twelve) with sides rounded up to 64 (fp32: 32), of about 4 GiB of buffers at a time. */
size_t wn_orthogonalize_workspace_bytes(int32_t n_arrays, const wn_ortho_array* arrays);

#ifdef __cplusplus
}
#endif

#endif /* WN_TRAIN_H_ */
