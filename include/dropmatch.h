/*
 * dropmatch.h -- C ABI of the B200 (sm_100a) DropMatch verification library.
 *
 * DropMatch (arXiv 2603.03333) verifies draft tokens of speculative decoding by
 * Monte-Carlo dropout on the LM head only.  For every draft position t the target
 * model's final hidden state h_t[d] is copied K times, each copy multiplied by an
 * independent Bernoulli(1-p) keep mask and rescaled by 1/(1-p) (Eq. 1, Eq. 2);
 * each copy is projected through the shared head W[V,d] (Eq. 3) and decoded to its
 * argmax token (Sec. 3.2).  The K tokens of a position form an empirical token
 * distribution; a draft token is accepted when it is one of them (naive
 * token-matching criterion, Sec. 3.2) or when it is their most frequent token
 * (majority criterion, Eq. 6).  Positions are accepted left to right and the first
 * rejection rejects everything after it (Sec. 2, lossless-decoding paragraph);
 * for draft trees (Sec. 4.4) the result is the longest accepted root-to-leaf path.
 *
 * Conventions that hold for every entry point
 *   - Unless a parameter says "host", every tensor pointer is a DEVICE pointer on
 *     the context's device, owned by the caller, dense row-major, and must stay
 *     valid until the work queued on `stream` has finished.
 *   - H (and W) must be 16-byte aligned (DM_EINVAL otherwise).
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default
 *     stream).  Device-pointer entry points only enqueue work: they never
 *     synchronise, never allocate and never free.
 *     The context-based verify calls (dropmatch_verify, _batched, _tree, _batched_next, _js)
 *     can therefore be captured into a CUDA graph; the seed and all sizes are then fixed.
 *   - The library allocates device memory only in dm_create, dm_set_head,
 *     dm_enable_js and dm_enable_score (its workspace) and frees it in dm_set_head / dm_destroy.
 *   - Every function returns DM_OK or a negative status; nothing throws, aborts
 *     or prints.  A CUDA error raised by earlier asynchronous work is reported by
 *     the next call as DM_ECUDA.  A kernel that gives up on an internal wait sets
 *     the context's device error word, which dm_device_error() reads.
 *   - Masks: element j of path i at position t of sequence s is dropped iff word
 *     (j mod 4) of Philox4x32-10(counter = (j/4, i, t, s mod 2^32),
 *     key = (seed low 32 bits, seed high 32 bits)) is < floor(p * 2^32).
 *     Results depend on (seed, s, t, i, j) only, never on batching or launch shape.
 *     (dm_set_mask_mode can take t out of the key.)
 *   - Row order: path i of hidden row q (q = b*T + t) is "row" q*K + i.
 *   - A context is not thread-safe; use one per host thread or lock around it.
 */
#ifndef DROPMATCH_H_
#define DROPMATCH_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dm_ctx dm_ctx; /* opaque: device id, head description, workspace, TMA descriptors */

enum {
    DM_OK = 0,
    DM_EINVAL = -1,       /* bad argument (null pointer, size < 1, p outside [0,1), bad enum)   */
    DM_EUNSUPPORTED = -2, /* shape the kernels cannot handle (see dm_set_head)                  */
    DM_ECUDA = -3,        /* a CUDA runtime or driver call failed                               */
    DM_EWORKSPACE = -4,   /* call needs more rows than dm_set_head reserved                     */
    DM_EDEVICE = -5,      /* device is not compute capability 10.x                              */
    DM_ENOHEAD = -6,      /* dm_set_head has not been called                                    */
    DM_ESTATICLIMIT = -7  /* call exceeds DM_STATIC_MAX_ROWS of dropmatch_verify_batched_static */
};
enum { DM_F32 = 0, DM_BF16 = 1 };             /* storage type of W and H (accumulation is fp32) */
enum { DM_RULE_NAIVE = 0, DM_RULE_MAJORITY = 1 };
enum { DM_IMPL_AUTO = 0, DM_IMPL_SIMT = 1, DM_IMPL_TCGEN05 = 2 };
enum { DM_MASK_PER_POSITION = 0, DM_MASK_PER_PATH = 1 };
enum { DM_TAIL_RENORM = 0, DM_TAIL_BUCKET = 1 };   /* what a teacher's mass outside its given tokens becomes (dropmatch_distill) */
#define DM_MAX_TOP 128                             /* alternatives, and teacher tokens, per row */

/* Create a context on CUDA device `device` (must be sm_100).  *out is set on success. */
int dm_create(dm_ctx** out, int device);
/* Free the context and its workspace.  Synchronises the device first.  NULL is allowed. */
int dm_destroy(dm_ctx* ctx);

/* Describe the LM head (Eq. 3): W is a device pointer to V*d elements, row-major [V,d],
 * 16-byte aligned, caller-owned; it is read, never written, by every verify call until the
 * next dm_set_head, and it must be complete before a call is enqueued: the tensor-core kernel
 * is launched with programmatic stream serialization and starts streaming W while the kernel
 * ahead of it in the stream is still finishing (H, the drafts and all outputs are only touched
 * after that kernel has completed).  Reserves workspace for calls of up to `max_rows` rows (rows = B*T*K, or
 * B*N_h*K for trees) and `max_hidden_rows` = rows/K hidden rows (used only by the *_host entry
 * point's staging buffers).  Requirements: V >= 1; d >= 4 and d % 4 == 0 (fp32) or d % 8 == 0
 * (bf16), else DM_EUNSUPPORTED.  bf16 heads with d % 64 == 0 run on the tcgen05 tensor-core
 * kernel, everything else on the CUDA-core kernel, which also needs one hidden row to fit
 * 200 KB of shared memory (d <= 51200 fp32, 102400 bf16; verify calls report DM_EUNSUPPORTED
 * beyond).  Synchronises the device (re-allocation); pins host memory for the *_host call. */
int dm_set_head(dm_ctx* ctx, const void* W, int V, int d, int dtype, int max_rows, int max_hidden_rows);

/* Programmatic stream serialization of the tensor-core kernel, on by default: the kernel starts
 * streaming W while the kernel ahead of it in the stream is still finishing, which is only right
 * if nothing ahead in the stream writes W.  A caller that refreshes W in stream order (a weight
 * reload, a dequantisation into the head buffer) and verifies right behind it on the same stream
 * switches it off with dm_set_pdl(ctx, 0): every verify kernel then starts after all earlier work
 * of the stream has completed, at the cost of about 2 us of launch latency per call. */
int dm_set_pdl(dm_ctx* ctx, int enable);

/* Force a kernel family (DM_IMPL_*) for later calls; DM_IMPL_AUTO restores the default choice.
 * DM_IMPL_TCGEN05 on a head it cannot handle makes verify calls return DM_EUNSUPPORTED. */
int dm_set_impl(dm_ctx* ctx, int impl);

/* How Eq. 1's masks are keyed for later calls.  DM_MASK_PER_POSITION (default): an independent
 * mask per (sequence, position, path).  DM_MASK_PER_PATH: the position is left out of the key, so
 * path i of a sequence applies one and the same mask m^(i) at every position (for trees: at every
 * hidden row) -- the K paths then behave as K persistent heads, which is how Eq. 1 and the
 * per-head table of Sec. 3.1 can also be read.  Everything else is unchanged. */
int dm_set_mask_mode(dm_ctx* ctx, int mode);

/* Verify one chain of T draft tokens (sequence id 0): Eq. 1-3, per-path argmax, token counts,
 * acceptance scan.
 *   H[T,d]           hidden state whose head output predicts draft[t] (storage type of the head)
 *   draft[T]         draft token ids (ids outside [0,V) simply never match)
 *   K                paths per position, 1 <= K <= 1024;  p in [0,1): drop probability;  seed: Philox key
 *   rule             DM_RULE_NAIVE (Sec. 3.2 token matching) or DM_RULE_MAJORITY (Eq. 6)
 *   out_tokens[T,K]  argmax token of every path (ties: smallest id)
 *   out_counts[T,K]  out_counts[t,i] = number of paths i' with out_tokens[t,i'] == out_tokens[t,i]
 *   out_accept_len[1] number of leading accepted draft tokens, in [0,T] */
int dropmatch_verify(dm_ctx* ctx, const void* H, const int32_t* draft, int T, int K, float p,
                     uint64_t seed, int rule, int32_t* out_tokens, int32_t* out_counts,
                     int32_t* out_accept_len, void* stream);

/* B independent chains in one pass over W; sequence b has id seq_base + b.
 *   H[B,T,d], draft[B,T] -> out_tokens[B,T,K], out_counts[B,T,K], out_accept_len[B];
 *   out_draft_hits[B,T] (may be NULL) = number of paths whose token equals draft[b,t].
 * Equals B calls of dropmatch_verify with the matching sequence ids, bit for bit. */
int dropmatch_verify_batched(dm_ctx* ctx, const void* H, const int32_t* draft, int B, int T, int K,
                             float p, uint64_t seed, uint64_t seq_base, int rule,
                             int32_t* out_tokens, int32_t* out_counts, int32_t* out_draft_hits,
                             int32_t* out_accept_len, void* stream);

/* dropmatch_verify_batched with the sampling decode rule: Sec. 3.2 lets the per-path token be the
 * top-1 token "or" one selected by nucleus sampling, without giving parameters.  Here path i of
 * position t draws y from Softmax(l / temperature) by the Gumbel-max construction,
 *   y = argmax_v ( l[v] / temperature - log(-log(u[v])) ),   equal keys -> smaller id,
 * with u[v] = (n + 0.5) / 2^23, n = top 23 bits of word (v mod 4) of
 * Philox4x32-10(counter = (v/4, i + 2^31, t, s mod 2^32), key = seed): the same generator as the
 * masks, on counters the masks never use, so a call is reproducible from (seed, s, t, i) alone.
 *   temperature > 0;  top_p in (0,1]: the nucleus mass.
 * top_p = 1 (temperature sampling): the noise is generated in the epilogue of the head kernel (one
 * Philox call and two logarithms per logit); no logit is written to memory.
 * top_p < 1 (nucleus sampling): the nucleus is the tokens in order of decreasing
 * Softmax(l / temperature) (equal probabilities: increasing id) up to and including the one whose
 * cumulative probability reaches top_p, and the draw is restricted to it.  The cut needs all logits
 * of a path at once: the head kernel writes them to the buffer that dm_enable_js reserves (call it
 * first with room for B*T*K rows, else DM_EWORKSPACE), and a second kernel, one thread-block cluster per path,
 * finds the boundary by mass (fixed-point sums: the result does not depend on the order of
 * additions) and draws the token.  Sharded heads (dm_set_vocab_offset) are not supported here: the
 * nucleus is taken over this context's head.
 * Counts, per-position test and scan are unchanged; everything else as for dropmatch_verify_batched. */
int dropmatch_verify_batched_sampled(dm_ctx* ctx, const void* H, const int32_t* draft, int B, int T, int K,
                                     float p, uint64_t seed, uint64_t seq_base, int rule, float temperature,
                                     float top_p, int32_t* out_tokens, int32_t* out_counts,
                                     int32_t* out_draft_hits, int32_t* out_accept_len, void* stream);

/* dropmatch_verify_batched plus the token the engine emits after the accepted prefix.  Every
 * hidden row gets, in the same pass over W, one more path without dropout: the target model's own
 * greedy token (the paper does not say how DropMatch picks the correction or bonus token; this
 * is the choice of plain speculative decoding with greedy verification).
 *   H[B, T + bonus_row, d]   bonus_row = 1: one more hidden row per sequence, the state after the
 *                            last draft token, so that a fully accepted draft yields a bonus token
 *   draft[B,T]               as before; positions 0..T-1 are scanned
 *   out_tokens, out_counts   [B, T + bonus_row, K] (the extra row's paths are computed too)
 *   out_draft_hits           [B,T] or NULL
 *   out_plain_tokens         [B, T + bonus_row]: argmax of the undropped head per hidden row
 *   out_next_token[B]        out_plain_tokens[b, accept_len[b]], or -1 if that row does not exist
 * Counts B*(T+bonus_row)*(K+1) rows against max_rows of dm_set_head.  K <= 1023. */
int dropmatch_verify_batched_next(dm_ctx* ctx, const void* H, const int32_t* draft, int B, int T, int bonus_row,
                                  int K, float p, uint64_t seed, uint64_t seq_base, int rule,
                                  int32_t* out_tokens, int32_t* out_counts, int32_t* out_draft_hits,
                                  int32_t* out_accept_len, int32_t* out_plain_tokens, int32_t* out_next_token,
                                  void* stream);

/* Same as dropmatch_verify_batched, but H, draft and all outputs are HOST pointers (pinned or
 * pageable).  Pinned buffers (cudaHostAlloc, cudaHostRegister, torch pin_memory) are used where
 * they are: the first kernel of the call (the mask pass, or a small copy kernel) fetches the
 * inputs over the host link while the head kernel already streams W, and the results are
 * written by the device straight into the caller's arrays.  Pageable buffers go through the
 * context's own pinned buffers (one memcpy each way).  The call returns once every result is in
 * place: the block that finishes the call writes a word into host memory behind its results and
 * the host waits for that word (or, where several blocks finish the call, for `stream` to
 * drain), so the call's last kernel may still be retiring on `stream` for a few microseconds
 * after the return; work queued on `stream` afterwards is ordered behind it as usual.  Whether a pointer is pinned is
 * looked up once and remembered (the last eight pointers): do not unpin or free a buffer and
 * reuse its address as pageable memory without a dm_set_head in between.  Needs
 * B*T <= max_hidden_rows of dm_set_head; H_host 16-byte aligned.  out_draft_hits may be NULL. */
int dropmatch_verify_batched_host(dm_ctx* ctx, const void* H_host, const int32_t* draft_host, int B,
                                  int T, int K, float p, uint64_t seed, uint64_t seq_base, int rule,
                                  int32_t* out_tokens_host, int32_t* out_counts_host,
                                  int32_t* out_draft_hits_host, int32_t* out_accept_len_host,
                                  void* stream);

/* JS-divergence criterion (Sec. 3.2: Eq. 4, Eq. 5, Algorithm 1).  dm_enable_js reserves, after
 * dm_set_head, the buffers this criterion needs for calls of up to max_rows = B*T*K paths and
 * max_hidden_rows = B*T positions: fp32 logits of every path (max_rows * V * 4 bytes) and small
 * partial sums.  Allocates; synchronises the device; a later dm_set_head drops the buffers. */
int dm_enable_js(dm_ctx* ctx, int max_rows, int max_hidden_rows);

/* Chain verification under Algorithm 1: position t is accepted iff
 *   JS(phat_t || pbar_t) <= max_i JS(p_t^(i) || pbar_t)                         (Eq. 5), or
 *   draft[t] is the most frequent of the K path tokens                           (Eq. 6),
 * where p_t^(i) = Softmax(l_t^(i)), pbar_t = Softmax(mean_i l_t^(i)) (Eq. 4) and phat_t is the
 * draft model's distribution; then the left-to-right rule.  Natural logarithm; fp32 arithmetic
 * on fp32 logits.
 *   draft_prob[B,T,V]   device, fp32 probabilities of the draft model (used as given)
 *   out_js[B,T,K+1]     device, fp32: JS(p^(i) || pbar) for i < K, then JS(phat || pbar)
 *   out_js_ok[B,T]      device, 1 iff Eq. 5 holds (may be NULL)
 *   the rest            as for dropmatch_verify_batched
 * Needs dm_enable_js with room for the call, else DM_EWORKSPACE; B*T <= 65535, else
 * DM_EUNSUPPORTED (checked before anything is launched).  Only enqueues work. */
int dropmatch_verify_js(dm_ctx* ctx, const void* H, const int32_t* draft, const float* draft_prob, int B, int T,
                        int K, float p, uint64_t seed, uint64_t seq_base, int32_t* out_tokens,
                        int32_t* out_counts, float* out_js, int32_t* out_js_ok, int32_t* out_accept_len,
                        void* stream);

/* ---- log-probabilities, and training the draft model ---------------------------------------------
 * The paper decides on tokens; an engine around it also wants their log-probabilities, and a draft
 * model whose tokens get accepted has to be trained towards the target.  The calls below cover
 * that: dropmatch_score reads the target's head (and gives a teacher's top tokens), dropmatch_distill
 * trains the draft's logits towards them, dropmatch_logprobs and its gradient work on any logits.
 * Results do not depend on the order in which CTAs run: equal calls give equal bits.
 *
 * Definitions, for a row of logits l[0..V) and a temperature T > 0:
 *   z = l / T;  lse = log sum_v exp(z[v]);  log p[v] = z[v] - lse;  entropy = - sum_v p[v] log p[v].
 * Natural logarithms.  Outputs (float32, one per row, each may be NULL):
 *   out_logprob   log p[tokens[r]]; 0 where tokens[r] is outside [0,V) (a row without a token);
 *                 needs `tokens`
 *   out_lse, out_entropy
 *   out_top_ids, out_top_logprob [rows, n_top]   the n_top largest entries in decreasing order, equal
 *                 entries: smaller id first.  Both or, with n_top = 0, neither.  n_top <= min(V, DM_MAX_TOP)
 * Masked entries: -inf has probability 0 (log p = -inf) and never yields a NaN; a large negative
 * number is just a number.  A row of nothing but -inf: lse = -inf, entropy 0, every log p = -inf.
 * A row that holds a NaN or +inf: lse, entropy and every log-probability of the row are NaN (top ids
 * list NaN first).  Sums are fp32; they are kept without the row's largest entry, so that
 * log-probabilities close to 0 keep their relative precision. */

/* Score hidden rows against the context's head, without dropout: l = H W^T (Eq. 3).
 * dm_enable_score reserves, after dm_set_head, the workspace for calls of up to max_rows rows (at most
 * dm_set_head's) and max_top alternatives: records of every vocabulary slice and, with alternatives, fp32
 * logits of at most 512 rows at a time.  Allocates; synchronises the device; a later dm_set_head or
 * dm_enable_score drops the buffers (graphs captured with them must not be replayed).
 *   H[n_rows,d]      storage type of the head, 16-byte aligned; finite, as W (what a row reports that a NaN
 *                    or an infinity in either reaches is unspecified; it is never a fault)
 *   tokens[n_rows]   device, may be NULL (then out_logprob must be NULL)
 * n_rows = 0 is allowed and does nothing.  DM_EWORKSPACE beyond what dm_enable_score reserved.
 * Sharded heads (dm_set_vocab_offset) are not supported: DM_EUNSUPPORTED.  Like every context-based
 * call it uses the context's workspace: order the calls (and captured graphs) of one context.
 * If a kernel gives up on a wait (dm_device_error), the outputs are NaN and ids -1. */
int dm_enable_score(dm_ctx* ctx, int max_rows, int max_top);
int dropmatch_score(dm_ctx* ctx, const void* H, const int32_t* tokens, int n_rows, int n_top, float temperature,
                    float* out_logprob, float* out_lse, float* out_entropy, int32_t* out_top_ids,
                    float* out_top_logprob, void* stream);

/* The same on logits in memory.  Needs no head and no workspace: calls of one context may overlap.
 *   logits[n_rows][ld]   dtype DM_F32 or DM_BF16, row stride ld >= V entries, aligned to one entry
 *                        (16-byte aligned rows of the same alignment are the fastest)
 * n_rows = 0 is allowed and does nothing.  V <= 2^30.
 * Error word (dm_device_error) 8, this call and the gradients: a cluster's wait for the answer to its request
 * for another row ran out (dm_debug_set_wait_limit).  It waits once more, for a second, and goes on with the
 * answer: the outputs are complete.  Only where that wait runs out too are rows that it would have taken unwritten. */
int dropmatch_logprobs(dm_ctx* ctx, const void* logits, int dtype, int64_t ld, int n_rows, int V,
                       const int32_t* tokens, int n_top, float temperature, float* out_logprob, float* out_lse,
                       float* out_entropy, int32_t* out_top_ids, float* out_top_logprob, void* stream);

/* Gradient of sum_r ( g_logprob[r] * logprob[r] + g_entropy[r] * entropy[r] ) with respect to the
 * logits:  dl[v] = (1/T) ( g_logprob (1[v = token] - p[v]) - g_entropy p[v] (log p[v] + entropy) ).
 *   g_logprob, g_entropy [n_rows]   float32; either may be NULL (zero); `tokens` is needed with g_logprob
 *   out_grad[n_rows][ld_grad]       same type as the logits, rounded once; may be the logits themselves
 *                                   (same pointer, ld_grad = ld), else the two ranges, from the first row's
 *                                   first entry to the last row's last, must not overlap.
 *                                   Entries V..ld_grad of a row are left as they are
 * A row whose two factors are 0 (or that has no token and g_entropy = 0) gets a gradient of 0 whatever
 * its logits hold; so does a row of nothing but -inf.  An entry of less than 2^-126 (1.2e-38) of the row's
 * largest probability counts as 0.  Recomputes the row's sums: one read of the logits, one write. */
int dropmatch_logprobs_grad(dm_ctx* ctx, const void* logits, int dtype, int64_t ld, int n_rows, int V,
                            const int32_t* tokens, float temperature, const float* g_logprob,
                            const float* g_entropy, void* out_grad, int64_t ld_grad, void* stream);

/* Distillation of a teacher that is known by k tokens per row: loss[r] = KL(teacher || student) and the
 * gradient of sum_r weight[r] * loss[r] with respect to the student's logits, in one pass.
 *   teacher_ids[n_rows,k], teacher_logprob[n_rows,k]   1 <= k <= DM_MAX_TOP.  An id outside [0,V) is an
 *       absent entry.  Values are taken at the teacher's temperature: dropmatch_score at temperature T
 *       gives them for a student temperature T.  -inf is probability 0.  An id that occurs twice counts
 *       with both values.
 *   tail  DM_TAIL_RENORM: q = Softmax(teacher_logprob) over the present entries (any common offset cancels:
 *         logits / T will do);   loss = sum q (log q - log p)
 *         DM_TAIL_BUCKET: q = exp(teacher_logprob) and the rest q_t = max(0, 1 - sum q) is matched as one
 *         outcome against the student's mass p_t outside the teacher's tokens:
 *         loss = sum q (log q - log p) + q_t (log q_t - log p_t)   (no rest where the tokens cover V)
 *   weight[n_rows]   float32 or NULL (1): a mask, 1/n, or the upstream gradient of loss[r]
 *   out_loss[n_rows] float32 (without the weight) or NULL;  out_grad as above, or NULL; not both NULL
 *   dl[v] = weight / T * ( M p[v] - q[v] - [v is no teacher token] q_t p[v] / p_t ),  M = sum q + q_t
 * No factor T^2 is applied.  A row without a present entry: loss 0 and gradient 0, whatever it holds.  A teacher token
 * the student gives probability 0: loss +inf; so does a tail of less than 2^-126 (1.2e-38) of the row's mass,
 * whose gradient is left out.  A row of nothing but -inf: gradient 0.  A row of weight 0
 * gets a gradient of 0 whatever it holds.  DM_EUNSUPPORTED beyond V of about 12 million (bf16) or 6 million
 * (fp32) with DM_TAIL_BUCKET or a gradient. */
int dropmatch_distill(dm_ctx* ctx, const void* logits, int dtype, int64_t ld, int n_rows, int V,
                      const int32_t* teacher_ids, const float* teacher_logprob, int k, int tail, float temperature,
                      const float* weight, float* out_loss, void* out_grad, int64_t ld_grad, void* stream);

/* ---- verification against the target's own distribution --------------------------------------------
 * The lossless rule of speculative decoding (Sec. 2), from random numbers that the caller draws: what DropMatch's
 * criteria are measured against, and what an engine falls back to.  For sequence b and drafted position t, with
 *   p = Softmax(target[b,t] / temperature),   q = Softmax(draft_logits[b,t] / draft_temperature),
 * the drafted token x is accepted iff u_accept[b,t] * q(x) < p(x); n is the length of the accepted prefix.  The
 * next token is drawn from r = max(p - q, 0) of row n (p, if r is 0 everywhere) where a token was rejected, and
 * from p of row n where all were accepted: the smallest v with  r(0) + ... + r(v) > u_next[b] * sum r.
 * Decisions and draws are those of 64-bit arithmetic on the given logits (exponentials to 2^-42; a difference p - q of
 * less than 2^-41 p counts as 0, of less than 2^-40 p may); out_accept_prob is fp32.
 *   target[B][T + bonus_row][ld_target]   dtype DM_F32 or DM_BF16; row stride ld_target >= V entries, aligned to one
 *                                entry (16-byte aligned rows are the fastest).  bonus_row = 1: one more row per
 *                                sequence, behind the last drafted token
 *   draft_logits[B][T][ld_draft] draft_dtype, as above; NULL: a drafter without a distribution (q is 1 on x, draft_dtype,
 *                                ld_draft and draft_temperature are not looked at)
 *   draft[B,T]                   ids outside [0,V) have p = 0
 *   draft_len[B]                 drafted tokens of each sequence, in [0,T] (clamped), or NULL: T.  Rows and tokens behind
 *                                them are not read, but for row draft_len[b] of the target, which the next token is drawn from
 *   u_accept[B,T], u_next[B]     float32 in [0,1).  Outputs must not overlap inputs
 *   out_accept_len[B], out_next_token[B]   -1 if every one of T tokens was accepted and there is no bonus row
 *   out_accept_prob[B,T]         float32, min(1, p(x) / q(x)); 0 behind draft_len.  Read by the call's second kernel.  Its
 *                                sums are split by B, T and V: a position's last bits may differ with the B and T of the
 *                                call, decisions and tokens only where 64-bit sums round apart
 * Masked entries: -inf has probability 0; a row of nothing but -inf has probability 0 everywhere.  A row that holds a
 * NaN or +inf: accept_prob NaN, the token is not accepted, next token -1; next token -1 too where there is nothing to draw from.
 * T = 0 with a bonus row draws one token per sequence (draft, u_accept and out_accept_prob may be NULL).  B = 0 is
 * allowed and does nothing.  V <= 2^30 and B (T + bonus_row) <= 2^27, else DM_EUNSUPPORTED.  Needs no head and no
 * workspace: calls of one context may overlap. */
int dropmatch_verify_lossless(dm_ctx* ctx, const void* target, int dtype, int64_t ld_target, const void* draft_logits,
                              int draft_dtype, int64_t ld_draft, const int32_t* draft, const int32_t* draft_len, int B,
                              int T, int bonus_row, int V, float temperature, float draft_temperature,
                              const float* u_accept, const float* u_next, int32_t* out_accept_len,
                              int32_t* out_next_token, float* out_accept_prob, void* stream);

/* ---- dropout as an operator ------------------------------------------------------------------------
 * Eq. 1 and Eq. 2 on rows in memory, with the masks of the verify calls (same key, same counters, dm_set_mask_mode
 * included): a head or a draft model is trained under the dropout that it is verified with.  No mask is stored; the
 * gradient generates it again from the same arguments.
 *   dropmatch_dropout       x[B*T][ld] -> out[B*T*K][ld_out]:  out[(b*T+t)*K+i, j] = keep ? x[b*T+t, j] * s : 0
 *   dropmatch_dropout_grad  grad[B*T*K][ld] -> out_grad[B*T][ld_out]:  s * sum_i (keep ? grad[(b*T+t)*K+i, j] : 0)
 * with s = 1 / (1 - p) in fp32; fp32 arithmetic, rounded once to dtype (DM_F32 or DM_BF16).  Dropped entries are +0
 * and add nothing whatever they hold.  Plain dropout of n rows: B = 1, T = n, K = 1.
 *   1 <= K <= 1024, B*T*K < 2^30, 1 <= d <= 2^30, strides >= d entries, pointers aligned to one entry (16-byte aligned
 *   rows are the fastest); entries d..ld_out of a row are left as they are.  The output must not overlap the input, each
 *   from its first entry to the last row's last (so not its neighbouring columns either), but for K = 1 may be the
 *   input itself (same pointer and stride).  B*T = 0 is allowed and does nothing.
 * A row's results do not depend on the other rows of the call.  Needs no head and no workspace: calls of one context
 * may overlap.  dm_set_mask_mode's value is taken at the call (and fixed in a captured graph). */
int dropmatch_dropout(dm_ctx* ctx, const void* x, int dtype, int64_t ld, int B, int T, int K, int d, float p,
                      uint64_t seed, uint64_t seq_base, void* out, int64_t ld_out, void* stream);
int dropmatch_dropout_grad(dm_ctx* ctx, const void* grad, int dtype, int64_t ld, int B, int T, int K, int d, float p,
                           uint64_t seed, uint64_t seq_base, void* out_grad, int64_t ld_out, void* stream);

/* ---- a head in 8-bit integers ----------------------------------------------------------------------
 * Projections through a matrix W[V,d] held in 8-bit integers with a scale for each row (vocabulary entry, channel), of
 * rows quantised to 8 bits with a scale for each row (token): half the bytes of a bf16 head, which bound a projection of few
 * rows.  The calls on a context's head (dm_set_head) take fp32 and bf16 only.
 * The logits go where any logits go (dropmatch_verify_lossless, _logprobs, _distill).
 *   dropmatch_quantize_i8  x[n_rows][ld] (DM_F32 or DM_BF16) -> out_q[n_rows][ld_q], out_scale[n_rows]:
 *                          scale = max(max_j |x[j]| / 127, 2^-126),  q[j] = x[j] / scale rounded to the nearest whole number,
 *                          ties to even; both quotients in fp32.  For W once and for tokens at every call.  A row that
 *                          holds a NaN or an infinity: scale NaN, q = 0 (its products are NaN).
 *   dropmatch_matmul_i8    out[r, v] = a_scale[r] * w_scale[v] * sum_j a[r, j] * w[v, j], out[n_rows][ld_out] in out_dtype
 *                          (DM_F32 or DM_BF16).  The sum is exact (32-bit integers); it is converted to fp32, multiplied
 *                          by w_scale, then by a_scale, and rounded once to out_dtype.
 *   dropmatch_linear_i8    both: quantises x into out_q / out_scale (the caller's, contents of no further use) and
 *                          multiplies; W and w_scale must be complete before the call is enqueued or be written by
 *                          earlier work of the same stream.
 * 8-bit matrices: any value in [-128, 127], 16-byte aligned, row strides (bytes) a multiple of 16; bytes d..ld of a row are
 * neither read nor written.  x, scales and out are aligned to one entry, strides at least the row's length; columns V..ld_out
 * are left as they are.  Products: d <= 131071, V and n_rows <= 2^30; quantisation: n <= 2^30; else DM_EUNSUPPORTED.  Outputs
 * must not overlap inputs, each from its first entry to the last row's last.
 * n_rows = 0 is allowed and does nothing.  Need no head and no workspace: calls of one context may overlap (linear's with
 * their own out_q and out_scale).  If a kernel gives up on a wait (dm_device_error), outputs that it did not reach are NaN. */
int dropmatch_quantize_i8(dm_ctx* ctx, const void* x, int dtype, int64_t ld, int n_rows, int n, int8_t* out_q,
                          int64_t ld_q, float* out_scale, void* stream);
int dropmatch_matmul_i8(dm_ctx* ctx, const int8_t* a, int64_t ld_a, const float* a_scale, int n_rows, const int8_t* w,
                        int64_t ld_w, const float* w_scale, int V, int d, void* out, int out_dtype, int64_t ld_out,
                        void* stream);
int dropmatch_linear_i8(dm_ctx* ctx, const void* x, int dtype, int64_t ld, int n_rows, const int8_t* w, int64_t ld_w,
                        const float* w_scale, int V, int d, int8_t* out_q, int64_t ld_q, float* out_scale, void* out,
                        int out_dtype, int64_t ld_out, void* stream);

/* Vocabulary-sharded heads (the deployment of Sec. 4.1 is tensor-parallel: every GPU holds a
 * slice of the LM head).  A context whose head is rows [offset, offset+V) of the full head reports
 * global token ids after dm_set_vocab_offset(ctx, offset) (call it after dm_set_head; default 0).
 * The masks are keyed on indices only, so every shard draws the same masks without any exchange.
 *
 * dropmatch_partial_best runs Eq. 1-3 and the vocabulary reduction on this context's head and
 * writes one packed word per path, out_packed[B*T*K] (device): (ordered fp32 key of the best logit
 * << 32) | (2^32-1 - token id).  The elementwise maximum of such arrays from all shards is the
 * result for the full head (equal logits resolve to the smaller token id).
 *
 * dropmatch_finalize_packed takes n_parts such arrays back to back, packed[n_parts][B*T*K]
 * (device) -- the layout an all-gather over the shards produces -- merges them and runs the
 * histogram and the acceptance scan as dropmatch_verify_batched does.  Needs no head.
 * Both only enqueue work on `stream`. */
int dm_set_vocab_offset(dm_ctx* ctx, int offset);
int dropmatch_partial_best(dm_ctx* ctx, const void* H, int B, int T, int K, float p, uint64_t seed,
                           uint64_t seq_base, uint64_t* out_packed, void* stream);
int dropmatch_finalize_packed(dm_ctx* ctx, const uint64_t* packed, int n_parts, const int32_t* draft, int B, int T,
                              int K, int rule, int32_t* out_tokens, int32_t* out_counts, int32_t* out_draft_hits,
                              int32_t* out_accept_len, void* stream);

/* The paper has no counterpart to this entry point; it exists for the way the library gets
 * deployed.  Some hosts of this code cannot ask CUDA for device memory at the time they verify:
 * a serving process that hands all of HBM to its own pool at start-up (a later cudaMalloc fails
 * or eats into the KV cache), a latency-critical decode loop (cudaMalloc and cudaFree stall the
 * whole device), or a plug-in that is handed tensors but may not set up a context with a
 * workspace of its own.  For them this call does what dropmatch_verify_batched does on the
 * CUDA-core kernel family, for fp32 and bf16 heads alike, but needs no dm_ctx and never
 * allocates or frees: the per-slice partial argmaxes go to a fixed array inside the library
 * image (about 0.6 MB, held by every GPU that loads the library until the process exits).
 *   device           CUDA device of all the pointers (compute capability 10.x)
 *   W[V,d], dtype    the LM head, as for dm_set_head (device pointer, 16-byte aligned)
 *   the rest         as for dropmatch_verify_batched; out_draft_hits may be NULL
 * Limits and rules:
 *   - B*T*K <= DM_STATIC_MAX_ROWS, else DM_ESTATICLIMIT and nothing is launched.
 *   - The first call on a device looks the array's device address up (once per device and
 *     process).  With CUDA's lazy module loading that first call is also when the driver loads
 *     the code and sets the 0.6 MB array aside, which can fail (DM_ECUDA) once a pool owns all
 *     of the device's memory: make one call per device at start-up, before the pool takes the
 *     memory and before any stream capture begins.  The remembered address does not survive a
 *     cudaDeviceReset.
 *   - All calls on a device share the one array, which keeps the previous call's contents; the
 *     call itself clears the part that must start at zero.  Two calls whose kernels can overlap
 *     on the GPU (different streams, or host threads racing on one device) corrupt each other:
 *     issue them on one stream, or order them with events.
 *   - Only enqueues work on `stream`; results are ready when the stream reaches that point. */
#define DM_STATIC_MAX_ROWS 256
int dropmatch_verify_batched_static(int device, const void* W, int V, int d, int dtype, const void* H,
                                    const int32_t* draft, int B, int T, int K, float p, uint64_t seed,
                                    uint64_t seq_base, int rule, int32_t* out_tokens, int32_t* out_counts,
                                    int32_t* out_draft_hits, int32_t* out_accept_len, void* stream);

/* Draft trees (Sec. 4.4).  Per sequence: N_h hidden rows H[b,q,:] and N nodes in topological
 * order.  Node n has a token, a parent node (node_parent[n] < n; -1 = child of the committed
 * prefix) and node_hrow[n] in [0,N_h): the hidden row whose head output predicts it (children
 * of one parent share one row).  Paths of hidden row q use position index t = q in the mask key.
 *   node_ok[n] = (parent is the prefix or node_ok[parent]) and token[n] passes `rule` against the
 *                K tokens of row node_hrow[n];
 *   out_accept_len[b] = depth of the deepest ok node (0 if none);
 *   out_best_node[b]  = smallest-index ok node of that depth (-1 if none).
 *   out_tokens[B,N_h,K], out_counts[B,N_h,K]; out_node_ok[B,N] may be NULL.
 * Node arrays are not validated on the device beyond clamping out-of-range indices to "rejected". */
int dropmatch_verify_tree(dm_ctx* ctx, const void* H, const int32_t* node_token,
                          const int32_t* node_parent, const int32_t* node_hrow, int B, int N_h, int N,
                          int K, float p, uint64_t seed, uint64_t seq_base, int rule,
                          int32_t* out_tokens, int32_t* out_counts, int32_t* out_node_ok,
                          int32_t* out_best_node, int32_t* out_accept_len, void* stream);

/* dropmatch_verify_tree plus, in the same pass over W, the target's own greedy token of every
 * hidden row (one more path without dropout, as in dropmatch_verify_batched_next):
 * out_plain_tokens[B,N_h].  The token to emit after the accepted path is the entry of the hidden
 * row that the best node owns (the caller knows which row that is; it need not exist for a leaf).
 * Counts B*N_h*(K+1) rows against max_rows.  K <= 1023. */
int dropmatch_verify_tree_next(dm_ctx* ctx, const void* H, const int32_t* node_token, const int32_t* node_parent,
                               const int32_t* node_hrow, int B, int N_h, int N, int K, float p, uint64_t seed,
                               uint64_t seq_base, int rule, int32_t* out_tokens, int32_t* out_counts,
                               int32_t* out_node_ok, int32_t* out_best_node, int32_t* out_accept_len,
                               int32_t* out_plain_tokens, void* stream);

/* Debug: full logits (Eq. 3 with Eq. 2's scale) of selected paths, computed by the same kernel
 * family a verify call would use.  H[B,T,d]; row_sel[n_sel,3] holds (b, t, i) triples with
 * 0 <= b < B, 0 <= t < T, i >= 0 (checked on the device: a bad triple yields a row of NaN);
 * sequence b has id seq_base + b.  out_logits[n_sel,V] fp32.  1 <= n_sel <= max_rows. */
int dm_debug_logits(dm_ctx* ctx, const void* H, int B, int T, const int32_t* row_sel, int n_sel,
                    float p, uint64_t seed, uint64_t seq_base, float* out_logits, void* stream);

/* Debug: the keep masks of Eq. 1, bit-packed.  out_bits[B,T,K,ceil(d/32)]: bit (j mod 32) of
 * word j/32 is 1 iff element j is kept.  Needs no head. */
int dm_debug_masks(dm_ctx* ctx, int B, int T, int K, int d, float p, uint64_t seed,
                   uint64_t seq_base, uint32_t* out_bits, void* stream);

/* Debug: the masked hidden rows themselves (Eq. 1 and Eq. 2 without the 1/(1-p) factor), exactly
 * as the tensor-core kernel stages them for calls of more than 64 paths or so: out[B*T*K, d] in
 * the head's storage type, row (b*T+t)*K+i = H[b,t,:] with the dropped elements set to zero.
 * bf16 heads only (DM_EUNSUPPORTED otherwise); out is a device pointer, 16-byte aligned. */
int dm_debug_masked_operand(dm_ctx* ctx, const void* H, int B, int T, int K, float p, uint64_t seed,
                            uint64_t seq_base, void* out, void* stream);

/* Measurement aid: enqueues one read-only pass over `bytes` bytes at device pointer `ptr` (16-byte
 * aligned; the bytes beyond a multiple of 16 are not read).  Timed over a buffer much larger than
 * L2 it gives the read-only HBM rate of the part, the ceiling of any kernel that streams W. */
int dm_debug_read_stream(dm_ctx* ctx, const void* ptr, size_t bytes, void* stream);

/* Reads and clears the context's device error word (0 = none); synchronises `stream` first.
 * Non-zero means a kernel abandoned an internal wait.  The outputs of that call, and of every
 * later call until this function has cleared the word, are then the fail-safe values written on
 * the device, so that no consumer further down the stream mistakes them for results:
 * tokens -1, counts and hits 0, accepted length 0, best node -1, node_ok 0, plain/next tokens -1
 * (the left-to-right rule of Sec. 2 with nothing accepted). */
int dm_device_error(dm_ctx* ctx, void* stream, uint32_t* out_code);

/* Debug: how many clock cycles a kernel of this context waits on one of its internal barriers
 * before it gives up, sets the device error word and winds down (0 restores the default, about
 * one second; the time a call spends queued behind the kernel ahead of it counts).  A limit of
 * a few cycles makes the first wait that is not satisfied at once run out: the tests use that
 * to exercise the wind-down and the fail-safe outputs without hanging or faulting anything.  The wait of the calls
 * on logits in memory for their next row, long satisfied as a rule, counts as run out at a limit of 1. */
int dm_debug_set_wait_limit(dm_ctx* ctx, uint64_t cycles);

/* Timing of the head kernel alone (the dominant kernel).  While enabled, every verify call
 * records a CUDA event on `stream` before and after its masked-head kernel launch(es) (not
 * around the finalize kernel); at most 4096 calls are kept between reads, later ones are not
 * recorded.  dm_profile_read waits for the recorded events, returns the summed elapsed time in
 * milliseconds and the number of calls it covers, and clears the record.  Creating the events
 * allocates driver resources, so enable it outside latency-critical code. */
int dm_profile_head(dm_ctx* ctx, int enable);
int dm_profile_read(dm_ctx* ctx, double* out_ms_total, int* out_calls);

/* Bytes of device workspace the context holds; which kernel family the last verify call used
 * (DM_IMPL_SIMT or DM_IMPL_TCGEN05, 0 before any call); kernels launched by the last call. */
size_t dm_workspace_bytes(const dm_ctx* ctx);
int dm_last_impl(const dm_ctx* ctx);
int dm_last_launches(const dm_ctx* ctx);

const char* dm_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* DROPMATCH_H_ */
