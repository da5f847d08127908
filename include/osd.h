/*
 * osd.h -- C ABI of the MI355X (gfx950) library for the vocabulary-wide logits
 * path of online speculative decoding (Liu et al., "Online Speculative
 * Decoding", ICML 2024, arXiv:2310.07177).
 *
 * Two operations (and their fused, sampling and vocabulary-sharded forms):
 *   osd_verify             speculative-sampling verification of k proposed
 *                          tokens against the target (Appendix A.1, Eq. 5;
 *                          Algorithm 1, the verification step);
 *   osd_distill_loss_grad  the distillation divergence of Eq. 3 (forward KL,
 *                          reverse KL, JSD[beta]) and its gradient with
 *                          respect to the draft (student) logits (Section 4.1,
 *                          Eq. 2-4);
 * and what the model does with drafted tokens in every layer between the two, on a
 * paged cache: osd_cache_append, osd_tree_attention, osd_cache_keep.
 *
 * Conventions shared by every entry point:
 *   - All array arguments are DEVICE pointers owned by the caller; the library
 *     never allocates, frees or synchronises.  Work is enqueued on `stream`
 *     (a hipStream_t passed as void*; NULL is the default stream) and the call
 *     returns without waiting for it.
 *   - Logit arrays are row-major with the vocabulary axis contiguous, in the
 *     dtype given by `dtype` (OSD_F32: IEEE float; OSD_BF16: bfloat16 bit
 *     patterns).  Rows may start at any element and have any length; reads
 *     are fastest from rows whose byte addresses are multiples of 16.
 *   - Host-checkable mistakes (null required pointer, non-positive sizes,
 *     K > OSD_MAX_K, V above osd_max_vocab, NaN or out-of-range scalars, an
 *     unknown enum, a workspace that is too small) return a negative status
 *     and enqueue nothing.  A failed launch returns OSD_ERR_DEVICE.
 *   - Workspaces: the caller allocates `*_workspace_bytes(...)` bytes of
 *     device memory and fills them with zeros ONCE before first use; every
 *     call leaves its workspace zeroed again when its kernels finish (those of
 *     osd_distill_topk_loss_grad, osd_verify_topk and osd_tree_attention keep
 *     scratch beside counters, and each serves its operator alone).  Calls that may run
 *     concurrently need distinct workspaces.  (A workspace that is not zero --
 *     fresh from an uninitialised allocation, or shared by calls in flight on
 *     two streams -- is not detected: the outputs are then wrong, with no
 *     status to say so.)
 *   - Thread-safe: apart from osd_verify_noalloc's per-GPU scratch array
 *     (see there), the library holds no mutable global state.  A call that is
 *     several launches holds a lock while it enqueues them, so threads may
 *     share a workspace as long as they share the stream too.
 */
#ifndef OSD_H
#define OSD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    OSD_OK = 0,
    OSD_ERR_INVALID_ARG = -1,
    OSD_ERR_UNSUPPORTED = -2,
    OSD_ERR_DEVICE = -3,
    OSD_ERR_WORKSPACE = -4,
    OSD_ERR_SCRATCH = -5
} osd_status;

typedef enum { OSD_F32 = 0, OSD_BF16 = 1 } osd_dtype;

typedef enum { OSD_FKL = 0, OSD_RKL = 1, OSD_JSD = 2 } osd_divergence;

#define OSD_MAX_K 16

/* Largest vocabulary size the row-resident kernels accept for `dtype`
 * (0 for an unknown dtype). */
int osd_max_vocab(int dtype);

/* Human-readable name of a status code (static storage). */
const char* osd_status_string(int status);

/* Workspace needed by osd_verify for B sequences of up to K proposals. */
size_t osd_verify_workspace_bytes(int B, int K);

/*
 * osd_verify -- one speculative-decoding verification step for B sequences
 * (Appendix A.1: with i rising from 1 to k, accept proposal y_i when
 * u < p(y_i)/q(y_i) and stop at the first rejection; Eq. 5: then draw one
 * more token from norm(max(0, p - q)) at the rejected position, or from p at
 * position k+1 when all k were accepted).
 *
 * target_logits [B, K+1, V]  row i (0-based) holds the target logits that
 *                            score proposal i, row k_b is the bonus row
 * draft_logits  [B, K, V]    row i holds the draft logits proposal i was
 *                            drawn from; may be NULL when temperature == 0
 * draft_tokens  [B, K] int32 the proposals y
 * draft_len     [B] int32    k_b in 1..K (ragged proposals), or NULL for K;
 *                            rows past k_b are padding and are never read
 * u_accept      [B, K] fp32  acceptance uniforms in [0,1); NULL iff T == 0
 * u_resample    [B] fp32     the uniform of the extra token; NULL iff T == 0
 * temperature   T > 0: logits are divided by T before the softmax (the same T
 *               for target and draft); T == 0: greedy verification, proposals
 *               are accepted while they equal the target argmax (lowest index
 *               on ties) and the extra token is that argmax
 * accepted_len  out [B] int32      a_b in 0..k_b, or -1 for an invalid row
 *                                  (k_b outside 1..K, a token outside [0,V),
 *                                  or a row that is read and has no finite
 *                                  logit)
 * out_tokens    out [B, K+1] int32 y_1..y_a, the extra token, then -1
 * reject_mask   out [B, K] uint8   nullable; 1 at i == a_b when a_b < k_b
 *                                  (the error index recorded for
 *                                  distillation), else 0
 * workspace     osd_verify_workspace_bytes(B, K) zero-initialised bytes
 *
 * Decisions are taken in fp32 arithmetic with fp64 scalars; they agree with
 * an exact computation except where u lies within about 1e-7 of p(y)/q(y) or
 * u*Z within about 1e-7 (in probability mass) of a CDF edge.
 */
int osd_verify(const void* target_logits, const void* draft_logits, int dtype,
               int B, int K, int V,
               const int32_t* draft_tokens, const int32_t* draft_len,
               const float* u_accept, const float* u_resample,
               float temperature,
               int32_t* accepted_len, int32_t* out_tokens,
               uint8_t* reject_mask,
               void* workspace, size_t workspace_bytes, void* stream);

/*
 * osd_verify_noalloc -- osd_verify for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): the same arguments without the workspace, and the same
 * results.  Its scratch is a device array the library holds, one per GPU, of
 * OSD_VERIFY_NOALLOC_SCRATCH_BYTES bytes, kept until the process ends; the
 * call itself allocates nothing.  Calls with
 * osd_verify_workspace_bytes(B, K) > OSD_VERIFY_NOALLOC_SCRATCH_BYTES
 * (about B * (K + 1) > 10000 rows) return OSD_ERR_SCRATCH and enqueue
 * nothing.  Every call on one GPU shares that GPU's array: each call clears
 * the part it needs on its own stream first, and calls that may overlap on
 * one GPU (concurrent streams, other host threads) race and must not be made
 * -- give those osd_verify with separate workspaces.  Other errors as
 * osd_verify.
 */
#define OSD_VERIFY_NOALLOC_SCRATCH_BYTES (4u << 20)
int osd_verify_noalloc(const void* target_logits, const void* draft_logits, int dtype,
                       int B, int K, int V,
                       const int32_t* draft_tokens, const int32_t* draft_len,
                       const float* u_accept, const float* u_resample,
                       float temperature,
                       int32_t* accepted_len, int32_t* out_tokens,
                       uint8_t* reject_mask, void* stream);

/* Workspace needed by osd_distill_loss_grad for B*K rows. */
size_t osd_distill_workspace_bytes(int B, int K);

/*
 * osd_distill_loss_grad -- masked distillation divergence between teacher
 * (target) and student (draft) distributions at temperature tau and its
 * gradient with respect to the student logits (Section 4.1, Eq. 3):
 *   FKL  KL(p || q)                 gradient (q - p) / tau
 *   RKL  KL(q || p)                 gradient q (log q - log p - KL(q||p)) / tau
 *   JSD  beta KL(p || m) + (1-beta) KL(q || m),  m = beta p + (1-beta) q,
 *                                   gradient (1-beta) q (log q - log m - KL(q||m)) / tau
 * with p = softmax(teacher / tau), q = softmax(student / tau), 0 log 0 = 0.
 *
 * teacher_logits  row (b, i) starts at element b*teacher_batch_stride + i*V
 *                 (pass (K+1)*V to distil the first K rows of a verify target)
 * student_logits  row (b, i) starts at element b*student_batch_stride + i*V
 * mask            [B, K] uint8 0/1, or NULL for all ones
 * kind            OSD_FKL / OSD_RKL / OSD_JSD;  beta in [0,1] weights the
 *                 teacher in the JSD mixture;  tau > 0
 * loss_out        out [2] fp32: {sum(mask*D)/sum(mask) (0 if the mask is
 *                 empty), sum(mask*D)} (Eq. 2's batch mean and Eq. 4's sum);
 *                 reduced in a fixed order in fp64, so bitwise deterministic
 * row_loss_out    out [B, K] fp32, nullable: D per row, 0 where mask is 0
 * grad_out        out [B, K, V] in `dtype`, contiguous, nullable: the
 *                 gradient of sum(mask*D); rows with mask 0 are written as 0.
 *                 It may take the student rows' own place for V up to 32768
 *                 (bf16) or 16384 (fp32); otherwise outputs and inputs must
 *                 not overlap
 * workspace       osd_distill_workspace_bytes(B, K) zero-initialised bytes
 *
 * Equal calls give equal bits.  Which kernel takes a row, and so the order of
 * its sums, depends on V, dtype and, for bf16 rows of 24577 to 32768 logits, on
 * whether the call has more than one row per two CUs: there a row's loss and
 * gradient may differ in their last bits between calls of few and of many rows.
 */
int osd_distill_loss_grad(const void* teacher_logits, int64_t teacher_batch_stride,
                          const void* student_logits, int64_t student_batch_stride,
                          int dtype, int B, int K, int V,
                          const uint8_t* mask, int kind, float beta, float tau,
                          float* loss_out, float* row_loss_out, void* grad_out,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Workspace needed by osd_verify_distill for B sequences of up to K proposals. */
size_t osd_verify_distill_workspace_bytes(int B, int K);

/*
 * osd_verify_distill -- one speculative step's verification and
 * distillation in a single pass over the row pairs (Algorithm 1 verifies the
 * proposals and records, at the error index, what distillation later trains
 * on; Section 4.1 and Eq. 2-4 give the divergence).  The results are those
 * of
 *   osd_verify(target, draft, ..., temperature, ...) and
 *   osd_distill_loss_grad(target, (K+1)*V, draft, K*V, dtype, B, K, V,
 *                         distill_mask, kind, beta, temperature, ...):
 * teacher = target rows 0..K-1, student = draft rows, tau = temperature.
 * Both read the same row pairs; done together they are read once and their
 * softmax normalisers are computed once.
 *
 * Arguments as in osd_verify and osd_distill_loss_grad, with:
 * temperature   T > 0: verification temperature and distillation tau
 * distill_mask  [B, K] uint8 0/1, or NULL for all rows: which rows are
 *               distilled (independent of the verification outcome)
 * workspace     osd_verify_distill_workspace_bytes(B, K) zero-initialised
 *               bytes
 *
 * Verification decisions have the same guarantee as osd_verify's (their
 * masses are formed from the distillation's cached exponents, so a draw that
 * sits within ~1e-7 of a CDF edge may differ from osd_verify's); losses and
 * gradients match osd_distill_loss_grad's within fp32 rounding (the fp64 loss
 * sum is taken in a different fixed order; a row's own values are the same bit
 * for bit, except in osd_distill_loss_grad's calls of few rows described there).
 */
int osd_verify_distill(const void* target_logits, const void* draft_logits, int dtype,
                       int B, int K, int V,
                       const int32_t* draft_tokens, const int32_t* draft_len,
                       const float* u_accept, const float* u_resample,
                       float temperature,
                       int32_t* accepted_len, int32_t* out_tokens, uint8_t* reject_mask,
                       const uint8_t* distill_mask, int kind, float beta,
                       float* loss_out, float* row_loss_out, void* grad_out,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * osd_verify_distill_rejected -- osd_verify_distill whose distilled rows are
 * the verification's own outcome: the row pair at each sequence's first
 * rejection a_b (the error index at which Algorithm 1 records the target for
 * distillation; Fig. 1: the positions where the draft proposed a wrong
 * token), and no other.  The results are those of
 *   osd_verify(target, draft, ..., temperature, ..., reject_mask, ...) then
 *   osd_distill_loss_grad(target, (K+1)*V, draft, K*V, dtype, B, K, V,
 *                         reject_mask, kind, beta, temperature, ...):
 * loss_out = {sum of D over the distilled rows / their number (0 if none),
 * that sum}; row_loss_out and grad_out hold zeros on every other row.  The
 * rejected row pair is read once: the workgroup that finds a sequence's
 * first rejection draws the correction and distils the row from what it
 * already holds.  (A workgroup that cannot learn in time whether an earlier
 * position rejected distils its row anyway; if it was not the first, the
 * call's last workgroup zeroes that row again.)
 *
 * Arguments as in osd_verify_distill, without distill_mask; reject_mask is
 * nullable.  workspace: osd_verify_distill_workspace_bytes(B, K)
 * zero-initialised bytes (one workspace serves both fused entry points).
 * Decisions, losses and gradients have osd_verify_distill's accuracy.
 */
int osd_verify_distill_rejected(const void* target_logits, const void* draft_logits, int dtype,
                                int B, int K, int V,
                                const int32_t* draft_tokens, const int32_t* draft_len,
                                const float* u_accept, const float* u_resample,
                                float temperature,
                                int32_t* accepted_len, int32_t* out_tokens, uint8_t* reject_mask,
                                int kind, float beta,
                                float* loss_out, float* row_loss_out, void* grad_out,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * osd_verify_tree -- multi-candidate (tree) verification.  The paper applies
 * its online updates to Medusa, which proposes several candidate tokens per
 * position arranged in a tree (Section 5, "OSD and Medusa", Table 4), and
 * states no verification rule for it; this call takes the rule that keeps
 * Appendix A.1's exactness (the emitted tokens follow the target): the
 * children of a node are candidates drawn independently from the draft
 * distribution q at that node and are tested in ascending node order,
 * candidate c accepted when u_c < R(y_c) / q(y_c), with R = p for the first
 * and, after each rejection, R <- norm(max(0, R - q)) (Eq. 5's residual).
 * The walk continues at the first accepted child; where every child is
 * rejected one token is drawn from the last residual max(0, R - q), and at a
 * node without children one token is drawn from p (the bonus token).  The
 * draws are the inverse CDF of osd_verify.  T == 0: the first child whose
 * token is the target argmax (lowest index on ties) is accepted and the
 * argmax is emitted where the walk stops.  A chain (one child per node) is
 * osd_verify.
 *
 * target_logits [B, N, V]  row n: target logits after the prefix ending at
 *                          node n (it scores node n's children; at a node
 *                          without children it is the bonus distribution)
 * draft_logits  [B, N, V]  row n: draft logits node n's children were drawn
 *                          from; not read at leaves; may be NULL at T == 0
 * parent        [B, N] int32  node 0 is the root (the accepted context; its
 *                          entry is ignored); 0 <= parent[n] < n for n >= 1
 * node_tokens   [B, N] int32  the candidate token of node n (node 0 ignored)
 * u_accept      [B, N] fp32  u_accept[b, n] tests node n; NULL iff T == 0
 * u_resample    [B] fp32    the extra token's uniform; NULL iff T == 0
 * accepted_len  out [B] int32  number of accepted candidates, or -1 for an
 *                          invalid tree (a parent or token out of range) or
 *                          a reached row without finite logits
 * out_tokens    out [B, N] int32  accepted tokens, the extra token, then -1
 * path_nodes    out [B, N] int32, nullable: the accepted nodes, then -1
 * workspace     osd_verify_tree_workspace_bytes(B, N) zero-initialised bytes
 *
 * N <= OSD_MAX_TREE_NODES; V up to 32768 (bf16) or 16384 (fp32), otherwise
 * OSD_ERR_UNSUPPORTED.  Every node's rows are read once, whether or not the
 * walk reaches it: at T > 0 about one workgroup per CU walks the nodes, at
 * T == 0 there is one workgroup per (sequence, node).
 */
#define OSD_MAX_TREE_NODES 64
size_t osd_verify_tree_workspace_bytes(int B, int N);
int osd_verify_tree(const void* target_logits, const void* draft_logits, int dtype,
                    int B, int N, int V,
                    const int32_t* parent, const int32_t* node_tokens,
                    const float* u_accept, const float* u_resample,
                    float temperature,
                    int32_t* accepted_len, int32_t* out_tokens, int32_t* path_nodes,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * osd_sample -- token sampling: the draft model's proposals y ~ q
 * (Algorithm 1) and the mixed sampling y ~ beta p + (1 - beta) q that
 * Section 4.1 uses to generate distillation data (beta weights the target
 * p).  For each row n:
 *   pi_n = beta softmax(p_n / T) + (1 - beta) softmax(q_n / T)
 * and out_tokens[n] is the smallest token id j whose running sum of pi_n
 * (ascending j) exceeds u[n] * sum(pi_n) -- the inverse CDF of osd_verify's
 * extra token.  T == 0 takes the argmax (lowest index on ties) of the row
 * with weight 1.
 *
 * p_logits      [N, V] dtype rows, row n at element offset n * p_row_stride;
 *               not read (may be NULL) when beta == 0
 * q_logits      [N, V] dtype rows, row stride q_row_stride elements; not read
 *               (may be NULL) when beta == 1
 * p_row_stride, q_row_stride  elements between rows, >= V (e.g. V for
 *               [N, V], or (K+1)*V for one position of every sequence of a
 *               [B, K+1, V] tensor)
 * temperature   T > 0 samples; T == 0 needs beta == 0 or beta == 1
 * beta          in [0, 1]
 * u             [N] float uniforms in [0, 1) (unused, may be NULL, at T == 0)
 * out_tokens    out [N] int32: the token, or -1 for a row with weight > 0
 *               that has no finite logit
 *
 * workspace     NULL, or at least osd_sample_workspace_bytes(N) bytes,
 *               16-byte aligned, zero before the first call; every call
 *               leaves it zero.  Calls that may overlap (other streams) need
 *               their own.  With a workspace, one-row sampling (T > 0, beta
 *               0 or 1) of fewer rows than two per CU splits each row over
 *               several workgroups that exchange two words each through it;
 *               every other call (and every call without one) runs one
 *               workgroup per row.  The token is the same rule's either way;
 *               the two can differ only where u * sum(pi) lies within fp32
 *               rounding of a boundary between tokens.
 *
 * Errors: OSD_ERR_INVALID_ARG for N <= 0, V <= 0, a bad dtype, T < 0, inf
 * or NaN, beta outside [0, 1], T == 0 with 0 < beta < 1, a needed pointer
 * NULL or a row stride < V; OSD_ERR_UNSUPPORTED for V > osd_max_vocab(dtype);
 * OSD_ERR_WORKSPACE for a workspace that is too small or misaligned;
 * OSD_ERR_DEVICE if the launch fails.  Nothing is enqueued on an error.
 */
size_t osd_sample_workspace_bytes(int N);
int osd_sample(const void* p_logits, int64_t p_row_stride,
               const void* q_logits, int64_t q_row_stride,
               int dtype, int N, int V, float temperature, float beta,
               const float* u, int32_t* out_tokens, void* workspace, size_t workspace_bytes,
               void* stream);

/*
 * The record of a row of logits: its k largest logits, and the mass of all
 * the others.  It is what a draft model that proposes from its top logits
 * needs to hand on, and what a replay buffer keeps of the teacher in place of
 * the row (Algorithm 1 stores the target's distribution at the error index; a
 * row of 32128 bf16 logits is 64256 bytes, its record with k = 64 388).
 *
 *   ids   [k] int32  token ids, largest logit first, the lowest id first among
 *                    equal logits (zeros of both signs are equal); -1 in slots
 *                    past the row's finite logits
 *   top   [k] dtype  their logits, -inf in slots without a token
 *   rest  fp32       log(sum over the tokens outside the record of
 *                    exp((x_j - top_0) / T)), -inf if they have no mass:
 *                    relative to the first slot's logit, at a temperature T
 *
 * A row with a NaN or +inf logit, or without a finite one, has the empty
 * record: ids -1, top -inf, rest -inf.
 *
 * osd_topk -- the record of each row and, with tokens_out, a token drawn
 * from it: rank r is the smallest whose running sum of exp(top_r / T), in slot
 * order, exceeds u * their total (a proposal y ~ q with q the softmax over
 * the record; Algorithm 1's proposal step with a truncated draft).
 *
 * logits        [N, V] dtype rows, row n at element offset n * row_stride
 *               (row_stride >= V)
 * k             1 .. min(V, OSD_MAX_TOPK)
 * temperature   T > 0; or T == 0, where the token is slot 0's (the argmax)
 *               and rest_out must be NULL
 * u             [N] float uniforms in [0, 1); NULL without tokens_out or at
 *               T == 0
 * ids_out       out [N, k] int32
 * top_out       out [N, k] dtype
 * rest_out      out [N] fp32, nullable
 * tokens_out    out [N] int32, nullable; -1 for an empty record
 *
 * Errors: OSD_ERR_INVALID_ARG for sizes or k out of range, a bad dtype, T < 0,
 * inf or NaN, rest_out at T == 0, a needed pointer NULL or a row stride < V;
 * OSD_ERR_UNSUPPORTED for V > osd_max_vocab(dtype); OSD_ERR_DEVICE if the launch
 * fails.  Nothing is enqueued on an error.
 */
#define OSD_MAX_TOPK 256
int osd_topk(const void* logits, int64_t row_stride, int dtype, int N, int V, int k, float temperature,
             const float* u, int32_t* ids_out, void* top_out, float* rest_out, int32_t* tokens_out,
             void* stream);

/*
 * osd_distill_topk_loss_grad -- osd_distill_loss_grad from teacher records.
 * The record's tokens are k buckets and all other tokens one more; over these
 *   p = softmax(top_1 / tau, .., top_k / tau, rest)      (teacher)
 *   q = the student's softmax(s / tau), the others summed
 * and D is Eq. 3's divergence between p and q:
 *   FKL  KL(p || q)          gradient of token j in bucket b  q_j (1 - p_b / q_b) / tau
 *   RKL  KL(q || p)                     q_j (log(q_b / p_b) - D) / tau
 *   JSD  beta KL(p || m) + (1 - beta) KL(q || m),  m = beta p + (1 - beta) q
 *                                       (1 - beta) q_j (log(q_b / m_b) - KL(q || m)) / tau
 * (0 log 0 = 0; a token with logit -inf outside the record has gradient 0; q_j / Q is taken of the
 * logits, so FKL's gradient holds however far the others lie below the record).  With a record
 * that holds the whole row this is osd_distill_loss_grad.
 *
 * teacher_ids   [.., k] int32, teacher_top [.., k] dtype, teacher_rest [..]
 *               fp32: records as osd_topk writes them (rest at T = tau).  The
 *               record of row (b, i) is number b * teacher_batch_rows + i (pass
 *               K + 1 to distil the first K of each sequence's K + 1 target
 *               rows).  The first slot holds the largest logit.  teacher_rest
 *               NULL: the teacher is its record alone (p of the last bucket is
 *               0); RKL, infinite there, is refused
 * student_logits  row (b, i) starts at element b * student_batch_stride + i*V
 * mask, kind, beta, tau, loss_out, row_loss_out   as osd_distill_loss_grad
 * grad_out      out [B, K, V] in `dtype`, contiguous, nullable: the gradient
 *               of sum(mask * D); rows with mask 0 are written as 0.  It may be
 *               the student rows themselves (the same address, rows without
 *               gaps); any other overlap with them is refused.  Outputs must not
 *               overlap the other inputs
 * workspace     osd_distill_topk_workspace_bytes(B, K) zero-initialised bytes
 *               for this operator alone (counters among them are left zero; the
 *               rest keeps scratch that later calls need not find cleared, at any B, K, V, k)
 *
 * A row whose record is empty, names a token outside [0, V) (-1: an empty slot)
 * or one token twice, or holds a NaN or +inf, and a student row with a NaN, +inf or
 * no finite logit, gives D = NaN and a gradient of NaN.  Equal calls give equal
 * bits.
 *
 * Errors as osd_distill_loss_grad, and OSD_ERR_INVALID_ARG for k outside
 * 1 .. min(V, OSD_MAX_TOPK), teacher_batch_rows < K with B > 1, RKL without
 * teacher_rest.
 */
size_t osd_distill_topk_workspace_bytes(int B, int K);
int osd_distill_topk_loss_grad(const int32_t* teacher_ids, const void* teacher_top, const float* teacher_rest,
                               int64_t teacher_batch_rows, int k, const void* student_logits,
                               int64_t student_batch_stride, int dtype, int B, int K, int V, const uint8_t* mask,
                               int kind, float beta, float tau, float* loss_out, float* row_loss_out,
                               void* grad_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * osd_verify_topk -- osd_verify for proposals drawn from the draft's record
 * (osd_topk with the same T): q is the softmax over the record's slots and 0
 * elsewhere, p the target's over the whole row, so the emitted tokens follow
 * the target exactly although the draft is truncated.  Acceptance, first
 * rejection, correction and bonus token as osd_verify (a proposal outside its
 * record has q = 0: accepted where p > 0).
 *
 * draft_ids     [B, K, k] int32, draft_top [B, K, k] dtype: the record that
 *               proposal i was drawn from (rest is not needed)
 * temperature   T > 0 (at T == 0 the draft's probabilities play no part: use
 *               osd_verify)
 * workspace     osd_verify_topk_workspace_bytes(B, K) zero-initialised bytes
 *               for this operator alone (counters among them are left zero; the
 *               rest keeps scratch that later calls need not find cleared, at any B, K, V)
 * the others    as osd_verify
 *
 * accepted_len is -1 as in osd_verify, and where the record of a position that
 * is tested is empty, names a token outside [0, V) (-1: an empty slot) or one
 * token twice, or holds a NaN or +inf.
 *
 * Tests agree with an exact computation except where u lies within about 1e-11
 * (relative) of p(y)/q(y), draws except within about 1e-11 of probability mass of
 * an edge: where u lies near the ratio, and a draw's point near an edge, they are
 * decided in fp64.
 */
size_t osd_verify_topk_workspace_bytes(int B, int K);
int osd_verify_topk(const void* target_logits, const int32_t* draft_ids, const void* draft_top, int k, int dtype,
                    int B, int K, int V, const int32_t* draft_tokens, const int32_t* draft_len,
                    const float* u_accept, const float* u_resample, float temperature, int32_t* accepted_len,
                    int32_t* out_tokens, uint8_t* reject_mask, void* workspace, size_t workspace_bytes,
                    void* stream);

/*
 * The paged cache of keys and values, and the attention that reads it: what a
 * step of speculative decoding runs the target over its drafted tokens with.
 * The candidate tree of osd_verify_tree (or the chain of osd_verify) goes
 * through osd_cache_append and osd_tree_attention in every layer; once its
 * tokens are verified, osd_cache_keep moves the accepted path of every layer to
 * where the context ends.
 *
 * The cache of one layer is two arrays of pages of page_size tokens,
 * [pages, kv_heads, page_size, head_dim] in `dtype`, with page_stride elements
 * between pages (so that K and V may share one allocation).  A sequence's
 * tokens lie on the pages that its row of page_table names: token j on page
 * page_table[b, j / page_size], slot j % page_size.  These calls have many
 * arguments, so they take them in a struct in host memory, which they have read
 * when they return.  osd_cache is what the three share:
 *
 * k_cache, v_cache   the caches
 * page_stride        elements between pages, >= kv_heads * page_size * head_dim
 * pages, page_size   pages of the cache, tokens of a page (any number)
 * kv_heads, head_dim head_dim a multiple of 8, at most OSD_MAX_HEAD_DIM
 * page_table         [B, table_len] int32; entries behind a sequence's last
 *                    token are not looked at
 * seq_len            [B] int32: tokens of the context, c_b; -1: no sequence
 *                    (a padded batch)
 * N                  new tokens of a sequence: node n of sequence b is token
 *                    c_b + n of the cache
 *
 * and two of them the tree:
 *
 * parent             [B, N] int32 as in osd_verify_tree (node 0 is the root,
 *                    0 <= parent[n] < n), or NULL: a chain, every node's parent
 *                    the one before it.  N <= OSD_MAX_TREE_NODES with a tree
 * new_len            [B] int32 or NULL: nodes that sequence b has, n_b <= N
 *                    (NULL: N); the nodes behind are padding
 *
 * Base addresses and strides of all arrays but the int32 ones are multiples of
 * 16 bytes; a sequence's table covers at most 2^30 tokens, a batch's 2^36, and 2^35
 * for osd_tree_attention (otherwise OSD_ERR_INVALID_ARG).  Unsupported head sizes
 * and batches above OSD_MAX_CACHE_BATCH give OSD_ERR_UNSUPPORTED.  Pages that
 * several sequences name are read correctly; a page that a call writes must belong
 * to one sequence alone.  Outputs must not overlap inputs, except as said.
 */
#define OSD_MAX_HEAD_DIM 256
#define OSD_MAX_CACHE_BATCH 4096

typedef struct {
    void* k_cache;
    void* v_cache;
    int64_t page_stride;
    const int32_t* page_table;
    const int32_t* seq_len;
    int32_t pages, page_size, kv_heads, head_dim, dtype, table_len, B, N;
} osd_cache;

/*
 * osd_cache_append -- new tokens' keys and values into the pages behind the
 * context, rotated by their positions on the way, and their queries rotated
 * along with them.
 *
 * A token's position is c_b + its depth (a tree: the number of its ancestors; a
 * chain: n), so that an accepted path needs no new rotation when it moves.  The
 * first rotary_dim values of a head are taken as pairs (x, y), element i with
 * element i + rotary_dim / 2 (OSD_ROTATE_HALVES) or elements 2i and 2i + 1
 * (OSD_ROTATE_PAIRS), and become (x cos - y sin, y cos + x sin); the others, and
 * all of V, are copied.
 *
 * q             [B, N, q_heads, head_dim], q_stride elements between tokens
 *               (token (b, n) at (b * N + n) * q_stride); NULL: keys and values
 *               alone
 * q_out         out, as q with q_out_stride between tokens; q itself with the
 *               same stride, or no part of it (with another stride: apart from the
 *               first to the last of q's tokens); NULL iff q is
 * k, v          [B, N, kv_heads, head_dim], k_stride and v_stride between tokens
 * rotation      [rotation_rows, rotary_dim] fp32: for each position the cosines
 *               of its rotary_dim / 2 angles, then the sines; NULL: no rotation
 * rotary_dim    even, 2 .. head_dim (ignored without rotation)
 *
 * Nothing is written for padding but zeros in q_out.  A token that has no place
 * (its page outside the cache or the table) or no position (beyond rotation_rows,
 * an invalid tree), and all of a sequence whose n_b is outside 0 .. N, is not
 * written to the cache; its q_out is NaN.
 */
typedef enum { OSD_ROTATE_HALVES = 0, OSD_ROTATE_PAIRS = 1 } osd_rotation;
typedef struct {
    osd_cache cache;
    const void* q;
    int64_t q_stride;
    void* q_out;
    int64_t q_out_stride;
    const void* k;
    int64_t k_stride;
    const void* v;
    int64_t v_stride;
    const int32_t* parent;
    const int32_t* new_len;
    const float* rotation;
    int32_t q_heads, rotation_rows, rotary_dim, rotation_style;
} osd_append;
int osd_cache_append(const osd_append* call, void* stream);

/*
 * osd_tree_attention -- attention of the drafted tokens: node n sees the context,
 * its ancestors and itself (all of them already in the cache),
 *   out = sum_j softmax_j(scale q . k_j) v_j,   j < c_b or j = c_b + an ancestor of n or n.
 * N = 1 is the decoding of single tokens, parent = NULL that of chains.
 *
 * q             [B, N, q_heads, head_dim], q_stride elements between tokens;
 *               query head h reads kv head h / (q_heads / kv_heads)
 * scale         finite, and so as a float times log2(e), too
 * out           out [B, N, q_heads, head_dim]
 * workspace     osd_tree_attention_workspace_bytes(...) zero-initialised bytes
 *               for this operator alone (counters among them are left zero; the
 *               rest keeps scratch that later calls need not find cleared, at any
 *               sizes)
 *
 * N <= OSD_MAX_TREE_NODES.  Padding, and sequences of length -1, get zeros.  A
 * sequence that is invalid (n_b outside 0 .. N, tokens beyond its table, a page
 * outside the cache, an invalid tree) gets NaN.  What the cache holds in tokens
 * that a node does not see (NaN, too) does not reach its output; an infinite value
 * that it sees gives that infinity, or NaN where its probability is less than fp32
 * holds (beside a score about 100 larger).  Finite values give finite outputs where
 * the |v| that a row sees sum to less than 2^127.  Scores, softmax and sums are
 * fp32; for the product with bf16 values a probability is taken as two bf16
 * numbers, off by 2^-15 of itself.  Work is divided over the GPU by the lengths in
 * device memory, so a captured call serves any lengths; how it is divided, and with
 * it the last bits, depends on all of the batch.  Equal calls give equal bits.
 */
typedef struct {
    osd_cache cache;
    const void* q;
    int64_t q_stride;
    const int32_t* parent;
    const int32_t* new_len;
    void* out;
    void* workspace;
    size_t workspace_bytes;
    int32_t q_heads;
    float scale;
} osd_attention;
size_t osd_tree_attention_workspace_bytes(int B, int N, int q_heads, int kv_heads, int head_dim);
int osd_tree_attention(const osd_attention* call, void* stream);

/*
 * osd_cache_keep -- the accepted path's keys and values move to where the context
 * ends: token c_b + path_nodes[b, i] to token c_b + 1 + i, i < accepted_len[b], in
 * the caches of all layers (the root, token c_b, is in place).  A chain needs no
 * move.
 *
 * layers, layer_stride  the caches are [layers, pages, ...], layer_stride elements
 *                       between layers, which share no memory
 * path_nodes            [B, N] int32 and
 * accepted_len          [B] int32: as osd_verify_tree returns them
 * new_seq_len           out [B] int32: c_b + 1 + accepted_len[b]; no part of seq_len
 *                       or of the other int32 arrays
 *
 * Nothing moves, and new_seq_len is c_b, where accepted_len is outside 0 .. N - 1
 * (-1: an invalid tree), the path is no ascending list of nodes in 1 .. N - 1, or
 * the root or a node on the path has no place.
 */
typedef struct {
    osd_cache cache;
    int64_t layer_stride;
    const int32_t* path_nodes;
    const int32_t* accepted_len;
    int32_t* new_seq_len;
    int32_t layers, reserved;
} osd_keep;
int osd_cache_keep(const osd_keep* call, void* stream);

/*
 * Vocabulary-sharded verification.  When the target and draft LM heads are
 * split by vocabulary over G ranks (tensor parallelism), rank g holds columns
 * [v_begin_g, v_begin_g + V_g) of every logit row, and no rank sees a whole
 * row.  The verification of osd_verify (Appendix A.1, Eq. 5) then runs in
 * three phases with one exchange after each:
 *
 *   1. osd_shard_verify_stats   each rank reduces its slice of every row to an
 *                               osd_shard_row_stats record;
 *      -> all-gather of the records over the G ranks, in rank order
 *         (stats_all [G, B, K+1]);
 *   2. osd_shard_verify_mass    every rank merges the G records of each row
 *                               (identically, in rank order), takes the
 *                               acceptance tests, finds the first rejection a_b,
 *                               and sums the extra draw's mass over its own
 *                               slice of row a_b into an osd_shard_mass record;
 *      -> all-gather of those records (mass_all [G, B]);
 *   3. osd_shard_verify_draw    every rank finds which slice holds the point
 *                               u * Z of the whole row's CDF; that rank draws
 *                               the token from its slice.  Every rank writes
 *                               the same accepted_len and reject_mask and an
 *                               out_tokens row whose extra token is -1 except
 *                               on the drawing rank;
 *      -> all-reduce MAX of out_tokens gives every rank the result.
 *
 * The result is osd_verify's on the whole rows: masses are summed in exact
 * fixed point, so how the vocabulary is split changes no decision beyond the
 * fp32 rounding that osd_verify documents.  The slices must partition
 * [0, V) in rank order (v_begin_0 = 0, v_begin_{g+1} = v_begin_g + V_g).
 * Greedy verification (T == 0) needs phases 1-3 too; its phase 2 finds the
 * extra token itself (the argmax) and phase 3 draws nothing.
 *
 * Shard logits are row-major [B, K+1, V_g] (target) and [B, K, V_g] (draft),
 * each row contiguous.  Arguments shared with osd_verify (draft_tokens as
 * global ids, draft_len, u_accept, u_resample, temperature, the outputs) have
 * its meaning.  Records are 8-byte aligned device arrays owned by the caller;
 * rows past k_b are neither read nor written.  No workspace.  Errors:
 * OSD_ERR_INVALID_ARG for a bad dtype, sizes <= 0, K > OSD_MAX_K, G outside
 * 1..OSD_MAX_SHARDS, shard outside [0, G), a slice outside [0, V), T < 0 or
 * not finite, a needed NULL pointer or a misaligned record array;
 * OSD_ERR_UNSUPPORTED for V_g above 65536 (bf16) or 32768 (fp32) -- a rank
 * holds its slice in registers -- or V > 524288 (the whole row's
 * fixed-point mass must stay below 2^63); OSD_ERR_DEVICE for a failed
 * launch.  Nothing is enqueued on an error.
 */
#define OSD_MAX_SHARDS 64

/* One rank's reduction of its slice of one logit row pair (40 bytes). */
typedef struct {
    double s_target;  /* T > 0: sum over the slice of 2^(t_j log2(e)/T - k_target) */
    double s_draft;   /* T > 0: the same for the draft row (proposal rows only)   */
    float k_target;   /* T > 0: whole-number shift >= max_j t_j log2(e)/T, -inf if
                         the slice has no finite logit; T == 0: max_j t_j      */
    float k_draft;    /* T > 0: the draft row's shift                           */
    float t_y, d_y;   /* T > 0: target and draft logits of the proposal y_i when
                         this slice holds it                                   */
    int32_t argmax;   /* T == 0: global id of the slice's largest target logit
                         (lowest id on ties), -1 if the slice has none           */
    int32_t flags;    /* bit 0: the slice holds y_i; bit 1: y_i lies outside [0, V) */
} osd_shard_row_stats;

/* One rank's part of a sequence's extra draw (48 bytes). */
typedef struct {
    uint64_t z;        /* mass of max(0, p - q) (of p at the bonus row) over the
                          slice, 2^-44 fixed point in units of the target row's
                          sum of exponentials                                  */
    uint64_t z_p;      /* mass of p over the slice, same units (used should the
                          whole row's residual mass round to 0)                 */
    double s_target, s_draft;  /* merged sums of row a_b (whole row)           */
    float k_target, k_draft;   /* their shifts                                 */
    int32_t accepted;  /* a_b, or -1 for an invalid sequence                   */
    int32_t token;     /* T == 0: the extra token (global id); else -1         */
} osd_shard_mass;

int osd_shard_verify_stats(const void* target_shard, const void* draft_shard, int dtype,
                           int B, int K, int V_shard, int v_begin, int V,
                           const int32_t* draft_tokens, const int32_t* draft_len,
                           float temperature,
                           osd_shard_row_stats* stats, /* out [B, K+1] */
                           void* stream);

int osd_shard_verify_mass(const void* target_shard, const void* draft_shard, int dtype,
                          int B, int K, int V_shard, int G,
                          const int32_t* draft_tokens, const int32_t* draft_len,
                          const float* u_accept, float temperature,
                          const osd_shard_row_stats* stats_all, /* [G, B, K+1] */
                          osd_shard_mass* mass,                 /* out [B]      */
                          void* stream);

int osd_shard_verify_draw(const void* target_shard, const void* draft_shard, int dtype,
                          int B, int K, int V_shard, int v_begin, int G, int shard,
                          const int32_t* draft_tokens, const int32_t* draft_len,
                          const float* u_resample, float temperature,
                          const osd_shard_mass* mass_all,       /* [G, B] */
                          int32_t* accepted_len, int32_t* out_tokens,
                          uint8_t* reject_mask, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* OSD_H */
