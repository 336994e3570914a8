/*
 * vt.h - C boundary of the trimmed-vocabulary draft head for NVIDIA B200 (sm_100a).
 *
 * The library computes, on one GPU, the part of a speculative-decoding draft step that
 * vocabulary trimming makes cheaper: the draft model's language-modelling head restricted to
 * a kept set V_d of V_trim token rows (the paper's k = |V_d|, Section 2.1), whose cost is the
 * 2*d*k term of the paper's cost model (Section 2.3, Eq. 3).
 *
 * Conventions that hold for every entry point
 *  - "dev" pointers are device memory of the current CUDA device, "host" pointers are host
 *    memory.  The caller owns every buffer; the library allocates and frees nothing and keeps
 *    no pointer after a call returns.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Unless stated
 *    otherwise a call only enqueues work on that stream and returns without synchronising.
 *  - bf16 tensors are row-major arrays of 16-bit patterns; ids and indices are int32.
 *  - Errors are return codes.  Argument errors are detected on the host before anything is
 *    launched.  No entry point throws, aborts or traps the device.
 *  - A call must run on the device whose memory it is given; the library does not switch devices.
 */
#ifndef VT_H_
#define VT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum vt_status {
    VT_OK = 0,
    VT_ERR_NULL = 1,       /* a required pointer is NULL                                              */
    VT_ERR_SHAPE = 2,      /* d < 8, d % 8 != 0, M < 1, V_trim < 1, V_trim > V_full, k < 1, k > V_trim,
                              k > VT_MAX_K, N < 0, a size beyond what an entry point states it takes  */
    VT_ERR_ALIGN = 3,      /* a bf16 matrix pointer is not 16-byte aligned, an id pointer not 4-byte  */
    VT_ERR_RANGE = 4,      /* a keep id lies outside [0, V_full), or a page id outside [0, n_pages)    */
    VT_ERR_DUP = 5,        /* keep_ids names an id twice (V_d is a set, Section 2.1)                  */
    VT_ERR_EMPTY = 6,      /* vt_coverage with N == 0: Eq. 2 would be 0/0                             */
    VT_ERR_WORKSPACE = 7,  /* workspace NULL, misaligned (256 B) or smaller than the size function says */
    VT_ERR_TIMEOUT = 8,    /* a bounded device-side wait ran out; outputs of that call are invalid    */
    VT_ERR_CUDA = 9,       /* a CUDA runtime or driver call failed (see vt_last_cuda_error)           */
    VT_ERR_UNSUPPORTED = 10 /* the requested path cannot run this shape (only with a forced path)     */
} vt_status;

#define VT_MAX_K 64        /* largest top-k per draft row */

/* Which contraction kernel vt_draft_head_path / vt_debug_logits run. */
typedef enum vt_path {
    VT_PATH_AUTO = 0,      /* chosen from M and d                                                     */
    VT_PATH_GEMV = 1,      /* CUDA-core streaming GEMV; 4 draft rows per pass, d <= 8192              */
    VT_PATH_MMA = 2,       /* tcgen05 tensor-core GEMM, draft rows on the TMEM lanes; any M            */
    VT_PATH_MMA_SMALL = 3  /* tcgen05 tensor-core GEMM, vocabulary rows on the TMEM lanes; any M, in passes
                              of 128 draft rows; of 256 when k <= 16 and M > 96 (M > 64 where a CTA owns at
                              most 128 vocabulary rows): pairs of CTAs then share each MMA            */
} vt_path;

#define VT_PATH_MASK 0xFF  /* the vt_path part of an `options` argument */

/* Option bits for vt_draft_head_path, ORed onto the vt_path value. */
#define VT_HEAD_STATIC_WEIGHTS 0x100 /* the caller declares W_trim a constant of the model: nothing earlier in the
                                        stream writes it (see vt_draft_head).  The kernels may then request weights
                                        ahead of the stream-order dependency wait.                                 */
#define VT_HEAD_D2T_OFFSETS    0x200 /* d2t holds offsets instead of ids: target id = draft index + d2t[draft index],
                                        the form an EAGLE-3 style checkpoint stores (Section 1)                     */

/* Text for a status code (static storage). */
const char* vt_strerror(vt_status s);

/* The last CUDA error code (cudaError_t or CUresult as int) this thread's calls ran into; 0 if none. */
int vt_last_cuda_error(void);

/* ------------------------------------------------------------------------------------------
 * Head compaction (Section 2.1: the draft vocabulary V_d is the kept tokens; the head keeps
 * only their rows).
 *
 *   W_trim[i, :] = W_full[keep_ids[i], :]      for i in [0, V_trim),  a bit copy of bf16 rows
 *
 *   W_full   dev  [V_full, d] bf16 row-major, 16-byte aligned
 *   keep_ids dev  [V_trim] int32, each in [0, V_full), pairwise distinct.  This call does not check that
 *                 (vt_validate_keep_ids does, and synchronises to do so); a row whose id is out of range
 *                 is left unwritten
 *   W_trim   dev  [V_trim, d] bf16 row-major, caller-allocated, 16-byte aligned, must not
 *                 overlap W_full
 * Asynchronous.  VT_ERR_NULL / VT_ERR_SHAPE / VT_ERR_ALIGN / VT_ERR_CUDA.
 */
vt_status vt_compact_head(const void* W_full, int V_full, int d,
                          const int32_t* keep_ids, int V_trim,
                          void* W_trim, void* stream);

/* Bytes of scratch vt_validate_keep_ids and vt_coverage need for a vocabulary of V_full ids
 * (a membership bitmap plus counters).  Returns 0 if V_full < 1. */
size_t vt_coverage_workspace_bytes(int V_full);

/* Checks that keep_ids is a set inside [0, V_full) (Section 2.1).  Builds the membership
 * bitmap in `workspace` (dev, 256-byte aligned, vt_coverage_workspace_bytes(V_full)) and
 * SYNCHRONISES the stream to read two counters back.
 * Returns VT_ERR_RANGE if any id is out of range, else VT_ERR_DUP if any id repeats, else VT_OK. */
vt_status vt_validate_keep_ids(const int32_t* keep_ids, int V_trim, int V_full,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Draft head over the trimmed vocabulary (Section 2.3: the d -> k linear head, the only
 * vocabulary-dependent cost of an EAGLE-style draft; Section 1: the draft-to-target buffer).
 *
 * For each draft row m in [0, M):
 *   x[m, i]   = sum_j h[m, j] * W_trim[i, j]            fp32 accumulation of exact bf16 products
 *   lse[m]    = log sum_{i < V_trim} exp(x[m, i])       natural log, over the kept rows only
 *   the k largest x[m, :] in descending order, equal logits ordered by ascending draft index
 *   logprobs[m, j]   = x[m, i_j] - lse[m]
 *   target_ids[m, j] = d2t[i_j]                         d2t holds absolute target-vocabulary ids
 * The logits are never written to memory.
 *
 *   h          dev [M, d] bf16, 16-byte aligned          W_trim dev [V_trim, d] bf16, 16-byte aligned
 *   d2t        dev [V_trim] int32
 *   target_ids dev [M, k] int32 (out)                    logprobs dev [M, k] float (out)
 *   draft_ids  dev [M, k] int32 (out) or NULL            lse      dev [M] float (out) or NULL
 *   workspace  dev, 256-byte aligned, at least vt_workspace_bytes(M, k) bytes, zero-filled once
 *              by vt_workspace_init before its first use.  It carries per-CTA partial results,
 *              an arrival counter and a status word; calls that share a workspace must be
 *              ordered on one stream.
 * d % 8 == 0, d >= 8; 1 <= k <= min(V_trim, VT_MAX_K); any M >= 1.  Inputs must be finite.
 * Stream order: the kernels are launched with programmatic dependent launch, i.e. their CTAs may become
 *   resident while the stream's previous kernel is finishing (for this library's own head kernels: while
 *   their last rows are still being merged).  They set up shared and tensor memory and then wait for that
 *   kernel to complete before they touch h, W_trim, d2t, the workspace or the outputs, so every input may be
 *   produced by earlier work on the same stream, whatever kind of kernel produced it.
 *   vt_draft_head_path with VT_HEAD_STATIC_WEIGHTS relaxes this for W_trim only: the caller declares that
 *   nothing earlier in the stream writes W_trim (it was written once, e.g. by vt_compact_head, and the
 *   stream or device was synchronised afterwards - the usual state of model weights in a serving loop).
 *   A kernel may then request weight tiles before the wait, which hides the first memory round trip behind
 *   the previous call's tail (the CUDA-core path for one or two draft rows does; the tensor-core paths
 *   measured no gain and ignore the option).  h, d2t, the workspace and the outputs keep full stream-order
 *   semantics.
 * Asynchronous: no host synchronisation.  A device-side wait that ran out is reported by
 * vt_last_status on the same workspace; after VT_ERR_TIMEOUT run vt_workspace_init again before
 * the workspace is reused (arrival counters may be left mid-count).
 */
size_t    vt_workspace_bytes(int M, int k);
vt_status vt_workspace_init(void* workspace, size_t workspace_bytes, void* stream);

vt_status vt_draft_head(const void* h, const void* W_trim, const int32_t* d2t,
                        int M, int d, int V_trim, int k,
                        int32_t* target_ids, float* logprobs,
                        int32_t* draft_ids, float* lse,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Same call with options: `options` = a vt_path value (a forced contraction kernel returns
 * VT_ERR_UNSUPPORTED if it cannot take the shape; VT_PATH_AUTO is what vt_draft_head uses), optionally ORed
 * with VT_HEAD_STATIC_WEIGHTS and / or VT_HEAD_D2T_OFFSETS.  vt_draft_head is this call with options = 0.
 * Unknown option bits give VT_ERR_SHAPE. */
vt_status vt_draft_head_path(const void* h, const void* W_trim, const int32_t* d2t,
                             int M, int d, int V_trim, int k,
                             int32_t* target_ids, float* logprobs,
                             int32_t* draft_ids, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream, int options);

/* End-to-end form of vt_draft_head for callers whose per-step data lives on the host:
 * h_host (host [M, d] bf16, ideally pinned) is copied to the device, the head runs, and
 * target_ids_host / logprobs_host (host [M, k]) are copied back, all on `stream`; the call
 * SYNCHRONISES the stream before returning so the host outputs are valid.  W_trim and d2t
 * stay device-resident (they are model state, not per-step input).  Pinned (page-locked, mapped) output
 * buffers are written by the kernel directly; pageable ones are filled by two copies after it.  Which kind a
 * buffer is is looked up once per buffer address and thread and remembered: keep an output buffer's kind
 * for as long as its address is passed.
 * workspace: dev, vt_host_workspace_bytes(M, d, k) bytes, initialised with vt_workspace_init. */
size_t    vt_host_workspace_bytes(int M, int d, int k);
vt_status vt_draft_head_host(const void* h_host, const void* W_trim, const int32_t* d2t,
                             int M, int d, int V_trim, int k,
                             int32_t* target_ids_host, float* logprobs_host,
                             void* workspace, size_t workspace_bytes, void* stream);

/* Reads the status word of a workspace.  SYNCHRONISES the stream.  Returns VT_OK, VT_ERR_TIMEOUT, VT_ERR_RANGE (vt_tree_attention met a
 * page id outside the cache) or VT_ERR_CUDA, and clears the word. */
vt_status vt_last_status(void* workspace, void* stream);

/* ------------------------------------------------------------------------------------------
 * Feature fusion of an EAGLE-style draft (Section 2.3, component 1: the layer that projects the concatenated
 * hidden states of several target-model layers into the hidden dimension; Table 1, first row, 2 * 3d * d
 * FLOPs - part of the fixed cost F_fixed of Eq. 3, independent of the vocabulary):
 *
 *   fused[m, i] = bf16( sum_j h3[m, j] * W_fuse[i, j] )     fp32 accumulation of exact bf16 products, rounded
 *                                                           once, to nearest-even
 *
 *   h3      dev [M, d_in]  bf16, 16-byte aligned (d_in = 3d for three concatenated layers)
 *   W_fuse  dev [d_out, d_in] bf16, 16-byte aligned, row-major (one row per output feature)
 *   fused   dev [M, d_out] bf16 (out)
 *   workspace  a draft-head workspace of at least vt_workspace_bytes(M, 1) bytes (only its status word is used)
 * d_in % 8 == 0, d_in >= 8.  It runs the head's contraction kernels with an epilogue that only stores, so the
 * fixed part of a draft step can be timed on the same footing as the vocabulary-dependent part.
 * Asynchronous; stream order as for vt_draft_head. */
vt_status vt_fuse_features(const void* h3, const void* W_fuse, int M, int d_in, int d_out,
                           void* fused, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Cross-row candidate selection of a tree-style draft step (Section 1 describes the draft proposing candidate
 * tokens that the target verifies; the paper gives no formula for expanding several rows at once, so this is the
 * plain reading, stated here in full):
 *
 *   score[m, j] = parent_scores[m] + logprobs[m, j]        one fp32 addition
 *   the T largest scores over all M * k pairs, in descending order; equal scores by ascending m * k + j
 *   out_rows[t], out_slots[t] = the pair (m, j);  out_tokens[t] = target_ids[m, j];  out_scores[t] = its score
 *
 *   logprobs, target_ids  dev [M, k] (the outputs of vt_draft_head)      parent_scores  dev [M] float
 *   out_rows, out_slots, out_tokens  dev [T] int32 (out)                 out_scores     dev [T] float (out)
 * M * k <= 8192, 1 <= T <= M * k.  Asynchronous. */
vt_status vt_tree_select(const float* logprobs, const int32_t* target_ids, const float* parent_scores,
                         int M, int k, int T,
                         int32_t* out_rows, int32_t* out_slots, int32_t* out_tokens, float* out_scores,
                         void* stream);

/* ------------------------------------------------------------------------------------------
 * Token scoring: log probabilities of given tokens under a head, with entropy and the best alternatives.  The target
 * model needs it to verify what the draft proposed (over W_full), a draft to be trained on its kept vocabulary (over
 * W_trim, with the gradient below).  For each row m in [0, M):
 *
 *   x[m, v]     = sum_j h[m, j] * W[v, j]               fp32 accumulation of exact bf16 products;  z = scale * x
 *   lse[m]      = log sum_{v < V} exp(z[m, v])
 *   logprobs[m] = z[m, tokens[m]] - lse[m]
 *   entropy[m]  = -sum_v p log p,   p = exp(z - lse)
 *   top_ids[m, :], top_logprobs[m, :]   the k largest x[m, :] in descending order, equal ones by ascending id, and
 *                                       their z - lse
 * A row whose token lies outside [0, V) - a padded position, a token the trimmed vocabulary does not keep - is not
 * scored: logprobs, entropy, lse and top_logprobs are 0 and top_ids -1, whatever its hidden state holds.  With
 * tokens == NULL every row is scored and logprobs must be NULL.  (The workspace may hold logits: where k is large or the
 * rows are few, never more than 40 MB of them unless k > 20.)
 *
 *   h       dev [M, d] bf16, rows ldh elements apart (ldh >= d, a multiple of 8), 16-byte aligned
 *   W       dev [V, d] bf16, 16-byte aligned              tokens dev [M] int32 or NULL
 *   logprobs, entropy, lse  dev [M] float (out), each may be NULL
 *   top_ids, top_logprobs   dev [M, k] int32, float (out); ignored when k == 0
 *   workspace  dev, 256-byte aligned, vt_score_workspace_bytes(M, d, V, k) bytes; it needs no initialisation except for
 *              vt_last_status, which reads a status word that vt_workspace_init clears
 * d % 8 == 0, d >= 8, 0 <= k <= min(V, VT_MAX_K), scale finite and > 0, else VT_ERR_SHAPE; any M >= 1.  Inputs must be
 * finite in the rows that are scored, and x and z there finite in fp32 and, within a row, no further apart than 2e38; a NaN stays in
 * its row.  Asynchronous; results do not depend on timing. */
size_t    vt_score_workspace_bytes(int M, int d, int V, int k);
vt_status vt_score_tokens(const void* h, int64_t ldh, const void* W, const int32_t* tokens,
                          int M, int d, int V, float scale, int k,
                          float* logprobs, float* entropy, float* lse, int32_t* top_ids, float* top_logprobs,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Gradient of vt_score_tokens.  With upstream gradients gl of the log probability and ge of the entropy:
 *
 *   G[m, v]      = scale * ( gl[m] * (1[v == tokens[m]] - p) - ge[m] * p * (log p + entropy[m]) )
 *   grad_h[m, :] = sum_v G[m, v] * W[v, :]        grad_W[v, :] = sum_m G[m, v] * h[m, :]
 *
 * p comes from the logits, multiplied out again, and lse; G is rounded once to bf16 (it is an operand of both products; what
 * that takes from the given tokens' entries, its largest, is added to the sums), the sums are fp32 and rounded once to
 * bf16.  A row that is not scored has G = 0 and adds nothing to grad_W.
 *
 *   h, ldh, W, tokens, M, d, V, scale   as in the forward call (tokens required);   lse, entropy  dev [M], its outputs
 *   grad_logprobs  dev [M] float        grad_entropy  dev [M] float or NULL (then entropy may be NULL, too)
 *   grad_h  dev [M, d] bf16 (out) or NULL      grad_W  dev [V, d] bf16 (out) or NULL; at least one; 16-byte aligned
 *   workspace  dev, 256-byte aligned, vt_score_backward_workspace_bytes(M, d, V) bytes (it holds G, 2 M V bytes, and 6 M d + 8 V
 *              more)
 * Asynchronous.  Gradients are overwritten, not added to. */
size_t    vt_score_backward_workspace_bytes(int M, int d, int V);
vt_status vt_score_tokens_backward(const void* h, int64_t ldh, const void* W, const int32_t* tokens,
                                   const float* lse, const float* entropy,
                                   const float* grad_logprobs, const float* grad_entropy,
                                   int M, int d, int V, float scale, void* grad_h, void* grad_W,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Gated feed-forward block of a draft layer (Table 1, the feed-forward row of the fixed cost F_fixed of Eq. 3):
 *
 *   g = x W_gate^T     u = x W_up^T     a = act(g) * u     y = a W_down^T
 *
 * fp32 accumulation throughout; a is rounded once to bf16 (it is an operand of the second product), y once to bf16.
 *
 *   x       dev [M, d] bf16, rows ldx elements apart (ldx >= d, a multiple of 8)
 *   W_gate, W_up  dev [f, d] bf16       W_down  dev [d, f] bf16       y  dev [M, d] bf16 (out)
 *   saved   dev 2 M f floats (out) or NULL: g and u for the backward pass, in fp32, in a layout of the library's own
 *   workspace  dev, 256-byte aligned, vt_gated_ffn_workspace_bytes(M, d, f) bytes; no initialisation needed (see above)
 * All matrices 16-byte aligned.  d % 8 == 0, f % 8 == 0, both >= 8, any M >= 1; act a vt_act.  Asynchronous. */
typedef enum vt_act {
    VT_ACT_SILU = 0,       /* g / (1 + e^-g)                                                 */
    VT_ACT_GELU = 1        /* g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2               */
} vt_act;

size_t    vt_gated_ffn_workspace_bytes(int M, int d, int f);
vt_status vt_gated_ffn(const void* x, int64_t ldx, const void* W_gate, const void* W_up, const void* W_down,
                       int M, int d, int f, int act, void* y, float* saved,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Backward pass of vt_gated_ffn, from its `saved`:
 *
 *   da = grad_y W_down      du = da act(g)      dg = da u act'(g)         (fp32; a, dg and du each rounded once to bf16)
 *   grad_x = dg W_gate + du W_up      grad_W_gate = dg^T x      grad_W_up = du^T x      grad_W_down = grad_y^T a
 *
 *   grad_y  dev [M, d] bf16, rows ld_grad_y elements apart (>= d, a multiple of 8)
 *   grad_x [M, d], grad_W_gate, grad_W_up [f, d], grad_W_down [d, f]  dev bf16 (out), each may be NULL, not all
 *   workspace  dev, 256-byte aligned, vt_gated_ffn_backward_workspace_bytes(M, d, f) bytes
 * Asynchronous.  Gradients are overwritten, not added to. */
size_t    vt_gated_ffn_backward_workspace_bytes(int M, int d, int f);
vt_status vt_gated_ffn_backward(const void* x, int64_t ldx, const void* W_gate, const void* W_up, const void* W_down,
                                const float* saved, const void* grad_y, int64_t ld_grad_y,
                                int M, int d, int f, int act,
                                void* grad_x, void* grad_W_gate, void* grad_W_up, void* grad_W_down,
                                void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Rotary positions (the attention of a draft layer, Table 1): each pair of a head's first rot_dim elements is turned by an angle
 * that grows with the token's position,
 *
 *   angle[n, i] = positions[n] * w_i          y1 = a (x1 cos - x2 sin)     y2 = a (x2 cos + x1 sin)       i < rot_dim / 2
 *
 * pair i being elements (i, i + rot_dim / 2) of a head, or (2 i, 2 i + 1) with VT_ROPE_INTERLEAVED; the other elements are
 * copied.  The gradient's way back is the turn by the opposite angle (VT_ROPE_INVERSE; `a` stays).  Sums in fp32, rounded once.
 *
 * vt_rope_table writes the frequencies, as fractions of a turn per position in 64-bit fixed point: position * entry modulo 2^64 is
 * then the angle without its whole turns, exactly, so that far positions are as good as near ones.  With base^(-2 i / rot_dim) = f_i:
 *
 *   VT_ROPE_NONE        w_i = f_i
 *   VT_ROPE_LINEAR      w_i = f_i / factor
 *   VT_ROPE_BASE        w_i = (base * factor^(rot_dim / (rot_dim - 2)))^(-2 i / rot_dim)
 *   VT_ROPE_WAVELENGTH  w_i = f_i s + f_i / factor (1 - s),  s = (turns - low) / (high - low) within [0, 1],
 *                       turns = original_len f_i / (2 pi)
 *   VT_ROPE_RAMP        w_i = f_i (1 - s) + f_i / factor s,  s = (i - i0) / (i1 - i0) within [0, 1],
 *                       i0 = floor(e(high)), i1 = ceil(e(low)) within [0, rot_dim - 1],
 *                       e(turns) = rot_dim log(original_len / (2 pi turns)) / (2 log base): the pair that makes so many turns
 *                       (its usual amplitude is a = 0.1 log(factor) + 1, and 1 for factors up to 1)
 *
 *   table  dev [rot_dim / 2] uint64 (out), 8-byte aligned
 * rot_dim a multiple of 16, 16 <= rot_dim <= 1024; base > 1, factor > 0, original_len > 0 and finite; low < high for WAVELENGTH,
 * 0 < low < high for RAMP; else VT_ERR_SHAPE.  Asynchronous. */
typedef enum vt_rope_scaling {
    VT_ROPE_NONE = 0,
    VT_ROPE_LINEAR = 1,
    VT_ROPE_BASE = 2,
    VT_ROPE_WAVELENGTH = 3,
    VT_ROPE_RAMP = 4
} vt_rope_scaling;

#define VT_ROPE_INTERLEAVED 1  /* pairs side by side */
#define VT_ROPE_INVERSE     2  /* turn back: the gradient of the call without it */

vt_status vt_rope_table(uint64_t* table, int rot_dim, double base, int scaling, double factor, double low, double high,
                        double original_len, void* stream);

/* A [tokens, heads, D] bf16 tensor: element (n, h, j) at ptr[n * token_stride + h * head_stride + j].  ptr 16-byte aligned, strides
 * multiples of 8. */
typedef struct vt_heads {
    void* ptr;
    int64_t token_stride, head_stride;
} vt_heads;

/* Turns q [N, Hq, D] into q_out and k [N, Hkv, D] into k_out (k, k_out NULL and Hkv = 0: queries alone).
 *   positions dev [N] int32 (any value)     table as above     amplitude: a, finite     options: VT_ROPE_* bits
 * Outputs may be the inputs themselves (same pointer and strides); otherwise they must not overlap them.
 * D a multiple of 16, rot_dim <= D <= 1024; N >= 0, Hq >= 1.  Asynchronous. */
vt_status vt_rope(const vt_heads* q, const vt_heads* k, const int32_t* positions, const uint64_t* table, int N, int Hq, int Hkv, int D,
                  int rot_dim, float amplitude, int options, const vt_heads* q_out, const vt_heads* k_out, void* stream);

/* ------------------------------------------------------------------------------------------
 * A paged cache of keys and values.  Page p, place i, head h, element j of the keys lies at
 * k[p * k_page_stride + i * k_token_stride + h * k_head_stride + j] (the values alike); position `at` of request b is place
 * at % page_size of page page_table[b * table_stride + at / page_size].  lens[b] positions of request b hold earlier tokens; the
 * tokens of a call are its positions lens[b], lens[b] + 1, ...
 *
 *   k, v        dev bf16, 16-byte aligned, strides multiples of 8 (elements)
 *   page_table  dev [B, max_pages] int32, rows table_stride apart        lens  dev [B] int32
 * page_size 8, 16, 32, 64 or a multiple of 128.  Neither the table nor the lengths are read before the stream's earlier work is done,
 * so both may be written by it. */
typedef struct vt_cache {
    void* k;
    void* v;
    const int32_t* page_table;
    const int32_t* lens;
    int64_t k_page_stride, k_token_stride, k_head_stride;
    int64_t v_page_stride, v_token_stride, v_head_stride;
    int64_t table_stride;
    int32_t n_pages, page_size, heads, head_dim, B, max_pages;
} vt_cache;

/* vt_rope for serving: queries are turned into q_out, keys are turned and stored in the cache, values [N, Hkv, D] are stored beside them.
 * Token n belongs to the request b with cu_tokens[b] <= n < cu_tokens[b + 1] and goes to position lens[b] + n - cu_tokens[b]; lens
 * itself stays as it is.
 *   cu_tokens  dev [B + 1] int32, ascending, within [0, N] (below 0 counts as 0)
 *   positions  dev [N] int32: what the angles go by (in a tree the depth, not the place)
 * Tokens outside [cu_tokens[0], cu_tokens[B]) are padding: nothing of theirs is written.  A token whose position lies past the table, or
 * whose page id lies outside [0, n_pages), is not stored (its query is still turned).  Asynchronous. */
vt_status vt_rope_append(const vt_heads* q, const vt_heads* k, const vt_heads* v, const int32_t* positions, const int32_t* cu_tokens,
                         const uint64_t* table, int N, int Hq, int rot_dim, float amplitude, int options, const vt_heads* q_out,
                         const vt_cache* cache, void* stream);

/* ------------------------------------------------------------------------------------------
 * Attention of drafted tokens over a paged cache that holds them at its end (their keys and values stored by vt_rope_append).  A
 * request's tokens may be a tree (mask), a chain (mask NULL: each sees itself and those before it), or one alone.  For token t of
 * request b, head h, and the positions i it attends - all i < lens[b], and lens[b] + u where bit u % 32 of word u / 32 of its mask row is
 * set (mask NULL: where u <= t) -
 *
 *   x_i = scale * q . k_i      lse = log sum_i exp(x_i)      out = sum_i exp(x_i - lse) v_i
 *
 * query head h reads key head h / (Hq / heads).  A token that attends nothing has out = 0 and lse = -infinity.  Keys and values of
 * positions that nobody attends, behind a request's end or out of every token's mask, may hold anything; where only some tokens attend one, the
 * others are not touched by it, but for those its value must be finite (infinities and NaN act as the largest finite number).  Queries of
 * requests, attended keys and values, their products q . k_i and the scores x_i must be finite, scores and scale below 2^127.  Products are
 * exact, sums fp32; the weights exp(x_i - m) are rounded to bf16 as an operand of the second product (not in lse), out once to bf16.
 *
 *   q        [N, Hq, D] as vt_heads                     out      [N, Hq, D] as vt_heads (out)      lse  dev [N, Hq] float (out) or NULL
 *   cu_tokens  dev [B + 1] int32, ascending, within [0, N]; rows outside all requests are left as they were
 *   mask     dev [N, mask_words] int32 or NULL; tokens from 32 * mask_words on are attended by nobody
 *   max_tokens  the most tokens a request has (a bound; what a request has beyond it is not computed and not attended)
 *   workspace   dev, 256-byte aligned, vt_tree_attention_workspace_bytes(Hq, heads, D, max_tokens) bytes; needs no initialisation but for
 *               vt_last_status (below).  Calls that share one must be ordered on one stream
 * D (the cache's head_dim) 64 or 128; Hq a multiple of heads, Hq / heads <= 128; max_tokens >= 1; scale finite and > 0; 0 <= N.
 * Positions past the table's max_pages pages are not attended.  A page id outside [0, n_pages) reads as keys and values of zeros and is reported
 * by vt_last_status as VT_ERR_RANGE.  Asynchronous; results do not depend on timing. */
size_t    vt_tree_attention_workspace_bytes(int Hq, int heads, int D, int max_tokens);
vt_status vt_tree_attention(const vt_heads* q, const int32_t* cu_tokens, const vt_cache* cache, const int32_t* mask, int mask_words,
                            int N, int Hq, int max_tokens, float scale, const vt_heads* out, float* lse,
                            void* workspace, size_t workspace_bytes, void* stream);

/* The mask and the positions of drafted trees from their parents: parents[n] is the index, within its request, of the token that
 * token n follows (an earlier one), or -1.  A token's mask row has the bits of itself and of all tokens on its way up; its depth is the
 * number of those above it.
 *   parents dev [N] int32        mask dev [N, mask_words] int32 (out) or NULL        positions dev [N] int32 (out) or NULL:
 *   lens[b] + depth (lens NULL: the depth)                cu_tokens dev [B + 1] int32, ascending, within [0, N] (below 0 counts as 0)
 * A parent that is not an earlier token of the request counts as -1.  Bits from 32 * mask_words on are dropped; rows outside all requests
 * are left as they were.  mask_words >= 1 where there is a mask.  Asynchronous. */
vt_status vt_tree_mask(const int32_t* parents, const int32_t* cu_tokens, const int32_t* lens, int N, int B, int32_t* mask, int mask_words,
                       int32_t* positions, void* stream);

/* ------------------------------------------------------------------------------------------
 * Verification of drafted tokens: which of a request's drafted tree stay, and the token that follows them, distributed exactly as if the
 * target had generated them alone.  Token 0 of a request is its root (already certain); probs[n, :] is the target's distribution
 * of what follows token n.  From the root on, at token x with p = probs[x]:
 *
 *   the children c of x are taken in ascending order; c is accepted if   u_accept[c] * q(c) * Z < r(c)   and r(c) > 0, and becomes x;
 *   otherwise what is left of p changes:
 *     drawn    (draft_probs given: the children of x were drawn from q = draft_probs[x], each alone)
 *              S += Z;  r(v) = max(p(v) - S q(v), 0);  Z = sum_v r(v)                    (S = 0, Z = 1, r = p at first)
 *     chosen   (draft_probs NULL: they were picked without chance; q(c) = 1)
 *              Z -= r(c);  r(c) = 0
 *   with no child left, the token that follows is the smallest v with  sum_{w <= v} r(w) > u_sample[b] * sum_w r(w).
 *
 * All of it in 64 bits.  (Where rounding leaves no r at all, p itself is drawn from.)
 *
 *   probs       dev [N, V] float, rows ld_probs apart     tokens  dev [N] int32: ids in the target's vocabulary
 *   parents     dev [N] int32: index within the request   cu_tokens  dev [B + 1] int32, ascending, within [0, N]
 *   u_accept    dev [N] float in [0, 1)                   u_sample   dev [B] float in [0, 1)
 *   draft_probs dev [N, Vd] float or NULL, rows ld_draft apart        draft_ids  dev [N] int32: tokens as draft indices (what d2t maps to tokens[n])
 *   d2t         dev [Vd] int32: the draft-to-target map, distinct ids (NULL: a draft index is the target's id)
 *   n_accepted  dev [B] int32 (out)       path  dev [B, max_tokens] int32 (out): the accepted tokens' indices within the request, then -1
 *   out_tokens  dev [B, max_tokens] int32 (out): the accepted tokens, the one that follows them, then -1
 * A token whose parent is not an earlier one of its request, or whose token or draft index lies outside its vocabulary, is left out, with all
 * that hangs on it.  A request without tokens accepts 0 and has -1 everywhere; one with more than max_tokens loses those past it.
 * Negative and NaN probabilities count as 0; a row without any positive entry gives -1 as the token that follows.
 * 1 <= max_tokens <= 1024; V <= 4194304, with draft_probs V <= 393216; Vd >= 1.  Asynchronous; results do not depend on timing. */
vt_status vt_verify_tokens(const float* probs, int64_t ld_probs, const int32_t* tokens, const int32_t* parents, const int32_t* cu_tokens,
                           const float* u_accept, const float* u_sample, const float* draft_probs, int64_t ld_draft,
                           const int32_t* draft_ids, const int32_t* d2t, int N, int B, int V, int Vd, int max_tokens,
                           int32_t* n_accepted, int32_t* path, int32_t* out_tokens, void* stream);

/* ------------------------------------------------------------------------------------------
 * Coverage of a token stream by the kept set (Eq. 2 with f(v) = occurrences of v in the
 * stream; the "frequency coverage" of Table 4):
 *
 *   covered = #{ t in [0, N) : token_ids[t] in keep_ids },   fraction = covered / N
 *
 *   token_ids dev [N] int32; ids outside [0, V_full) count in N and are never covered
 *   keep_ids  dev [V_trim] int32 in [0, V_full) (out-of-range entries are ignored)
 *   covered_out, fraction_out: host (either may be NULL)
 *   workspace dev, 256-byte aligned, vt_coverage_workspace_bytes(V_full) bytes; contents are
 *             overwritten, no initialisation needed
 * SYNCHRONISES the stream once to return the count.  N == 0 gives VT_ERR_EMPTY.
 */
vt_status vt_coverage(const int32_t* token_ids, int64_t N,
                      const int32_t* keep_ids, int V_trim, int V_full,
                      uint64_t* covered_out, double* fraction_out,
                      void* workspace, size_t workspace_bytes, void* stream);

/* The same count (Eq. 2) in two steps, for callers that must not synchronise where the work is enqueued:
 * vt_coverage_enqueue puts the bitmap build and the count on the stream and returns at once (same arguments and
 * errors as vt_coverage, minus the outputs); vt_coverage_result SYNCHRONISES the stream and reads the count
 * that the last enqueue on this workspace left in it (N = that call's N, for the fraction). */
vt_status vt_coverage_enqueue(const int32_t* token_ids, int64_t N,
                              const int32_t* keep_ids, int V_trim, int V_full,
                              void* workspace, size_t workspace_bytes, void* stream);
vt_status vt_coverage_result(void* workspace, int64_t N,
                             uint64_t* covered_out, double* fraction_out, void* stream);

/* ------------------------------------------------------------------------------------------
 * Vocabulary-size selection (the paper's method, Sections 2.1-2.5), as an exhaustive scan over k:
 *
 *   f(v)  = occurrences of id v in token_ids (the stream is taken as already restricted to assistant
 *           tokens, Section 2.2); ids outside [0, V_full) are ignored
 *   order = ids by (f descending, id ascending)                     top-k most frequent, Section 2.1
 *   C(k)  = (sum of the k largest f) / (sum of all f)               Eq. 2
 *   R(k)  = 1 - (F_fixed + 2 d k) / (F_fixed + 2 d V_full)          Eq. 3
 *   U(k)  = alpha C(k) + (1 - alpha) R(k);  U~(k) = U(k) if C(k) >= c_min, else -1       Eq. 4, 5
 *   k*    = argmax of U~(k) over k_min <= k <= k_max, the smallest k among equal maxima   Eq. 1
 *
 * The paper searches k with 100 trials of a TPE optimiser; every k is evaluated here, which gives the exact
 * optimum of the same objective.  All arithmetic is IEEE double without fused multiply-add.
 *
 *   token_ids  dev [N] int32            ranked_ids dev [V_full] int32 (out): ranked_ids[:k*] is the draft
 *                                       vocabulary, i.e. keep_ids / d2t for the calls above
 *   cum_counts dev [V_full] uint64 (out) or NULL: cum_counts[k-1] = occurrences covered by the top k
 *   k_star     host (out);  C_star, R_star, U_star  host (out), each may be NULL
 *   unique_star host (out) or NULL: of the distinct ids that occur in the stream, the fraction that the top k*
 *              keeps (the "unique coverage" Table 4 reports beside Eq. 2's frequency-weighted coverage)
 *   workspace  dev, 256-byte aligned, vt_select_workspace_bytes(V_full); contents are overwritten
 * 1 <= k_min <= k_max <= V_full, 0 <= alpha <= 1, F_fixed >= 0, d >= 1, N < 2^32 (frequencies are counted in
 * 32 bits; a longer stream gives VT_ERR_SHAPE).  SYNCHRONISES the stream.
 * VT_ERR_EMPTY if N == 0 or no id falls inside [0, V_full). */
size_t    vt_select_workspace_bytes(int V_full);
vt_status vt_select_vocab(const int32_t* token_ids, int64_t N, int V_full, int d, double F_fixed,
                          double alpha, double c_min, int k_min, int k_max,
                          int32_t* ranked_ids, uint64_t* cum_counts,
                          int* k_star, double* C_star, double* R_star, double* U_star, double* unique_star,
                          void* workspace, size_t workspace_bytes, void* stream);

/* vt_coverage for callers that must not allocate device memory.  (The paper has no counterpart: this
 * entry point exists for integration, not for the method.)
 *
 * Who needs it: code that runs inside someone else's serving loop - an engine plugin that is handed a
 * stream and device pointers but does not own an allocator, or a process whose memory pool has been
 * reserved up front so that a late cudaMalloc would either fail or stall every stream on the device
 * while it runs.  vt_coverage asks such a caller for a scratch buffer it cannot provide; this variant
 * keeps the membership bitmap and the counters in a fixed array inside the library instead, and makes
 * no cudaMalloc / cudaFree call of its own.
 *
 * Same arguments, results and errors as vt_coverage, minus the workspace, with these differences:
 *  - V_full may be at most 262,144 (the built-in bitmap is 32 KiB; with its counters the array takes
 *    33,024 bytes on every device that loads the library, until the process ends).  A larger V_full
 *    returns VT_ERR_SHAPE and launches nothing.
 *  - The first call on a device looks up the array's device address and remembers it.
 *  - Every call ends by synchronising the stream to read the count back, so it cannot be part of a stream
 *    capture at all (neither can vt_coverage).
 *  - All calls on a device share the one array.  Each call clears it before use, so results do not
 *    depend on earlier calls, but two calls whose GPU work can overlap (different streams, different
 *    host threads) race on it: keep them ordered.
 * SYNCHRONISES the stream once to return the count, like vt_coverage. */
vt_status vt_coverage_static(const int32_t* token_ids, int64_t N,
                             const int32_t* keep_ids, int V_trim, int V_full,
                             uint64_t* covered_out, double* fraction_out, void* stream);

/* ------------------------------------------------------------------------------------------
 * Test and inspection entry points (same kernels as the calls above).
 */

/* The head contraction alone (Section 2.3), with the epilogue storing x[m, i] as fp32:
 * logits dev [M, V_trim] row-major (out).  Runs the same contraction code as vt_draft_head
 * on the chosen path; workspace as for vt_draft_head with k = 2 (vt_workspace_bytes(M, 2)). */
vt_status vt_debug_logits(const void* h, const void* W_trim, int M, int d, int V_trim,
                          float* logits, void* workspace, size_t workspace_bytes,
                          void* stream, int path);

/* The draft-to-target map alone (Section 1): target_ids[t] = d2t[draft_ids[t]] for t < n.
 * A draft id outside [0, V_trim) writes -1.  All pointers dev. */
vt_status vt_remap(const int32_t* draft_ids, const int32_t* d2t, int64_t n, int V_trim,
                   int32_t* target_ids, void* stream);

/* The two index buffers an EAGLE-3 style draft stores with its weights (the draft-to-target and the
 * target-to-draft map of Section 1), derived from keep_ids:
 *   d2t_offsets[i] = keep_ids[i] - i        (target id = draft index + offset), dev [V_trim] int32 or NULL
 *   t2d_mask[v]    = 1 if v is kept else 0,                                      dev [V_full] uint8 or NULL
 * At least one output must be given.  The head calls above take absolute ids (keep_ids itself as d2t) unless
 * VT_HEAD_D2T_OFFSETS is set, in which case they take the d2t_offsets this call writes.  Asynchronous. */
vt_status vt_vocab_maps(const int32_t* keep_ids, int V_trim, int V_full,
                        int32_t* d2t_offsets, uint8_t* t2d_mask, void* stream);

/* Number of kernels the last call of this thread launched (for launch accounting). */
int vt_last_launch_count(void);

/* Failure-path probe: one tiny kernel posts an mbarrier transaction that no copy will ever complete and
 * waits on it with the same bounded wait the head kernels use, limited to `limit_us` microseconds
 * (1 .. 1,000,000).  When the limit runs out it sets the time-out bit in the workspace's status word and
 * exits normally - nothing is in flight, nothing faults - so vt_last_status(workspace) then reports
 * VT_ERR_TIMEOUT, exactly as after a head call whose wait ran out.  workspace: a draft-head workspace.
 * Asynchronous. */
vt_status vt_test_timeout_probe(void* workspace, int limit_us, void* stream);

/* Failure path of the scoring and feed-forward products: until the calling thread passes 0 again, each of its products counts on
 * 16 bytes more than its copies bring and gives up waiting after `limit_us` microseconds (1 .. 100,000).  The product then
 * lets what is in flight end, sets the time-out bit in its workspace's status word and returns without a valid result, as after a copy
 * that never came; the call's other kernels run on what is there.  Nothing faults, and every wait is bounded. */
vt_status vt_test_withhold_copies(int limit_us);

/* The forms that the scoring and feed-forward products launched by the calling thread took since the last time this was asked, at
 * most `max` and 16: five ints each - CTA pairs (1) or single CTAs, accumulator columns of a tile, CTAs that divide a tile's sum,
 * tiles (scoring: runs of tiles), and how many of these the grid takes at once.  Returns their number and forgets them (out ==
 * NULL: only forgets). */
int vt_test_products(int* out, int max);

/* Stream-order probe: a kernel that releases its programmatic dependents at once, idles for `delay_us`
 * microseconds (0 .. 10,000) and only then copies n_bytes (a multiple of 16; dev pointers, 16-byte aligned)
 * from src to dst.  A head call enqueued right behind it must still see the copied bytes. Asynchronous. */
vt_status vt_test_late_copy(void* dst, const void* src, size_t n_bytes, int delay_us, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VT_H_ */
