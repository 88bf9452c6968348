/*
 * coreinfer.h -- C ABI of libcoreinfer.so: the data-parallel hot path of
 * CoreInfer (arXiv 2410.18311) for one AMD MI355X (gfx950).
 *
 * The path has two halves.
 *   Prefill (once per sentence and FFN layer): the dense FFN produces the
 *   activation matrix A (one row per prompt token); coreinfer_select turns it
 *   into the sentence-wise core neuron set S (Sec. 3.1, Def. 1-2, Eq. 1-3);
 *   coreinfer_compact gathers the weights of S into contiguous buffers
 *   (Sec. 5.3, "deploying the necessary neurons during pre-filling").
 *   Decode (every generated token): coreinfer_ffn_decode runs the FFN over
 *   the frozen set S only (Sec. 4.1 stability-guided prediction; Sec. 4.2).
 *
 * Conventions, valid for every entry point unless stated otherwise:
 *   - Every tensor pointer is a DEVICE pointer owned by the caller.  The
 *     library allocates and frees nothing; scratch memory is the caller's
 *     workspace, sized by the matching *_workspace_size query (a pure host
 *     function that needs no GPU).  Two exceptions are static device memory
 *     that the library holds on every GPU it runs on until the process ends:
 *     the array of coreinfer_ffn_decode_static, and 4 MiB for the decode of
 *     small layers (see coreinfer_ffn_decode).  Inputs are never modified.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     All work is enqueued on it; no call synchronises the device, so outputs
 *     are valid only after the caller synchronises the stream.
 *   - Arguments are validated on the host before any HIP call.  The return
 *     value is CI_OK (0) or a negative ci_status; coreinfer_strerror names it.
 *     No exception crosses the boundary.
 *   - Matrices are row-major and dense (leading dimension = row length) unless
 *     an `ld` argument says otherwise.  Weights use the nn.Linear convention of
 *     the models the paper runs: w_up, w_gate are [N, d]; w_down is [d, N]
 *     (CI_DOWN_OUT_MAJOR) or its transpose [N, d] (CI_DOWN_NEURON_MAJOR).
 *   - d = d_model, N = d_ff (neurons per layer), M = prompt tokens,
 *     K = |S|, B = sentences decoded together.
 *   - Element types: CI_F32, CI_F16 (IEEE half), CI_BF16.  Every sum is
 *     accumulated in fp32.  The decode entry points and the scores A handed
 *     to the selection keep the hidden activations in fp32 (Sec. 5, "Models":
 *     fp16 parameters, fp32 intermediate activations); the two places that
 *     round them to the element type say so (the Y of coreinfer_ffn_dense for
 *     M > 4, and the H of coreinfer_ffn_dense_hidden).
 *   - Pointers must be 16-byte aligned, and d must be a multiple of
 *     16 / sizeof(element) (8 for 16-bit types, 4 for fp32); otherwise
 *     CI_ERR_BAD_LAYOUT.
 *   - Calls are deterministic: the same bits in give the same bits out.
 */
#ifndef COREINFER_H_
#define COREINFER_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CI_OK = 0,
  CI_ERR_INVALID_ARG = -1, /* null pointer, size out of range, fraction outside (0,1] */
  CI_ERR_BAD_DTYPE = -2,   /* dtype / activation enum not recognised               */
  CI_ERR_BAD_LAYOUT = -3,  /* alignment, leading dimension or layout enum          */
  CI_ERR_WORKSPACE = -4,   /* workspace null or smaller than the query says        */
  CI_ERR_HIP = -5,         /* a HIP runtime call or kernel launch failed           */
  CI_ERR_UNSUPPORTED = -6  /* valid request that this build does not implement     */
} ci_status;

typedef enum { CI_F32 = 0, CI_F16 = 1, CI_BF16 = 2 } ci_dtype;
typedef enum { CI_ACT_RELU = 0, CI_ACT_SWIGLU = 1 } ci_act;
typedef enum { CI_DOWN_OUT_MAJOR = 0, CI_DOWN_NEURON_MAJOR = 1 } ci_down_layout;

/* Upper limits accepted by the entry points. */
#define CI_MAX_TOKENS 65535     /* M: counts fit 16 bits                */
#define CI_MAX_NEURONS 1048576  /* N                                   */
#define CI_MAX_DMODEL 32768     /* d                                   */
#define CI_MAX_UNION_SENTENCES 8 /* sentences of a union-batched decode */

/* Human-readable name of a status code (static storage, never NULL). */
const char* coreinfer_strerror(int status);

/* Library ABI version (increases when a signature changes). */
int coreinfer_version(void);

/*
 * Size of "the top `frac` share of n items", the rule every selection below
 * uses: k = ceil(q * n / 10^6) with q = floor(frac * 10^6 + 0.5), in integer
 * arithmetic (Def. 1 and Def. 2 leave the rounding open; this is the smallest
 * set that covers at least the fraction).  Host-only, needs no GPU; lets the
 * caller size core_idx without a device round trip.
 * frac outside (0, 1] (or below 1e-6), n < 0 or k == NULL: CI_ERR_INVALID_ARG.
 */
int coreinfer_keep_count(double frac, int64_t n, int64_t* k);

/*
 * Sentence-wise core neuron selection for one FFN layer of one sentence
 * (Sec. 3.1; Fig. 1 "top-k selection ... top-k commonly activated").
 *
 *   act      [M, N] fp32, row stride ld >= N elements: A, the activation of
 *            every neuron for every prompt token (ReLU output, or
 *            |SiLU(gate)*up| for gated FFNs).
 *   step 1   (Def. 1 / Eq. 1) per token m: P = #{a > 0};
 *            C_m = the keep_count(alpha, P) largest positive entries,
 *            equal values resolved towards the lower neuron index.
 *            NaN and values <= 0 are never selected.
 *   step 2   (Eq. 3) counts[n] = #{m : n in C_m}.
 *   step 3   (Def. 2 / Eq. 2) S = the K = keep_count(beta, N) neurons that
 *            come first in the order (count descending, index ascending).
 *   core_idx [K] int32 out: S in ascending index order.
 *   counts   [N] int32 out, may be NULL (then it lives in the workspace).
 *   ws       coreinfer_select_workspace_size(M, N) bytes.  For N <= 40960 the
 *            last min(M, 512) * N of them (N rounded up to 4096) let long
 *            prompts read their activations once instead of twice; a workspace
 *            without them is accepted too, with the same results.
 * Limits: 1 <= M <= CI_MAX_TOKENS, 1 <= N <= CI_MAX_NEURONS.
 */
int coreinfer_select_workspace_size(int64_t M, int64_t N, size_t* bytes);
int coreinfer_select(const float* act, int64_t M, int64_t N, int64_t ld,
                     double alpha, double beta,
                     int32_t* core_idx, int32_t* counts,
                     void* ws, size_t ws_bytes, void* stream);

/*
 * The same selection for B sentences at once (independent sentences batched,
 * each with its own core set): sentence b is rows [b M, (b + 1) M) of
 * act [B M, N]; core_idx [B, K] and counts [B, N] (may be NULL) hold its
 * results, exactly those of coreinfer_select on its rows.  One set of launches
 * serves all sentences where Def. 2 runs in parallel (M < 2048 and
 * N <= 65536); otherwise the sentences are taken one after the other.
 * ws: at least coreinfer_select_batch_workspace_size(B, M, N) bytes.
 * Limits: 1 <= B <= 65535, B * M <= CI_MAX_TOKENS * 64.
 */
int coreinfer_select_batch_workspace_size(int64_t B, int64_t M, int64_t N, size_t* bytes);
int coreinfer_select_batch(const float* act, int64_t B, int64_t M, int64_t N, int64_t ld,
                           double alpha, double beta, int32_t* core_idx, int32_t* counts,
                           void* ws, size_t ws_bytes, void* stream);

/*
 * The same selection on the hidden matrix as the FFN holds it, in the layer's
 * element type, so that no fp32 copy of the activations has to be written for
 * it (Sec. 1 calls the prefill-stage selection free of extra cost; Def. 1
 * ranks "the activation", and a 16-bit model holds 16-bit activations).
 *   hidden [M, N] of `dtype` (row stride ld >= N elements), as written by
 *   coreinfer_ffn_dense_hidden: max(z, 0) for CI_ACT_RELU, SiLU(gate) * up for
 *   CI_ACT_SWIGLU.  The value ranked is the element itself for CI_ACT_RELU and
 *   its magnitude for CI_ACT_SWIGLU; 16-bit values are compared exactly (their
 *   fp32 images).  Everything else -- keep counts, ties towards the lower
 *   index, outputs, workspace, limits -- as for coreinfer_select; with
 *   CI_F32 / CI_ACT_RELU the two calls are the same.  Equal activations are far
 *   more frequent among 16-bit values; they are resolved towards the lower
 *   neuron index like any other tie.
 */
int coreinfer_select_hidden(const void* hidden, int dtype, int act, int64_t M, int64_t N, int64_t ld,
                            double alpha, double beta, int32_t* core_idx, int32_t* counts, void* ws,
                            size_t ws_bytes, void* stream);

/*
 * The two halves of coreinfer_select as separate calls, for callers that keep
 * running counts while a sentence grows (Fig. 1 names a "stability estimation"
 * that decides how the set is updated but does not specify it; Eq. 3 is a sum
 * over tokens, so counts of new tokens simply add to the old ones):
 *   coreinfer_count_tokens  steps 1-2 of coreinfer_select over the M rows of
 *                           act; counts [N] is overwritten unless
 *                           accumulate != 0, in which case it is added to;
 *                           ws: coreinfer_select_workspace_size(M, N) bytes.
 *   coreinfer_count_select  step 3 on given counts (every value must lie in
 *                           [0, max_count], max_count <= CI_MAX_TOKENS);
 *                           core_idx [keep_count(beta, N)] ascending;
 *                           ws: at least 256 bytes.
 */
int coreinfer_count_tokens(const float* act, int64_t M, int64_t N, int64_t ld, double alpha,
                           int32_t* counts, int accumulate, void* ws, size_t ws_bytes, void* stream);
int coreinfer_count_select(const int32_t* counts, int64_t N, int64_t max_count, double beta,
                           int32_t* core_idx, void* ws, size_t ws_bytes, void* stream);

/*
 * Similarity-guided prediction, group step (Sec. 4.1): the core neurons of a
 * semantic group are the top gamma share of neurons that appear most often in
 * the core sets of the group's sentences.
 *   core_sets [G, K] int32: the G sentences' core sets (any order; entries
 *             outside [0, N) are ignored);  counts[n] = #{g : n in set g}
 *             (out, may be NULL);  core_idx [keep_count(gamma, N)] ascending,
 *             ties towards the lower index as in coreinfer_select.
 *   ws: at least coreinfer_select_workspace_size(G, N) bytes.  G <= CI_MAX_TOKENS.
 * How sentences are grouped (labels, K-Means; App. A.2.3) is outside this library.
 */
int coreinfer_group_select(const int32_t* core_sets, int64_t G, int64_t K, int64_t N, double gamma,
                           int32_t* core_idx, int32_t* counts, void* ws, size_t ws_bytes, void* stream);

/*
 * Core-neuron similarity of two sets (Sec. 3.2, Insight-2: identical neurons
 * over all neurons involved).  set_a [Ka], set_b [Kb]: ascending, duplicate
 * free.  out [2] int32 (device): out[0] = |a and b|, out[1] = |a or b|; the
 * similarity is out[0] / out[1] (1 if both are empty).
 */
int coreinfer_core_similarity(const int32_t* set_a, int64_t Ka, const int32_t* set_b, int64_t Kb,
                              int32_t* out, void* stream);

/*
 * Similarity-guided prediction, choosing the group (Sec. 4.1 says only "once
 * the input sentence's group is determined"; the rule here is a reading): the
 * group whose core set is most similar to the prompt's own core set under the
 * metric above.  set [K] and every row of group_sets [G, Kg]: ascending,
 * duplicate free.  Out (device): inter_union [G, 2] int32 as for
 * coreinfer_core_similarity, best [1] int32 = the group with the largest
 * identical / involved ratio, compared exactly; equal ratios go to the lower
 * index; two empty sets count as ratio 1.  G <= CI_MAX_TOKENS.
 */
int coreinfer_assign_group(const int32_t* set, int64_t K, const int32_t* group_sets, int64_t G, int64_t Kg,
                           int32_t* best, int32_t* inter_union, void* stream);

/*
 * Similarity-guided prediction, choosing the group when the groups are K-Means
 * clusters of one layer's activation (App. A.2.3): the K-Means assignment
 * step.  The prompt's feature vector is the mean over its M tokens of the
 * activation rows act [M, N] (fp32, row stride ld >= N; the same matrix that
 * coreinfer_select ranks) -- the paper does not say how a sentence's tokens
 * are summarised, this is a reading.  centroids [G, N] fp32, row-major.
 * Out (device): dist [G] fp32 = squared Euclidean distance of the feature to
 * every centroid; best [1] int32 = the nearest centroid, equal distances going
 * to the lower index (a NaN distance is never nearest; group 0 if all are).
 * All sums in fp32, in an order that does not depend on scheduling.
 *   ws: at least coreinfer_assign_centroid_workspace_size(N) bytes (holds the
 *       feature vector, N floats from its start, readable after the call).
 * Limits: 1 <= M <= CI_MAX_TOKENS, 1 <= N <= CI_MAX_NEURONS, 1 <= G <= CI_MAX_TOKENS.
 */
int coreinfer_assign_centroid_workspace_size(int64_t N, size_t* bytes);
int coreinfer_assign_centroid(const float* act, int64_t M, int64_t N, int64_t ld, const float* centroids,
                              int64_t G, int32_t* best, float* dist, void* ws, size_t ws_bytes, void* stream);

/*
 * Deploy the core neurons (Sec. 5.3): gather rows S of w_up (and w_gate),
 * entries S of b_up and columns S of w_down into contiguous buffers:
 *   w_up_c   [K, d] = w_up[S, :]        w_gate_c [K, d] = w_gate[S, :]
 *   b_up_c   [K]    = b_up[S]
 *   w_down_c, by down_c_layout:
 *     CI_DOWN_NEURON_MAJOR  [K, d]  = (w_down[:, S])^T
 *     CI_DOWN_OUT_MAJOR     [d, ld] = w_down[:, S], ld = K rounded up to whole
 *                           16-byte vectors (coreinfer_compact_down_ld); the
 *                           columns K .. ld-1 are written as zeros.  This is
 *                           the layout the single-launch decode reads.
 * w_gate / w_gate_c must be non-NULL exactly when act == CI_ACT_SWIGLU;
 * b_up / b_up_c are both NULL or both non-NULL, and NULL for CI_ACT_SWIGLU
 * (the gated FFNs of the paper's models have no biases; CI_ERR_INVALID_ARG).
 * core_idx [K] must be strictly ascending with values in [0, N); an entry that
 * violates this yields an all-zero row / column and sets *status (device
 * int32, may be NULL; the caller zeroes it beforehand) to 1 -- it never causes
 * an out-of-bounds access.  Output buffers are caller-allocated and must not
 * overlap the inputs.  With CI_DOWN_OUT_MAJOR b_up_c holds ld elements (the
 * entries K .. ld-1 are left as they are).
 *
 * coreinfer_compact_preferred_layout names, in *down_c_layout (host), the
 * layout of w_down_c that decodes faster for K core neurons of a layer of width
 * d: both are correct for every shape; small layers decode faster through the
 * neuron-major path (two launches), large ones through the output-major path
 * (one launch), and where the single-launch path does not apply
 * (coreinfer_ffn_decode would return CI_ERR_UNSUPPORTED) the answer is
 * CI_DOWN_NEURON_MAJOR.
 */
int coreinfer_compact_down_ld(int64_t K, int dtype, int64_t* ld);
int coreinfer_compact_preferred_layout(int64_t K, int64_t d, int dtype, int act, int* down_c_layout);
int coreinfer_compact(const void* w_up, const void* w_gate, const void* b_up,
                      const void* w_down, int down_layout, int dtype, int act,
                      int64_t d, int64_t N, const int32_t* core_idx, int64_t K,
                      void* w_up_c, void* w_gate_c, void* b_up_c, void* w_down_c,
                      int down_c_layout, int32_t* status, void* stream);

/*
 * Re-deploying after the core set changed (Fig. 1 names a stability estimation
 * that decides "how to update" the set but gives no rule; this call rewrites
 * as little as possible).  The compact buffers written by coreinfer_compact
 * (or by an earlier update) are changed in place so that they hold exactly the
 * neurons of new_idx: a neuron that stays keeps its row; the rows of neurons
 * that left, in ascending row order, take the neurons that entered, in
 * ascending neuron order.  Only those rows are copied.
 *   new_idx [K] int32 ascending, duplicate free, the new core set (same K as
 *   the buffers).  slot_idx [K] int32, in/out: the neuron held by each row;
 *   after coreinfer_compact it equals that call's core_idx.  The decode entry
 *   point does not care about the order of the rows.  changed [1] int32
 *   (device, may be NULL): number of rows rewritten.  Weights, layouts
 *   (down_c_layout names the layout of w_down_c: rows or columns are rewritten
 *   accordingly) and dtypes as for coreinfer_compact.
 *   ws: coreinfer_compact_update_workspace_size.
 */
int coreinfer_compact_update_workspace_size(int64_t N, int64_t K, size_t* bytes);
int coreinfer_compact_update(const void* w_up, const void* w_gate, const void* b_up, const void* w_down,
                             int down_layout, int dtype, int act, int64_t d, int64_t N,
                             const int32_t* new_idx, int64_t K, int32_t* slot_idx, void* w_up_c,
                             void* w_gate_c, void* b_up_c, void* w_down_c, int down_c_layout,
                             int32_t* changed, void* ws, size_t ws_bytes, void* stream);

/*
 * Weights of one FFN layer as the decode kernel reads them.
 *   core_idx == NULL: compacted -- the buffers written by coreinfer_compact;
 *                     K rows each, shared by all B inputs.  down_layout says
 *                     how w_down_c was written: CI_DOWN_NEURON_MAJOR [K, d], or
 *                     CI_DOWN_OUT_MAJOR [d, ld_down].
 *   core_idx != NULL: gathered -- the resident dense weights, all neuron-major
 *                     (w_up, w_gate, w_down are [N, d], b_up is [N];
 *                     down_layout must be CI_DOWN_NEURON_MAJOR);
 *                     core_idx is [B, K], row b naming sentence b's core set.
 *                     Entries outside [0, N) contribute nothing.
 */
typedef struct {
  const void* w_up;        /* [K, d] or [N, d]                          */
  const void* w_gate;      /* same shape; NULL unless CI_ACT_SWIGLU     */
  const void* b_up;        /* [K] or [N]; may be NULL; NULL for SwiGLU  */
  const void* w_down;      /* [K, d] / [N, d], or [d, ld_down]          */
  const void* b_down;      /* [d]; may be NULL                          */
  const int32_t* core_idx; /* NULL (compacted) or [B, K] (gathered)     */
  int64_t K;               /* core neurons per sentence                 */
  int64_t d;               /* d_model                                   */
  int64_t N;               /* rows of the resident weights (gathered)   */
  int64_t ld_down;         /* row length of an output-major w_down (>= K, whole 16-byte vectors;
                              the columns K .. ld_down-1 must hold finite values, e.g. the zeros
                              coreinfer_compact writes: they are multiplied by zero) */
  int32_t down_layout;     /* ci_down_layout of w_down                  */
} ci_ffn_weights;

/*
 * Decode-stage FFN over the frozen core set (Sec. 4.2):
 *   ReLU:    y = w_down_c^T max(w_up_c x + b_up_c, 0) + b_down
 *   SwiGLU:  y = w_down_c^T (SiLU(w_gate_c x) * (w_up_c x)) + b_down
 * x [B, d] in, y [B, d] out, element type `dtype`; K = 0 gives y = b_down.
 * b_up with CI_ACT_SWIGLU: CI_ERR_INVALID_ARG.
 * ws: at least coreinfer_ffn_decode_workspace_size(B, K, d) bytes.
 *
 * Two kernel paths, chosen by the layout of the compact down matrix:
 *   CI_DOWN_NEURON_MAJOR (and every gathered call): neuron slices produce fp32
 *     partial outputs in ws, a second launch sums them in a fixed order.  ws
 *     needs no initialisation.  Compacted layers of up to 128 K elements in
 *     w_up (and w_gate) and up to four sentences run in one launch instead and
 *     leave ws as it is (a rule on sizes and types; not where y lies over x);
 *     the outputs are the same to the bit.  From 64 K elements on, unless the
 *     stream is being captured, its workgroups may hand the hidden values to
 *     each other through 4 MiB of static device memory.  Calls from any number
 *     of threads and streams may use it at the same time: a value carries the
 *     tag of its call, and a workgroup whose values are overwritten, or do not
 *     come within 20 us, computes them itself.  A gathered call of up to
 *     CI_MAX_UNION_SENTENCES large, overlapping lists reads each row of their
 *     union once, as coreinfer_ffn_decode_union does (a rule on B, K, N, d and
 *     the types; a neuron that a list names r times still counts r times).
 *   CI_DOWN_OUT_MAJOR: one launch, no partial outputs; the hidden values cross
 *     workgroups through ws as self-validating words.  For this path ws must
 *     have been ZEROED ONCE (hipMemsetAsync) before its first use and must not
 *     be written by anything else afterwards; every call leaves it ready for
 *     the next one, also when replayed from a HIP graph.  A workspace that has
 *     served a neuron-major or gathered call (which fills it with partial sums)
 *     must be zeroed again before an output-major call.  The launch needs one workgroup per compute unit resident at
 *     the same time; if other work keeps compute units busy for long, a
 *     workgroup gives up waiting after a bounded number of polls, the call's
 *     output is then unspecified and the int32 at ws + 4 is set to 1 (it is 0
 *     otherwise; coreinfer_ffn_decode_status copies it out).
 * Calls that share a workspace must not overlap in time.
 */
int coreinfer_ffn_decode_workspace_size(int64_t B, int64_t K, int64_t d, size_t* bytes);
int coreinfer_ffn_decode(const void* x, int64_t B, const ci_ffn_weights* w,
                         int dtype, int act, void* y,
                         void* ws, size_t ws_bytes, void* stream);
/* Enqueues a copy of the workspace's error word (see above) to *status_out, a
 * device int32; valid after the stream has been synchronised. */
int coreinfer_ffn_decode_status(const void* ws, int32_t* status_out, void* stream);

/*
 * coreinfer_ffn_decode for callers that cannot allocate device memory or have
 * none to pass: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Same arguments, same kernels and same results as
 * coreinfer_ffn_decode, but the workspace is a static array inside the library
 * (17 MiB of device memory on every GPU the library runs on, held until the
 * process ends); the call allocates nothing.  Limits: output-major compact
 * buffers: K <= 131024; neuron-major and gathered calls: B * slices * d * 4
 * bytes <= 16 MiB, slices = min(K, compute units / B) (e.g. B = 8, d = 9216 on
 * 256 compute units needs 9 MiB).  Beyond them: CI_ERR_WORKSPACE, nothing is
 * launched.  status_out: NULL, or a device int32 that receives the call's error
 * word (0, or 1 if a single-launch call gave up waiting; see above) by a copy
 * enqueued after the kernels.
 * All calls on one GPU share that GPU's array: calls that overlap in time on
 * one GPU (different streams, different host threads) race and give wrong
 * results; calls on one stream are fine.  Nothing needs zeroing by the caller.
 */
int coreinfer_ffn_decode_static(const void* x, int64_t B, const ci_ffn_weights* w,
                                int dtype, int act, void* y, int32_t* status_out, void* stream);

/*
 * Union-batched decode.  Several sentences, each with its own frozen core set
 * (stability-guided prediction, Sec. 4.1), decode one token each against the
 * same resident weights (the large-model scenario of Sec. 5.3).  Each row of
 * the UNION of the core sets is read once and applied to the sentences that
 * own it; per sentence the result is exactly the sparse FFN of Sec. 4.2 over
 * its own set, i.e. what coreinfer_ffn_decode computes with core_idx = [B, K].
 *
 * coreinfer_union_build: core_idx [B, K] int32 (device; any order, entries
 *   outside [0, N) are ignored, duplicates allowed), B <= CI_MAX_UNION_SENTENCES.
 *   Out (device, caller-owned): union_idx [max_rows] int32, ascending, the
 *   neurons in at least one set; union_mask [max_rows] uint32, bit s set iff
 *   sentence s owns the row; union_count [1] int32, the number of rows.
 *   max_rows >= min(N, B*K) (CI_ERR_INVALID_ARG otherwise).  Entries past
 *   union_count are left untouched.  ws: coreinfer_union_workspace_size(N) bytes.
 *
 * coreinfer_ffn_decode_union: x [B, d], y [B, d] of `dtype`; w->w_up,
 *   w->w_gate (SwiGLU), w->b_up, w->b_down as for the gathered decode: the full
 *   resident matrices, w_up / w_gate [N, d], w_down NEURON-MAJOR [N, d];
 *   w->core_idx, w->K, w->ld_down and w->down_layout are ignored.  union_idx / union_mask / union_count as
 *   written by coreinfer_union_build with the same max_rows; the row count is
 *   read on the device, so no host synchronisation is needed between the two
 *   calls.  ws: coreinfer_ffn_decode_union_workspace_size bytes, 16-byte aligned.
 *   Deterministic (fixed summation order).  Errors as for coreinfer_ffn_decode.
 */
int coreinfer_union_workspace_size(int64_t N, size_t* bytes);
int coreinfer_union_build(const int32_t* core_idx, int64_t B, int64_t K, int64_t N, int64_t max_rows,
                          int32_t* union_idx, uint32_t* union_mask, int32_t* union_count, void* ws,
                          size_t ws_bytes, void* stream);
int coreinfer_ffn_decode_union_workspace_size(int64_t B, int64_t max_rows, int64_t d, int dtype, int act,
                                              size_t* bytes);
int coreinfer_ffn_decode_union(const void* x, int64_t B, const ci_ffn_weights* w,
                               const int32_t* union_idx, const uint32_t* union_mask,
                               const int32_t* union_count, int64_t max_rows, int dtype, int act,
                               void* y, void* ws, size_t ws_bytes, void* stream);

/*
 * Dense FFN over all N neurons (Def. 1: the activation vector A(x) of every
 * prompt token; with M = 1 also the dense decode baseline).
 *   ReLU:    H = max(X w_up^T + b_up, 0),           A = H
 *   SwiGLU:  H = SiLU(X w_gate^T) * (X w_up^T),     A = |H|
 *   Y = H w_down^T + b_down
 * X [M, d]; Y [M, d] (element type `dtype`, may be NULL); A [M, N] fp32 (may
 * be NULL); at least one of Y, A must be given.  b_up may be NULL and must be
 * NULL for CI_ACT_SWIGLU (CI_ERR_INVALID_ARG).  For Y, H is rounded to
 * `dtype` before the second product when M > 4 (matrix-core path).
 * ws: coreinfer_ffn_dense_workspace_size(M, d, N, dtype) bytes.  For M > 4 what
 * goes beyond the hidden matrix (4 M N bytes, whole 256-byte blocks, and 256)
 * holds partial sums of Y where tiles are split along N; a workspace without
 * room for them is accepted, and no tile is split.
 */
int coreinfer_ffn_dense_workspace_size(int64_t M, int64_t d, int64_t N, int dtype, size_t* bytes);
int coreinfer_ffn_dense(const void* X, int64_t M,
                        const void* w_up, const void* w_gate, const void* b_up,
                        const void* w_down, const void* b_down, int down_layout,
                        int dtype, int act, int64_t d, int64_t N,
                        void* Y, float* A,
                        void* ws, size_t ws_bytes, void* stream);

/*
 * Dense FFN that hands out the hidden matrix instead of fp32 scores: the
 * prefill pass for coreinfer_select_hidden.  H [M, N] (caller-allocated, of
 * `dtype`, 16-byte aligned) receives max(X w_up^T + b_up, 0) or
 * SiLU(X w_gate^T) * (X w_up^T), rounded once from the fp32 accumulator; Y
 * (nullable) = H w_down^T + b_down as in coreinfer_ffn_dense.  No fp32 matrix
 * of size M x N is written.  Arguments, layouts and errors as for
 * coreinfer_ffn_dense; the workspace (at least 256 bytes) only holds partial
 * sums of Y where tiles are split along N.
 */
int coreinfer_ffn_dense_hidden_workspace_size(int64_t M, int64_t d, int64_t N, int dtype, size_t* bytes);
int coreinfer_ffn_dense_hidden(const void* X, int64_t M, const void* w_up, const void* w_gate,
                               const void* b_up, const void* w_down, const void* b_down, int down_layout,
                               int dtype, int act, int64_t d, int64_t N, void* Y, void* H, void* ws,
                               size_t ws_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * Serving in 4 bits: weights and a key-value cache that take a quarter of the
 * 16-bit bytes, for decode steps, which are bound by the bytes they read.
 *
 * Both are held in groups of `group` (32, 64 or 128) neighbouring elements of a
 * row.  A group x_0 .. x_{g-1} has
 *     low  = fp16(min x),   step = fp16((max x - min x) / 15),
 *     n_i  = rint((x_i - low) / step) within 0 .. 15   (0 where step is 0),
 * differences and quotients in fp32 and values beyond +-65504 held there, and
 * stands for low + step n_i.  A NaN makes low and step, and so the whole group, NaN.
 * A last group that the row does not fill ranges over what there is of it.
 * ---------------------------------------------------------------------------
 */
#define CI_MAX_W4_ROWS 64            /* M of coreinfer_w4_matvec                  */
#define CI_MAX_CACHE_SLOTS 16777216  /* slots of a sentence in a cache            */
#define CI_ACT_NONE 2                /* no activation: coreinfer_w4_matvec only   */

/*
 * Weights in 4 bits.  The packed form is the library's own (the order in which
 * the matrix cores take it), 16-byte aligned, coreinfer_w4_size bytes.
 *   coreinfer_w4_quantize  w [R, C] (row stride ld >= C elements, of `dtype`,
 *                          any alignment of whole elements) -> packed.
 *   coreinfer_w4_read      packed -> the values it stands for, in `dtype`.
 * E.g. the buffers of coreinfer_compact: w_up_c / w_gate_c [K, d] and, with
 * CI_DOWN_OUT_MAJOR, w_down_c [d, K] with row stride ld.
 * Limits: 1 <= R, C <= CI_MAX_NEURONS.  A group that is none of the three:
 * CI_ERR_UNSUPPORTED.
 */
int coreinfer_w4_size(int64_t R, int64_t C, int group, size_t* bytes);
int coreinfer_w4_quantize(const void* w, int64_t R, int64_t C, int64_t ld, int dtype, int group, void* packed,
                          void* stream);
int coreinfer_w4_read(const void* packed, int64_t R, int64_t C, int group, void* w, int64_t ld, int dtype, void* stream);

/*
 * y = act(x W^T + b) for one to 64 rows x [M, C] over weights in 4 bits, W [R, C]:
 *   CI_ACT_NONE, CI_ACT_RELU (gate NULL; bias [R] of `bias_dtype` or NULL), or
 *   CI_ACT_SWIGLU: y = SiLU(x G^T) * (x W^T), gate packed as W is (same R, C,
 *   group); a bias is CI_ERR_INVALID_ARG as everywhere for gated layers.
 * x [M, C] of x_dtype (row stride ldx >= C) and y [M, R] of y_dtype (row stride
 * ldy >= R) may be of different types, so that the hidden values between two
 * products stay in fp32; both are aligned to their elements.  16-bit x is multiplied
 * as it is, fp32 x in three bf16 pieces (24 bits); sums in fp32, in a fixed order,
 * for 16-bit x of the codes plus 16 (1.4 of the 24 bits are the 16's).
 * A row of x with an infinity or a NaN gives NaN.  y must not overlap x.
 * ws: coreinfer_w4_matvec_workspace_size bytes, 16-byte aligned; NULL where that is
 * 0: up to 16 rows of 64 KB together, at 2 bytes an element (fp32: 6) of rows filled up to
 * 128s (one row: C <= 32768, fp32 10880).  The size is asked of longer 16-bit rows too, but
 * up to 16 of them leave it alone where x, C and ldx are whole words, ldx <= 2^26 and
 * (M - 1) ldx + C < 2^29.
 */
int coreinfer_w4_matvec_workspace_size(int64_t M, int64_t C, int x_dtype, size_t* bytes);
int coreinfer_w4_matvec(const void* x, int64_t M, int64_t ldx, int x_dtype, const void* w, const void* gate,
                        const void* bias, int bias_dtype, int act, int64_t R, int64_t C, int group, void* y,
                        int64_t ldy, int y_dtype, void* ws, size_t ws_bytes, void* stream);

/*
 * A layer's keys and values in 4 bits: B sentences, H heads of D = 64 or 128
 * channels, room for `cap` slots a sentence (a multiple of 32).  The buffers are
 * the caller's, 16-byte aligned, of the sizes that coreinfer_kv4_sizes states, and
 * need no initialisation: no call uses what lies behind a sentence's last slot.
 * Which slots are in use is not part of the struct; the calls are told by `lens` [B]
 * int32 on the device, so that a captured step can be replayed while sentences grow.
 * D or group not supported (group must divide D): CI_ERR_UNSUPPORTED.
 * B * H <= 65535.
 */
typedef struct {
  void* k;           /* B H cap D / 2 bytes                              */
  void* v;           /* B H cap D / 2 bytes                              */
  uint32_t* k_scale; /* B H (D / group) cap: step and low                */
  uint32_t* v_scale; /* the same                                         */
  float* weight;     /* [B, H, cap] accumulated attention weight, or NULL  */
  int32_t* pos;      /* [B, H, cap] position of a slot's token, or NULL    */
  int64_t B, H, cap;
  int32_t D, group;
} ci_kv4;
int coreinfer_kv4_sizes(int64_t B, int64_t H, int64_t cap, int D, int group, size_t* codes_bytes, size_t* scale_bytes);

/*
 * Writes S tokens' keys and values, k and v [B, S, H, D] of `dtype` with the
 * element strides stride[0 .. 2] of b, s and h (host array, shared by both; a row of D is
 * contiguous), e.g. slices of one fused projection.  lens [B] counts the new
 * tokens already: token i goes to slot lens[b] - S + i.  start [B] (or NULL):
 * the first slot that may be written, so that sentences with fewer than S new tokens
 * have theirs at the end of the S; slots outside 0 .. cap - 1 are not written either.
 * weight of a written slot becomes 0, pos (where the cache has them) next[b] - S + i;
 * next [B]: the sentence's tokens so far, evicted ones included, NULL = lens.
 * 1 <= S <= 2^19.
 */
int coreinfer_kv4_append(const ci_kv4* cache, const void* k, const void* v, int64_t S, const int64_t* stride, int dtype,
                         const int32_t* start, const int32_t* lens, const int32_t* next, void* stream);

/*
 * Slots first .. first + count - 1 as the values they stand for: k and v
 * [B, H, count, D] of `dtype`, 16-byte aligned; zeros from lens[b] on.
 */
int coreinfer_kv4_read(const ci_kv4* cache, const int32_t* lens, int64_t first, int64_t count, void* k, void* v,
                       int dtype, void* stream);

/*
 * Attention of S tokens a sentence over the cache, q [B, S, Hq, D] (element
 * strides as above; Hq a multiple of H, query head i reads head i / (Hq / H)):
 *     out[b, s, i] = sum_t p_t v_t,   p = softmax over t of scale (q . k_t).
 * The S tokens are the sentence's last ones: row s sees the slots t < lens[b] and
 * t <= lens[b] - S + s.  A row that sees none gives zeros.  lens beyond
 * 0 .. max_len are taken as its ends; max_len <= cap sizes the launches.
 *   out [B, S, Hq, D] of `dtype`, contiguous, 16-byte aligned, not overlapping q.
 *   lse [B, S, Hq] fp32 or NULL: log of the sum of exp(scale q . k_t) over t
 *       (-infinity for a row that sees nothing).
 *   weight_out [B, H, cap] fp32 or NULL: cache->weight plus, for every slot t <
 *       lens[b], the p_t of all rows and heads that read it; other slots are left as
 *       they are.  May be cache->weight itself, which must not be NULL then.
 * scale > 0 and finite, also times log2(e).  Softmax statistics and sums in fp32; keys and values enter
 * as they are held, q as it is (fp32 q in three bf16 pieces), probabilities in
 * two bf16 pieces (fp32 q: three).  The order of the sums is fixed.
 * ws: coreinfer_kv4_attend_workspace_size bytes, 16-byte aligned (weights != 0: for
 * calls with weight_out).  Calls that share a workspace must not overlap in time.
 * Limits: Hq / H <= 4096, S * (Hq / H) <= 2^20.
 */
int coreinfer_kv4_attend_workspace_size(int64_t B, int64_t H, int D, int64_t S, int64_t Hq, int64_t max_len, int weights,
                                        size_t* bytes);
int coreinfer_kv4_attend(const ci_kv4* cache, const void* q, int64_t S, int64_t Hq, const int64_t* stride, int dtype,
                         float scale, const int32_t* lens, int64_t max_len, void* out, float* lse, float* weight_out,
                         void* ws, size_t ws_bytes, void* stream);

/*
 * Eviction by accumulated attention weight: of every head with more than `budget`
 * slots in use, `budget` stay, first those of the sentence's last `recent`
 * positions (pos >= next[b] - recent), then those with the largest weight; equal
 * weights go to the lower slot, a NaN counts least.
 * As in coreinfer_compact_update a slot that stays below the budget keeps its place and
 * those that stay from above it take the places of the others, both in ascending
 * order, so only they are moved: one row a head for a cache that is cut by one at
 * every step.  cache->weight and cache->pos must not be NULL.
 *   weight_out, pos_out [B, H, cap]: of the new contents; slots from the budget to
 *     lens[b] - 1 get weight 0 and pos -1, others are left.  May be
 *     cache->weight and cache->pos.
 *   lens_out [B] or NULL: min(lens[b], budget); may be lens (apart from lens and next, calls
 *     of few moves and max_len <= 32768 take one launch instead of two).
 * The order of slots is no longer that of positions, which attention does not ask for.
 * ws: coreinfer_kv4_evict_workspace_size bytes, 16-byte aligned.
 * 1 <= budget, 0 <= recent <= budget, 1 <= max_len <= cap.
 */
int coreinfer_kv4_evict_workspace_size(int64_t B, int64_t H, int64_t max_len, int64_t budget, size_t* bytes);
int coreinfer_kv4_evict(const ci_kv4* cache, const int32_t* lens, const int32_t* next, int64_t max_len, int64_t budget,
                        int64_t recent, float* weight_out, int32_t* pos_out, int32_t* lens_out, void* ws,
                        size_t ws_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * Serving from a cache in pages, in the layer's own type, for packed batches.
 *
 * The new tokens of B sentences are T rows one behind the other: those of sentence b
 * are the rows first[b] .. first[b + 1] - 1 (first [B + 1] int32 on the device,
 * ascending from 0), so that a prompt's chunk and other sentences' single tokens
 * go together; a sentence may have none.  lens [B] int32 on the device: a sentence's
 * slots in use, its new tokens included, which are its last ones: row i of n is in slot
 * lens[b] - n + i.  Rows from first[B] on belong to no sentence: what they would
 * write stays as it is.  Entries of first outside 0 .. T are taken as its ends.
 * Strides are in elements, of a row (token) and of a head; a head's channels are
 * contiguous.  T = 0 is CI_OK and does nothing (no pointer is looked at).
 * ---------------------------------------------------------------------------
 */
#define CI_MAX_PACKED_ROWS 1048576 /* T                     */
#define CI_MAX_ROPE_CHANNELS 512   /* D of coreinfer_rope   */

/*
 * Rotary positions.  Of a head's D channels the first `rot` are turned, in pairs
 * i = 0 .. rot / 2 - 1 of the channels
 *     CI_ROPE_HALF          i and i + rot / 2,
 *     CI_ROPE_INTERLEAVED   2 i and 2 i + 1,
 * a pair (a, c) at position p becomes scale (a cos - c sin, c cos + a sin) of the angle
 * 2 pi turns[i] p / 2^64.  In whole 2^-64ths of a turn an angle is exact at every
 * position, however far.  The other channels stay as they are.
 */
typedef enum { CI_ROPE_HALF = 0, CI_ROPE_INTERLEAVED = 1 } ci_rope_style;
typedef struct {
  const uint64_t* turns; /* [rot / 2] device, 8-byte aligned; NULL where rot is 0 */
  float scale;           /* of the turned channels, finite                        */
  int32_t rot;           /* even, 0 .. D; 0 turns nothing                         */
  int32_t style;
} ci_rope;

/*
 * turns [rot / 2] (HOST array) of the frequencies f_i = base^(-2 i / rot) radians a
 * position (Su et al. 2021), or of those scaled for a context `factor` times as long:
 *     CI_ROPE_LINEAR  f_i / factor (positions are squeezed)
 *     CI_ROPE_BASE    base factor^(rot / (rot - 2)) in the place of base (the slowest pair is squeezed, the
 *                     fastest stays)
 *     CI_ROPE_PARTS   f_i (g + (1 - g) / factor), g = (original f_i / (2 pi) - slow) /
 *                     (fast - slow) within 0 .. 1: pairs that turn more than `fast` times in the
 *                     `original` context stay, those below `slow` are squeezed (Peng et al.
 *                     2023, who also scale by 0.1 ln(factor) + 1 where factor > 1: ci_rope's scale)
 * Host-only.  rot even, 2 .. 512; base > 0; factor > 0 (not looked at for CI_ROPE_PLAIN);
 * original > 0 and fast > slow for CI_ROPE_PARTS only; everything finite.
 */
typedef enum { CI_ROPE_PLAIN = 0, CI_ROPE_LINEAR = 1, CI_ROPE_BASE = 2, CI_ROPE_PARTS = 3 } ci_rope_scaling;
int coreinfer_rope_turns(int64_t rot, double base, int scaling, double factor, double original, double fast, double slow,
                         uint64_t* turns);

/*
 * y = x [T, H, D] normed by head and turned by its positions, in one pass:
 *   norm [D] of `dtype` or NULL: n = x / sqrt(mean over the head of x^2 + eps) norm, eps >= 0;
 *   then rope (NULL: nothing is turned) at positions pos [T] int32 (may be negative;
 *   NULL where nothing is turned).
 * backward != 0: the angles' signs are turned, which is the gradient (the transpose) of
 * the rotation and, up to scale^2, its inverse; with a norm CI_ERR_INVALID_ARG.
 * Everything in fp32, rounded once.  y (any strides at which its rows lie apart, none between another's
 * heads) may be x itself with x's strides, and must not overlap it otherwise.  x and y are aligned to their elements; it is fastest
 * where they and norm are aligned to 16 bytes, strides included, and D and rot are multiples of 32 bytes.
 * 1 <= H <= 65535, 1 <= D <= CI_MAX_ROPE_CHANNELS.
 */
int coreinfer_rope(const void* x, const int64_t* stride, int64_t T, int64_t H, int64_t D, int dtype, const void* norm,
                   float eps, const ci_rope* rope, const int32_t* pos, int backward, void* y, const int64_t* y_stride,
                   void* stream);

/*
 * A layer's keys and values in pages of `page` slots (16, 32, 64, 128 or 256), H heads of
 * D = 64 or 128 channels (other D or page: CI_ERR_UNSUPPORTED).  table [B, most]: slot t of
 * sentence b is slot t % page of page table[b][t / page]; the caller gives pages
 * out, and may give a page to several sentences that begin alike.  An entry outside 0 .. pages - 1
 * is no page: nothing is written there and no row sees its slots.  The buffers need no
 * initialisation: no result depends on what lies behind a sentence's last slot.
 * most * page <= CI_MAX_CACHE_SLOTS, B * H <= 65535.
 */
typedef struct {
  void* k;              /* [pages, H, page, D] of dtype, 16-byte aligned */
  void* v;              /* the same                                      */
  const int32_t* table; /* [B, most] device                              */
  int64_t pages, most, B;
  int32_t H, page, D, dtype;
} ci_kvp;

/*
 * Writes the packed tokens' keys and values, k and v [T, H, D] of the cache's type (strides
 * shared by both, e.g. slices of one fused projection), to their slots; slots that have no page, or outside
 * 0 .. most * page - 1, are not written.  On the way the keys are normed by head
 * (k_norm [D], NULL: not) and turned by their positions (rope, NULL: not), as
 * coreinfer_rope does; pos [T] or NULL: a token's position is its slot.  q [T, Hq, D] (or NULL, with
 * Hq = 0) goes the same way, with q_norm, to q_out [T, Hq, D] contiguous, 16-byte aligned, not
 * overlapping q (CI_ERR_BAD_LAYOUT).  Values are copied.  No two tokens may go to the same slot.
 */
int coreinfer_kvp_append(const ci_kvp* cache, const void* k, const void* v, const int64_t* stride, int64_t T,
                         const int32_t* first, const int32_t* lens, const int32_t* pos, const ci_rope* rope,
                         const void* k_norm, float eps, const void* q, int64_t Hq, const int64_t* q_stride,
                         const void* q_norm, void* q_out, void* stream);

/*
 * Attention of packed rows q [T, Hq, D] of the cache's type (Hq a multiple of H, query head
 * i reads head i / (Hq / H)) over their sentences' slots:
 *     out[r, i] = sum_t p_t v_t,   p = softmax over t of scale (q . k_t).
 * The row in slot p sees the slots t <= p; with window > 0 of those only t > p - window
 * and t < sinks.  A row that sees none gives zeros.  What it does not see, infinities and NaN
 * included, does not touch it.  A logit of +infinity or NaN that it sees gives NaN, in lse too;
 * where all that it sees are -infinity, it gives NaN, and lse -infinity.
 * An infinite value that it sees gives that infinity, whatever its weight; values that are not finite cost
 * the rows that meet them, seen or not, a second time through, of a few times the first's time.
 *   max_rows  the most rows of a sentence, max_len the most slots (<= most * page): they choose
 *             and size the launches.  lens beyond 0 .. max_len are taken as its ends; rows
 *             of a sentence from max_rows on are left as they are.
 *   out [T, Hq, D] contiguous, 16-byte aligned, not overlapping q (CI_ERR_BAD_LAYOUT).
 *   lse [T, Hq] fp32 or NULL: log of the sum of exp(scale q . k_t) (-infinity where nothing is seen).
 * scale > 0 and finite, also times log2(e).  Softmax statistics and sums in fp32, in a fixed order.
 * Probabilities enter the product with 16-bit values in two pieces of that type where few
 * rows share a head, and rounded to it once in prompts: with R = min(max_rows, T) Hq / H, where
 * R > 64, or R > 16 and B H ceil(R / 16) max_len >= 196608, but for sentences of up to 16 rows a head
 * if T < B max_rows.  max_rows and max_len choose the last bits of a result by that rule.
 * ws: coreinfer_kvp_attend_workspace_size bytes, 16-byte aligned; NULL where that is 0.  Calls
 * that share a workspace must not overlap in time.
 * window, sinks >= 0.  Hq / H <= 4096, T * Hq <= 2^30.
 */
int coreinfer_kvp_attend_workspace_size(const ci_kvp* cache, int64_t T, int64_t Hq, int64_t max_rows, int64_t max_len,
                                        int64_t window, int64_t sinks, size_t* bytes);
int coreinfer_kvp_attend(const ci_kvp* cache, const void* q, int64_t Hq, const int64_t* stride, int64_t T,
                         const int32_t* first, const int32_t* lens, int64_t max_rows, int64_t max_len, int64_t window,
                         int64_t sinks, float scale, void* out, float* lse, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* COREINFER_H_ */
