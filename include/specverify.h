/*
 * specverify: one batched speculative-decoding tree-verify step on an
 * AMD Instinct MI355X (gfx950).
 *
 * The operation (RLHFSpec, Section 2.2 "Speculative Decoding"; Section 5.2
 * names its two costs, attention over the KV cache and the FFN matrix
 * products; Section 6.2 fixes that a step never rewrites verified KV):
 *
 *   For every live sample b the caller hands in a committed KV length S_b
 *   and a draft token tree of T_b nodes (node 0 = root = the token decided
 *   by the previous step, whose K/V are not cached yet).  The target model,
 *   a Llama-style decoder, runs one forward pass over all N = sum T_b
 *   nodes: node i sits at position S_b + depth(i) and attends to the whole
 *   committed prefix plus its own ancestors in the tree (itself included).
 *   Greedy acceptance then takes g_i = argmax of node i's logits (lowest
 *   token id on ties), accepts a node when every edge on its branch carries
 *   the token its parent predicted (the root is always accepted), and
 *   picks the deepest accepted node (lowest node index on ties):
 *   accepted_len = its depth, next_token = its g.  Committing moves the K/V
 *   of the accepted branch to cache positions S_b .. S_b + accepted_len and
 *   the committed length becomes S_b + accepted_len + 1.
 *
 * Conventions for every entry point:
 *   - Return value: SPEC_OK (0) or a negative spec_status.  On a validation
 *     failure nothing has been enqueued and no output or KV byte has been
 *     written; spec_last_error() then describes the failure.
 *   - Work is enqueued on the caller's HIP stream (passed as void*; NULL is
 *     the null stream) and is asynchronous: device outputs are valid once
 *     the stream has been synchronised.
 *   - "host" / "device" below says where a pointer must point.  All device
 *     memory (weights, KV pool, workspace, outputs) is allocated and owned
 *     by the caller; the library never allocates device memory.  The only
 *     allocations it makes are its opaque handle and a small pinned host
 *     staging area inside it.
 *   - One spec_kv handle must not be used from two threads or two streams
 *     at once.
 *   - Numerics: bf16 weights, bf16 activations at GEMM inputs, bf16 KV
 *     cache; fp32 accumulation, softmax, norms and residual stream.
 *   - Supported shapes: head_dim 64 or 128; hidden, n_heads*head_dim and
 *     ffn multiples of 128; n_kv_heads*head_dim a multiple of 128; vocab a
 *     multiple of 128; n_heads a multiple of n_kv_heads; 1 <= T_b <=
 *     SPEC_MAX_TREE.  Anything else returns SPEC_ERR_UNSUPPORTED.
 */
#ifndef SPECVERIFY_H
#define SPECVERIFY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPEC_MAX_TREE 256
/* 64-bit words of one node's ancestor set (spec_debug.anc). */
#define SPEC_ANC_WORDS (SPEC_MAX_TREE / 64)

typedef enum {
  SPEC_OK = 0,
  SPEC_ERR_INVALID = -1,     /* null pointer, non-positive size, bad config or sample id */
  SPEC_ERR_TREE = -2,        /* parents[0] != -1, parent not before child, token out of range */
  SPEC_ERR_CAPACITY = -3,    /* S_b + T_b exceeds the sample's KV capacity, or buffer too small */
  SPEC_ERR_WORKSPACE = -5,   /* workspace smaller than the call needs */
  SPEC_ERR_UNSUPPORTED = -6, /* shape outside the supported set (see above) */
  SPEC_ERR_HIP = -7          /* a HIP runtime call or kernel launch failed */
} spec_status;

/* Llama-style decoder shape.  rope_theta: base of the rotary frequencies,
 * frequency j = rope_theta^(-2j/head_dim), half-split rotation (element j
 * pairs with j + head_dim/2).  rms_eps: RMSNorm epsilon. */
typedef struct {
  int32_t n_layers, hidden, n_heads, n_kv_heads, head_dim, ffn, vocab;
  float rope_theta, rms_eps;
} spec_model_config;

/* Weights: device pointers to row-major bf16 matrices in [out][in] layout
 * (a GEMM computes x . W^T), read-only, owned by the caller.  The per-layer
 * fields are HOST arrays of n_layers device pointers. */
typedef struct {
  const void* tok_embed;        /* [vocab][hidden] */
  const void* final_norm;       /* [hidden] RMSNorm gain */
  const void* lm_head;          /* [vocab][hidden] (untied) */
  const void* const* attn_norm; /* [hidden] */
  const void* const* wq;        /* [n_heads*head_dim][hidden] */
  const void* const* wk;        /* [n_kv_heads*head_dim][hidden] */
  const void* const* wv;        /* [n_kv_heads*head_dim][hidden] */
  const void* const* wo;        /* [hidden][n_heads*head_dim] */
  const void* const* ffn_norm;  /* [hidden] */
  const void* const* w_gate;    /* [ffn][hidden] */
  const void* const* w_up;      /* [ffn][hidden] */
  const void* const* w_down;    /* [hidden][ffn] */
} spec_weights;

/* Opaque KV-pool handle (host memory, owned by the library). */
typedef struct spec_kv spec_kv;

/* Optional device dumps for tests; any field may be NULL.  N = sum T_b,
 * rows in batch order (sample 0's nodes first, each tree in its own node
 * order). */
typedef struct {
  float* logits;      /* [N][vocab] fp32 */
  int32_t* argmax;    /* [N] greedy token after each node */
  int32_t* depth;     /* [N] depth of each node (root 0) */
  int32_t* pos;       /* [N] position S_b + depth */
  uint64_t* anc;      /* [N][SPEC_ANC_WORDS] ancestor set: bit t % 64 of word t / 64 is node t
                         of the same tree; own bit set, bits of nodes >= T_b clear */
} spec_debug;

/* ---- KV pool (Section 6.2: verified KV is never rewritten) -------------
 *
 * Layout: sample s owns one contiguous block of
 *   n_layers * 2 * n_kv_heads * capacity[s] * head_dim  bf16 values,
 * ordered [layer][K=0,V=1][kv_head][position][head_dim]; blocks follow each
 * other in sample order, each starting at a 256-byte aligned offset.
 * Positions [0, S_s) hold committed K/V (K already rotated). */

/* Bytes a pool for n_samples samples with the given host capacities needs,
 * or 0 if an argument is invalid. */
size_t spec_kv_bytes(const spec_model_config* cfg, int32_t n_samples, const int32_t* capacity);

/* Create a handle over caller memory device_buf (device, >= spec_kv_bytes,
 * 256-byte aligned).  capacity: host [n_samples].  *out receives the handle. */
int spec_kv_alloc(const spec_model_config* cfg, int32_t n_samples, const int32_t* capacity,
                  void* device_buf, size_t buf_bytes, spec_kv** out);

/* Release the handle (not device_buf).  Waits for the handle's pending
 * staging copies. */
int spec_kv_free(spec_kv* kv);

/* Byte offset of sample's block inside device_buf and its capacity. */
int spec_kv_sample_layout(const spec_kv* kv, int32_t sample, int64_t* byte_offset,
                          int32_t* capacity);

/* ---- The verify step ---------------------------------------------------- */

/* Workspace bytes spec_verify needs for up to max_batch samples and
 * max_tokens tree nodes in total; 0 if an argument is invalid. */
size_t spec_workspace_bytes(const spec_model_config* cfg, int32_t max_batch, int32_t max_tokens);

/* One tree-verify step over `batch` live samples.
 *   sample_ids   host [batch]   pool sample of each live sample (distinct)
 *   tree_offsets host [batch+1] tree_offsets[0] = 0, T_b = diff, 1..SPEC_MAX_TREE
 *   tree_tokens  host [N]       token of every node, in [0, vocab)
 *   tree_parents host [N]       parent node index within the same tree;
 *                               -1 for node 0, 0 <= parent < node otherwise
 *   seq_lens     host [batch]   committed length S_b, S_b + T_b <= capacity
 *   workspace    device, ws_bytes >= spec_workspace_bytes(cfg, batch, N)
 * Outputs (device, int32):
 *   accepted_len   [batch]                  depth of the deepest accepted node
 *   next_token     [batch]                  greedy token after that node
 *   accepted_nodes [batch][SPEC_MAX_TREE]   node ids of the accepted branch,
 *                                           root first, then -1
 * KV effect: writes the nodes' K/V to positions S_b + node of each sample
 * (never below S_b).  dbg may be NULL. */
int spec_verify(const spec_model_config* cfg, const spec_weights* w, spec_kv* kv,
                int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets,
                const int32_t* tree_tokens, const int32_t* tree_parents, const int32_t* seq_lens,
                void* workspace, size_t ws_bytes, void* stream,
                int32_t* accepted_len, int32_t* next_token, int32_t* accepted_nodes,
                const spec_debug* dbg);

/* ---- Acceptance at a sampling temperature, and end of sequence ---------
 *
 * Speculative decoding is lossless (Section 2.2): at temperature T > 0 the
 * verified tokens follow the target model's sampling distribution
 * p_u = softmax(z_u / T) (z_u: the logits after node u).  This assumes the
 * draft drew the children of every node u independently from its own
 * distribution q_u.  The acceptance walk (multi-draft speculative sampling):
 * at the current node u, with the unnormalised residual P = p_u (total R =
 * its fp64 sum), try u's children in node order; child c with token x is
 * accepted when uniforms[c][0] * q_u(x) * R < P(x); a rejected child sets
 * P = max(P - R q_u, 0) and R = sum P.  An accepted child becomes u.  When no
 * child of u is accepted (or u has none) the next token is the smallest y
 * with P(0) + ... + P(y) > uniforms[u][1] * R.  Residuals, sums and the CDF
 * are fp64.  accepted_len = depth of the final u, accepted_nodes = the path.
 *
 * End of sequence (eos_token >= 0, RLHF rollouts end at it): an accepted node
 * carrying the EOS token ends the branch, its children are not tried and
 * next_token = -1.  With temperature 0 the acceptance is spec_verify's greedy
 * rule with that truncation (an accepted EOS node accepts no children).
 *
 * spec_sampling:
 *   temperature  >= 0, finite
 *   eos_token    -1 (none) or a token id
 *   draft_probs  device [N][vocab] fp32, row i = q of node i (sums to 1;
 *                read for nodes with children); unused when temperature == 0
 *   uniforms     device [N][2] fp32 in [0, 1): column 0 = node i's
 *                acceptance draw as a child, column 1 = the draw that samples
 *                the next token if the walk ends at node i; unused at T == 0
 * The random draws are inputs so that the caller owns the randomness. */
typedef struct {
  float temperature;
  int32_t eos_token;
  const float* draft_probs;
  const float* uniforms;
} spec_sampling;

/* Workspace bytes spec_verify_sampled needs at temperature > 0 (the logits
 * [N][vocab] fp32, the nodes' decisions and a [batch][vocab] fp64 residual on
 * top of spec_workspace_bytes); 0 if an argument is invalid.  At temperature
 * 0 spec_workspace_bytes suffices. */
size_t spec_workspace_bytes_sampled(const spec_model_config* cfg, int32_t max_batch,
                                    int32_t max_tokens);

/* spec_verify with the acceptance above.  Same arguments and outputs; samp
 * must not be NULL.  dbg->logits, when given, receives the logits the
 * sampling reads. */
int spec_verify_sampled(const spec_model_config* cfg, const spec_weights* w, spec_kv* kv,
                        int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets,
                        const int32_t* tree_tokens, const int32_t* tree_parents,
                        const int32_t* seq_lens, void* workspace, size_t ws_bytes, void* stream,
                        const spec_sampling* samp, int32_t* accepted_len, int32_t* next_token,
                        int32_t* accepted_nodes, const spec_debug* dbg);

/* ---- Verify without a caller workspace ---------------------------------
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation):
 * spec_verify with its workspace taken from a static device array of
 * SPEC_NOALLOC_SCRATCH_BYTES, one per device, held by the library from the
 * first call on that device until the process ends.  Arguments, outputs, KV
 * effect and results are spec_verify's (bitwise: the same plan and kernels),
 * without workspace and ws_bytes.  The call makes no device or pinned host
 * allocation; its per-call descriptors go to the device from pageable host
 * memory (hipMemcpyAsync, which may block the calling thread until the copy
 * is done).  Returns SPEC_ERR_WORKSPACE, before enqueueing anything, when
 * spec_workspace_bytes(cfg, batch, N) exceeds SPEC_NOALLOC_SCRATCH_BYTES (at
 * the Llama-3-8B shape, 128 samples with 1024 tree nodes in total fit).
 * Every call on one device shares that device's array and leaves its
 * contents behind: calls that overlap on one device (two streams, two
 * threads) race and must be serialised by the caller.  The calling thread's
 * current device must be the stream's; SPEC_ERR_HIP if the array's address
 * cannot be looked up on it. */
#define SPEC_NOALLOC_SCRATCH_BYTES ((size_t)320 << 20)

int spec_verify_noalloc(const spec_model_config* cfg, const spec_weights* w, spec_kv* kv,
                        int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets,
                        const int32_t* tree_tokens, const int32_t* tree_parents,
                        const int32_t* seq_lens, void* stream, int32_t* accepted_len,
                        int32_t* next_token, int32_t* accepted_nodes, const spec_debug* dbg);

/* Commit the accepted branches of the preceding spec_verify (same batch,
 * sample_ids and seq_lens, same stream): the K/V of node accepted_nodes[b][d]
 * moves to position S_b + d for d = 1..accepted_len[b] (all layers, K and
 * V), and new_seq_lens[b] = S_b + accepted_len[b] + 1.
 *   accepted_len, accepted_nodes: device, as written by spec_verify
 *   new_seq_lens: device [batch] int32 output */
int spec_kv_commit(spec_kv* kv, int32_t batch, const int32_t* sample_ids,
                   const int32_t* seq_lens, const int32_t* accepted_len,
                   const int32_t* accepted_nodes, int32_t* new_seq_lens, void* stream);

/* ---- KV transfer for sample migration ----------------------------------
 * (Section 6.2, "Two-stage Sample Migration": phase 1 copies the K/V of the
 * migrating samples out of the cache store into one contiguous buffer, so
 * that the transfer is a single copy; phase 3 parses such a buffer and
 * appends its K/V to the destination store.  Verified K/V never changes
 * (the Markov property the paper relies on), so stage 1 can move the
 * verified prefix [0, S) while the sample keeps running and stage 2 only the
 * tokens verified since: both are a token range [begin, end) per sample.)
 *
 * Buffer layout, the paper's model -> layer -> sample order (this library
 * holds one model, the LLM):
 *   [layer][K=0,V=1][sample j in call order][kv_head][token begin_j .. end_j-1][head_dim]
 * bf16, no padding; its size is spec_kv_transfer_bytes.
 *
 *   sample_ids host [n]  distinct pool samples, 1 <= n <= pool samples
 *   tok_begin  host [n]  first token of each range, 0 <= begin
 *   tok_end    host [n]  one past the last, begin <= end <= capacity
 *                        (empty ranges are allowed and contribute nothing)
 *   buf        device, 16-byte aligned, buf_bytes >= spec_kv_transfer_bytes
 * The buffer belongs to the caller.  Returns SPEC_ERR_CAPACITY for a range
 * outside a sample's capacity or a buffer that is too small; nothing is
 * enqueued then. */

/* Bytes of the transfer buffer for these ranges (0 if an argument is invalid). */
size_t spec_kv_transfer_bytes(const spec_kv* kv, int32_t n, const int32_t* tok_begin,
                              const int32_t* tok_end);

/* Phase 1: copy positions [begin_j, end_j) of every layer, K and V and KV
 * head of sample sample_ids[j] into buf.  Reads the pool only. */
int spec_kv_pack(spec_kv* kv, int32_t n, const int32_t* sample_ids, const int32_t* tok_begin,
                 const int32_t* tok_end, void* buf, size_t buf_bytes, void* stream);

/* Phase 3: the reverse: write buf's runs to positions [begin_j, end_j) of
 * sample sample_ids[j] of this pool (the destination of the migration; the
 * caller raises its committed lengths afterwards).  Reads buf only. */
int spec_kv_unpack(spec_kv* kv, int32_t n, const int32_t* sample_ids, const int32_t* tok_begin,
                   const int32_t* tok_end, const void* buf, size_t buf_bytes, void* stream);

/* ---- Products with weights in 4 bits -----------------------------------
 *
 * Few rows through a model cost the bytes of its weights.  These products take
 * them in 4.25 bits per number: x . W^T as every GEMM here, with W quantised once.
 * spec_verify_w4, below, runs a whole step with them.
 *
 * Numbers.  E2M1 codes times a power of two 2^e that 32 consecutive numbers of a
 * row share, as in the 4-bit cache below, with e >= -120: the smallest exponent in
 * [-120, 125] with which no magnitude of the group exceeds 6 * 2^e (125 if none is;
 * larger numbers take 6 * 2^125), the nearest code, the even one of two equally
 * near, and code 0 for zero.  A group with an infinity or NaN reads as NaN.
 *
 * Layout (spec_w4_bytes).  Rows in tiles of 16, columns in tiles of 128, both
 * padded with zeros.  A row tile holds, for its T column tiles,
 *   codes   [T][64 lanes][16 bytes]: lane l has row l % 16, columns 32 (l / 16)
 *           .. + 31 of the tile, column 2n and 2n + 1 in the low and high half of
 *           byte n: what a lane of the matrix cores takes, in one load
 *   scales  [T][64 lanes] bytes e + 127 (255: none), padded to 256 */
typedef struct {
  const void* data;       /* device, spec_w4_bytes(rows, cols), 256-byte aligned */
  int32_t rows, cols;     /* W is [rows][cols]: cols inputs, rows outputs */
} spec_w4;

/* Bytes of a [rows][cols] matrix in 4 bits; 0 if an argument is invalid (rows >= 1,
 * cols a positive multiple of 32, both at most 2^24). */
size_t spec_w4_bytes(int32_t rows, int32_t cols);

/* Quantise w (device bf16, row r at r * stride; stride in values, a multiple of 8;
 * 16-byte aligned) into data (device, 256-byte aligned, bytes >= spec_w4_bytes). */
int spec_w4_pack(const void* w, int64_t stride, int32_t rows, int32_t cols, void* data, size_t bytes,
                 void* stream);

/* What the matrix stands for, exactly, as bf16 rows of w (as in spec_w4_pack). */
int spec_w4_unpack(const spec_w4* m, void* w, int64_t stride, void* stream);

enum {
  SPEC_W4_BF16 = 0,       /* out = bf16(x W^T) */
  SPEC_W4_F32 = 1,        /* out = x W^T, fp32 (logits) */
  SPEC_W4_ADD = 2         /* out += x W^T, fp32 (a residual stream) */
};

/* Workspace bytes that a product of up to max_n rows of x with one such matrix (or, in
 * spec_w4_gate_up, with two) may need.  May be 0, also if an argument is invalid.  (A search
 * over n, about a microsecond for each, up to 4096 of them: for setting up, not for every call.) */
size_t spec_w4_workspace_bytes(int32_t rows, int32_t cols, int32_t max_n);

/* What a product of n rows needs, with one matrix or (pair 1) two: at most the above for
 * max_n = n, without the search.  May be 0, also if an argument is invalid. */
size_t spec_w4_product_bytes(int32_t rows, int32_t cols, int32_t n, int32_t pair);

/* Products of 0 <= n <= 2^20 rows (n * rows <= 2^34).  The weights enter as the numbers they stand for, sums are
 * fp32, in an order that depends on the shapes and n alone.
 *   x          device bf16 [n][cols], row i at i * x_stride (a multiple of 8, at most 2^28;
 *              16-byte aligned)
 *   out        device, row i at i * out_stride (in values, any stride >= rows; aligned
 *              as its type), of type `kind`
 *   workspace  device, 256-byte aligned; may be NULL where no bytes are needed.  Calls
 *              that can run at once need workspaces of their own.
 * A row of x with an infinity or NaN changes no other row's outputs.  Only launches
 * kernels: can be captured into a graph. */
int spec_w4_linear(const spec_w4* m, const void* x, int64_t x_stride, int32_t n, void* out,
                   int64_t out_stride, int32_t kind, void* workspace, size_t ws_bytes, void* stream);

/* out = bf16(silu(x Wg^T) * (x Wu^T)), out [n][rows]: an FFN's first half.  Both
 * matrices have the same shape; the rest as above. */
int spec_w4_gate_up(const spec_w4* gate, const spec_w4* up, const void* x, int64_t x_stride, int32_t n,
                    void* out, int64_t out_stride, void* workspace, size_t ws_bytes, void* stream);

/* ---- The choice of beams ------------------------------------------------
 *
 * One step of beam search, or the next level of a draft tree: of `groups` samples,
 * each with `width` beams (or tree nodes) that have a score and logits, the k best
 * continuations.
 *   logits       device [groups * width] rows of vocab values, row r at r * row_stride
 *                (in values, >= vocab), fp32 (bf16 = 0) or bf16 (1)
 *   scores       device fp32 [groups][width], e.g. log probabilities so far
 *   last_tokens  device int32 [groups][width], or NULL: the beams' last tokens, read
 *                when eos_token >= 0
 * Candidate (w, y) scores scores[w] + (logits of w)[y] - lse_w in fp64.  The beam's lse_w =
 * log sum exp(logits of w) is one fp64 number, right to 1e-9 (and to its own rounding, which
 * counts more beside logits above 2^22), and the same for equal rows.  A beam whose last
 * token is eos_token has ended: it offers (w, eos_token) alone, at scores[w].  No candidates:
 * tokens whose logit is -infinity; beams whose score is not finite; live beams with a logit
 * that is NaN or +infinity.
 * Outputs, per group the k best, best first, the lower (w, y) of equal scores first:
 *   parents      device int32 [groups][k]  w
 *   tokens       device int32 [groups][k]  y
 *   new_scores   device fp32 [groups][k]   (rounded to fp32 once)
 * Where a group has fewer candidates, the rest is -1, -1 and -infinity.  new_scores may
 * be scores and tokens last_tokens (k == width).
 * 1 <= k <= SPEC_MAX_BEAMS, 1 <= width <= SPEC_MAX_BEAMS, eos_token < vocab.  Only
 * launches kernels; the workspace (device, 256-byte aligned, spec_beam_workspace_bytes) is
 * the call's until they are done. */
#define SPEC_MAX_BEAMS 64

size_t spec_beam_workspace_bytes(int32_t groups, int32_t width, int32_t vocab, int32_t k);
int spec_beam_select(const void* logits, int64_t row_stride, int32_t bf16, int32_t groups, int32_t width,
                     int32_t vocab, const float* scores, const int32_t* last_tokens, int32_t eos_token,
                     int32_t k, int32_t* parents, int32_t* tokens, float* new_scores, void* workspace,
                     size_t ws_bytes, void* stream);

/* ---- The cache rows that follow the beams ------------------------------
 *
 * Beam j of group g, pool sample sample_ids[g][j], continues beam p = parents[g][j]:
 * the K/V of its positions [begin[g], end[g]), all layers, become what sample
 * sample_ids[g][p] holds there before the call, all beams at once (p may be any beam of
 * the group, the same for several).  A p outside [0, width), as spec_beam_select gives
 * where there is no candidate, or equal to j leaves the beam as it is.  Positions before
 * begin (a prompt that all beams share) are not touched.
 *   sample_ids  host [groups][width]   distinct
 *   begin, end  host [groups]          0 <= begin <= end <= every beam's capacity
 *   parents     device int32 [groups][width]
 * 1 <= width <= SPEC_MAX_BEAMS.  A capturing stream is refused: samples and ranges are the
 * call's host values, which a replay would not see change, and large calls upload them. */
int spec_kv_reorder(spec_kv* kv, int32_t groups, int32_t width, const int32_t* sample_ids,
                    const int32_t* begin, const int32_t* end, const int32_t* parents, void* stream);

/* ---- A KV cache in 4 bits, in pages ------------------------------------
 *
 * The bf16 pool above gives every sample one block of fixed capacity.  This
 * one holds K and V in about 4.2 bits per number, in pages of
 * SPEC_KV4_PAGE positions that the caller hands out: a sample grows page by
 * page, and samples of one prompt can share the pages of their common prefix.
 *
 * Numbers.  A number is an E2M1 code (sign, 2 exponent bits, 1 mantissa bit:
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 and negatives) times a power of two 2^e.  32
 * consecutive numbers of a K row share their e, so do all head_dim numbers of
 * a V row.  e is the smallest exponent in [-126, 125] with which no
 * magnitude of the group exceeds 6 * 2^e (125 if none is: 6 * 2^125 is the
 * largest number here, and larger ones take it); a number takes the code
 * nearest to x / 2^e, the even one (0, 1, 2, 4) of two equally near; zero, also
 * a negative one, takes code 0.  A group with an infinity or NaN has no e: it
 * reads as NaN, and rows that see it attend to NaN or infinities.
 * Every reader sees the same numbers, whether a key is a tree node of this
 * step or was committed long ago, so a verified tree gives what one-token
 * steps over the same cache give, up to the attention's roundings.
 *
 * Pages.  Page p lies at byte p * spec_kv4_page_bytes(cfg); in it, layer l
 * and KV head g take 64 * (head_dim + head_dim / 32 + 2) bytes at
 * (l * n_kv_heads + g) times that:
 *   K codes   [2 blocks of 32 keys][head_dim / 32][32 keys][16 bytes]: numbers
 *             2n and 2n + 1 of the 32 in the low and high half of byte n
 *   V codes   [8 octets of keys][32][head_dim / 32][4 bytes]: word (m, i) holds
 *             number 32 i + m of the octet's 8 keys, keys 2n and 2n + 1 in the
 *             low and high half of byte n
 *   K scales  [64 keys][head_dim / 32] bytes e + 127 (255: none)
 *   V scales  [64 keys] bf16 2^e (NaN: none)
 *
 * Use, per model step:
 *   spec_kv4_step_begin    plans the step's rows: once
 *   spec_kv4_append        every layer: the rows' K/V into the cache
 *   spec_kv4_attend        every layer: their attention
 *   spec_kv4_commit        after acceptance, for trees
 * or spec_verify_kv4, which does all but the commit.  spec_kv4_append,
 * _read and _attend only launch kernels: they can be captured into a graph and
 * replayed while the step, its workspace and its pages stay as they are.
 * _step_begin, _commit and spec_verify_kv4 upload descriptors and refuse a
 * capturing stream. */
#define SPEC_KV4_PAGE 64

typedef struct spec_kv4 spec_kv4;             /* opaque pool handle (host, owned by the library) */
typedef struct spec_kv4_step spec_kv4_step;   /* opaque plan of one step */

/* Bytes of one page (all layers and KV heads); 0 if cfg is invalid. */
size_t spec_kv4_page_bytes(const spec_model_config* cfg);

/* Bytes of a pool of n_pages pages for n_samples samples: the pages, padded to
 * 256 bytes, then a control area of 32 bytes per sample, padded alike; 0 if an
 * argument is invalid. */
size_t spec_kv4_bytes(const spec_model_config* cfg, int32_t n_samples, int32_t n_pages);

/* Create a handle over caller memory device_buf (device, >= spec_kv4_bytes,
 * 256-byte aligned).  No sample has pages at first.  One handle must not be used
 * from two threads or two streams at once. */
int spec_kv4_alloc(const spec_model_config* cfg, int32_t n_samples, int32_t n_pages,
                   void* device_buf, size_t buf_bytes, spec_kv4** out);

/* Release the handle (not device_buf, and after its steps).  Waits for the
 * handle's pending uploads. */
int spec_kv4_free(spec_kv4* kv);

/* Set the pages of one sample: positions [64 i, 64 i + 64) lie in page pages[i].
 *   pages  host [n_pages]  distinct ids in [0, pool pages); n_pages may be 0
 * A page may belong to several samples (a shared prefix): it is then read only,
 * and a step or commit that would write to it is refused with
 * SPEC_ERR_INVALID.  Host bookkeeping only: contents stay as they are, and steps
 * begun before keep the pages they were begun with. */
int spec_kv4_map(spec_kv4* kv, int32_t sample, int32_t n_pages, const int32_t* pages);

/* Workspace bytes of a step of up to max_batch samples and max_rows rows, whose
 * keys (committed and new) lie in up to max_pages pages, summed over the
 * samples; 0 if an argument is invalid. */
size_t spec_kv4_step_bytes(const spec_model_config* cfg, int32_t max_batch, int32_t max_rows,
                           int32_t max_pages);

/* Plan a step: sample sample_ids[b] has S_b = seq_lens[b] committed positions and
 * gets T_b = row_offsets[b + 1] - row_offsets[b] >= 1 new rows, in slots S_b + i.
 *   sample_ids   host [batch]    distinct
 *   row_offsets  host [batch+1]  row_offsets[0] = 0
 *   parents      host [N]        trees as in spec_verify (T_b <= SPEC_MAX_TREE):
 *                                row i sits at position S_b + depth(i) and sees the
 *                                committed keys and its ancestors, itself included.
 *                                NULL: runs, of any length: row i sits at position
 *                                S_b + i and sees the keys [0, S_b + i]
 *   seq_lens     host [batch]    S_b >= 0, S_b + T_b <= 64 * (pages of the sample)
 *   workspace    device, 256-byte aligned; the step's until its last launch is done
 * The plan is uploaded on `stream`: launches on another stream are the caller's to order
 * after it.  *out receives the plan; spec_kv4_step_free releases it (host memory only: call
 * it once no more launches are to be made). */
int spec_kv4_step_begin(spec_kv4* kv, int32_t batch, const int32_t* sample_ids,
                        const int32_t* row_offsets, const int32_t* parents, const int32_t* seq_lens,
                        void* workspace, size_t ws_bytes, void* stream, spec_kv4_step** out);
int spec_kv4_step_free(spec_kv4_step* step);

/* Write the K/V of the step's N rows into their slots of one layer.
 *   k, v       device bf16; row r, KV head g, number j at r * stride + g * head_dim + j
 *              (strides in values, multiples of 8; 16-byte aligned), so that a slice
 *              of a fused projection's output can be passed as it is
 *   rotate     nonzero: k is rotated by its position first (rope_theta of the pool's
 *              config; angles, products and sums in double precision, rounded once,
 *              to the code); zero: k has been rotated already
 * Bytes of positions outside the rows' slots are not changed. */
int spec_kv4_append(const spec_kv4_step* step, int32_t layer, const void* k, int64_t k_stride,
                    const void* v, int64_t v_stride, int32_t rotate, void* stream);

/* What the cache holds for the step's rows, exactly, as bf16 (same layout of k and
 * v, which are written). */
int spec_kv4_read(const spec_kv4_step* step, int32_t layer, void* k, int64_t k_stride, void* v,
                  int64_t v_stride, void* stream);

/* Attention of the step's rows over one layer of the cache, their own K/V included
 * (append them first): softmax(q . K / sqrt(head_dim)) V over the keys that each
 * row sees.
 *   q    device bf16, rotated; row r, query head i at r * q_stride + i * head_dim
 *        (q_stride a multiple of 8, 16-byte aligned)
 *   out  device bf16 [N][n_heads * head_dim], 16-byte aligned
 * K and V enter as the numbers they stand for; probabilities are rounded to bf16,
 * sums and softmax statistics are fp32.  Query numbers less than 2^9 below their
 * row's largest are exact; what the others are off by (2^-17 of the largest each at
 * most) comes, summed, to at most 2^-12 of the row's numbers that are more than 16
 * times below the largest, or is 2^-34 of the largest at most each.  V is summed before the
 * division by the softmax's sum: values past 2^96 may overflow fp32 there.  Bitwise
 * the same for the same step, one attend of which runs at a time. */
int spec_kv4_attend(const spec_kv4_step* step, int32_t layer, const void* q, int64_t q_stride,
                    void* out, void* stream);

/* Workspace bytes spec_verify_kv4 needs; max_pages as in spec_kv4_step_bytes, sampled
 * nonzero for a temperature > 0; 0 if an argument is invalid. */
size_t spec_workspace_bytes_kv4(const spec_model_config* cfg, int32_t max_batch, int32_t max_tokens,
                                int32_t max_pages, int32_t sampled);

/* spec_verify (samp NULL) or spec_verify_sampled over this pool: the same arguments
 * and outputs, committed positions in kv's pages (S_b + T_b <= 64 * pages, the pages
 * of positions from S_b on not shared), workspace 256-byte aligned.  K and V leave the
 * projection as bf16 (rotated) and enter the cache, and the attention, in 4 bits. */
int spec_verify_kv4(const spec_model_config* cfg, const spec_weights* w, spec_kv4* kv, int32_t batch,
                    const int32_t* sample_ids, const int32_t* tree_offsets, const int32_t* tree_tokens,
                    const int32_t* tree_parents, const int32_t* seq_lens, void* workspace,
                    size_t ws_bytes, void* stream, const spec_sampling* samp, int32_t* accepted_len,
                    int32_t* next_token, int32_t* accepted_nodes, const spec_debug* dbg);

/* ---- The verify step with weights in 4 bits ----------------------------
 *
 * spec_verify's step with these products in place of the bf16 ones: a draft model's
 * steps, or a target's where its weights' bytes are the cost.  Norm gains and the
 * embedding stay bf16.  Pointers of matrices as in spec_weights, 256-byte aligned. */
typedef struct {
  const void* tok_embed;        /* device bf16 [vocab][hidden] */
  const void* final_norm;       /* device bf16 [hidden] */
  spec_w4 lm_head;              /* [vocab][hidden] */
  const void* const* attn_norm; /* host [n_layers] of device bf16 [hidden] */
  const spec_w4* wqkv;          /* host [n_layers]: [(n_heads + 2 n_kv_heads) * head_dim][hidden],
                                   the rows of q, then of k, then of v */
  const spec_w4* wo;            /* host [n_layers]: [hidden][n_heads*head_dim] */
  const void* const* ffn_norm;  /* host [n_layers] of device bf16 [hidden] */
  const spec_w4* w_gate;        /* host [n_layers]: [ffn][hidden] */
  const spec_w4* w_up;          /* host [n_layers]: [ffn][hidden] */
  const spec_w4* w_down;        /* host [n_layers]: [hidden][ffn] */
} spec_weights_w4;

/* Workspace bytes spec_verify_w4 needs: max_pages 0 for a bf16 pool, otherwise as in
 * spec_workspace_bytes_kv4; 0 if an argument is invalid.  (It holds all nodes' logits in
 * fp32, 525 MB of 1024 nodes and 128256 tokens, for greedy steps too.) */
size_t spec_workspace_bytes_w4(const spec_model_config* cfg, int32_t max_batch, int32_t max_tokens,
                               int32_t max_pages, int32_t sampled);

/* spec_verify (samp NULL) or spec_verify_sampled with w, over the bf16 pool kv (kv4
 * NULL) or the 4-bit one kv4 (kv NULL): otherwise the same arguments, outputs and
 * commit as theirs or spec_verify_kv4's, at most 65535 nodes in all.  Refuses a
 * capturing stream. */
int spec_verify_w4(const spec_model_config* cfg, const spec_weights_w4* w, spec_kv* kv, spec_kv4* kv4,
                   int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets,
                   const int32_t* tree_tokens, const int32_t* tree_parents, const int32_t* seq_lens,
                   void* workspace, size_t ws_bytes, void* stream, const spec_sampling* samp,
                   int32_t* accepted_len, int32_t* next_token, int32_t* accepted_nodes,
                   const spec_debug* dbg);

/* spec_kv_commit for this pool: the codes and scales of node accepted_nodes[b][d]
 * move to position S_b + d for d = 1 .. accepted_len[b], all layers, and
 * new_seq_lens[b] = S_b + accepted_len[b] + 1. */
int spec_kv4_commit(spec_kv4* kv, int32_t batch, const int32_t* sample_ids, const int32_t* seq_lens,
                    const int32_t* accepted_len, const int32_t* accepted_nodes,
                    int32_t* new_seq_lens, void* stream);

/* spec_kv_reorder for this pool: codes and scales move.  The pages of positions
 * [begin[g], end[g]) of every beam must not be shared (SPEC_ERR_INVALID).
 *   workspace  device, 256-byte aligned, spec_kv4_reorder_bytes(kv, groups, width, pages) with
 *              pages >= those that any group's range touches (0 for a small call: it may
 *              be NULL then); the call's until it has run */
size_t spec_kv4_reorder_bytes(const spec_kv4* kv, int32_t groups, int32_t width, int32_t max_pages);
int spec_kv4_reorder(spec_kv4* kv, int32_t groups, int32_t width, const int32_t* sample_ids,
                     const int32_t* begin, const int32_t* end, const int32_t* parents, void* workspace,
                     size_t ws_bytes, void* stream);

/* ---- Drafting-strategy selection (Section 5) ----------------------------
 *
 * Verification-cost predictor (Section 5.2, "the execution time"): a
 * regression on the verification features, in milliseconds,
 *   t_sd = c0 + c_seq * N_seq + c_draft * N_draft + c_tree * TK
 * with N_seq = sum of committed lengths S_b (the KV the attention loads),
 * N_draft = sum of tree sizes T_b (the rows of the FFN products) and
 * TK = sum of T_b * S_b (the attention work that grows with both).  The
 * coefficients are fitted offline on measured steps of this library.
 * Bucket cache: with bucket_ratio r > 0, every feature x > 0 falls in bucket
 * floor(log(x) / log(1 + r)) (0 has its own bucket); all feature triples in
 * one bucket share the prediction at the buckets' geometric midpoints, which
 * is computed once and then read from the cache.  r = 0 disables it. */
typedef struct {
  double c0, c_seq, c_draft, c_tree;
  double bucket_ratio;
} spec_cost_coeffs;

typedef struct spec_cost_model spec_cost_model;   /* opaque, host, owned by the library */

int spec_cost_model_create(const spec_cost_coeffs* coeffs, spec_cost_model** out);
int spec_cost_model_free(spec_cost_model* model);
/* Predicted step time in ms, or a negative value for a negative feature. */
double spec_cost_predict(spec_cost_model* model, int64_t n_seq, int64_t n_draft, int64_t tree_kv);
/* Cache hits and misses since creation. */
int spec_cost_model_stats(const spec_cost_model* model, int64_t* hits, int64_t* misses);

/* Choose the draft token num n (tree nodes per sample, root included) of the
 * next step for a batch (Sections 5.1 and 5.3): n maximises
 * al(n) / t_sd(n), where al(n) = sum over samples of the weights of S_b(n)
 * and t_sd is the predictor above at the features of trees of min(n, |tree|)
 * nodes.  S_b(1) = {root}; S_b(n+1) adds the heaviest unselected node of the
 * sample's candidate tree, taken from a max-priority queue that receives the
 * nodes of layer m (depth m) when the search reaches layer m; equal weights
 * go to the shallower node, then the lower index.  Since weights never grow
 * from parent to child, S_b(n) is a connected tree.  The search over n stops
 * after `patience` consecutive falls of the objective.
 *   seq_lens      host [batch]    committed length S_b of each sample
 *   tree_offsets  host [batch+1]  candidate trees, offsets[0] = 0, sizes >= 1
 *   parents       host [total]    parent within the tree, -1 for node 0,
 *                                 0 <= parent < node otherwise
 *   weights       host [total]    w(u) = F(dl(u)) >= 0, w(child) <= w(parent)
 *   n_max         1 .. SPEC_MAX_TREE
 * Outputs (host): *n_out; selected [batch][n_max], sample b's nodes in the
 * order they joined S_b (the first n form S_b(n)), -1 past the tree's size;
 * objective [n_max] (may be NULL): al(n) / t_sd(n), 0 past the stop. */
int spec_select_draft_count(spec_cost_model* model, int32_t batch, const int32_t* seq_lens,
                            const int32_t* tree_offsets, const int32_t* parents,
                            const float* weights, int32_t n_max, int32_t patience, int32_t* n_out,
                            int32_t* selected, double* objective);

/* Message of the last failure on the calling thread ("" if none). */
const char* spec_last_error(void);

/* ---- Kernel timing (measurement only) ----------------------------------
 * While enabled, every launch of the named kernel class is bracketed by a
 * pair of HIP events on its stream.  spec_profile_end synchronises those
 * events, returns the summed duration in ms and the launch count, and
 * disables timing.  Kernel classes: */
enum {
  SPEC_K_GEMM_QKV = 0,
  SPEC_K_ATTENTION = 1,
  SPEC_K_GEMM_O = 2,
  SPEC_K_GEMM_GATE_UP = 3,
  SPEC_K_GEMM_DOWN = 4,
  SPEC_K_LM_HEAD = 5,
  SPEC_K_COMMIT = 6,
  SPEC_K_TRANSFER = 7,   /* spec_kv_pack / spec_kv_unpack */
  SPEC_K_ACCEPT = 8,     /* tree acceptance: greedy, greedy with EOS, or sampled */
  SPEC_K_KV4_APPEND = 9, /* spec_kv4_append (SPEC_K_ATTENTION: spec_kv4_attend too) */
  SPEC_K_W4 = 10,        /* spec_w4_linear / spec_w4_gate_up.  spec_verify_w4's products are in 0
                            and 2 .. 5, by themselves: what joins their splits, rotates, adds,
                            normalises or takes maxima, which these classes hold in the other
                            steps, is in none */
  SPEC_K_BEAM = 11,      /* spec_beam_select */
  SPEC_K_REORDER = 12,   /* spec_kv_reorder / spec_kv4_reorder */
  SPEC_K_COUNT = 13
};
int spec_profile_begin(int32_t kernel_class, int32_t max_launches);
int spec_profile_end(float* total_ms, int32_t* launches);

/* How a verify step of n_tokens rows runs one of its products (kernel_class
 * SPEC_K_GEMM_QKV, _O, _GATE_UP, _DOWN or SPEC_K_LM_HEAD; host arithmetic, for
 * tests and measurement): rows and columns of its output tile and its K
 * splits.  The few-rows kernel reports a tile of 16 columns and 0 rows. */
int spec_gemm_plan(const spec_model_config* cfg, int32_t kernel_class, int32_t n_tokens,
                   int32_t* tile_rows, int32_t* tile_cols, int32_t* splits);

#ifdef __cplusplus
}
#endif

#endif /* SPECVERIFY_H */
