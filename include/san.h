/*
 * san.h -- C ABI of the shared-attention (SAN) decode library for NVIDIA B200 (sm_100a).
 *
 * The library implements the cached attention of auto-regressive Transformer decoding
 * when attention weights are shared inside blocks of adjacent decoder layers
 * ("Sharing Attention Weights for Fast Transformer", arXiv 1906.11024).
 *
 * Notation follows the paper: S = Softmax(Q.K^T / sqrt(d_k)) are the attention WEIGHTS
 * (Eq. 1) and the attention OUTPUT is S.V (Eq. 2; the paper calls it A, this header calls
 * it O).  In a block of pi adjacent layers only the lowest layer m computes S^m from its
 * own queries and keys; layers m+1 .. m+pi-1 reuse S^m and apply it to their own values
 * (Eq. 3-4).  Hence only block-first layers keep a key cache (Section 3.2, memory note).
 *
 * General rules
 *  - Every function returns a status (SAN_OK = 0).  Nothing throws or traps, and no kernel
 *    spins on another kernel, CTA or rank.  The only device-side waits are a CTA's waits for
 *    its OWN asynchronous copies or tensor-core operations (mbarrier waits in the kernels
 *    behind san_decode_step, san_full_block, san_window_block, san_prefix_attn and san_packed_block), the CTAs of a
 *    cluster meeting one another (san_cache_evict) and the end of
 *    the kernel before on the same stream; an mbarrier wait gives up after about a second and makes
 *    the kernel stop early.  san_decode_step reports it as SAN_ERR_TIMEOUT through
 *    san_device_status, which then also clears the context's split-row tickets so that later
 *    steps start clean; san_prefix_attn and san_packed_block report it in their status words (their outputs are then
 *    undefined); san_full_block and san_window_block have no status word, and a tile whose wait
 *    ran out leaves its output rows unwritten.
 *  - All `d_` pointers are DEVICE pointers owned by the caller; all others are HOST
 *    pointers.  The library allocates no device memory: the cache arena and the
 *    workspace are caller buffers handed to san_create.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  No hot call
 *    synchronises the host.  Calls on one context must be ordered on the device (same
 *    stream, or events between streams): they share the context's workspace.
 *  - Host-checkable mistakes (null pointers, shapes, an invalid policy, a layer outside
 *    the block, capacity) are reported before anything is launched.  Mistakes visible
 *    only on the device (an id out of range, a length < 1 or beyond capacity) make the
 *    kernel skip that item and record the first such error in a device word, read back
 *    with san_device_status.
 *  - Element type is SAN_F32 or SAN_BF16 for q/k/v/x/outputs; S, where it is given or taken, is
 *    always float32; products, sums and the softmax are float32.  d_head must be 64.  Of bf16 inputs the
 *    weights enter their product with the values in bf16 (at most half a step off, 2^-8 relative; their sum is that of
 *    the float32 ones) in san_window_block, san_window_attn, san_prefix_attn, san_packed_block, san_quant_attn (there
 *    times a row's step), the 128-query tiles of san_full_block and kernels 2 and 3 of san_decode_step (san_step_kernel_select): outputs are off by 1.2 to 1.4
 *    times what their own rounding alone is.  The per-warp step kernel and the 64-query tiles of san_full_block
 *    add what the rounding of a weight left as a second bf16 number.
 *  - Sequences are numbered 0 .. max_sent*beam-1; sequence s belongs to sentence
 *    s / beam (the beams of a sentence read the same encoder memory, Section 2).
 *
 * Cache layout inside the arena (head-major; every (id, head) panel is contiguous and
 * each row is 64 elements = 128 B bf16 / 256 B f32, 16-byte aligned).  bf16 rows are stored
 * with their eight 16-byte chunks permuted: chunk c of the row at position pos sits at chunk
 * c ^ (pos & 7), so that a tile of rows copied verbatim into shared memory can be read eight
 * rows at a time without bank conflicts; callers never see this unless they read the arena
 * directly.  float32 rows are stored in natural order.
 *    self K   [self block ][sequence][head][max_tgt_len][64]   (block-first layers only)
 *    self V   [layer      ][sequence][head][max_tgt_len][64]
 *    memory K [encdec block][sentence][head][max_src_len][64]
 *    memory V [layer       ][sentence][head][max_src_len][64]  (one plane per BLOCK when
 *                                                               encdec_shared_context)
 *    AAN sum  [layer][sequence][n_heads*64] float32             (only when self_is_aan)
 */
#ifndef SAN_H_
#define SAN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct san_ctx san_ctx; /* opaque; lives in host memory */

enum {
    SAN_OK = 0,
    SAN_ERR_NULL = 1,         /* a required pointer is NULL */
    SAN_ERR_SHAPE = 2,        /* a size or count is out of range */
    SAN_ERR_POLICY = 3,       /* block sizes / block map do not describe a valid policy */
    SAN_ERR_CAPACITY = 4,     /* a caller buffer is too small, or more blocks than key planes */
    SAN_ERR_DTYPE = 5,
    SAN_ERR_RANGE = 6,        /* layer/block/position outside what the policy or config allows */
    SAN_ERR_CUDA = 7,         /* a CUDA runtime call failed (launch configuration, bad stream...) */
    SAN_ERR_DEVICE_CHECK = 8, /* a kernel met an invalid id/length/position and skipped the item */
    SAN_ERR_TIMEOUT = 9,      /* a kernel's bounded wait for its own copies ran out (see General rules) */
    SAN_ERR_UNSUPPORTED = 10
};
enum { SAN_F32 = 0, SAN_BF16 = 1, SAN_Q4 = 2 }; /* SAN_Q4: cached rows in four bits, see san_planes; no call takes it elsewhere */
enum { SAN_SELF = 0, SAN_ENCDEC = 1 };

#define SAN_MAX_LAYERS 64
#define SAN_MAX_BEAM 32

typedef struct {
    int32_t n_layers;    /* M, 1..SAN_MAX_LAYERS */
    int32_t n_heads;     /* H */
    int32_t d_head;      /* must be 64 */
    int32_t max_sent;    /* sentences the caches have room for */
    int32_t beam;        /* sequences per sentence, 1..SAN_MAX_BEAM */
    int32_t max_tgt_len; /* self-attention cache rows per sequence */
    int32_t max_src_len; /* encoder-memory rows per sentence */
    int32_t dtype;       /* SAN_F32 or SAN_BF16 */
    int32_t self_is_aan; /* 1: decoder self-attention is the cumulative average (san_aan_step) */
    int32_t encdec_shared_context; /* 1: Eq. 5, one O (and one V plane) per enc-dec block */
} san_config;

/* Bytes the caller must provide for a configuration whose self / enc-dec policies have
 * n_self_blocks / n_encdec_blocks blocks (the key-cache planes; Section 3.2: layers that
 * take their weights from another layer keep no keys).  Either output may be NULL. */
int32_t san_query_bytes(const san_config* cfg, int32_t n_self_blocks, int32_t n_encdec_blocks,
                        size_t* cache_bytes, size_t* workspace_bytes);

/* Creates a context over caller-owned device buffers (256-byte aligned).  The sharing
 * policies are given as block sizes {pi_1..pi_N} bottom-up (Section 3.3); their block
 * counts fix the number of key planes carved out of the arena.  Zeroes the workspace
 * header on the default stream and waits for it (the one synchronising call besides
 * san_device_status).  The arena is not cleared. */
int32_t san_create(const san_config* cfg, const int32_t* self_sizes, int32_t n_self,
                   const int32_t* encdec_sizes, int32_t n_encdec, void* d_cache, size_t cache_bytes,
                   void* d_workspace, size_t workspace_bytes, san_ctx** out);
int32_t san_destroy(san_ctx* ctx);

/* Sharing policy (Section 3.3): block sizes bottom-up with sum = n_layers and every size
 * >= 1, or the same thing as a per-layer block id (starts at 0; each next layer keeps the
 * id or raises it by one).  A policy with more blocks than the context has key planes is
 * refused with SAN_ERR_CAPACITY.  Changing the policy does not move cached rows. */
int32_t san_policy_set_sizes(san_ctx* ctx, int32_t kind, const int32_t* sizes, int32_t n_blocks);
int32_t san_policy_set_map(san_ctx* ctx, int32_t kind, const int32_t* block_of_layer, int32_t n_layers);
/* Any output may be NULL.  block_of_layer[n_layers], first_layer_of_block[n_blocks]. */
int32_t san_policy_get_map(const san_ctx* ctx, int32_t kind, int32_t* block_of_layer,
                           int32_t* first_layer_of_block, int32_t* n_blocks);

/* Attention cache (Section 4.1 uses one; Section 2: enc-dec keys/values come from the
 * encoder output).  Copies new rows into the caches of layers [layer_begin, layer_end):
 *   kind = SAN_SELF   d_ids = sequence ids, rows go to the self-attention K/V caches;
 *   kind = SAN_ENCDEC d_ids = sentence ids, rows go to the encoder-memory K/V.
 * Item i writes d_nrows[i] rows (1 if d_nrows is NULL) starting at row d_pos[i] (0 if
 * d_pos is NULL).  Source layout, `rows_per_item` = row capacity of one item (>= every
 * d_nrows[i]; 1 for a decode step):
 *   d_v_new [layers in range          ][n_items][rows_per_item][H][64]
 *   d_k_new [block-first layers in range][n_items][rows_per_item][H][64]   (in layer order)
 * d_k_new must be NULL iff the range holds no block-first layer.  With
 * encdec_shared_context only block-first layers may be in an ENCDEC range.
 * Not allowed for SAN_SELF when self_is_aan.  Payload is copied bit for bit. */
int32_t san_cache_append(san_ctx* ctx, int32_t kind, int32_t layer_begin, int32_t layer_end,
                         const void* d_k_new, const void* d_v_new, const int32_t* d_ids,
                         const int32_t* d_pos, const int32_t* d_nrows, int32_t n_items,
                         int32_t rows_per_item, void* stream);

/* Eq. 1 for one decode step, at the lowest layer of `block` (Eq. 3):
 *   S[j] = exp(z_j - max z) / sum_j exp(z_j - max z),  z_j = (q . K_j) / sqrt(64),
 * over cached rows j in [0, d_lens[i]).
 *   kind = SAN_SELF    d_ids sequence ids; d_q [n_items][H][64]; d_S [n_items][H][ld_s]
 *   kind = SAN_ENCDEC  d_ids sentence ids; d_q [n_items][beam][H][64];
 *                      d_S [n_items][beam][H][ld_s]; d_lens[i] = source length; every
 *                      key tile is read once for all beams of the sentence.
 * max_len is a host-side upper bound on d_lens (1..capacity; 0 = capacity) used to size
 * the launch; a longer length is a device-check error.  ld_s >= max_len.  Entries of a
 * row beyond its length are left untouched.  Long rows are split over several warps
 * (partial max/sum in the workspace, combined by the last warp to finish; nothing waits). */
int32_t san_attn_weights(san_ctx* ctx, int32_t kind, int32_t block, const void* d_q,
                         const int32_t* d_ids, const int32_t* d_lens, int32_t n_items,
                         int32_t max_len, float* d_S, int64_t ld_s, void* stream);

/* Eq. 2 with Eq. 4: for every layer l in [layer_begin, layer_end), all inside `block`,
 *   O_l = sum_{j in [p0, p1)} S[j] * V_l[j]
 * with the block's weights S (layout as written by san_attn_weights) and each layer's own
 * cached values, in one launch; S is staged on chip once per work item and reused for
 * every layer.  p0 = d_pos_begin[i] (0 if NULL), p1 = d_pos_end[i].
 *   d_out [layer_end-layer_begin][n_items]([beam])[H][64], element type = cfg.dtype
 *         (rounded to nearest even from float32 for bf16).
 * accumulate != 0 adds to what d_out holds (for finishing a layer whose newest value row
 * arrived after the block's history was applied).  With encdec_shared_context (Eq. 5) an
 * ENCDEC call must name exactly the block's first layer; the one output serves the block.
 * max_len bounds d_pos_end as in san_attn_weights. */
int32_t san_attn_apply(san_ctx* ctx, int32_t kind, int32_t block, int32_t layer_begin,
                       int32_t layer_end, const float* d_S, int64_t ld_s, const int32_t* d_ids,
                       const int32_t* d_pos_begin, const int32_t* d_pos_end, int32_t n_items,
                       int32_t max_len, void* d_out, int32_t accumulate, void* stream);

/* Average attention in place of decoder self-attention (the AAN model the paper combines
 * with SAN in Table 6): for layers [layer_begin, layer_end) and item i with sequence
 * d_ids[i] at 1-based target position d_t[i]:
 *   sum_l[seq] += x_l[i];  out_l[i] = sum_l[seq] / d_t[i]      (mean of positions 1..t)
 * d_t[i] == 1 restarts the sum from x.  d_x, d_out: [layers in range][n_items][H*64]. */
int32_t san_aan_step(san_ctx* ctx, int32_t layer_begin, int32_t layer_end, const void* d_x,
                     const int32_t* d_ids, const int32_t* d_t, int32_t n_items, void* d_out,
                     void* stream);

/* Forget the history of the listed sequences under average attention (Table 6 pairing): the
 * running sums of every layer are set to zero for each sequence d_seq_ids[i], i < n, so that
 * a cache slot can be handed to another hypothesis or sentence at any point of its count.
 * After the call the next san_aan_step at position t returns x / t for such a sequence, as
 * if its earlier inputs had been zero; restarting the count at t = 1 needs no reset (that
 * step overwrites the sum).  Only for contexts with self_is_aan (else SAN_ERR_UNSUPPORTED).
 * An id outside 0 .. max_sent*beam-1 is skipped and reported through san_device_status. */
int32_t san_seq_reset(san_ctx* ctx, const int32_t* d_seq_ids, int32_t n, void* stream);

/* One whole decode step in ONE launch: for every block of both attention kinds, append
 * this step's rows (Section 4.1 cache), compute the block's weights at its lowest layer
 * (Eq. 1, Eq. 3) and apply them to the values of every layer of the block (Eq. 2, Eq. 4;
 * Eq. 5 with encdec_shared_context); with self_is_aan the cumulative average replaces
 * the self-attention part.  Same arithmetic and outputs as the sequence
 *     san_cache_append(SELF, 0..M) ; per block san_attn_weights + san_attn_apply
 * for inputs laid out for all layers at once (a caller that has every layer's q/k/v of
 * the step up front, e.g. a benchmark or a speculative/batched front end):
 *   d_q_self, d_k_new [n_self_blocks][n_seqs][H][64]   rows of the block-first layers
 *   d_v_new           [n_layers][n_seqs][H][64]
 *   d_seq_ids, d_pos  sequence ids and the row each writes this step (length = pos + 1)
 *   d_S_self          [n_self_blocks][n_seqs][H][ld_t] float32, or NULL if not wanted
 *   d_O_self          [n_layers][n_seqs][H][64]
 *   d_q_enc           [n_encdec_blocks][n_sent][beam][H][64]
 *   d_sent_ids, d_src_lens   sentence ids and their source lengths
 *   d_S_enc           [n_encdec_blocks][n_sent*beam][H][ld_s] float32, or NULL
 *   d_O_enc           [n_layers (or n_encdec_blocks with Eq. 5)][n_sent*beam][H][64]
 *   d_x_aan, d_t      [n_layers][n_seqs][H*64] and 1-based positions (self_is_aan only;
 *                     the averages go to d_O_self)
 * n_seqs == 0 skips the self/AAN part, n_sent == 0 the enc-dec part.  max_len / max_src
 * are host bounds on pos+1 / source lengths (0 = capacity).  Rows longer than the on-chip
 * score buffer are split into at most 32 spans; a bound that would need more returns
 * SAN_ERR_UNSUPPORTED (use the separate calls).  The kernel's waits on its own copies are
 * bounded: if one runs out the step reports SAN_ERR_TIMEOUT through san_device_status.  A beam
 * wider than 8 takes one launch per group of 8 query rows. */
typedef struct {
    const void* d_q_self; const void* d_k_new; const void* d_v_new;
    const int32_t* d_seq_ids; const int32_t* d_pos; int32_t n_seqs; int32_t max_len;
    float* d_S_self; int64_t ld_t; void* d_O_self;
    const void* d_q_enc; const int32_t* d_sent_ids; const int32_t* d_src_lens; int32_t n_sent; int32_t max_src;
    float* d_S_enc; int64_t ld_s; void* d_O_enc;
    const void* d_x_aan; const int32_t* d_t;
} san_step_args;
int32_t san_decode_step(san_ctx* ctx, const san_step_args* args, void* stream);

/* Which kernel san_decode_step launches, and (for testing and tuning) how its rows are cut.
 * The library has three implementations of the one-launch step (same arithmetic, Eq. 1-5):
 *   which = 1  per-warp pipeline: every warp streams the tiles of its own row (float32 and bf16);
 *   which = 2  team pipeline (bf16): four producer warps each stream bundles of two units to a team
 *              of two warps, a unit being up to four heads of one sequence or one of two spans of
 *              a long row; SAN_ERR_UNSUPPORTED from the step if a shape does not fit;
 *   which = 3  short rows (bf16, max_len and max_src at most 96): a warp fetches whole planes of 1, 2
 *              or 4 heads (heads_per_unit; fewer where they would not fit its ring) and keeps the
 *              scores in registers; layers_per_unit as below; SAN_ERR_UNSUPPORTED from the step
 *              if the bounds are larger;
 *   which = 0  automatic (the default): the team pipeline for steps whose rows are long enough to be
 *              split over the warps of a team, the short-rows kernel for launches that hold
 *              encoder-decoder attention alone (where each measured faster), else the per-warp one.
 * A value may carry a second one for encoder-decoder attention in its bits 8 and up, as (v + 1) << 8.
 * spans_log2 >= 0 overrides the automatic cut of the team pipeline: every row is dealt to
 * 1 << spans_log2 warps (0..1); with one span up to heads_per_unit (1, 2 or 4) heads of one
 * sequence or sentence go to a warp where the head count allows (at most 2 where several
 * beams share a key tile); tiles hold tile_pos positions (a multiple of 16);
 * layers_per_unit > 0 caps the layers one warp applies (the block's other layers go to
 * further warps, which recompute S); grab_mult >= 1 makes the bundles shrink earlier towards
 * the end of the launch.  spans_log2 < 0 restores the automatic cut. */
int32_t san_step_kernel_select(san_ctx* ctx, int32_t which, int32_t spans_log2, int32_t heads_per_unit,
                               int32_t tile_pos, int32_t layers_per_unit, int32_t grab_mult);

/* Which kernel the last san_decode_step of this context launched (1, 2 or 3 as above, 0 before the
 * first step) and, for the team pipeline and the short-rows kernel, how many heads of one sequence / sentence it gave
 * to one warp: rows_per_unit[0] for self-attention, [1] for encoder-decoder attention (may
 * be NULL).  For tests and benchmarks that must know what they measured. */
int32_t san_step_kernel_used(const san_ctx* ctx, int32_t* which, int32_t* rows_per_unit);

/* san_decode_step for a caller whose step inputs and outputs live in HOST memory (pinned
 * memory if the copies are to overlap anything): the same step (Eq. 1-5, Section 4.1) with
 * the transfers issued by the library on `stream`, in order: every input array named in
 * `host` is copied into the array of the same field in `dev`, san_decode_step(ctx, dev) is
 * launched, then O_self and O_enc (and S_self / S_enc where both structs name a buffer) are
 * copied back into `host`.  `dev` is a complete argument block of caller-owned device
 * buffers and carries the counts, bounds and leading dimensions; the pointer fields of
 * `host` are HOST pointers of the same shapes (its scalar fields are ignored).  Nothing is
 * allocated and the host is not synchronised: `host` outputs are valid once `stream` has
 * reached this point, and `host` inputs must stay untouched until then. */
int32_t san_decode_step_host(san_ctx* ctx, const san_step_args* host, const san_step_args* dev, void* stream);

/* Beam-search cache reorder (Section 4.1: decoding runs a beam of hypotheses per sentence;
 * after a step each surviving hypothesis continues the attention cache of the hypothesis it
 * extends).  For item i = sentence d_sent_ids[i] and beam slot s, the sequence
 * sentence*beam + s takes over the first d_lens[i*beam + s] cached rows of the sequence
 * sentence*beam + d_parent[i*beam + s], in every self-attention key plane (one per block:
 * Section 3.2, shared layers keep no keys, so sharing shrinks this step too) and every
 * value plane; with self_is_aan it takes over the parent's running sum instead (when the
 * length is > 0).  d_parent holds beam slots 0..beam-1 of the SAME sentence, which is what
 * lets the gather run in place: all rows are read before any is written, as if copied
 * through a snapshot.  Slots with d_parent == s keep their rows and cost nothing.
 * Encoder memory is per sentence and is not touched.  max_len is a host bound on d_lens
 * (0 = capacity).  A parent outside 0..beam-1, a length outside 0..max_len or a sentence id
 * out of range skips that slot and is reported through san_device_status.  Bit copy. */
int32_t san_beam_reorder(san_ctx* ctx, const int32_t* d_sent_ids, const int32_t* d_parent,
                         const int32_t* d_lens, int32_t n_sent, int32_t max_len, void* stream);

/* Full-sequence shared attention (the encoder-side use of Table 5; with causal != 0 the
 * prefill of a decoder prompt): for every sequence i and head, the l x l weights
 *   S = Softmax(Q.K^T / sqrt(64)),  l = d_lens[i],  query row a over keys 0..l-1 (0..a when causal)
 * are computed once from the queries and keys of the block's lowest layer (Eq. 1, Eq. 3) and
 * applied to the values of each of the block's n_layers layers (Eq. 2, Eq. 4) in the same
 * launch.  Needs no context and allocates nothing.
 *   d_q, d_k  [n_seq][cap_len][n_heads][64]            (the order a projection writes them)
 *   d_v       [n_layers][n_seq][cap_len][n_heads][64]
 *   d_out     [n_layers][n_seq][cap_len][n_heads][64]  rows at or beyond d_lens[i] are not written
 *   d_S       optional [n_seq][n_heads][cap_len][ld_s] float32; entries a row does not attend
 *             to (causal) are written as 0, entries at or beyond d_lens[i] are not written
 * dtype must be SAN_BF16 (SAN_F32 is refused with SAN_ERR_UNSUPPORTED: tensor-core products
 * of float32 inputs would not meet the float32 tolerance).  max_len is a host bound on d_lens
 * (0 = cap_len); a longer length is cut to max_len.  It also selects the kernel: a bound of
 * 128 or more with n_layers <= 6 runs 128-query tiles on the tcgen05 tensor cores with the
 * accumulators in tensor memory (any length); otherwise 64-query tiles on mma.sync, for which
 * max_len above 512 is SAN_ERR_UNSUPPORTED. */
int32_t san_full_block(int32_t dtype, int32_t n_heads, int32_t n_layers, int32_t causal, const void* d_q,
                       const void* d_k, const void* d_v, const int32_t* d_lens, int32_t n_seq, int32_t cap_len,
                       int32_t max_len, float* d_S, int64_t ld_s, void* d_out, void* stream);

/* Policy learning (Section 3.1, Section 3.3, Eq. 6).
 *
 * san_js_matrix: the Jensen-Shannon divergence between the attention weights of every pair
 * of layers, JS(p,q) = (KL(p||m) + KL(q||m))/2 with m = (p+q)/2 and natural logarithms, one
 * value per (row, head) distribution and averaged over all of them (heads count as separate
 * channels).  d_S holds the weights of n_layers layers of an unshared model (block size 1) as
 * the decode step writes them: layer l at d_S + l*layer_stride, each [n_rows][n_heads][ld_s]
 * float32 with d_lens[row] valid positions (clamped to 0..ld_s).  d_js receives the
 * n_layers x n_layers symmetric matrix (float64, zero diagonal); it is cleared first.  Needs
 * no context and allocates nothing.
 *
 * san_block_similarity (host): Eq. 6 for the block of layers m..n (0-based, m < n),
 *   sim(m,n) = sum_{i != j in m..n} (ln 2 - JS(i,j)) / ((n-m+1)(n-m)).
 * san_policy_search (host): the bottom-up search of Section 3.3; starting at the lowest layer
 * a block grows while the similarity of the block with the next layer added is >= theta and
 * closes at the first failure (a block of one layer always qualifies); sizes[] (room for
 * n_layers entries) receives {pi_i}, ready for san_policy_set_sizes. js is a HOST matrix. */
int32_t san_js_matrix(int32_t n_layers, const float* d_S, int64_t layer_stride, int64_t ld_s,
                      int32_t n_rows, int32_t n_heads, const int32_t* d_lens, double* d_js, void* stream);
int32_t san_block_similarity(const double* js, int32_t n_layers, int32_t m, int32_t n, double* sim);
int32_t san_policy_search(const double* js, int32_t n_layers, double theta, int32_t* sizes, int32_t* n_blocks);

/* ------------------------------------------------------------------------------------------
 * Around the decode step of a beam decoder with long prompts.  None of these calls needs a
 * context or allocates: workspaces are caller buffers (256-byte aligned, contents of no importance between calls; calls
 * whose kernels may overlap on the device need a workspace each).  The *_bytes functions give the size that a call with
 * these arguments makes full use of.  A workspace sized for the largest batch serves smaller ones: san_beam_select needs no
 * more for fewer sentences, beams or tokens; the attention calls take any size from two partial results a query
 * row (one for a prefix and one for own rows; none for san_window_attn) on and cut rows into fewer runs where it is less than
 * they would use.  `d_status` is an optional device int32[8] that the caller has
 * zeroed: the first item skipped because of its id, length or position is recorded there as
 * [0] = SAN_ERR_DEVICE_CHECK, [1..4] = kernel tag, item, value, limit, and stays until the
 * caller clears it.  The current device at the call is the one that owns the stream and the
 * buffers.  All may be captured into a CUDA graph. */

/* Beam search's selection (Section 4.1 decodes with beam 4, Figure 5 with 4 to 20): the `beam` best
 * continuations of every sentence, chosen over all of its hypotheses and the vocabulary.
 * Hypothesis b of sentence s is row s*beam + b of every array.
 *   - a hypothesis that is not done offers every token v with the score
 *         d_score[row] + log Softmax(d_logits[row])[v]          and the length d_len[row] + 1;
 *   - one that is done (d_done != 0) offers itself alone, unchanged; its token counts as eos;
 *   - one whose score is not finite (a beam slot not in use yet: -inf) offers nothing.
 * Candidates are ranked by score / ((5 + length) / 6)^alpha (alpha = 0: by score), ties go to the
 * lowest slot, then the lowest token.  A logit of -inf or NaN is a masked token: it is never
 * chosen and adds nothing to the sum; logits of +inf share the row's probability among them.
 * Outputs, best first:
 *   d_parent[row]     the slot (0..beam-1) it descends from: what san_beam_reorder takes
 *   d_next[row]       its newest token (eos for a hypothesis that was done)
 *   d_score_out, d_len_out, d_done_out   its state (done: it was, or the new token is eos)
 *   d_tokens_out      its history: the parent's first len tokens and, unless the parent was done,
 *                     the new one; entries from the new length on are not written
 * Where a sentence has fewer candidates than slots, the slots left over come out as done, with
 * score -inf, parent = the slot itself, token eos (0 without eos) and the slot's old length and history.
 * Outputs may be the inputs' own buffers (d_tokens_out = d_tokens with the same ld_tokens, ...).
 * Scores are compared in double.  A row's sum of exponentials has float32 terms, added in float32 within
 * a thread's 8 to 32 logits of a step and in double beyond: within 3e-6 relative at worst, whatever the vocabulary.
 * Rows that hold the same logits in another order, or all of them moved by a constant, may differ by that and then do
 * not tie; a row of one token (the others masked) offers it at the hypothesis' score, exactly.
 * A length outside 0..ld_tokens, ld_tokens itself where a token has to be added, or a length whose ((5 + length) / 6)^alpha
 * is not within 10^-250 .. 10^250 (an alpha far from 0), skips the sentence (its outputs are not written) and is reported. */
typedef struct {
    int32_t dtype;            /* of d_logits: SAN_F32 or SAN_BF16 */
    int32_t n_sent, beam, vocab;      /* beam 1..SAN_MAX_BEAM */
    const void* d_logits;     /* [n_sent*beam][ld_logits], any element-aligned address */
    int64_t ld_logits;        /* >= vocab */
    int32_t eos;              /* 0..vocab-1, or -1: no token ends a hypothesis */
    float alpha;              /* length exponent, finite */
    const float* d_score; const int32_t* d_len; const int32_t* d_done;       /* [n_sent*beam] */
    const int32_t* d_tokens; int64_t ld_tokens;     /* [n_sent*beam][ld_tokens], or both token arrays NULL; 1..0x7fff0000 */
    float* d_score_out; int32_t* d_len_out; int32_t* d_done_out; int32_t* d_tokens_out;
    int32_t* d_parent; int32_t* d_next;
    void* d_workspace; size_t workspace_bytes;
    int32_t* d_status;        /* optional */
} san_select_args;
int32_t san_beam_select_bytes(int32_t n_sent, int32_t beam, int32_t vocab, size_t* workspace_bytes);
int32_t san_beam_select(const san_select_args* args, void* stream);

/* Where a context keeps the cached rows of a block: the key plane of the block's lowest layer, the value
 * plane of the same layer, and the distance between the value planes of successive layers in elements
 * (kind SAN_SELF: planes [sequence][head][max_tgt_len][64]; SAN_ENCDEC: [sentence][head][max_src_len][64]).
 * With encdec_shared_context (Eq. 5) an encoder-decoder block has a single value plane and a single output: the distance
 * is 0, and the calls below take such a block with n_layers = 1 alone (SAN_ERR_SHAPE otherwise).
 * SAN_ERR_UNSUPPORTED for SAN_SELF with self_is_aan.  The addresses stay valid until the policy changes. */
int32_t san_cache_planes(const san_ctx* ctx, int32_t kind, int32_t block, void** d_k, void** d_v, int64_t* v_stride);

/* Query rows of one decode step and the cached rows behind them, for san_window_attn and
 * san_prefix_attn: item i is sequence d_ids[i] with d_lens[i] cached rows (this step's row among them).
 * The planes have the context's layout (san_cache_planes; chunk-permuted bf16 rows).  n_heads is a
 * multiple of n_kv_heads: query head h reads key head h / (n_heads / n_kv_heads). */
typedef struct {
    int32_t dtype, n_heads, n_kv_heads;
    int32_t n_layers;         /* layers that share the weights (Eq. 4): value planes and outputs */
    const void* d_q;          /* [n_items][n_heads][64], 16-byte aligned as all of these */
    const void* d_k;          /* [max_ids][n_kv_heads][cap_len][64] */
    const void* d_v;          /* [n_layers] planes like d_k, v_stride elements apart (a multiple of 64) */
    int64_t v_stride;
    int32_t max_ids, cap_len;
    const int32_t* d_ids; const int32_t* d_lens;
    int32_t n_items;
    int32_t max_len;          /* host bound on d_lens (0 = cap_len) */
    void* d_out;              /* [n_layers][n_items][n_heads][64] */
    int32_t* d_status;        /* optional */
} san_cached_rows;

/* Prefixes shared by rows of the batch: prefix g stands in front of the items d_first[g] ..
 * d_first[g+1]-1 (items before d_first[0] or from d_first[n_prefix] on have none).  Rows in the order a
 * projection (and san_full_block, san_window_block) has them, so that a prompt's keys and values
 * can be used where they are. */
typedef struct {
    const void* d_k;          /* [n_prefix][cap_len][n_kv_heads][64], 16-byte aligned */
    const void* d_v;          /* [n_layers] arrays like d_k, v_stride elements apart (a multiple of 64) */
    int64_t v_stride;
    int32_t n_prefix, cap_len;
    const int32_t* d_lens;    /* [n_prefix], 0..max_len */
    int32_t max_len;          /* host bound on d_lens (0 = cap_len) */
    const int32_t* d_first;   /* [n_prefix + 1], ascending */
    int32_t max_group;        /* host bound on the items of a prefix (0 = n_items).  Kernels and cuts are chosen by it, so that a
                                 close one is worth giving where there are several prefixes: results do not depend on it */
} san_shared_prefix;

/* One decode step of attention over a sliding window with sinks: with len = d_lens[i], row j is seen if
 *     j >= len - window   or   j < n_sink,
 *     S = Softmax(q . K^T / 8) over the rows seen,   O_l = sum_j S[j] V_l[j]   for every layer l.
 * Rows that are not seen are not read.  window >= 1, n_sink >= 0.  len = 0 gives zeros, and so does a row whose scores
 * are all -infinity (here and in the two calls below).  An id or length out
 * of range leaves the item's output as it was and is reported. */
int32_t san_window_attn_bytes(const san_cached_rows* rows, int32_t window, int32_t n_sink, size_t* workspace_bytes);
int32_t san_window_attn(const san_cached_rows* rows, int32_t window, int32_t n_sink, void* d_workspace,
                        size_t workspace_bytes, void* stream);

/* One decode step of attention for rows behind shared prefixes: softmax and outputs as above over the
 * prefix's rows and all of the item's own ones together.  A prefix is read from memory once for all of its
 * items (eight query rows at a time, from L2 after the first; 256 with tensor-core tiles).  A row that sees nothing
 * (no prefix rows, len 0) gives zeros.  A prefix whose length, first item or number of items is out of range
 * leaves the outputs of its items as they were and is reported. */
int32_t san_prefix_attn_bytes(const san_cached_rows* rows, const san_shared_prefix* prefix, size_t* workspace_bytes);
int32_t san_prefix_attn(const san_cached_rows* rows, const san_shared_prefix* prefix, void* d_workspace,
                        size_t workspace_bytes, void* stream);

/* The whole-sequence form of san_window_attn, for prompts: san_full_block with causal != 0 and a window. Query
 * row a of a sequence sees key row b <= a if b > a - window or b < n_sink.
 *   d_q, d_out  [n_seq][cap_len][n_heads][64] and [n_layers][n_seq][cap_len][n_heads][64]
 *   d_k, d_v    [n_seq][cap_len][n_kv_heads][64] and [n_layers][n_seq][cap_len][n_kv_heads][64]
 * (16-byte aligned).  Rows at or beyond d_lens[i] are neither read nor written; a length is cut to
 * 0..max_len (0 = cap_len) as in san_full_block.  SAN_BF16 only (SAN_F32: SAN_ERR_UNSUPPORTED, for the reason
 * given there).  What a row does not see does not reach it, infinities and NaN included. */
int32_t san_window_block(int32_t dtype, int32_t n_heads, int32_t n_kv_heads, int32_t n_layers, int32_t window,
                         int32_t n_sink, const void* d_q, const void* d_k, const void* d_v, const int32_t* d_lens,
                         int32_t n_seq, int32_t cap_len, int32_t max_len, void* d_out, void* stream);

/* ------------------------------------------------------------------------------------------
 * Long prompts, and a cache that is kept small: prompts without padding, cached rows in four bits a number, and the rows that
 * receive least attention given up.  The rules of the calls above hold for these too: no context, nothing allocated, caller's
 * workspaces (256-byte aligned, contents of no importance between calls, one for each call that may overlap another; sized by the *_bytes
 * functions, and one sized for the largest batch serves smaller ones), optional d_status, all may be captured into a CUDA graph.  An id is named by one item of a call at most,
 * except where rows are only read. */

/* Causal attention of whole prompts laid end to end: sequence s is the tokens d_first[s] .. d_first[s+1]-1, and token a sees the
 * tokens b <= a of its sequence,
 *     S = Softmax(Q . K^T / 8) over those,   O_l = S . V_l   for every layer l of the block (Eq. 1 - 4).
 * Query head h reads key head h / (n_heads / n_kv_heads).  Tokens may lie further apart than their numbers are long (q, k and v of
 * one fused projection): ld_q, ld_k, ld_v are elements between tokens, multiples of 8.  Sequences may be empty.  Tokens that belong to no
 * sequence keep their outputs as they were.  What a token does not see does not reach it, infinities and NaN included (rows beside such values are
 * computed a second time, one by one: some 30 ms for 32 of them in a sequence of 32768).  A quarter of the exponentials of bounds of 128 and more are
 * off by up to 1.0e-4, which the rounding of the weights to bf16 covers; the others, and all of shorter bounds, by 2^-22.
 * SAN_BF16 only (SAN_F32: SAN_ERR_UNSUPPORTED, for the reason given for san_full_block).  A sequence that does not lie within the
 * tokens or is longer than max_len is skipped and reported, and so is a tile of sequences that overlap in more tokens than there are. */
typedef struct {
    int32_t dtype, n_heads, n_kv_heads, n_layers;
    const void* d_q; int64_t ld_q;        /* [n_tokens][n_heads][64], ld_q elements between tokens; 16-byte aligned as all of these */
    const void* d_k; int64_t ld_k;        /* [n_tokens][n_kv_heads][64] */
    const void* d_v; int64_t ld_v; int64_t v_stride;        /* [n_layers] of those, v_stride elements apart (a multiple of 8) */
    const int32_t* d_first;               /* [n_seq + 1], ascending */
    int32_t n_seq, n_tokens;              /* 2^28 each at most */
    int32_t max_len;                      /* host bound on the lengths (0 = n_tokens); kernels are chosen by it: below 128
                                             n_seq times the layers' groups of four is at most 65535, from there on (n_tokens / 256 + n_seq) *
                                             n_heads times the groups of two below 2^31 */
    void* d_out;                          /* [n_layers][n_tokens][n_heads][64] */
    int32_t* d_status;                    /* optional */
} san_packed_args;
int32_t san_packed_block_bytes(const san_packed_args* args, size_t* workspace_bytes);
int32_t san_packed_block(const san_packed_args* args, void* d_workspace, size_t workspace_bytes, void* stream);

/* Planes of cached rows of a block: its keys and each layer's values.
 *   SAN_F32, SAN_BF16   [max_ids][n_kv_heads][cap_len][64], as a context keeps them (san_cache_planes)
 *   SAN_Q4              codes [max_ids][n_kv_heads][cap_len][32 bytes] and scales [max_ids][n_kv_heads][cap_len][2] bf16, in the
 *                       caller's own buffers: 36 bytes a row.  Dim d is in byte d / 2, even ones in its low half.  A row reads as
 *                           low + step * n,   n its codes 0..15, (step, low) its scales.
 * v_stride: elements between the layers' value planes, 64 a row in every format (a multiple of 64). */
typedef struct {
    int32_t dtype, n_kv_heads, n_layers;
    void* d_k; void* d_v; int64_t v_stride;         /* 16-byte aligned */
    void* d_k_scale; void* d_v_scale;               /* SAN_Q4 alone: [n_layers] of the latter, v_stride / 64 rows apart */
    int32_t max_ids, cap_len;
} san_planes;

/* Rows into a cache of four bits, and back as numbers.  Item i's rows are n = d_nrows[i] (rows_per_item where d_nrows is NULL) from
 * row d_pos[i] (0 where it is NULL) of id d_ids[i] on; the other side is in the order a projection writes it,
 *     keys [n_items][rows_per_item][n_kv_heads][64],   values [n_layers][n_items][rows_per_item][n_kv_heads][64]   of `dtype`
 * (SAN_F32 or SAN_BF16; rows beyond n are neither read nor written; rows_per_item may be more than cap_len where d_nrows is given).
 * Of a row x:  low = min x rounded down to bf16, step = (max x - low) / 15 rounded up to bf16 and, unless it is 0, to 2^-50 at least,
 * n = (x - low) / step rounded to the nearest, half to even (0 where step is 0), of the exact quotients: no number is off by more than
 * step / 2.  A row with a NaN or a number of 2^40 or more reads as NaN.  san_quant_read gives the float32 number next to low + step * n, rounded
 * once more where `dtype` is bf16.
 * An id, a number of rows or a place out of range skips the item and is reported.  (1 + n_layers) * n_items * rows_per_item *
 * n_kv_heads is below 2^31. */
int32_t san_quant_append(const san_planes* cache, int32_t dtype, const void* d_k_new, const void* d_v_new, const int32_t* d_ids,
                         const int32_t* d_pos, const int32_t* d_nrows, int32_t n_items, int32_t rows_per_item,
                         int32_t* d_status, void* stream);
int32_t san_quant_read(const san_planes* cache, int32_t dtype, void* d_k, void* d_v, const int32_t* d_ids, const int32_t* d_pos,
                       const int32_t* d_nrows, int32_t n_items, int32_t rows_per_item, int32_t* d_status, void* stream);

/* One decode step of attention over a cache of four bits: item i is one query position over the first d_lens[i] rows of id d_ids[i]
 * (this step's row among them; several items may read one id),
 *     S = Softmax(q . K^T / 8),   O_l = S . V_l   for every layer l of the block,
 * K and V being what the rows read as.  len = 0 gives zeros, and so does a row whose scores are all -infinity; rows behind the length are not
 * read.  A query row with a NaN or a number of 2^40 or more gives NaN; scales are such as san_quant_append writes.  d_S, where it is given, receives the weights as san_attn_weights writes
 * them (entries behind a row's length are left as they were): what san_weight_mass takes.
 * float32 queries are answered in float32's accuracy: the cache's codes are whole numbers, nothing else is rounded. */
typedef struct {
    int32_t dtype, n_heads;               /* SAN_F32 or SAN_BF16; n_heads a multiple of the planes' n_kv_heads */
    const void* d_q;                      /* [n_items][n_heads][64], 16-byte aligned */
    const int32_t* d_ids; const int32_t* d_lens;
    int32_t n_items;
    int32_t max_len;                      /* host bound on d_lens (0 = cap_len) */
    float* d_S; int64_t ld_s;             /* optional: [n_items][n_heads][ld_s], ld_s >= max_len */
    void* d_out;                          /* [n_layers][n_items][n_heads][64], 16-byte aligned */
    int32_t* d_status;                    /* optional */
} san_step_rows;
int32_t san_quant_attn_bytes(const san_planes* cache, const san_step_rows* rows, size_t* workspace_bytes);
int32_t san_quant_attn(const san_planes* cache, const san_step_rows* rows, void* d_workspace, size_t workspace_bytes, void* stream);

/* The mass of cached rows: what they have received of the weights.  For item i with len = d_lens[i], key head k and j < len
 *     m[j] = (decay * m[j] where j < d_begin[i], else 0) + sum over r < rows and the query heads h of k of S[i][r][h][j],
 * m = d_mass[d_ids[i]][k]; entries behind len are left as they were.  d_begin (0 .. len; NULL: len) is where rows begin that the mass does
 * not know yet.  S is what any call of this library writes, by its strides in elements:
 *     san_attn_weights, san_decode_step, san_quant_attn    item_stride H * ld_s, head_stride ld_s, n_rows 1
 *     the same for encoder memory, rows = beam             item_stride beam * H * ld_s, row_stride H * ld_s, head_stride ld_s
 *     san_full_block, rows = positions                     item_stride H * cap_len * ld_s, head_stride cap_len * ld_s, row_stride ld_s
 * S[i][r][h][j] is read for j < len alone.  d_rows: rows of each item, 0 .. n_rows (NULL: n_rows).  Sums are float32, in an order that
 * n_rows and the heads of a group alone decide.  An id, length, number of rows or begin out of range skips the item and is reported. */
typedef struct {
    int32_t n_heads, n_kv_heads;
    const float* d_S; int64_t item_stride, row_stride, head_stride;
    int32_t n_rows; const int32_t* d_rows;          /* n_rows 0 .. 2^20 */
    const int32_t* d_ids; const int32_t* d_lens; const int32_t* d_begin;
    int32_t n_items;                      /* at most 65535 */
    int32_t max_len;                      /* host bound on d_lens, at most 2^28 (0 = ld_mass) */
    float decay;                          /* finite */
    float* d_mass; int64_t ld_mass;       /* [max_ids][n_kv_heads][ld_mass], ld_mass >= max_len */
    int32_t max_ids;
    int32_t* d_status;                    /* optional */
} san_mass_args;
int32_t san_weight_mass(const san_mass_args* args, void* stream);

/* A cache cut back to its heaviest rows, in place.  Of an item with len = d_lens[i] > n_keep rows, each key head keeps n_keep: the
 * first n_sink, the last n_recent, and of those between the ones of the largest mass (ties: the lowest row; NaN counts as -infinity).  They
 * move to the front in their order, in the key plane, every layer's value plane and the mass; what lies behind them is left as it
 * was.  Shorter items stay as they are.  d_lens_out[i] = min(len, n_keep) (may be d_lens).  d_kept, where it is given, receives
 * the rows that were kept, min(len, n_keep) of them in ascending order.  Key heads choose for themselves, layers of a block share their
 * weights and so the choice.  An id or length out of range skips the item (d_lens_out too) and is reported. */
typedef struct {
    const int32_t* d_ids; const int32_t* d_lens;
    int32_t n_items;                      /* at most 65535 */
    int32_t max_len;                      /* host bound on d_lens (0 = cap_len) */
    int32_t n_keep, n_sink, n_recent;     /* n_keep >= 1, n_sink + n_recent <= n_keep <= 2^26 */
    float* d_mass; int64_t ld_mass;       /* [max_ids][n_kv_heads][ld_mass], ld_mass >= max_len */
    int32_t* d_kept; int64_t ld_kept;     /* optional: [n_items][n_kv_heads][ld_kept], ld_kept >= n_keep */
    int32_t* d_lens_out;                  /* [n_items] */
    int32_t* d_status;                    /* optional */
} san_evict_args;
int32_t san_cache_evict_bytes(const san_planes* cache, const san_evict_args* args, size_t* workspace_bytes);
int32_t san_cache_evict(const san_planes* cache, const san_evict_args* args, void* d_workspace, size_t workspace_bytes, void* stream);

/* Reads (and clears) the device error word: *first_error = SAN_OK or the first
 * device-check error since the last read; detail[0..3] (optional) = kernel tag, item,
 * offending value, limit.  Synchronises `stream`. */
int32_t san_device_status(san_ctx* ctx, int32_t* first_error, int32_t* detail, void* stream);

/* The weights step of san_attn_weights for callers that cannot allocate device memory.
 * (The paper has no counterpart: this entry point exists for deployment reasons only.)
 *
 * A decode loop inside a serving process often may not call cudaMalloc: the server's
 * cache manager has reserved all of HBM, a plug-in contract forbids allocation while
 * serving, or the stall that cudaMalloc/cudaFree impose on every stream of the device is
 * not acceptable.  Such a caller cannot create a san_ctx, which needs a workspace buffer.
 * This call needs neither: it takes the key panel directly and keeps the scratch of
 * split rows (tickets, partial max/sum) in a fixed 1 MiB array inside the library image,
 * present on every GPU that loads the library until the process exits.  It calls no
 * cudaMalloc, cudaFree or other allocating routine.
 *
 *   dtype      SAN_F32 or SAN_BF16 (element type of d_q and d_K)
 *   n_queries  query rows sharing each key panel: 1 for self-attention, the beam size for
 *              encoder memory (1..8)
 *   d_q        [n_items][n_queries][n_heads][64]
 *   d_K        key plane [max_ids][n_heads][cap_len][64], the layout of the context's planes
 *   d_ids, d_lens, n_items, max_len, d_S, ld_s   as in san_attn_weights;
 *              d_S is [n_items][n_queries][n_heads][ld_s]
 *   d_status   optional device int32[8]: cleared, then [0] = SAN_ERR_DEVICE_CHECK and
 *              [1..4] = kernel tag, item, value, limit if an item was skipped
 *
 * Limits: n_items * n_heads <= 65536 rows, else SAN_ERR_CAPACITY (use a context instead).
 * The device that owns `stream` and every buffer must be the current device at the call, on
 * every call and not only the first (the call uses that device's copy of the array and does
 * not check whose stream it was given).  The first call on each device looks up the array's
 * device address; make that first call before any stream capture begins.  Every call on a
 * device uses the same array and finds what the previous call left there; the call clears
 * the tickets and status words it needs on `stream` before launching.  Two calls whose
 * kernels may overlap on one GPU (different streams without an event between them, or
 * different host threads doing so) race on the array: order them. */
int32_t san_attn_weights_static(int32_t dtype, int32_t n_heads, int32_t n_queries, const void* d_q,
                                const void* d_K, int32_t max_ids, int32_t cap_len,
                                const int32_t* d_ids, const int32_t* d_lens, int32_t n_items,
                                int32_t max_len, float* d_S, int64_t ld_s, int32_t* d_status,
                                void* stream);

const char* san_status_string(int32_t status);

#ifdef __cplusplus
}
#endif
#endif /* SAN_H_ */
