/*
 * conserve_attn.h -- C ABI of the paged-KV attention hot path under conversation-level
 * disaggregated serving (arxiv 2606.01839, "Observation, Not Prediction").
 *
 * The paper (Section 4 and Fig. 9) binds each agentic conversation to one decoder for its whole
 * life: the turn-1 prompt is prefilled (on the prefiller), the resulting KV cache is transferred
 * exactly once, and the first decode plus every later turn's incremental prefill ("append") and
 * decode run on the decoder against the conversation's ever-growing KV cache (Section 1; Section
 * 3.1 "prefix caching" and "KV cache transfer"; Section 3.2 "memory-bound" decode). This library is
 * the data-parallel part of that: a pool of 16-token KV pages per GPU, conversations that own pages,
 * and the kernels that append KV, attend (turn-1 prefill, extend, batched decode) and move a
 * conversation's KV out of / into a pool (the one-time transfer).
 *
 * Conventions for every call
 * --------------------------
 *  - Device pointers: every `void*` named k, v, q, out, dst, src, kv_base, ws_base is a device
 *    address on the current HIP device; the caller owns that memory and keeps it alive until the
 *    stream reaches the call. Host pointers: cs_conv arrays, q_lens, and the out-parameters.
 *  - Element type: bf16 (IEEE binary32 with the low 16 bits dropped) everywhere; accumulation fp32.
 *    A pool may hold K and V in 4 bits instead (cs_pool_create_as); what goes in and out stays bf16.
 *  - Append-then-attend: a conversation's K/V are written by the append calls (cs_kv_append, its batched,
 *    rotated and tree forms, the mixed steps), by cs_kv_unpack, which makes the conversation, and by
 *    cs_kv_keep, which moves tokens within it; attention only reads them. Attention calls (but for
 *    cs_attn_tree and cs_attn_cross) take queries for the LAST q_len positions of each conversation; query i of a conversation of
 *    length L sits at position p = L - q_len + i and sees keys 0..p (itself included). Softmax
 *    scale is exactly 1/sqrt(head_dim). Query head h reads KV head h / (n_q_heads / n_kv_heads).
 *  - Errors: every call validates all arguments before changing any state; on error it returns a
 *    negative cs_status, changes nothing, and sets a thread-local message (cs_last_error). Nothing
 *    aborts or throws across this ABI. CS_EHIP reports a failing HIP runtime call, CS_ENOMEM also host
 *    memory that ran out; an append that fails so still changes no length and no page (its reserved
 *    pages return to the free list); cs_mixed_step's append is complete when a later attention launch
 *    fails; after either the outputs of the failing call are undefined. What such an append stored behind a
 *    conversation's end is seen by no row, but where its values are not finite, prefill and extend give
 *    NaN until a later append has overwritten them.
 *  - Asynchrony: host metadata (lengths, page tables) is committed when the call returns; kernels
 *    and the small metadata uploads they need are enqueued on `stream` (a hipStream_t, 0 = null
 *    stream). No call synchronises the device, except that switching a pool to another stream
 *    makes the new stream wait (hipStreamWaitEvent) for work already enqueued on the previous one.
 *  - A pool is not thread-safe: one host thread at a time.
 */
#ifndef CONSERVE_ATTN_H
#define CONSERVE_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cs_pool cs_pool;   /* opaque; library-owned host metadata */
typedef int32_t cs_conv;          /* conversation handle (>= 0) */
typedef void* cs_stream;          /* hipStream_t */
typedef int32_t cs_status;

enum {
  CS_OK = 0,
  CS_EINVAL = -1,  /* bad argument: null pointer, bad size, duplicate conversation, wire mismatch */
  CS_ENOMEM = -2,  /* too few free pages / no free conversation slot / ring too small / no host memory */
  CS_ENOENT = -3,  /* unknown or destroyed conversation handle */
  CS_ESTATE = -4,  /* call not valid in the conversation's state (e.g. q_len > length) */
  CS_ERANGE = -5,  /* index out of range (layer, page capacity of a conversation) */
  CS_EHIP = -6,    /* a HIP runtime call failed */
  CS_EBUSY = -7    /* placement refused: the prefiller is saturated (conserve_sched.h) */
};

#define CS_PAGE_TOKENS 16

typedef struct {
  int32_t n_layers;            /* >= 1 */
  int32_t n_q_heads;           /* multiple of n_kv_heads; n_q_heads/n_kv_heads in {1,2,4,8} */
  int32_t n_kv_heads;          /* >= 1 */
  int32_t head_dim;            /* 64 or 128 */
  int32_t max_convs;           /* live conversations at once, 1 .. 2^20 */
  int32_t max_pages_per_conv;  /* longest conversation, in 16-token pages */
  int64_t n_pages;             /* pool capacity in pages; a page holds 16 tokens of every layer */
} cs_pool_desc;

/*
 * KV pool layout (device, caller-allocated, cs_pool_kv_bytes(desc) bytes, 256-byte aligned):
 *   pool[layer][page][kv_head] = one 4*16*head_dim-byte block:
 *     K part: head_dim/32 sub-blocks, sub-block s = K[16 tokens][dims 32s .. 32s+31] token-major
 *             (each sub-block 1 KiB: what one matrix-core operand load of 16 keys reads), then
 *     V^T[head_dim][16] dimension-major (each row holds one dimension of the page's 16 tokens).
 * Token slots >= length in a conversation's last page always hold zeros (append and unpack write
 * them), so a page is never read past the conversation's end with undefined contents.
 */
size_t cs_pool_kv_bytes(const cs_pool_desc* desc);

/* Device workspace bytes the pool needs: page-table mirror, decode partials, records of extend tiles
 * whose keys are cut into pieces (head_dim 128: 69 MB, 208 MB in a pool of several layers; about half at
 * 64; none where no conversation can exceed 512 tokens), metadata ring (8 MiB). */
size_t cs_pool_workspace_bytes(const cs_pool_desc* desc);

/*
 * Create a pool over caller memory. Physical pages are handed out from a free list shuffled by
 * `placement_seed`, so page placement is random (results never depend on it). Pinned host staging
 * memory for metadata uploads is allocated by the pool's first device call (an append, unpack or
 * attention call) and freed by cs_pool_destroy.
 * Errors: CS_EINVAL (bad descriptor, null/short/misaligned buffers), CS_EHIP.
 */
cs_status cs_pool_create(const cs_pool_desc* desc, void* kv_base, size_t kv_bytes, void* ws_base,
                         size_t ws_bytes, uint64_t placement_seed, cs_pool** out);

/*
 * What a pool's pages hold.
 * CS_KV_BF16: K and V as they are appended (the layout above).
 * CS_KV_FP4: K and V in 4 bits, 17 head_dim bytes a block instead of 64 head_dim: 3.76 times the tokens in
 *   the same memory, and as many fewer bytes for a decode step to read and for a transfer to move. Values
 *   are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times a power of two: for K one for every 32
 *   dims of a token and kv head, for V one for every token and kv head. With a the largest magnitude of
 *   such a group the power is 2^(floor(log2 a) - 2), at least 2^-126; a value is rounded to the nearest
 *   e2m1 value times it (ties to the even code) and at most to 6 times it. K and V must be finite: a group
 *   with an infinity or NaN is held, read back and attended as NaN. Attention is that of the held values:
 *   every call below does on such a pool what it does on a bf16 one, with the same arguments, asynchrony and
 *   errors. Scores take a query as three 3-bit parts for every 32 dims (head_dim 64, decode: 16 dims): exactly
 *   where its magnitude is at least 2^-8 of the largest of them, else to within 2^-16 of that largest, so a
 *   query with outliers far over the dims that matter loses bits that a bf16 pool keeps.
 *   Block (layer, page, kv head), two codes a byte, the first in the low bits: K[d/32 groups][16 tokens][32
 *   dims], V[4][16][d/16][4]: part i, row c, tile t hold dim 16 t + c of tokens 4 i .. 4 i + 3; then bytes e
 *   (the power 2^(e - 127); 255: NaN, V's codes then zeros): K[16 tokens][d/32 groups], V[16 tokens], zeros
 *   up to 17 d. Token slots >= length are zeros.
 */
enum { CS_KV_BF16 = 0, CS_KV_FP4 = 1 };

/* As cs_pool_kv_bytes and cs_pool_create, for a pool of the given format (CS_KV_BF16: the same as those;
 * the workspace is cs_pool_workspace_bytes either way). cs_pool_kv_bytes_as returns 0 and cs_pool_create_as
 * CS_EINVAL for an unknown format. */
size_t cs_pool_kv_bytes_as(const cs_pool_desc* desc, int32_t format);
cs_status cs_pool_create_as(const cs_pool_desc* desc, int32_t format, void* kv_base, size_t kv_bytes, void* ws_base,
                            size_t ws_bytes, uint64_t placement_seed, cs_pool** out);

/* Destroy host state; never frees caller memory. Waits for the pool's enqueued work first. */
cs_status cs_pool_destroy(cs_pool* pool);

/* Pages held by live conversations and pages still free (the decoder's active KV occupancy that
 * the paper's reactive scheduler reads, Section 4.2; freed when a conversation ends). */
cs_status cs_pool_occupancy(const cs_pool* pool, int64_t* used_pages, int64_t* free_pages);

/* New empty conversation (Section 4.2: a conversation enters at its first turn).
 * Errors: CS_EINVAL (null out), CS_ENOMEM (max_convs live). */
cs_status cs_conv_create(cs_pool* pool, cs_conv* out);

/* End a conversation and return its pages to the pool (Section 4.2: occupancy is decremented at
 * termination). The caller must not destroy a conversation that enqueued work still reads.
 * Errors: CS_ENOENT. */
cs_status cs_conv_destroy(cs_pool* pool, cs_conv conv);

/* Current length in tokens. Errors: CS_ENOENT, CS_EINVAL. */
cs_status cs_conv_len(const cs_pool* pool, cs_conv conv, int64_t* tokens);

/* Copy the conversation's physical page ids (logical order) into out[0..cap); *n = page count.
 * Errors: CS_ENOENT, CS_EINVAL (null), CS_ERANGE (cap < page count; *n still set). */
cs_status cs_conv_pages(const cs_pool* pool, cs_conv conv, int32_t* out, int64_t cap, int64_t* n);

/*
 * Append n_new tokens of K and V for every layer (Section 2.1: decode appends one KV entry per
 * generated token; Section 3.1: a later turn adds the entries of its appended tokens).
 * k, v: device, [n_layers][n_new][n_kv_heads][head_dim] bf16, contiguous.
 * Reserves ceil((len+n_new)/16) - ceil(len/16) new pages first; on CS_ENOMEM nothing changes.
 * n_new == 0 is a no-op. Errors: CS_ENOENT, CS_EINVAL, CS_ENOMEM, CS_ERANGE, CS_EHIP.
 */
cs_status cs_kv_append(cs_pool* pool, cs_conv conv, int32_t n_new, const void* k, const void* v,
                       cs_stream stream);

/*
 * Batched append: conversation convs[i] receives n_new[i] tokens; k, v are
 * [n_layers][sum(n_new)][n_kv_heads][head_dim] with the conversations' tokens concatenated in
 * batch order. All-or-nothing page reservation. Conversations must be distinct.
 */
cs_status cs_kv_append_batch(cs_pool* pool, int32_t n_convs, const cs_conv* convs,
                             const int32_t* n_new, const void* k, const void* v, cs_stream stream);

/*
 * Rotary positions. Of every head the first rotary_dim dims turn with the token's position p (0 for a
 * conversation's first token), pair i = 0 .. rotary_dim/2 - 1 by p inv_freq[i] radians:
 *   (a, b) -> amplitude (a cos - b sin, a sin + b cos)
 * where a pair is dims (i, i + rotary_dim/2), or (2 i, 2 i + 1) with interleaved; the other dims stay.
 * The angle, kept as a 64-bit fraction of a turn and rounded to fp32, is within 2^-25 turns of the exact
 * one at any position. The rotated value is computed in fp32, within 2^-21 amplitude (|a| + |b|), and
 * rounded once, to bf16 or to the pool's 4 bits.
 */
typedef struct {
  int32_t rotary_dim;   /* 16, 32, .., head_dim */
  int32_t interleaved;  /* 0 or 1 */
  double amplitude;     /* factor on rotated dims */
  double inv_freq[64];  /* radians per position; the first rotary_dim/2 are used */
} cs_rope;

/*
 * Fill *out: inv_freq[i] = f_i = base^(-2 i / rotary_dim), amplitude 1, changed for contexts `factor` times
 * longer than those a model was trained on (original_len tokens):
 *   CS_ROPE_PLAIN   not at all (the last four arguments are not read)
 *   CS_ROPE_LINEAR  f_i / factor
 *   CS_ROPE_NTK     base factor^(rotary_dim / (rotary_dim - 2)) in place of base
 *   CS_ROPE_PARTS   f_i (g + (1 - g) / factor) with g = (n - low) / (high - low), between 0 and 1, where pair i
 *                   makes n = original_len f_i / 2 pi turns over the original context: pairs of fewer than
 *                   `low_turns` turns slow down, of more than `high_turns` do not; amplitude 0.1 ln(factor) + 1
 * A caller may change any field afterwards. Host only.
 * Errors: CS_EINVAL (null, rotary_dim no multiple of 16 in 16 .. 128, interleaved not 0 or 1, base <= 1,
 * unknown scaling, factor < 1, for PARTS original_len <= 0 or low_turns >= high_turns, not finite).
 */
enum { CS_ROPE_PLAIN = 0, CS_ROPE_LINEAR = 1, CS_ROPE_NTK = 2, CS_ROPE_PARTS = 3 };
cs_status cs_rope_init(cs_rope* out, int32_t rotary_dim, int32_t interleaved, double base, int32_t scaling,
                       double factor, double original_len, double low_turns, double high_turns);

/*
 * cs_kv_append_batch with rotated keys: a token's K enters the cache turned by its position. With q (may be
 * null) the queries of the same tokens, [n_layers][sum(n_new)][n_q_heads][head_dim], are rotated in the same
 * call into q_out (same shape; q itself, or no overlap with it), ready for the attention calls.
 * Errors: as cs_kv_append_batch; CS_EINVAL for a null or invalid rope (rotary_dim no multiple of 16 in
 * 16 .. head_dim, interleaved not 0 or 1, amplitude or an inv_freq in use not finite), q without q_out, q of more
 * than 2^28 - 16 rows; CS_ENOMEM for q of more than 2^18 conversations. After CS_EHIP q_out is undefined: queries
 * rotated in place may or may not have turned.
 */
cs_status cs_kv_append_rope(cs_pool* pool, const cs_rope* rope, int32_t n_convs, const cs_conv* convs, const int32_t* n_new,
                            const void* k, const void* v, const void* q, void* q_out, cs_stream stream);

/*
 * Queries of the last q_lens[i] positions of each conversation (those the attention calls take), rotated:
 * q, out [n_layers][sum(q_lens)][n_q_heads][head_dim] for any n_layers >= 0; out may be q itself, otherwise
 * they do not overlap. May be captured into a graph, as cs_attn_decode_batch_noalloc. Errors: as cs_attn_extend,
 * and as cs_kv_append_rope for rope, rows, conversations and after CS_EHIP; CS_EINVAL (n_layers < 0).
 */
cs_status cs_rope_q(cs_pool* pool, const cs_rope* rope, int32_t n_convs, const cs_conv* convs, const int32_t* q_lens,
                    int32_t n_layers, const void* q, void* out, cs_stream stream);

/*
 * Read tokens [starts[i], starts[i] + n[i]) of each conversation back from the cache: k, v
 * [n_layers][sum(n)][n_kv_heads][head_dim], conversations in batch order. A bf16 pool gives the bits that
 * were appended (rotated, if they were); a 4-bit pool the values it holds, exact in bf16 (below 2^-126 in magnitude
 * as far as bf16 holds them). The conversations must be distinct. n[i] == 0 is allowed.
 * Errors: CS_EINVAL (null, negative, duplicate conversation, too many tokens), CS_ENOENT, CS_ERANGE (past
 * the conversation's end), CS_EHIP.
 */
cs_status cs_kv_read(cs_pool* pool, int32_t n_convs, const cs_conv* convs, const int64_t* starts, const int32_t* n, void* k,
                     void* v, cs_stream stream);

/*
 * Turn-1 causal prefill (Section 3.1: the compute-bound first-turn prefill). For each conversation
 * q_lens[i] must equal its length (its whole content is the prompt just appended).
 * q:   device [sum(q_lens)][n_q_heads][head_dim] bf16, conversations in batch order.
 * out: device, same shape; bf16 (round to nearest even) of softmax(q k^T / sqrt(d)) v, causal.
 * The result is bitwise deterministic and independent of physical page placement. It depends on the
 * call's batch as far as rounding goes: a call with few queries cuts the keys into pieces, whose size
 * follows from the whole batch, and sums them piece by piece. The same queries in another batch, or
 * chunk by chunk, agree to the rounding of bf16 weights (measured: 3e-3 in the 2-norm), and bit for bit
 * only where neither call cuts its keys.
 * Errors: CS_EINVAL (null, duplicate conv, q_len < 0), CS_ENOENT, CS_ESTATE (q_len != length),
 * CS_ERANGE (layer), CS_ENOMEM (metadata larger than the ring), CS_EHIP.
 */
cs_status cs_attn_prefill_turn1(cs_pool* pool, int32_t n_convs, const cs_conv* convs,
                                const int32_t* q_lens, int32_t layer, const void* q, void* out,
                                cs_stream stream);

/*
 * Extend-prefill of a later turn (Section 3.1 "prefix caching": the appended tokens attend to the
 * whole cached history and causally among themselves; Section 4: it runs on the pinned decoder).
 * Same arguments as cs_attn_prefill_turn1 but 0 <= q_lens[i] <= length (q_len == length is a full
 * prefill, q_len == 1 a decode), and the same holds for its bits. Errors as above, CS_ESTATE when
 * q_len > length.
 */
cs_status cs_attn_extend(cs_pool* pool, int32_t n_convs, const cs_conv* convs,
                         const int32_t* q_lens, int32_t layer, const void* q, void* out,
                         cs_stream stream);

/*
 * Attention of drafted tokens over the cache that holds them, to verify them in one call (a step of several guesses in
 * place of one token). The last q_lens[i] tokens of conversation i are a tree: parents[..], one for each query row in batch
 * order, is -1 (the token follows the last cached one) or the index of an earlier token of the same tree, counted from
 * its first. Row j sees the length - q_lens[i] cached tokens, its ancestors and itself, and no other branch: a NaN or infinity in
 * a branch it does not see (keys or values) does not reach it. An infinite value that a row sees makes that dim of it the same
 * infinity, or NaN where it sees both signs or the key's weight underflows (below 2^-126 of the row's largest). A tree that is a chain
 * (parents -1, 0, 1, ..) is cs_attn_extend.
 * At most CS_MAX_DRAFT tokens a tree. Pages of either format. Several lengths, and none, in one batch are fine.
 * q, out: device [sum(q_lens)][n_q_heads][head_dim] bf16. Deterministic and independent of page placement; a row's last bits
 * depend on the batch, as with cs_attn_extend. May be captured into a graph, as cs_attn_decode_batch_noalloc.
 * Errors: as cs_attn_extend; CS_ERANGE (a tree too large), CS_EINVAL (null parents, a parent that is no earlier token).
 */
#define CS_MAX_DRAFT 1024
cs_status cs_attn_tree(cs_pool* pool, int32_t n_convs, const cs_conv* convs, const int32_t* q_lens, const int32_t* parents,
                       int32_t layer, const void* q, void* out, cs_stream stream);

/*
 * cs_kv_append_rope for the drafted tokens of such trees: token j of conversation i takes the next slot, as with any
 * append, but turns by its position in the tree, length + depth (depth 0 for a parent of -1), and so does its query. `parents`
 * as in cs_attn_tree, one for each new token. (Without rotary positions cs_kv_append_batch appends a draft.)
 * Errors: as cs_kv_append_rope; CS_ERANGE and CS_EINVAL for the trees, as cs_attn_tree.
 */
cs_status cs_kv_append_tree(cs_pool* pool, const cs_rope* rope, int32_t n_convs, const cs_conv* convs, const int32_t* n_new,
                            const int32_t* parents, const void* k, const void* v, const void* q, void* q_out, cs_stream stream);

/*
 * Keep the accepted tokens of a draft: of the last n_last[i] tokens of conversation i those stay whose indexes (0 for
 * the first of them) the next n_keep[i] entries of `keep` give, increasing, and follow the tokens before them in that order; the
 * others are dropped, and pages that end up empty return to the pool. Of a tree the indexes are those of an accepted path:
 * its tokens were turned by their depth, which is now their slot. n_keep = 0 takes the conversation back to what it was before
 * its last n_last tokens, whatever they were; n_keep == n_last changes nothing. All layers; pages of either format, whose
 * bytes move as they are. Where the kept tokens are the first ones nothing moves.
 * After CS_EHIP the last n_last tokens are undefined, the lengths unchanged. Not under stream capture (CS_ESTATE).
 * Errors: CS_EINVAL (null, duplicate conversation, n_keep not in 0 .. n_last, keep not increasing in 0 .. n_last - 1),
 * CS_ENOENT, CS_ESTATE (n_last > length), CS_ENOMEM (more than one metadata upload holds, some 250,000 moved tokens or 20,000
 * conversations; nothing is changed), CS_EHIP.
 */
cs_status cs_kv_keep(cs_pool* pool, int32_t n_convs, const cs_conv* convs, const int32_t* n_last, const int32_t* n_keep,
                     const int32_t* keep, cs_stream stream);

/*
 * Cross attention: q_lens[i] rows see ALL tokens of conversation i, which holds the K and V of an encoder's states (or any other
 * context), appended like any tokens. No mask, no relation between a row and a position: any number of rows, more
 * than the conversation has tokens too, one for each of several hypotheses or a whole text. A conversation may appear several
 * times in a batch (rows of its entries are computed one by one; as one entry they share the reading). Rows of a conversation
 * without tokens are zeros. q, out, the result's bits, infinite values, and capture: as cs_attn_tree.
 * Errors: CS_EINVAL (null, q_len < 0, too many rows), CS_ENOENT, CS_ERANGE (layer), CS_ENOMEM, CS_EHIP.
 */
cs_status cs_attn_cross(cs_pool* pool, int32_t n_convs, const cs_conv* convs, const int32_t* q_lens, int32_t layer, const void* q,
                        void* out, cs_stream stream);

/*
 * Batched single-token decode (Section 2.1 / 3.2: each step reads the whole cache of every
 * conversation in the batch; memory-bound). The query of convs[i] is its last position.
 * q, out: device [n_convs][n_q_heads][head_dim] bf16. Conversations distinct, length >= 1.
 * Split-K over fixed logical token ranges plus a fixed-order log-sum-exp merge: the result is
 * bitwise deterministic and independent of physical page placement.
 * Errors: CS_EINVAL, CS_ENOENT, CS_ESTATE (length 0), CS_ERANGE, CS_ENOMEM, CS_EHIP.
 */
cs_status cs_attn_decode_batch(cs_pool* pool, int32_t n_convs, const cs_conv* convs,
                               int32_t layer, const void* q, void* out, cs_stream stream);

/*
 * Allocation-free variant of cs_attn_decode_batch, for callers that cannot allocate device memory
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc). Same
 * arguments, semantics and output bits as cs_attn_decode_batch; the only difference is where the
 * decode split keeps its partial records: in a static device array of the library (16 MiB =
 * 4,194,304 floats on each GPU, held until the process ends) instead of the pool's workspace.
 * The call allocates no device or pinned memory and creates no HIP objects (the device address of
 * the array is looked up once per device); host-side planning uses the C++ heap. It launches
 * untimed: cs_profile_* does not see it.
 * Every call on one GPU shares that GPU's array: calls that overlap on one GPU (on different
 * streams, or from different pools on different host threads) race and must not be issued.
 * Captured into a graph, the batch's descriptors are part of the graph, of whatever size. A replay is work
 * of the pool: it must not overlap the pool's other calls or another graph's replay, and it decodes at the
 * lengths that the conversations had at the capture.
 * Errors: as cs_attn_decode_batch; CS_ENOMEM when the batch's partial records
 * (n_items * n_q_heads * (head_dim + 4) floats; batches whose conversations are each one work item
 * need none) exceed the array; CS_ESTATE when the pool has made no device call yet (its first one
 * allocates its metadata ring; an append or unpack that filled it always has); CS_EINVAL when the
 * current device is not the pool's.
 */
cs_status cs_attn_decode_batch_noalloc(cs_pool* pool, int32_t n_convs, const cs_conv* convs,
                                       int32_t layer, const void* q, void* out, cs_stream stream);

/*
 * One step of a decoder serving agentic conversations (Section 4: after the one-time transfer a
 * conversation's later turns -- incremental prefill of appended tokens and decoding -- run on its
 * decoder; Section 2.1: dynamic batching lets requests join and leave every iteration). In one
 * call: conversations ext_convs[i] append an extend chunk of ext_lens[i] >= 1 tokens and
 * conversations dec_convs[j] append one decoded token (all layers), then for every layer the extend
 * queries attend (as cs_attn_extend) and the decode queries attend (as cs_attn_decode_batch).
 * All conversations must be distinct.
 *   k, v:     [n_layers][sum(ext_lens) + n_dec][n_kv_heads][head_dim], extend tokens first
 *   q_ext:    [n_layers][sum(ext_lens)][n_q_heads][head_dim];  out_ext same shape
 *   q_dec:    [n_layers][n_dec][n_q_heads][head_dim];          out_dec same shape
 * The batch metadata is uploaded once and reused by every layer's launches. Work enqueued on
 * `stream` after the call (and a synchronisation of `stream`) sees every output of the step.
 * flags = 0: every layer's queries are inputs of the call, so no layer waits for another: the extend
 *   work of all layers is one launch and the decode work of all layers another (several where the
 *   workspace has no room for the records of all layers), each followed by its merge. With both parts
 *   present the extend launches run beside the decode on a second stream owned by the pool, forked
 *   from `stream` after the append and joined back into it before the call returns.
 * flags = CS_MIXED_LAYER_ORDERED: the order of a model forward pass, where layer l+1's queries
 *   depend on layer l's output: layer l's extend and decode overlap each other, and layer l+1
 *   starts only when both are complete. With both parts present a layer is one launch holding its
 *   extend tiles and its decode split, then one that merges what they left in pieces.
 * (Extend plans larger than a 2 MiB upload -- some 65,000 chunks or more -- take the second stream in
 * layer order too; larger than three uploads, everything runs on `stream`.)
 * Outputs are bitwise the same either way (and the same as the separate calls).
 * Errors: as cs_kv_append_batch, cs_attn_extend and cs_attn_decode_batch; CS_EINVAL for unknown
 * flags.
 */
enum { CS_MIXED_LAYER_ORDERED = 1 };
cs_status cs_mixed_step(cs_pool* pool, int32_t n_ext, const cs_conv* ext_convs,
                        const int32_t* ext_lens, int32_t n_dec, const cs_conv* dec_convs,
                        const void* k, const void* v, const void* q_ext, void* out_ext,
                        const void* q_dec, void* out_dec, uint32_t flags, cs_stream stream);

/*
 * The same step of a model with rotary positions: the new tokens' keys enter the cache turned by their positions (as
 * cs_kv_append_rope) and every query attends turned by its own (as cs_rope_q). q_ext and q_dec are left as they are,
 * unless the outputs are the same tensors (out_ext == q_ext, out_dec == q_dec), which is allowed; otherwise
 * inputs and outputs do not overlap. Errors: as cs_mixed_step, and as cs_kv_append_rope for rope and rows; a batch
 * that the pool cannot take is refused before a query turns, but after CS_EHIP the outputs are undefined.
 */
cs_status cs_mixed_step_rope(cs_pool* pool, const cs_rope* rope, int32_t n_ext, const cs_conv* ext_convs,
                             const int32_t* ext_lens, int32_t n_dec, const cs_conv* dec_convs, const void* k, const void* v,
                             const void* q_ext, void* out_ext, const void* q_dec, void* out_dec, uint32_t flags,
                             cs_stream stream);

/*
 * Version of the transfer wire format of cs_kv_pack / cs_kv_unpack below. The format is frozen at
 * this version: it is the pool's block format as of version 1, and a later change of the pool's
 * private block layout keeps pack and unpack reading and writing exactly this format (a new format
 * would take a new version number).
 */
#define CS_WIRE_FORMAT_VERSION 1

/* Wire size of a conversation's KV: n_layers * ceil(len/16) * n_kv_heads * 64 * head_dim bytes (a 4-bit
 * pool: 17 * head_dim, see cs_kv_pack_fp4). */
cs_status cs_kv_pack_size(const cs_pool* pool, cs_conv conv, size_t* bytes);

/*
 * Gather a conversation's pages in logical order into a contiguous wire buffer (the sending half
 * of the one-time turn-1 KV transfer, Section 4 and Section 3.1 "KV cache transfer").
 * Wire layout: [layer][logical page][kv_head] blocks in the pool's block format (K part in
 * 32-dim token-major sub-blocks, then V^T[d][16]); token slots >= length are written as zeros. dst: device, dst_bytes must equal
 * cs_kv_pack_size. Errors: CS_ENOENT, CS_EINVAL, CS_EHIP.
 */
cs_status cs_kv_pack(const cs_pool* pool, cs_conv conv, void* dst, size_t dst_bytes,
                     cs_stream stream);

/*
 * The transfer into a 4-bit pool: cs_kv_pack_fp4 gathers a conversation into the wire that such a pool unpacks,
 * [layer][logical page][kv_head] blocks of CS_KV_FP4, token slots >= length zeros. From a bf16 pool the values
 * are rounded as an append to a 4-bit pool rounds them, so a prefiller that attends in bf16 sends 3.76 times
 * fewer bytes and the decoder holds what it would had the same K and V been appended there. (From a 4-bit pool
 * it is cs_kv_pack.) cs_kv_pack_fp4_size: n_layers * ceil(len/16) * n_kv_heads * 17 * head_dim bytes.
 * Errors: as cs_kv_pack_size and cs_kv_pack. The format is frozen at CS_WIRE_FP4_VERSION.
 */
#define CS_WIRE_FP4_VERSION 1
cs_status cs_kv_pack_fp4_size(const cs_pool* pool, cs_conv conv, size_t* bytes);
cs_status cs_kv_pack_fp4(const cs_pool* pool, cs_conv conv, void* dst, size_t dst_bytes, cs_stream stream);

/*
 * Receiving half of the transfer: create a conversation of n_tokens tokens in `pool`, take fresh
 * pages from its (randomly placed) free list and scatter the wire buffer into them. src_bytes must
 * equal the wire size for n_tokens with this pool's shape; tail slots are written as zeros.
 * Errors: CS_EINVAL (size mismatch, n_tokens < 1), CS_ENOMEM, CS_ERANGE, CS_EHIP.
 */
cs_status cs_kv_unpack(cs_pool* pool, const void* src, size_t src_bytes, int64_t n_tokens,
                       cs_conv* out_conv, cs_stream stream);

/*
 * Instrumentation (per-kernel timing; not part of the attention path). Between cs_profile_start
 * and cs_profile_stop every kernel the pool launches is bracketed by two HIP timing events on its
 * stream, except that in cs_mixed_step one pair of events brackets the extend launches of all layers
 * (their time then includes the gaps between those launches). cs_profile_stop waits for the events, writes the
 * summed milliseconds and the launch count per kernel kind into ms[CS_PROF_KINDS] and
 * launches[CS_PROF_KINDS], and disables timing.
 * Errors: CS_EINVAL (null), CS_EHIP.
 */
enum {
  CS_PROF_APPEND = 0,        /* kv append kernel */
  CS_PROF_PACK = 1,          /* kv pack kernel */
  CS_PROF_UNPACK = 2,        /* kv unpack kernel */
  CS_PROF_DECODE_SPLIT = 3,  /* decode split-K kernel */
  CS_PROF_DECODE_MERGE = 4,  /* decode merge kernel; in a layer-ordered mixed step also the extend merge */
  CS_PROF_ATTN_FWD = 5,      /* prefill / extend attention kernel and the merge of cut tiles */
  CS_PROF_MIXED_LAYER = 6,   /* one layer's extend tiles + decode split in one launch */
  CS_PROF_KINDS = 7
  /* queries rotated by cs_rope_q and cs_kv_keep count as CS_PROF_APPEND, cs_kv_read as CS_PROF_UNPACK, cs_attn_tree
   * and cs_attn_cross as CS_PROF_ATTN_FWD */
};
cs_status cs_profile_start(cs_pool* pool);
cs_status cs_profile_stop(cs_pool* pool, double* ms, int64_t* launches);

/*
 * Instrumentation: properties of a HIP device that measurements are logged with (from
 * hipGetDeviceProperties). Errors: CS_EINVAL (null), CS_EHIP (no such device).
 */
typedef struct {
  char name[256];
  char arch[64];                 /* gcnArchName, e.g. "gfx950:sramecc+:xnack-" */
  int32_t cu_count;              /* compute units */
  int32_t clock_khz;             /* peak engine clock */
  int32_t memory_clock_khz;      /* peak memory clock */
  int32_t memory_bus_width_bits;
  int64_t lds_per_cu_bytes;      /* shared memory per compute unit */
  int64_t lds_per_block_bytes;   /* shared memory one workgroup may use */
  int64_t l2_bytes;              /* L2 cache size the runtime reports */
  int64_t total_mem_bytes;
} cs_device_info_t;
cs_status cs_device_info(int32_t device, cs_device_info_t* out);

/*
 * Instrumentation: read `bytes` (a multiple of 16) of device memory at `src` once with the
 * non-temporal 16-byte loads the decode and pack kernels use, on 8 workgroups per compute unit of
 * the current device, enqueued on `stream`; `sink` is 4 bytes of device memory that the kernel
 * writes only if the XOR of everything read equals 0x9E3779B9 (it exists so the loads stay live).
 * Time it with events on `stream` to get what streaming reads reach on the part.
 * Errors: CS_EINVAL (null pointers, bytes not a multiple of 16), CS_EHIP.
 */
cs_status cs_probe_stream_read(const void* src, size_t bytes, void* sink, cs_stream stream);

/*
 * Test instrumentation of the error paths: after `after` more kernel launches of this pool
 * succeed, every later launch of the pool reports CS_EHIP ("failure injected") without launching
 * anything, until the call is made again with after < 0 (off, the default). The failing call
 * behaves as on a real HIP launch failure at that point. Errors: CS_EINVAL (null pool).
 */
cs_status cs_debug_fail_launches(cs_pool* pool, int64_t after);

/* Message of the last failing call on this thread ("" if none). Valid until the next call. */
const char* cs_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* CONSERVE_ATTN_H */
