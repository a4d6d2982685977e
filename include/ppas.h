/*
 * ppas.h -- C ABI of libppas.so: one mixed scheduler step's attention over a
 * paged KV cache on an AMD Instinct MI355X (gfx950).
 *
 * A scheduler iteration batches prefill chunks and single-token decode rows of
 * different requests under one token budget (P-PAS paper, Section 2: continuous
 * batching with chunked prefill; Section 6.2: prefill and decode tokens sharing
 * an iteration). Prefill and decode store each token's key and value in the KV
 * cache (Section 2), which is paged (Section 7, PagedAttention). A step is two
 * calls on one stream: ppas_kv_append writes the step's new keys/values into
 * the pages (or ppas_rope_kv_append, which first rotates the new query and key
 * rows by their positions), then ppas_attn_step computes the attention of
 * every query row.
 *
 * Conventions shared by every entry point
 *   - bf16 means IEEE bfloat16 bit patterns (uint16 in memory).
 *   - Device pointers are HIP device memory on the current device; host pointers
 *     are ordinary host memory. The caller owns every buffer. The library
 *     allocates no device memory; it keeps a pool of pinned host buffers that
 *     hold its work lists (read by the kernels directly), released at process
 *     exit, and ppas_attn_step_noalloc uses one fixed device array per device.
 *   - No state is shared between calls other than that pool and that array:
 *     planning choices and profiling events are arguments of the calls that
 *     use them.
 *   - All device work is enqueued on `hip_stream` (a hipStream_t, NULL = the
 *     null stream) and the call returns without synchronising the host. Calls
 *     on the same stream execute in order; append before attending.
 *   - The appends and attention calls, planned or not, read a step's lists, which
 *     return to that pool: on a stream that captures a HIP graph they are
 *     PPAS_EUNSUPPORTED and leave the capture as it was. The other calls, and
 *     ppas_attn_step_noalloc, can be captured.
 *   - Every argument is validated on the host before anything is enqueued; a
 *     failed validation enqueues nothing. No C++ exception crosses the ABI.
 *   - Compiled shapes: head_dim 128, page_size 16, n_q_heads / n_kv_heads == 8
 *     (grouped-query attention; query head h reads KV head h / 8). Anything else
 *     returns PPAS_EUNSUPPORTED.
 *
 * Layouts
 *   q, out      [T][n_q_heads][128] bf16, row t = query token t of the step.
 *   k_new,v_new [T][n_kv_heads][128] bf16, the step's new keys/values, same rows.
 *   k_pages     [num_pages][n_kv_heads][16][16][8] bf16: per page and KV head,
 *               16 chunks of 8 consecutive features; chunk c holds the 16
 *               tokens' features 8c..8c+7, token after token (chunk-major).
 *   v_pages     [num_pages][n_kv_heads][128][16] bf16: per page and KV head,
 *               128 feature rows of 16 contiguous tokens.
 *   block_table [n_seqs][bt_stride] int32: entry j of request s is the physical
 *               page holding its positions 16j..16j+15. Entries past the
 *               request's last page are ignored (conventionally -1).
 *   seqs        host array of n_seqs descriptors (query_start, n_query,
 *               cached_len). Request s owns rows query_start..query_start+n-1,
 *               at positions cached_len..cached_len+n-1; query_start must start
 *               at 0 and be contiguous (query_start[s+1] = query_start[s] + n[s]),
 *               so T = sum of n_query. n_query == 1 is a decode row.
 */
#ifndef PPAS_H
#define PPAS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum ppas_status {
  PPAS_OK = 0,
  PPAS_EINVAL = -1,        /* malformed argument: null pointer, bad descriptor, bad stride */
  PPAS_ERANGE = -2,        /* a block-table entry outside [0, num_pages), a length overflow, or a step
                               too large for the int32 work list */
  PPAS_ENOSPACE = -3,      /* workspace smaller than ppas_attn_workspace_bytes(), or a step too large
                               for the fixed array of ppas_attn_step_noalloc */
  PPAS_EHIP = -4,          /* a HIP runtime call or kernel launch failed */
  PPAS_EUNSUPPORTED = -5   /* shape outside the compiled set, no gfx950 device, or a capturing stream
                               where the call reads a step's lists */
} ppas_status;

typedef struct ppas_shape {
  int32_t n_q_heads;    /* query heads (16 for the Qwen2.5-3B attention shape) */
  int32_t n_kv_heads;   /* KV heads; n_q_heads / n_kv_heads must be 8 */
  int32_t head_dim;     /* must be 128 */
  int32_t page_size;    /* tokens per page; must be 16 */
  int32_t num_pages;    /* pages in each of the K and V pools */
  float scale;          /* softmax scale applied to q.k (1/sqrt(head_dim) by convention) */
} ppas_shape;

typedef struct ppas_seq {
  int32_t query_start;  /* first query row of this request in q/out/k_new/v_new */
  int32_t n_query;      /* new tokens of this request in the step, >= 1 */
  int32_t cached_len;   /* tokens already in the cache before this step, >= 0 */
} ppas_seq;

/*
 * Planning choices of one call (this library's own tuning, not a quantity of
 * the paper). A zeroed struct, or NULL where a pointer is taken, selects the
 * automatic choice for every field.
 */
typedef struct ppas_plan_opts {
  int32_t prefill_split;    /* > 0: at most this many keys per prefill work item (rounded up to a
                               multiple of 64); 0: about two prefill items per compute unit */
  int32_t decode_split;     /* > 0: at most this many keys per decode work item (rounded up to a
                               multiple of 32, capped at 16384); 0: automatic */
  int32_t tile_positions;   /* 16 or 32: prefill tiles of that many positions (four- or eight-wave
                               kernel); 0: chosen per step. Any other value is PPAS_EINVAL */
  int32_t num_cus;          /* > 0: plan for a device with this many compute units; 0: the current
                               device's count (ppas_plan_items: 256) */
} ppas_plan_opts;

/*
 * HIP events (hipEvent_t handles created by the caller) that a call's kernel
 * launches record as they start and end, so a kernel's own duration can be
 * read with hipEventElapsedTime. Each pair is either both NULL (not recorded)
 * or both set (PPAS_EINVAL otherwise).
 *   start, stop              the call's main kernel: the packed attention
 *                            launch, or the page-write launch of an append
 *   merge_start, merge_stop  the split-merge launch of an attention call; not
 *                            recorded when the call merges no split row
 *                            (ppas_step_plan_info tells whether it does)
 */
typedef struct ppas_events {
  void* start;
  void* stop;
  void* merge_start;
  void* merge_stop;
} ppas_events;

/* Human-readable name of a status code. Never NULL; the string is static. */
const char* ppas_status_string(ppas_status status);

/*
 * Host-only check of a step description (no HIP call; usable without a GPU).
 * The description is the one of a scheduler iteration in Section 2: each
 * request contributes n_query new tokens (a prefill chunk, or one decode
 * token) after cached_len tokens already in the KV cache, stored in pages
 * (Section 7, PagedAttention) that the block table names. The checks
 * themselves are this library's own:
 * the shape (PPAS_EUNSUPPORTED outside the compiled set, PPAS_EINVAL for
 * non-positive sizes or a non-finite scale), each descriptor (n_query >= 1,
 * cached_len >= 0, contiguous query_start from 0, cached_len + n_query fitting in
 * int32: PPAS_EINVAL / PPAS_ERANGE), bt_stride >= ceil((cached_len+n_query)/16)
 * for every request (PPAS_EINVAL), and, when block_table_host is not NULL, that
 * every entry a request uses lies in [0, num_pages) (PPAS_ERANGE) and that no
 * two requests write the same (page, slot) in this step (PPAS_EINVAL). The cost
 * grows with the pages the requests use, not with num_pages.
 * n_seqs == 0 is a valid empty step.
 */
ppas_status ppas_validate_step(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                               const int32_t* block_table_host, int32_t bt_stride);

/*
 * Append the step's new keys and values to the paged cache (Section 2: the
 * processed tokens' keys and values are stored in the KV cache).
 * For every request s and i < n_query: position p = cached_len + i,
 * page = block_table[s][p / 16], slot = p % 16;
 *   k_pages[page][g][d / 8][slot][d % 8] = k_new[query_start + i][g][d]
 *   v_pages[page][g][:][slot] = v_new[query_start + i][g][:]   for every KV head g.
 * Bit-exact copies; no other byte of the pools is written. One kernel launch
 * for any number of requests. block_table_dev is the device copy of the table;
 * block_table_host (nullable) is a host copy used only for validation (range
 * and overlap checks are skipped when it is NULL, and out-of-range device
 * entries then give undefined results).
 * Returns PPAS_OK or a validation / PPAS_EHIP status.
 */
ppas_status ppas_kv_append(const ppas_shape* shape, void* k_pages, void* v_pages,
                           const void* k_new, const void* v_new,
                           const ppas_seq* seqs, int32_t n_seqs,
                           const int32_t* block_table_dev, int32_t bt_stride,
                           const int32_t* block_table_host, void* hip_stream);

/*
 * Rotary position embedding of the step's new rows, fused with the append.
 * The paper does not describe positional encoding; the operation is the
 * standard rotary embedding (RoPE) in rotate-half form over the whole head,
 * applied to the new query and key rows of a decoder block's attention
 * (Section 6.1) before they are used and cached. For every request s and
 * i < n_query: row r = query_start + i at position p = cached_len + i; for
 * every pair j < 64 the angle is a = p * rope_theta^(-2j/128), and a head row x
 * becomes (x_j cos a - x_{j+64} sin a) at j and (x_{j+64} cos a + x_j sin a) at
 * j + 64.
 *   q [T][n_q_heads][128] bf16: every query head row r is rotated in place.
 *   k_new [T][n_kv_heads][128] bf16: rotated and written to k_pages at (page,
 *     slot) exactly as ppas_kv_append writes keys; k_new itself is not modified.
 *   v_new: copied to v_pages unrotated, bit-exact, as ppas_kv_append does.
 * Angles are reduced in fp64, cos/sin taken in fp32, the rotation computed in
 * fp32 and rounded to bf16 nearest-even. Nothing else in q or the pools is
 * written. rope_theta must be finite and > 0 (else PPAS_EINVAL); q must not
 * be NULL. Validation, ownership and errors otherwise as ppas_kv_append. Call
 * it in place of ppas_kv_append, before ppas_attn_step, on the same stream.
 */
ppas_status ppas_rope_kv_append(const ppas_shape* shape, float rope_theta, void* q,
                                void* k_pages, void* v_pages,
                                const void* k_new, const void* v_new,
                                const ppas_seq* seqs, int32_t n_seqs,
                                const int32_t* block_table_dev, int32_t bt_stride,
                                const int32_t* block_table_host, void* hip_stream);

/*
 * Rotary positions in their general form (the paper does not describe positional
 * encoding; the operation is the library's own offer to models that need more than
 * ppas_rope_kv_append). Pair j < rotary_dim / 2 of a head at position p turns by
 * a = p w_j, and both results are multiplied by the magnitude m:
 *   x_a <- m (x_a cos a - x_b sin a),  x_b <- m (x_b cos a + x_a sin a)
 * with (x_a, x_b) features (j, j + rotary_dim / 2) in the half layout and
 * (2j, 2j + 1) in the interleaved one. Features from rotary_dim on are copied bit for
 * bit. With u_j = theta^(-2j / rotary_dim):
 *   PLAIN   w_j = u_j
 *   LINEAR  w_j = u_j / factor (positions squeezed into the learned length)
 *   BASE    w_j = (theta factor^(R / (R - 2)))^(-2j / R), R = rotary_dim (a larger base,
 *           which leaves the first pair as it is and divides the last by factor; R = 2: u_j)
 *   BANDS   by turns over the learned length, n_j = original_len u_j / (2 pi): pairs of at
 *           least `high` turns keep u_j, those of at most `low` get u_j / factor, and
 *           between them w_j = u_j (s + (1 - s) / factor), s = (n_j - low) / (high - low)
 *   RAMP    by pair numbers: with d(b) = R ln(original_len / (2 pi b)) / (2 ln theta), the
 *           pair of b turns, first = max(floor d(high), 0), last = min(ceil d(low), R - 1):
 *           w_j = u_j (1 - t + t / factor), t = (j - first) / (last - first) kept within
 *           0..1 (t = 0 up to `first` where last <= first, 1 behind it)
 * Frequencies and angles are computed in fp64 (whole turns removed), cos and sin in
 * fp32, the turn in fp32, and results rounded to bf16 nearest-even. A pair of more than
 * 4,096 turns per position, or of none, is PPAS_EINVAL: fp64 would not hold its angle at
 * far positions.
 */
enum { PPAS_ROPE_HALF = 0, PPAS_ROPE_INTERLEAVED = 1 };
enum { PPAS_ROPE_PLAIN = 0, PPAS_ROPE_LINEAR = 1, PPAS_ROPE_BASE = 2, PPAS_ROPE_BANDS = 3, PPAS_ROPE_RAMP = 4 };

typedef struct ppas_rope {
  int32_t layout;       /* PPAS_ROPE_HALF or PPAS_ROPE_INTERLEAVED */
  int32_t rotary_dim;   /* features that turn: even, 2..head_dim */
  int32_t scaling;      /* PPAS_ROPE_PLAIN .. PPAS_ROPE_RAMP */
  int32_t original_len; /* BANDS, RAMP: the learned length in positions, >= 1 */
  double theta;         /* finite, > 0 (RAMP: > 1) */
  double factor;        /* unless PLAIN: finite, > 0 */
  double low, high;     /* BANDS, RAMP: turns over original_len, 0 < low < high, finite */
  double magnitude;     /* m, finite and > 0; 0 selects 1 */
} ppas_rope;

/* w_j in radians per position for every pair of a ppas_rope, to rotary_dim / 2 doubles
 * (host only, no HIP call). PPAS_EINVAL for a field out of range. */
ppas_status ppas_rope_frequencies(const ppas_rope* rope, int32_t head_dim, double* out);

/*
 * Rows of heads turned by given positions: row r < n_rows of x (n_heads heads of
 * head_dim features each, one after the other, at x + r * x_stride elements) to the
 * same row of y (y_stride), at position positions_dev[r] (device int32, any value,
 * negative ones included). bf16. `transposed` turns by -a instead: the gradient of the
 * turn, and for m = 1 its inverse. x == y with equal strides turns in place; otherwise
 * the two must not overlap. head_dim is even, 2..256; n_heads 1..65536; strides are at
 * least n_heads * head_dim (PPAS_EINVAL otherwise; PPAS_EUNSUPPORTED for a larger
 * head_dim). Pointers need their element's alignment only; bases and strides on 16
 * bytes, and a rotary_dim that is a multiple of 16 in the half layout, are faster.
 * n_rows == 0 is a no-op. One launch; it allocates nothing, keeps nothing, and may be
 * captured into a HIP graph. events may be NULL.
 */
ppas_status ppas_rope_rows(const ppas_rope* rope, const void* x, int64_t x_stride, void* y, int64_t y_stride,
                           const int32_t* positions_dev, int32_t n_rows, int32_t n_heads, int32_t head_dim,
                           int32_t transposed, const ppas_events* events, void* hip_stream);

/*
 * A step's new rows as the projection left them: bf16 rows of n_q_heads (q) or
 * n_kv_heads (k, v) heads of 128 features, at base + row * stride elements. Fused
 * QKV rows are three pointers into one buffer with one stride.
 */
typedef struct ppas_qkv {
  const void* q;
  const void* k;
  const void* v;
  int64_t q_stride, k_stride, v_stride;   /* elements between rows, at least a row's features */
} ppas_qkv;

/*
 * As ppas_rope_kv_append, with any ppas_rope and rows at any stride: the queries are
 * rotated to q_out [T][n_q_heads][128] (the layout ppas_attn_step reads), the rotated
 * keys and the values go to the pages; the rows themselves are not modified. q_out may
 * be rows->q where q_stride is n_q_heads * 128 (in place); otherwise it must not overlap
 * the rows (PPAS_EINVAL, as for strides below a row's features or pools off 16 bytes).
 * Validation, ownership, streams and errors otherwise as ppas_rope_kv_append
 * (PPAS_ERANGE from 2^24 touched pages on).
 */
ppas_status ppas_rope_qkv_append(const ppas_shape* shape, const ppas_rope* rope, const ppas_qkv* rows, void* q_out,
                                 void* k_pages, void* v_pages, const ppas_seq* seqs, int32_t n_seqs,
                                 const int32_t* block_table_dev, int32_t bt_stride,
                                 const int32_t* block_table_host, void* hip_stream);

/*
 * Norms of query and key heads before their turn, in the same pass (the library's own
 * offer to models that normalise them; the paper does not describe it). A head x of D
 * features becomes
 *   z_i = (x_i - mu) / sqrt(var + eps) * (offset + w_i),  var = mean_i (x_i - mu)^2
 * with mu its mean where `center` is not 0, and 0 otherwise (the root-mean-square form);
 * then z turns as the calls without a norm turn x. Statistics, norm and turn are fp32 and
 * rounded once to bf16 nearest-even; the magnitude of a ppas_rope is on the turned
 * features only. Every finite head has its finite norm (a head of zeros gives zeros); one
 * that holds an infinity or a NaN gives what the formula gives in IEEE arithmetic.
 */
typedef struct ppas_head_norm {
  const void* weight;   /* device bf16: head_dim weights, or a row of them per head; NULL: no weights
                           (z without its last factor) */
  int64_t head_stride;  /* elements between the heads' rows, at least head_dim; 0: one row for all heads */
  float eps;            /* finite, at least 2^-100 */
  float offset;         /* added to every weight (1 where a model holds differences from one), finite */
  int32_t center;
} ppas_head_norm;

/*
 * As ppas_rope_rows (without `transposed`) and ppas_rope_qkv_append, of normalised
 * heads: the rows' heads, or a step's queries and keys, each with their norm. Values are
 * copied as they are. PPAS_EINVAL also for a norm that is NULL or out of range, and for
 * outputs (the pools whole) that overlap the weights. Weights on 16 bytes with a
 * head_stride that is a multiple of 8 are faster.
 */
ppas_status ppas_norm_rope_rows(const ppas_head_norm* norm, const ppas_rope* rope, const void* x, int64_t x_stride,
                                void* y, int64_t y_stride, const int32_t* positions_dev, int32_t n_rows,
                                int32_t n_heads, int32_t head_dim, const ppas_events* events, void* hip_stream);

ppas_status ppas_norm_rope_qkv_append(const ppas_shape* shape, const ppas_head_norm* q_norm,
                                      const ppas_head_norm* k_norm, const ppas_rope* rope, const ppas_qkv* rows,
                                      void* q_out, void* k_pages, void* v_pages, const ppas_seq* seqs, int32_t n_seqs,
                                      const int32_t* block_table_dev, int32_t bt_stride,
                                      const int32_t* block_table_host, void* hip_stream);

/*
 * Requests first_seq .. first_seq + n_seqs - 1 of a step hold the same first `len`
 * positions in the same pages (a system prompt, a document, sampled continuations):
 * their block-table rows start with the same len / 16 entries. len is a multiple of 16
 * (whole pages) and at most every member's cached_len; 0 shares nothing. Prefixes of a
 * step are given in request order and do not overlap.
 */
typedef struct ppas_prefix {
  int32_t first_seq, n_seqs, len;
} ppas_prefix;

/*
 * Device workspace that ppas_attn_step needs for this step description on the
 * current device, with the automatic planning choices. This sizing call is the
 * library's own (the paper describes no workspace): the workspace holds the
 * fp32 partial results of rows whose keys are split across workgroups of the
 * launch (at least 256 bytes). Depends only on the shape, the descriptors and
 * the device's compute-unit count. Returns 0 if the description is invalid.
 */
size_t ppas_attn_workspace_bytes(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs);

/*
 * Attention of every query row of the step (Section 2 chunked prefill and
 * decode; Section 6.2 mixed iterations). For request s, row i at position
 * p = cached_len + i, query head h and KV head g = h / 8:
 *   out[query_start+i][h][:] = sum_{j<=p} softmax_j(scale * q[.][h] . K_s[j][g]) V_s[j][g][:]
 * where K_s/V_s are request s's keys/values at positions 0..p read from the
 * pages through block_table (the step's own keys must already be appended).
 * Prefill rows (n_query > 1) are causal within their chunk and see the whole
 * cached prefix; decode rows (n_query == 1) see cached_len + 1 keys. Inputs bf16,
 * fp32 accumulation, output rounded to bf16 (nearest even).
 * All rows of all requests run in one packed launch; rows whose keys were split
 * across workgroups are merged by a second, small launch.
 * workspace: device buffer of at least ppas_attn_workspace_bytes() bytes, owned
 * by the caller, not read before being written; it must not be used by another
 * call still in flight. The work list travels in pinned host memory from a pool
 * the library owns, read by the kernels directly; a buffer of the pool is
 * reused only after the launches that read it have completed; a replay would
 * read it later, so a call on a stream that captures a HIP graph is
 * PPAS_EUNSUPPORTED (ppas_attn_step_noalloc can be captured). Calls from several threads or on several streams are safe (each
 * with its own workspace). Equivalent to creating a step plan with default
 * options, ppas_attn_step_planned, and destroying the plan.
 * Returns PPAS_OK, a validation status, PPAS_ENOSPACE or PPAS_EHIP.
 */
ppas_status ppas_attn_step(const ppas_shape* shape, void* out, const void* q,
                           const void* k_pages, const void* v_pages,
                           const ppas_seq* seqs, int32_t n_seqs,
                           const int32_t* block_table_dev, int32_t bt_stride,
                           const int32_t* block_table_host,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Step plans. One scheduler iteration runs every decoder layer over the same
 * batch of requests (Section 2: an iteration processes the batch's tokens
 * through the model; Section 6.1 profiles one decoder block of it), so the
 * host work of a step (validation, the attention work list, the page-write
 * list) is the same for every layer. A plan holds that work once, for as many
 * launches as the caller makes with it: ppas_kv_append_planned,
 * ppas_rope_kv_append_planned and ppas_attn_step_planned then only launch
 * kernels. The plan keeps the shape, the descriptors' work and bt_stride; each
 * planned call takes the layer's device buffers and block table (same stride).
 *
 * ppas_step_plan_create validates as ppas_validate_step does (with the range
 * and overlap checks when block_table_host is not NULL), plans with `opts`
 * (NULL = automatic) for the current device, and stores the lists in pinned
 * host memory from the library's pool. *plan receives the handle (NULL on
 * error). Returns PPAS_OK, a validation status, PPAS_ERANGE for a step too
 * large for the int32 work list, PPAS_EUNSUPPORTED without a gfx950 device, or
 * PPAS_EHIP.
 */
typedef struct ppas_step_plan ppas_step_plan;

ppas_status ppas_step_plan_create(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                                  const int32_t* block_table_host, int32_t bt_stride,
                                  const ppas_plan_opts* opts, ppas_step_plan** plan);

/*
 * As ppas_step_plan_create, for a step some of whose requests share prefixes (the
 * library's own; the paper's requests share nothing). The plan's attention reads a
 * shared prefix once for all rows of its group, in tiles of matrix instructions that
 * hold rows of several requests, then each request's own keys, and merges the two by
 * their log-sum-exp. The results are those of ppas_attn_step but for the order of the
 * sums and the pieces of keys, within which probabilities are rounded to bf16 relative
 * to the largest: 64 decode rows behind 8,192 shared keys are 2.3e-3 of their size from
 * 64-bit sums with either call. Used are whole blocks of 64 keys of a prefix; requests
 * of more than 64 new tokens fill tiles of their own and read it for themselves, groups
 * that need as many tiles together as apart are not shared, and a step that would save
 * little, or with chunks in its groups take longer, is planned without sharing
 * (opts->prefill_split > 0 shares whatever it saves). Choosing the plan takes host time
 * (about 50 us for 64 decode rows, 20 without prefixes), so a plan made once for all
 * layers pays sooner than a call that plans for itself. The pages of a prefix are taken
 * from its first member's table row. PPAS_EINVAL for a prefix out of range, out of
 * order, of a length that is no multiple of 16 or longer than a member's cached_len, or,
 * when block_table_host is not NULL, whose members' entries differ. n_prefixes == 0
 * (prefixes may be NULL) is ppas_step_plan_create. Used and destroyed like any plan.
 */
ppas_status ppas_step_plan_create_shared(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                                         const ppas_prefix* prefixes, int32_t n_prefixes,
                                         const int32_t* block_table_host, int32_t bt_stride,
                                         const ppas_plan_opts* opts, ppas_step_plan** plan);

/* As ppas_attn_step and ppas_attn_workspace_bytes, for a step with shared prefixes:
 * equivalent to ppas_step_plan_create_shared with default options,
 * ppas_attn_step_planned, and destroying the plan. */
ppas_status ppas_attn_step_shared(const ppas_shape* shape, void* out, const void* q,
                                  const void* k_pages, const void* v_pages,
                                  const ppas_seq* seqs, int32_t n_seqs,
                                  const ppas_prefix* prefixes, int32_t n_prefixes,
                                  const int32_t* block_table_dev, int32_t bt_stride,
                                  const int32_t* block_table_host,
                                  void* workspace, size_t workspace_bytes, void* hip_stream);

size_t ppas_attn_shared_workspace_bytes(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                                        const ppas_prefix* prefixes, int32_t n_prefixes);

/* What a plan launches (host only). */
typedef struct ppas_plan_info {
  int32_t n_items;          /* workgroups of the packed attention launch */
  int32_t n_merge;          /* split-merge items (0: no merge launch) */
  int32_t tile_positions;   /* 16 or 32 */
  int32_t n_append;         /* (request, page) workgroups of a page-write launch */
  uint64_t workspace_bytes; /* workspace ppas_attn_step_planned needs */
} ppas_plan_info;

ppas_status ppas_step_plan_info(const ppas_step_plan* plan, ppas_plan_info* info);

/* As ppas_kv_append, with the plan's descriptors and validation; events may be NULL. */
ppas_status ppas_kv_append_planned(const ppas_step_plan* plan, void* k_pages, void* v_pages,
                                   const void* k_new, const void* v_new,
                                   const int32_t* block_table_dev, const ppas_events* events,
                                   void* hip_stream);

/* As ppas_rope_kv_append, with the plan's descriptors and validation; events may be NULL. */
ppas_status ppas_rope_kv_append_planned(const ppas_step_plan* plan, float rope_theta, void* q,
                                        void* k_pages, void* v_pages,
                                        const void* k_new, const void* v_new,
                                        const int32_t* block_table_dev, const ppas_events* events,
                                        void* hip_stream);

/* As ppas_rope_qkv_append, with the plan's descriptors and validation; events may be NULL. */
ppas_status ppas_rope_qkv_append_planned(const ppas_step_plan* plan, const ppas_rope* rope, const ppas_qkv* rows,
                                         void* q_out, void* k_pages, void* v_pages,
                                         const int32_t* block_table_dev, const ppas_events* events,
                                         void* hip_stream);

/* As ppas_norm_rope_qkv_append, with the plan's descriptors and validation; events may be NULL. */
ppas_status ppas_norm_rope_qkv_append_planned(const ppas_step_plan* plan, const ppas_head_norm* q_norm,
                                              const ppas_head_norm* k_norm, const ppas_rope* rope,
                                              const ppas_qkv* rows, void* q_out, void* k_pages, void* v_pages,
                                              const int32_t* block_table_dev, const ppas_events* events,
                                              void* hip_stream);

/*
 * As ppas_attn_step, with the plan's descriptors, validation and work list
 * (workspace of at least ppas_plan_info.workspace_bytes); events may be NULL.
 * Calls with one plan may run on several streams at once, each with its own
 * workspace.
 */
ppas_status ppas_attn_step_planned(const ppas_step_plan* plan, void* out, const void* q,
                                   const void* k_pages, const void* v_pages,
                                   const int32_t* block_table_dev,
                                   void* workspace, size_t workspace_bytes,
                                   const ppas_events* events, void* hip_stream);

/*
 * Release a plan (NULL is a no-op). Does not wait: the plan's pinned memory
 * returns to the pool and is reused only after every launch made with the plan
 * has completed.
 */
void ppas_step_plan_destroy(ppas_step_plan* plan);

/*
 * Work-list introspection for tests (host only, no HIP call). Plans the step
 * with `opts` (NULL = automatic; num_cus 0 = 256 compute units) and writes at
 * most `capacity` items of 8 int32 each to `items_out` (kind, seq, kv_head, row0,
 * pos0, npos, key_lo, key_hi per item, in launch order; kind 0 = prefill tile,
 * 1 = decode row). Returns the number of items, or a negative ppas_status
 * (PPAS_EINVAL also for an invalid opts field).
 */
int32_t ppas_plan_items(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                        const ppas_plan_opts* opts, int32_t* items_out, int32_t capacity);

/*
 * The same of a step with shared prefixes: items whose rows belong to several requests
 * come with their prefix's first request as seq and the prefix's used length as pos0, and
 * behind the launch's items, with kind 2, those decode rows that one wave takes.
 */
int32_t ppas_plan_shared_items(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                               const ppas_prefix* prefixes, int32_t n_prefixes,
                               const ppas_plan_opts* opts, int32_t* items_out, int32_t capacity);

/*
 * The fused gate-up projection of a decoder block's MLP, the other prefill
 * operation the paper profiles next to attention (Section 6.1: cumulative time
 * of eight 2k chunks against one 16k chunk, Fig. 4b; SM throughput, L2 hit rate
 * and DRAM throughput at both chunk sizes, Table 6). The gate and up
 * projections read the same hidden states and run as one linear layer whose
 * weight stacks the gate rows over the up rows:
 *   y[t][n] = sum_k x[t][k] * w[n][k]      t < n_tokens, n < n_out
 * x [n_tokens][hidden] bf16 (the chunk's normalised hidden states), w
 * [n_out][hidden] bf16 (row-major, gate rows 0..n_out/2-1 then up rows; any
 * n_out >= 1 is accepted), y [n_tokens][n_out] bf16, all device memory owned by
 * the caller. fp32 accumulation, output rounded to bf16 nearest-even; the
 * activation that follows is not applied. When a call's 256 x 256 output
 * tiles are fewer than the device's compute units, the reduction over hidden
 * may be split across several workgroups per tile; their fp32 partial sums go to
 * the caller's workspace (ppas_gateup_workspace_bytes, device memory, not read
 * before written, not shared with a call still in flight) and a second launch
 * adds them in a fixed order. A workspace smaller than that (NULL with 0 bytes
 * included) gives fewer splits, down to none. The kernel, and with it the order of
 * the sums, is chosen by the shape, the workspace size, the device's compute units
 * and whether x and w both start on a 16-byte boundary: results are deterministic
 * where these are the same, and every choice stays within the same rounding bound.
 * The kernels run on hip_stream (events: start on the first
 * launch, stop on the last, as for the other calls; may be NULL); no host sync.
 * hidden must be a positive multiple of 64 (PPAS_EUNSUPPORTED otherwise);
 * n_tokens == 0 is a no-op; NULL pointers (a NULL workspace with a non-zero
 * size included) or non-positive sizes are PPAS_EINVAL; n_tokens or n_out above
 * 2^31 - 513, or more than 2^31 - 1 output tiles of 256 x 256, is PPAS_ERANGE.
 */
ppas_status ppas_gateup_proj(const void* x, const void* w, void* y, int32_t n_tokens, int32_t hidden,
                             int32_t n_out, void* workspace, size_t workspace_bytes,
                             const ppas_events* events, void* hip_stream);

/* The most workspace ppas_gateup_proj can use for this shape on the current device
 * (0 when it does not split the reduction, or for an invalid shape): that of about
 * one workgroup per compute unit. Aligned operands often take fewer splits and
 * touch less of it. The library's own sizing call: the paper describes no
 * workspace. */
size_t ppas_gateup_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_out);

/*
 * The same projection with the MLP's gated activation applied on the way out:
 * the paper profiles the projection (Section 6.1, Fig. 4b, Table 6); in the
 * Qwen2.5 models it measures, the MLP then multiplies the SiLU of the gate half
 * by the up half, and doing that in the projection's epilogue writes half the
 * bytes and saves a pass over them (the library's own fusion). With n_inter
 * intermediate features and w [2 n_inter][hidden] (gate rows 0..n_inter-1, then
 * the up rows of the same features):
 *   y[t][f] = silu(g) * u,  g = sum_k x[t][k] w[f][k],  u = sum_k x[t][k] w[n_inter + f][k],
 *   silu(g) = g / (1 + e^-g),  t < n_tokens, f < n_inter
 * y [n_tokens][n_inter] bf16; g and u are accumulated in fp32 as in
 * ppas_gateup_proj, silu(g) * u is evaluated in fp32 and rounded to bf16
 * nearest-even. Workspace, splits, events, streams and status codes as for
 * ppas_gateup_proj with n_out = 2 n_inter; n_inter above (2^31 - 513) / 2 is
 * PPAS_ERANGE.
 */
ppas_status ppas_gateup_act(const void* x, const void* w, void* y, int32_t n_tokens, int32_t hidden,
                            int32_t n_inter, void* workspace, size_t workspace_bytes,
                            const ppas_events* events, void* hip_stream);

/* The most workspace ppas_gateup_act can use for this shape on the current device
 * (0 when it does not split the reduction, or for an invalid shape). The library's
 * own sizing call. */
size_t ppas_gateup_act_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_inter);

/*
 * 8-bit integers for the projections (the library's own; the paper's models run in
 * bf16). Rows of activations (one per token) or weights (one per output channel) to
 * 8-bit integers and a scale: for row r < n_rows of x (bf16, x_stride elements apart,
 * `hidden` of them), with m its largest magnitude,
 *   scale[r] = m / 127 (fp32),  xq[r][i] = 127 x[r][i] / m to the nearest integer, ties
 * to even, in -127..127. xq [n_rows][hidden] int8, scale [n_rows] fp32. A row whose m is
 * below 2^-110 gives zeros and scale 0; a row that holds an infinity or a NaN gives zeros
 * and a NaN scale, which makes every product with it NaN. hidden is any positive size;
 * multiples of 8 on 16 bytes (x and x_stride) are faster. n_rows == 0 is a no-op; NULL
 * pointers, an x_stride below hidden or non-positive sizes are PPAS_EINVAL. x and the
 * outputs must not overlap. One launch, no workspace, no host sync.
 */
ppas_status ppas_quant_i8(const void* x, int64_t x_stride, void* xq, float* scale, int32_t n_rows, int32_t hidden,
                          const ppas_events* events, void* hip_stream);

/*
 * ppas_gateup_proj and ppas_gateup_act on such rows: x [n_tokens][hidden] and w
 * [n_out][hidden] (or [2 n_inter][hidden]) int8, -128 included, with x_scale [n_tokens]
 * and w_scale [n_out] (or [2 n_inter]) fp32:
 *   s[t][n] = x_scale[t] w_scale[n] sum_k x[t][k] w[n][k]
 * written as y[t][n] = s[t][n], or as y[t][f] = silu(s[t][f]) s[t][n_inter + f], bf16
 * nearest-even. The sums are exact int32, so that results depend neither on the number
 * of tokens beside a token, nor on the workspace or kernel; the product of the scales,
 * the sum and their product are each rounded to fp32. hidden is 1..131071 (the sums
 * then fit; above: PPAS_ERANGE); multiples of 128 from 256 on, with x and w on 16 bytes,
 * are fast, and may be split over workgroups with int32 partial sums in the workspace
 * (optional, as in ppas_gateup_proj; any size, 16-byte aligned). x_scale and w_scale may be any fp32
 * values. n_tokens == 0 is a no-op. Other arguments, events, streams and errors as for
 * ppas_gateup_proj. No call allocates or keeps anything; each may be captured into a
 * HIP graph, and graphs that share a workspace must not run at once.
 */
ppas_status ppas_gateup_proj_i8(const void* x, const float* x_scale, const void* w, const float* w_scale, void* y,
                                int32_t n_tokens, int32_t hidden, int32_t n_out, void* workspace,
                                size_t workspace_bytes, const ppas_events* events, void* hip_stream);

ppas_status ppas_gateup_act_i8(const void* x, const float* x_scale, const void* w, const float* w_scale, void* y,
                               int32_t n_tokens, int32_t hidden, int32_t n_inter, void* workspace,
                               size_t workspace_bytes, const ppas_events* events, void* hip_stream);

/* The most workspace that such a call can use for this shape on the current device (0
 * when it does not split the reduction, or for an invalid shape). */
size_t ppas_gateup_i8_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_out);
size_t ppas_gateup_act_i8_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_inter);

/*
 * Low-rank adapters of many requests beside a shared projection (the library's own; the
 * paper's requests run the plain model). A set holds n_adapters adapters of one projection
 * from `hidden` to n_out features: A [n_adapters][rank][hidden] and B [n_adapters][n_out]
 * [rank] bf16, contiguous, and a scale each; ranks below the set's are padded with zeros. A
 * row t with adapter a gets
 *   out[t] = y[t] + scale[a] (x[t] A_a^T) B_a^T
 * on top of the projection's output y (any projection of this library or another, bf16),
 * and a row of no adapter out[t] = y[t]. The product with A is fp32, so is that with B
 * and its sum with y, which is rounded once to bf16 nearest-even. Weights have to be finite.
 *
 * Rows of one adapter may lie anywhere in a step: ppas_adapter_rows brings the row numbers
 * into the order of their adapters once per step, for every layer and projection that uses
 * as many adapters. row_adapter_dev [n_tokens] holds the rows' adapters; -1, like every
 * number outside 0..n_adapters - 1, is a row without one. `rows` is device memory of
 * ppas_adapter_rows_bytes(n_tokens, n_adapters) on 16 bytes, not over row_adapter_dev; the calls that read it have to
 * be given the n_tokens and adapters it was made for (others' results are undefined, but
 * stay inside the call's rows) and must come behind it on their stream.
 */
typedef struct ppas_adapters {
  const void* a;
  const void* b;
  const float* scale;    /* device fp32 [n_adapters]; NULL: 1 */
  int32_t n_adapters;    /* 1..1024 (PPAS_EUNSUPPORTED above) */
  int32_t rank;          /* 1..128 (PPAS_EUNSUPPORTED above) */
  int32_t hidden, n_out;
} ppas_adapters;

size_t ppas_adapter_rows_bytes(int32_t n_tokens, int32_t n_adapters);

ppas_status ppas_adapter_rows(const int32_t* row_adapter_dev, int32_t n_tokens, int32_t n_adapters, void* rows,
                              size_t rows_bytes, const ppas_events* events, void* hip_stream);

/*
 * The adapters' share added to y [n_tokens][n_out], x being the projection's input
 * [n_tokens][hidden]; strides are elements between rows, so that parts of fused rows may be
 * given. out may be y with the same stride: rows without an adapter are then not touched;
 * otherwise it must not overlap y, nor ever x, the set or `rows`; the workspace must not
 * overlap any of these (PPAS_EINVAL, as for strides below a row's features). `workspace` is device memory of ppas_adapter_workspace_bytes() on 16 bytes. That is
 * not the largest for the most rows: few rows split hidden further. A smaller one gives
 * fewer splits (one made for a server's largest step serves all of them), down to n_tokens
 * times the rank, rounded up to 16, 32, 64 or 128, in fp32; below that PPAS_ENOSPACE. Bases and strides on 16 bytes with hidden, rank and n_out
 * that are multiples of 8 are faster. Two launches (events: start on the first, stop on the
 * last); nothing is allocated or kept, and calls may be captured into a HIP graph; calls
 * that share a workspace must not run at once. A row's result may differ in the rounding
 * of its sums with n_tokens, n_adapters and the workspace, on which the split of hidden
 * depends.
 * n_tokens == 0 is a no-op, above 2^24 PPAS_ERANGE.
 */
ppas_status ppas_adapter_add(const ppas_adapters* set, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                             void* out, int64_t out_stride, int32_t n_tokens, const void* rows, size_t rows_bytes,
                             void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream);

/*
 * The same before the MLP's gated activation: y holds the gate and up halves [n_tokens]
 * [n_out] as ppas_gateup_proj (or ppas_gateup_proj_i8) writes them, B the rows of both, and
 *   out[t][f] = silu(g) u,  f < n_out / 2
 * with g and u the two halves of y[t] with the adapters' share, not rounded before; out
 * [n_tokens][n_out / 2] must not overlap y or x. n_out is even.
 */
ppas_status ppas_adapter_act(const ppas_adapters* set, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                             void* out, int64_t out_stride, int32_t n_tokens, const void* rows, size_t rows_bytes,
                             void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream);

/* The most workspace that such a call can use on the current device. */
size_t ppas_adapter_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t rank, int32_t n_adapters);

/*
 * Log probabilities of logit rows, as a request is answered with them: of a given token per
 * row (a sampled one, or a prompt's next), its rank, the row's entropy and the top
 * alternatives (the library's own; the paper's requests are measured, not read). Row r <
 * n_rows holds `vocab` logits x_i (type PPAS_BF16 or PPAS_F32, row_stride elements apart,
 * any alignment of their type); with l_i = scale x_i (scale: 1 / temperature) and
 * lse = ln sum_i e^(l_i):
 *   logprob[r] = l_t - lse, t = tokens_dev[r]
 *   rank[r]    = the number of tokens before t: of a larger x, or an equal one and a lower
 *                number; -1 if e^(l_t) is 0 because x_t is -infinity
 *   entropy[r] = lse - sum_i p_i l_i, p_i = e^(l_i - lse)
 *   top_ids[r][j], top_logprobs[r][j], j < top_k: the tokens in that order and their
 *                l - lse; -1 and -infinity behind the last token that is not masked
 * A logit of -infinity has probability 0 and adds nothing. A row with a NaN, a +infinity or
 * nothing but -infinity has no distribution: its results are NaN, its ids and ranks -1. A
 * token out of range (-1: none given) has logprob NaN and rank -1. Sums are fp32: up to 2^18
 * tokens, a log probability is within 2e-5 + 2^-20 D + 2^-22 of its own size, D the spread of
 * the row's l_i that are not masked, counted up to 104 (what is further down adds nothing).
 * The order is that of the logits themselves, before any rounding. Outputs may each be NULL, and
 * must not overlap the logits (PPAS_EINVAL) or each other; logprob and rank need
 * tokens_dev. top_k is 0..64 (PPAS_EUNSUPPORTED above); scale is 2^-100..2^100; vocab at
 * most 2^30 (PPAS_ERANGE). Few rows are split over workgroups that meet in the workspace
 * (ppas_logprobs_workspace_bytes, 16-byte aligned; a smaller one, NULL with 0 bytes
 * included, gives fewer splits), by which the sums' rounding, but no id or rank, may
 * differ. Nothing is allocated or kept; a call may be captured into a HIP graph, and calls
 * that share a workspace must not run at once. n_rows == 0 is a no-op.
 */
enum { PPAS_BF16 = 0, PPAS_F32 = 1 };

typedef struct ppas_logprob_out {
  float* logprob;        /* [n_rows] */
  int32_t* rank;         /* [n_rows] */
  float* entropy;        /* [n_rows] */
  int32_t* top_ids;      /* [n_rows][top_k] */
  float* top_logprobs;   /* [n_rows][top_k] */
} ppas_logprob_out;

ppas_status ppas_logprobs(const void* logits, int32_t type, int64_t row_stride, int32_t n_rows, int32_t vocab,
                          float scale, const int32_t* tokens_dev, int32_t top_k, const ppas_logprob_out* out,
                          void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream);

/* The most workspace that such a call can use on the current device (0 where rows are not
 * split, or for an invalid shape). */
size_t ppas_logprobs_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t top_k);

/*
 * Kernel choice of a projection call, for tests (host only, no HIP call): the
 * kernel that ppas_gateup_proj, or with `activation` ppas_gateup_act (n_out = 2
 * n_inter), takes for this shape and workspace size on a device of num_cus compute
 * units (0 = 256), `aligned` if x and w are. Writes 8 int32 to `choice`: kernel (0
 * tiles, 1 few rows, 2 general), token rows of a main tile (64: none, 64-row tiles
 * only) or few-row workgroup, main tiles and 64-row tiles along the tokens, weight-row tiles of a few-row
 * workgroup and their rows, reduction splits, 64-feature stages whose sum is added
 * to the total at a time (main tiles of 256 rows and the general kernel keep one
 * chain per split instead). PPAS_EINVAL for n_tokens == 0.
 */
ppas_status ppas_gateup_choice(int32_t n_tokens, int32_t hidden, int32_t n_out, int32_t activation,
                               int32_t aligned, size_t workspace_bytes, int32_t num_cus, int32_t* choice);

/*
 * The same of an 8-bit product: 16 int32, eight for each of its launches (a reducing one
 * apart): token rows (0: no second launch, else the call's last rows), kernel (0 tiles, 1
 * few rows, 2 general, 3 tiles of 128 x 128), then as above from the rows of a main tile to
 * the reduction splits.
 */
ppas_status ppas_gateup_i8_choice(int32_t n_tokens, int32_t hidden, int32_t n_out, int32_t activation,
                                  int32_t aligned, size_t workspace_bytes, int32_t num_cus, int32_t* choice);

/*
 * A plain streaming read of `bytes` bytes of device memory at `buf`: the
 * device's attainable HBM read rate, the measured ceiling beside the spec peak
 * for the memory-bound kernels above (the library's own measurement aid, not a
 * step of the method). Every 16-byte word is read once with nontemporal loads by
 * one 256-thread workgroup per compute unit, each wave reading contiguous 8 KB
 * runs; the XOR of all words, as four uint32 lanes, is XORed into the 16 bytes
 * of device memory at `sink` (zero it first to receive the XOR itself), so the
 * reads cannot be elided and the result is checkable. `buf` and `bytes` must be multiples of 16 and `sink`
 * 4-byte aligned (PPAS_EINVAL otherwise); bytes == 0 is a no-op. Enqueued on
 * hip_stream without a host sync; the launch records `events` if given.
 */
ppas_status ppas_stream_read(const void* buf, size_t bytes, void* sink, const ppas_events* events,
                             void* hip_stream);

/*
 * For callers that cannot allocate memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc. Computes exactly what
 * ppas_attn_step computes, with the same plan and kernels (bit-identical
 * output), but takes no workspace and uses neither a caller buffer nor the
 * library's pinned host pool: the step's work list (32 bytes per work item)
 * and, after it, the fp32 partials of rows split across workgroups live in a
 * fixed device array of PPAS_NOALLOC_SCRATCH_BYTES that every device the call
 * runs on holds until the process ends. The call allocates nothing
 * (no hipMalloc, hipFree, hipHostMalloc); the first call on a device looks up
 * that device's array (hipGetSymbolAddress).
 *
 * The work list is copied from host memory to the array with hipMemcpyAsync on
 * hip_stream during the call, then the attention and merge launches follow on
 * the same stream. Every call on one device shares that device's array, which
 * keeps the last call's contents (nothing in it needs to start at zero): calls
 * ordered on one stream are safe, but calls that overlap in time on one device
 * (other streams, other threads) race and give undefined results. A call may be
 * captured into a HIP graph, whose replays copy the list again: it stays in host
 * memory until the process ends.
 *
 * A step whose work list and partials do not fit the array returns
 * PPAS_ENOSPACE and enqueues nothing (steps of up to ~40 MB of partials fit,
 * e.g. two 1,024-token chunks plus 48 decode rows of 20k-30k keys).
 * Arguments, validation and other errors as ppas_attn_step.
 */
#define PPAS_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)

ppas_status ppas_attn_step_noalloc(const ppas_shape* shape, void* out, const void* q,
                                   const void* k_pages, const void* v_pages,
                                   const ppas_seq* seqs, int32_t n_seqs,
                                   const int32_t* block_table_dev, int32_t bt_stride,
                                   const int32_t* block_table_host, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* PPAS_H */
