/*
 * pic.h -- link-stage attention over position-independent chunk caches, on
 * one AMD Instinct MI355X (gfx950).
 *
 * The method (Comb, "You Need an Encoder for Native Position-Independent
 * Caching"): each static context chunk is compiled once into key/value
 * caches computed from position zero (Sec. 1, Fig. 1; Sec. 4.2 stores the
 * cross-attention K and V). A request is a question plus zero or more
 * contexts in any order (Sec. 3). In the link stage the request's chunk
 * caches are looked up by id (Sec. 3, step 1), concatenated in request order
 * along the document axis (Sec. 4.2), and the request's dynamic tokens
 * attend over them -- without a mask (cross-attention, Sec. 4.2 Eq. 7-8) --
 * and over their own KV under a causal mask (Sec. 4.1 Eq. 2-3), all under
 * one softmax here. The PIC allocator owns a pool of GPU memory reserved
 * when the system starts (Sec. 5.3).
 *
 * Math computed for request r, query row i (0 <= i < L_q), query head h:
 *   keys  = [ K_{c_1} ; ... ; K_{c_n} ; K_own[0 .. i + L_s - L_q] ]
 *   s_j   = softmax_scale * <q[i,h], keys_j[h / (H_q/H_kv)]>
 *   out[i,h] = sum_j softmax(s)_j * values_j[h / (H_q/H_kv)]
 *   lse[i,h] = log(sum_j exp(s_j))   (natural log; -inf and out = 0 if no key)
 * The query rows are the last L_q of the L_s own tokens (bottom-right causal
 * alignment): new tokens are appended to the query sequence (Sec. 4).
 * MLA (absorbed latent form, Sec. 5.1 DeepSeek-V2-Lite backbone): one KV
 * "head" whose rows are [latent | rope] (d_k wide); the value of a row is its
 * first d_v entries, and the output is the latent (d_v wide) per head.
 *
 * Conventions for every call:
 *   - Status codes are negative on error. All validation happens on the host
 *     before any device work: an error launches nothing and writes nothing.
 *     pic_last_error() gives a thread-local message about the last error.
 *   - Device pointers are HIP device allocations on the current device;
 *     "host" arrays are ordinary host memory, read before the call returns.
 *   - `stream` is a hipStream_t (NULL = the null stream). All device work is
 *     enqueued on it; calls return before it runs.
 *   - Tensors are dense, row-major, with no padding, in the store's dtype
 *     (fp32, or bf16 as raw 16-bit patterns) unless stated; lse is fp32.
 *   - One host thread uses a store at a time. Outputs of calls that are in
 *     flight on different streams must not alias.
 *   - Each pic_link_attn / pic_link_decode call gets a device workspace of
 *     its own (the request's own KV laid out for the kernels, and partial
 *     results of split key ranges): a store keeps eight, handed out in turn,
 *     and one is reused only once the call that last used it has completed,
 *     so calls may be in flight on different streams at once; a ninth call
 *     waits on the host for the oldest of the eight. Runs of one link plan
 *     share the plan's workspace instead (see pic_link_plan_run).
 */
#ifndef PIC_H
#define PIC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PIC_OK = 0,
  PIC_ERR_INVALID = -1,      /* bad argument, shape or layout */
  PIC_ERR_NOT_FOUND = -2,    /* a linked chunk id is not in the store */
  PIC_ERR_EXISTS = -3,       /* put of an id already stored (chunks are immutable) */
  PIC_ERR_OOM = -4,          /* the store's pool has no room */
  PIC_ERR_HIP = -5,          /* a HIP runtime call failed */
  PIC_ERR_UNSUPPORTED = -6   /* valid request this build has no kernel for */
} pic_status;

/* pic_store_desc.dtype. PIC_FP4: chunk caches are held in 4 bits (17 bytes per
 * 32 elements); see below. */
enum { PIC_F32 = 0, PIC_BF16 = 1, PIC_FP4 = 2 };
enum { PIC_GQA = 0, PIC_MLA = 1 };      /* pic_store_desc.kind  */

/* 4-bit stores (dtype PIC_FP4; GQA only, d_k = d_v of 64 or 128, else
 * UNSUPPORTED). Everything that goes in or out is bf16: k and v of pic_store_put
 * and pic_store_write_rows, q, k_self, v_self and out of the link calls, and
 * the values that pic_debug_gather returns. What a put rounds: a row (one
 * token of one head) is cut into blocks of 32 elements; a block keeps the
 * numbers 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, times 2^e, where e is the
 * smallest exponent in -126 .. 125 with max|x| < 7 * 2^e (125 where there is
 * none). Elements are rounded to the nearest such number, ties to the one
 * with the even index in that list; what lies above 6 * 2^e, infinities too,
 * becomes 6 * 2^e. A block with a NaN reads as NaN throughout. A row's numbers depend
 * on that row alone. The request's own KV is not rounded. Store calls, link
 * calls, plans and export work as for the other dtypes. Link calls round each
 * probability to bf16 for its product with the values (at most 2^-8 of it) and
 * the output once; sums are fp32. The output is a mean of the values that a row
 * sees and stays finite for every finite one, cached infinities (6 * 2^125)
 * among them, but for own values within 1% of bf16's largest; dot products have to
 * lie in the fp32 range. A NaN in the cached
 * or own V, or an infinity in the own V, may reach every row of the requests
 * that link it, also rows that a limit or the causal mask keeps from it; a
 * query row with a NaN or an infinity gives an output row of NaN or zeros. */

/* Shape of a store's chunk caches. d_k and d_v must be multiples of 8.
 * GQA: n_kv_heads >= 1, separate K [.., d_k] and V [.., d_v] per head.
 * MLA: n_kv_heads == 1, d_v <= d_k, the value is the first d_v of each key row.
 * n_layers: cross-attention layers per chunk, 0 or 1 for one. Comb
 *   interleaves L_cross cross-attention layers with the decoder (Sec. 4.2
 *   and 4.3, Fig. 3: 8 among 32 decoder layers; Eq. 12), and each reads its
 *   own K and V of every document; a chunk's caches of all layers are put
 *   together and each link call names its layer.
 * capacity_tokens: pool size in tokens per layer, in pages of 64 tokens.
 * Each chunk occupies its length rounded up to whole pages in every layer,
 * in one run of consecutive pages when a free run is long enough, else in
 * several (removal leaves holes; no copy ever moves a chunk). */
typedef struct pic_store_desc {
  int32_t kind;
  int32_t dtype;
  int32_t n_kv_heads;
  int32_t d_k;
  int32_t d_v;
  int32_t n_layers;          /* 0..256; 0 and 1 both mean one layer */
  int64_t capacity_tokens;
} pic_store_desc;

typedef struct pic_store pic_store;

/* Creates a chunk store on the current HIP device and reserves its pool
 * (the PIC allocator's reservation, Sec. 5.3): capacity_tokens per layer.
 * *out receives the handle.
 * Errors: INVALID (desc), UNSUPPORTED (shape), HIP (allocation failed). */
pic_status pic_store_create(const pic_store_desc *desc, pic_store **out);

/* Waits for the device, then frees the store and everything it owns.
 * NULL is accepted and ignored. Errors: INVALID while link plans or block
 * indexes of the store are alive (destroy them first). */
pic_status pic_store_destroy(pic_store *store);

/* Compile-stage entry (Sec. 3 steps 3-4): copies one chunk's caches into the
 * pool and records chunk_id -> slot in the store's hash table.
 *   k: device, [n_layers][n_tokens][n_kv_heads][d_k] (token-major per layer)
 *   v: device, [n_layers][n_tokens][n_kv_heads][d_v] for GQA; NULL for MLA
 * The copy (into the store's internal layout) is ordered on `stream`; the
 * caller may reuse k and v once the stream has passed it.
 * Errors: INVALID, EXISTS (id present), OOM (pool full), HIP. */
pic_status pic_store_put(pic_store *store, uint64_t chunk_id, int64_t n_tokens, const void *k,
                         const void *v, void *stream);

/* Removes a chunk from the store and frees its pages (the paper's allocator
 * hands out free memory, Sec. 5.3, and says nothing of eviction; removal is
 * the caller's policy). The pages are reused only after the work enqueued on
 * `stream` up to this call has completed: pass the stream of the link calls
 * that may still read the chunk. A removed id may be put again.
 * Errors: INVALID (NULL store, or a live link plan links the chunk),
 * NOT_FOUND, HIP. */
pic_status pic_store_remove(pic_store *store, uint64_t chunk_id, void *stream);

/* A chunk that differs from a stored one in a few rows, for the link stage
 * of post-training PIC, which recomputes selected tokens of each document
 * and attends over the cached KV with those rows replaced (Sec. 2: EPIC
 * recomputes the first tokens of every chunk, CacheBlend the tokens whose
 * cached KV deviates most; Sec. 6.1 runs CacheBlend at 20%).
 * pic_store_derive: new_id becomes a chunk with base_id's length and
 *   content. The 64-token pages that hold `rows` (host int32 [n_rows],
 *   strictly increasing, each below the base's length) are private copies
 *   made on `stream`; every other page is shared with the base (no copy).
 *   The base may be removed first: shared pages live while a chunk holds
 *   them (a run of pages allocated together is freed once no chunk holds
 *   any of its pages). Errors: INVALID, NOT_FOUND (base), EXISTS (new_id),
 *   OOM, HIP.
 * pic_store_write_rows: writes token-major K / V rows of one layer into a
 *   derived chunk: k device [n_rows][n_kv_heads][d_k], v device
 *   [n_rows][n_kv_heads][d_v] (GQA) or NULL (MLA); rows as above, each on a
 *   page the chunk holds alone (a page named at pic_store_derive and not
 *   shared since by a later derive). Ordered on `stream`; k and v are read
 *   before the stream passes the call. Link calls already enqueued on
 *   another stream may see either content.
 *   Errors: INVALID (not a derived chunk, a row on a shared page, bad
 *   arguments), NOT_FOUND, HIP. */
pic_status pic_store_derive(pic_store *store, uint64_t new_id, uint64_t base_id, int32_t n_rows,
                            const int32_t *rows, void *stream);
pic_status pic_store_write_rows(pic_store *store, uint64_t chunk_id, int32_t layer,
                                int32_t n_rows, const int32_t *rows, const void *k,
                                const void *v, void *stream);

/* Growing chunks: a request's own tokens kept in the store's pages, so that a decode
 * step hands over its new tokens only (a generated token is appended to the query
 * sequence, Sec. 4) and links the chunk behind its documents.
 * pic_store_open: chunk_id becomes an empty chunk with pages for max_tokens tokens
 *   reserved (1 .. 2^29 - 1). Host only. Errors: INVALID, EXISTS, OOM (pool full),
 *   UNSUPPORTED (a 4-bit store).
 * pic_store_append: tokens offsets[i] .. offsets[i+1]-1 of the sources become the next
 *   rows of growing chunk chunk_ids[i] in one layer (each layer of a chunk grows by
 *   calls of its own; a link call sees what its layer holds). With a rotary handle
 *   (pic_rope_create; its dtype the store's, its head_dim d_k) the keys, and the
 *   queries where q is given, are turned by their positions on the way, as by
 *   pic_rope_apply; v is not. Without one they are copied.
 *     chunk_ids, offsets  host, n_chunks and n_chunks + 1 entries; no id twice
 *     k  device [n][n_kv_heads][d_k], v [n][n_kv_heads][d_v] (NULL for MLA), n =
 *        offsets[n_chunks], token t at t * stride elements (0: dense; else at least a
 *        row: slices of a fused projection)
 *     q, q_out  device [n][n_q_heads][d_k] (strides alike) or both NULL; q_out may be q
 *        (same stride); buffers must not overlap otherwise
 *     positions  device int32 [n], any value (with a handle)
 *   Several chunks of a batch are one launch. Ordered on `stream`; link calls already
 *   enqueued on another stream may see either content of a chunk's last page. A captured
 *   call writes the same rows again when it is replayed, and zeros behind them to the end of a
 *   64-token page that it began: rows appended there since are lost, and a block index is not told
 *   of either. Errors: INVALID (not a growing chunk, one that a live plan links, bad arguments),
 *   NOT_FOUND, OOM (beyond max_tokens), HIP; on an error no chunk has grown.
 * pic_store_truncate: chunk chunk_ids[i] keeps at most its first n_tokens[i] tokens in
 *   every layer (n_tokens[i] at most what some layer holds): tokens that were proposed
 *   and not accepted. The rows taken back are cleared on `stream` as far as they share a page with
 *   rows that stay, by a captured call at each replay. Errors: INVALID, NOT_FOUND, HIP.
 * A growing chunk is linked, gathered, removed and exported like any other (one without
 * tokens adds no rows; pic_store_lookup: the fewest tokens of any layer, which is also what
 * an export holds); a link plan takes it as it stands, with as many tokens in every layer,
 * and it neither grows nor shrinks while the plan lives: a decode loop whose own tokens are in
 * growing chunks makes direct calls, and one that runs a plan hands them over as own KV.
 * pic_store_derive refuses it (INVALID). */
pic_status pic_store_open(pic_store *store, uint64_t chunk_id, int64_t max_tokens);
typedef struct pic_rope pic_rope;
typedef struct pic_append {
  int32_t layer;
  int32_t n_chunks;
  const uint64_t *chunk_ids;
  const int32_t *offsets;
  const void *k;
  const void *v;
  int64_t k_stride, v_stride;
  const pic_rope *rope;      /* or NULL */
  const int32_t *positions;
  const void *q;
  void *q_out;
  int64_t q_stride, q_out_stride;
  int32_t n_q_heads;
} pic_append;
pic_status pic_store_append(pic_store *store, const pic_append *append, void *stream);
pic_status pic_store_truncate(pic_store *store, int32_t n, const uint64_t *chunk_ids,
                              const int64_t *n_tokens, void *stream);

/* Handing a store to another process on the same GPU, in place: the PIC
 * manager of the paper sends the handles of the PICaches it collected to the
 * inference engine over the GPU's inter-process memory API, so tensors pass
 * between processes without copies (Sec. 5.3, System Details).
 * pic_store_export: waits for the device (every put and copy enqueued so far
 *   has landed), then writes a self-contained description of the store --
 *   its shape, an inter-process handle of its pool and its chunk index as it
 *   stands -- into buf (host, buf_bytes). *bytes_out receives the size
 *   needed; buf = NULL only asks for it. Chunks put or removed later are not
 *   in the description: the exporting process keeps the store and the
 *   exported chunks alive (no pic_store_remove, no pic_store_destroy) while
 *   importers use them. Errors: INVALID (NULL store or bytes_out, buffer too
 *   small, an imported store), UNSUPPORTED (pool of 2 GiB or more: the
 *   pool's n_layers * capacity_tokens * H_kv * (d_k + d_v) * esize must stay
 *   below 2^31 bytes), HIP.
 * pic_store_import: in another process on the same GPU (with that device
 *   current), maps the exported pool and rebuilds the chunk index. The result
 *   is a read-only store: link calls, link plans, pic_store_lookup,
 *   pic_store_usage and pic_debug_gather work as on the original;
 *   pic_store_put, pic_store_remove, pic_store_derive and
 *   pic_store_write_rows return INVALID. pic_store_destroy unmaps the pool
 *   (the exporter still owns it). Mapping a pool in the process that
 *   exported it is not supported. Errors: INVALID (not a description made by
 *   pic_store_export, or a corrupt one), HIP (the mapping failed), OOM. */
pic_status pic_store_export(pic_store *store, void *buf, size_t buf_bytes, size_t *bytes_out);
pic_status pic_store_import(const void *buf, size_t buf_bytes, pic_store **out);

/* Hash-table lookup (Sec. 3 step 1): *n_tokens_out = the chunk's length.
 * Errors: INVALID, NOT_FOUND. */
pic_status pic_store_lookup(const pic_store *store, uint64_t chunk_id, int64_t *n_tokens_out);

/* Pool usage in tokens of allocated 64-token pages (pages of removed chunks
 * count until their readers have finished; pages shared by derived chunks
 * count once), the capacity, and the number of stored chunks (derived ones
 * included). Any output pointer may be NULL. */
pic_status pic_store_usage(const pic_store *store, int64_t *used_tokens,
                           int64_t *capacity_tokens, int64_t *n_chunks);

/* A batch of requests (Sec. 3: a question plus zero or more contexts).
 * All arrays are host memory with batch+1 non-decreasing entries from 0.
 *   chunk_offsets/chunk_ids: the links of request r, in request order, are
 *     chunk_ids[chunk_offsets[r] .. chunk_offsets[r+1]-1]; an id may repeat.
 *   q_offsets: the query tokens of request r are rows q_offsets[r].. of q.
 *   self_offsets: own-KV tokens of request r (L_s >= L_q), or NULL for
 *     cross-attention only (no own KV, every row sees only the documents).
 *   chunk_starts: NULL (every link reads its whole chunk), or per link (same
 *     indexing as chunk_ids) the first token of the chunk the link reads: a
 *     multiple of 64 below the chunk's length. Lets a request splice chunk
 *     caches, e.g. the link of post-training PIC that recomputes the first
 *     tokens of every document (Sec. 1 and 2.2; Sec. 6.1 runs EPIC with 64
 *     per document): link [the recomputed tokens, put as a chunk of their
 *     own ; the cached chunk from token 64] for every document.
 *   q_doc_limits: NULL (every query token sees all of its request's linked
 *     rows), or per query token t (indexing as q) the number of leading
 *     linked rows it sees, 0 .. the request's linked rows. Recomputed
 *     tokens attend as in a prefill of the concatenated prompt (Sec. 2,
 *     post-training PIC): a token at position P of the linked rows passes
 *     P + 1 (and the call passes self_offsets = NULL). The own KV, if any,
 *     is not affected. */
typedef struct pic_link_req {
  int32_t batch;
  int32_t layer;             /* the store layer whose chunk caches are read (0 for one layer) */
  const int32_t *chunk_offsets;
  const uint64_t *chunk_ids;
  const int32_t *q_offsets;
  const int32_t *self_offsets;
  const int32_t *chunk_starts;
  const int32_t *q_doc_limits;
} pic_link_req;

/* Link-stage attention for prefill-shaped requests (Sec. 4.1-4.2).
 *   q      device [Tq][n_q_heads][d_k], Tq = q_offsets[batch]
 *   k_self device [Ts][n_kv_heads][d_k], Ts = self_offsets[batch] (NULL if none)
 *   v_self device [Ts][n_kv_heads][d_v] (GQA), NULL for MLA
 *   out    device [Tq][n_q_heads][d_v], store dtype
 *   lse    device [Tq][n_q_heads] fp32 natural-log log-sum-exp, or NULL
 * n_q_heads must be a multiple of n_kv_heads. softmax_scale (positive,
 * finite) multiplies the dot products (Eq. 2 and 7 use 1/sqrt(d)). The chunk table of the call is
 * copied to the device on `stream`; all host arrays are consumed on return.
 * When the batch has too few query rows to fill the GPU (short questions
 * over long documents), the library splits each request's keys and merges
 * the partial softmax states exactly, as pic_link_decode does; the result
 * is the same up to floating-point rounding order.
 * In bf16 GQA stores of d 128 and bf16 MLA stores of 576 / 512, values above
 * 2^61 / T in magnitude may give infinities, T the 64-token tiles that a row
 * sees (pic_link_decode, d 128: only with more than 16 query rows per kv head,
 * or limits that differ within a request).
 * UNSUPPORTED: one request's query rows alone pass what one launch holds
 * (2^23 - 1 workgroups of its row blocks; no limit of the batch).
 * Errors: INVALID, NOT_FOUND, UNSUPPORTED, HIP. */
pic_status pic_link_attn(pic_store *store, const pic_link_req *req, int32_t n_q_heads,
                         const void *q, const void *k_self, const void *v_self,
                         float softmax_scale, void *out, float *lse, void *stream);

/* Link-stage attention for decode-shaped requests (few query tokens each):
 * the same function as pic_link_attn (a generated token is treated like a
 * query token, Sec. 4), computed by splitting each request's keys into
 * num_splits ranges whose partial softmax states are merged exactly
 * (log-sum-exp). num_splits = 0 lets the library choose; otherwise 1..256
 * (a call within pic_link_decode_noalloc's limit may get fewer, see there).
 * Each request may have at most 16 query tokens.
 * Errors: as pic_link_attn. */
pic_status pic_link_decode(pic_store *store, const pic_link_req *req, int32_t n_q_heads,
                           const void *q, const void *k_self, const void *v_self,
                           float softmax_scale, int32_t num_splits, void *out, float *lse,
                           void *stream);

/* pic_link_decode for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc. Same arguments, kernels, split choice and result as
 * pic_link_decode, but the call's tables, own-KV layout and split partials
 * live in the library's static device scratch, a file-scope array of
 * 72 MiB that each GPU the library runs on holds until the process ends;
 * the call allocates nothing (no hipMalloc, hipFree, pinned staging or
 * event). The host tables are copied with hipMemcpyAsync from pageable
 * memory, which the runtime completes before returning (the host therefore
 * waits for the stream's earlier work). Small calls (at most 32 links and 8
 * requests, no per-query limits, any store but bf16 GQA of d 128, bf16
 * MLA of 576 / 512 and 4-bit ones) run the kernels pic_link_decode runs for them, which take
 * the tables as a kernel argument and read the own KV in place: they use the
 * scratch for split partials only and copy nothing. Every kernel writes what
 * it later reads, so nothing in the scratch has to start at zero.
 * All calls on one GPU share its scratch: calls must not overlap on a GPU
 * (enqueue them on one stream, or order them); calls that overlap race.
 * Errors: as pic_link_decode, and INVALID when the call is charged more than
 * 64 MiB: its tables (32 B per link and for a request's own KV, 36 B per
 * request, 4 B per query token where limits differ), ceil(L_s / 64) * 64 own tokens *
 * H_kv * (d_k + d_v) * esize per request (also where the kernel reads them in
 * place; nothing for a 4-bit store), and Tq * H_q * splits * (d_v + 2) * 4 B when the keys are split, with
 * one split count for all requests (num_splits, or for 0 about eight
 * workgroups per CU). Such a call launches nothing. A call within the charge
 * whose requests are cut into more pieces than that, or whose 64 B of work
 * item per piece do not fit the other 8 MiB, is cut into fewer pieces, here
 * and in pic_link_decode alike. */
pic_status pic_link_decode_noalloc(pic_store *store, const pic_link_req *req, int32_t n_q_heads,
                                   const void *q, const void *k_self, const void *v_self,
                                   float softmax_scale, int32_t num_splits, void *out, float *lse,
                                   void *stream);

/* A request batch resolved once for repeated calls. Comb runs the same
 * links in each of its cross-attention layers and again at every decode
 * step (generated tokens attend to the same documents, Sec. 4 and Eq. 12);
 * a plan looks the chunk ids up, chooses kernel and splits, and puts the
 * link tables of every layer and the call's workspace on the device once,
 * so that a run enqueues kernels only: no host-side lookup, no copy, no
 * allocation.
 * pic_link_plan_create: req as for pic_link_attn (req->layer must be 0);
 *   mode PIC_PREFILL (num_splits must be 0) computes as pic_link_attn,
 *   PIC_DECODE as pic_link_decode with the given num_splits (0 = auto),
 *   with the same kernels and split choice, so a run returns the bits the
 *   direct call returns (small calls, see pic_link_decode_noalloc, pass the
 *   tables as a kernel argument from the plan's host copy of each layer's
 *   table, as the direct calls do).
 *   Blocking: copies the tables to the device before returning. The plan
 *   keeps no pointer into req; the store must outlive it
 *   (pic_store_destroy refuses while plans are alive).
 * pic_link_plan_run: one call of the planned batch on cross-attention layer
 *   `layer`, with tensors as for pic_link_attn (sizes from the plan's
 *   offsets). Runs of one plan share its workspace: enqueue them on one
 *   stream, or order them.
 * pic_link_plan_destroy: waits for the device and frees the plan; NULL is
 *   ignored.
 * Errors: INVALID, NOT_FOUND, UNSUPPORTED, OOM, HIP. */
enum { PIC_PREFILL = 0, PIC_DECODE = 1 };   /* pic_link_plan_create mode */
typedef struct pic_link_plan pic_link_plan;
pic_status pic_link_plan_create(pic_store *store, const pic_link_req *req, int32_t n_q_heads,
                                int32_t mode, int32_t num_splits, pic_link_plan **out);
pic_status pic_link_plan_run(pic_link_plan *plan, int32_t layer, const void *q,
                             const void *k_self, const void *v_self, float softmax_scale,
                             void *out, float *lse, void *stream);
pic_status pic_link_plan_destroy(pic_link_plan *plan);

/* Link attention of requests that share linked chunks: users who ask about the same
 * documents. Group g is the requests request_offsets[g] .. request_offsets[g+1]-1 of the
 * batch; all of them see the group's shared links (chunk_offsets, chunk_ids, chunk_starts,
 * as in pic_link_req, by group), then their own links and own KV (req). The result is that of
 * pic_link_attn with the shared links put before each request's own ones, to
 * floating-point rounding order; but a group's shared rows are read once for all of its
 * query tokens, and every row's partial softmax states over both are merged exactly. Chunk
 * caches depend on no position, so any documents that the requests have in common can be
 * shared, in any order.
 *   req: as for pic_link_attn, own links and own KV may be empty; q_doc_limits count the
 *     rows of a request's own links (shared ones are seen by every query token).
 *   groups: host arrays, n_groups and n_groups + 1 entries, the last of request_offsets
 *     the batch. A group may be empty or share nothing.
 * Tensors, scale and lse as for pic_link_attn. Workspace: fp32 partials of every query row,
 * about 2 Tq * H_q * (d_v + 2) * 4 bytes or more where keys are split.
 * The range of the values and the rounding of lse are those of pic_link_attn: over bf16 GQA stores
 * of d 128 and bf16 MLA stores of 576 / 512 values up to 2^61 / T, for single tokens too, where
 * pic_link_decode takes larger ones. Over bf16 GQA stores with d_k = d_v = 128, or 64 and more than 16
 * query rows per kv head, the sums are of fp32 probabilities.
 * pic_link_shared_plan_create: the same, resolved once (req->layer must be 0), run and
 *   destroyed by pic_link_plan_run and pic_link_plan_destroy: a run enqueues kernels only, and may
 *   be captured.
 * Errors: as pic_link_attn; UNSUPPORTED also for pic_link_shared in a graph capture (its
 * workspace serves later calls); the plan's also OOM. */
typedef struct pic_link_groups {
  int32_t n_groups;
  const int32_t *request_offsets;
  const int32_t *chunk_offsets;
  const uint64_t *chunk_ids;
  const int32_t *chunk_starts;   /* or NULL */
} pic_link_groups;
pic_status pic_link_shared(pic_store *store, const pic_link_req *req,
                           const pic_link_groups *groups, int32_t n_q_heads, const void *q,
                           const void *k_self, const void *v_self, float softmax_scale, void *out,
                           float *lse, void *stream);
pic_status pic_link_shared_plan_create(pic_store *store, const pic_link_req *req,
                                       const pic_link_groups *groups, int32_t n_q_heads,
                                       pic_link_plan **out);

/* Link attention over selected blocks, for long document sets: each query token attends over
 * the linked blocks that a cheap score finds for it, and over its own KV. A block is 64 tokens of
 * a linked chunk, from its first linked token on (a chunk's last one may be shorter); a
 * request's blocks are counted over its links in order. fp32 and bf16 GQA stores, d_k = d_v of
 * 64 or 128 (else UNSUPPORTED).
 *   summary  of a block and kv head: the mean of its K rows, rounded to fp32 and then to bf16
 *   score    of a block for a query token and kv head: the largest dot product of the summary
 *            with a query head of that kv head's group (summed in 64 bits; NaN counts as -inf)
 *   taken    the first keep_first and the last keep_last of the request's blocks, then those of
 *            the largest scores, n_blocks in all (all blocks, if it has no more); of equal
 *            scores the lower block
 * A block index holds a store's summaries (n_layers * capacity / 64 * H_kv * d_k * 2 bytes):
 * pic_index_create: nothing indexed yet. The store must outlive the index
 *   (pic_store_destroy refuses while one is alive). Errors: INVALID, UNSUPPORTED, OOM, HIP.
 * pic_index_update: forms the summaries of the listed chunks (host, an id may repeat) in
 *   one layer, or in all of them for layer -1, as the chunks stand; ordered on `stream`. To be
 *   called again when a chunk has been written to, has grown (only blocks that grew are
 *   formed again) or has been put anew. A captured call forms the same blocks again when it
 *   is replayed. Errors: INVALID, NOT_FOUND, HIP.
 * pic_index_destroy: waits for the device and frees the index; NULL is ignored.
 * pic_link_sparse: tensors, scale and lse as for pic_link_attn; req->q_doc_limits must be
 *   NULL. blocks: device int32 [Tq][n_kv_heads][n_blocks] or NULL: receives the taken blocks,
 *   ascending, -1 behind them. n_blocks 1 .. 1024, a request's blocks at most 8192 (else
 *   UNSUPPORTED). One token a request is the ordinary use (a decode step); several are
 *   computed one by one. It is the faster call for long document sets, n_blocks a few tenths
 *   of them at most: with 16 or 24 blocks of 32/8 heads x 128, from about 128 blocks a request on for one or
 *   two requests, 64 for four and 32 for sixteen. A graph capture takes calls of up to 88 links and 32 query tokens in
 *   all (else UNSUPPORTED); a replay reads the rows that those links had, so their chunks have
 *   to stay. Errors: INVALID (also a linked chunk whose summaries in the layer are
 *   not those of its present content), NOT_FOUND, UNSUPPORTED, OOM, HIP. */
typedef struct pic_index pic_index;
pic_status pic_index_create(pic_store *store, pic_index **out);
pic_status pic_index_update(pic_index *index, int32_t layer, int32_t n, const uint64_t *chunk_ids,
                            void *stream);
pic_status pic_index_destroy(pic_index *index);
pic_status pic_link_sparse(pic_index *index, const pic_link_req *req, int32_t n_q_heads,
                           int32_t n_blocks, int32_t keep_first, int32_t keep_last, const void *q,
                           const void *k_self, const void *v_self, float softmax_scale, void *out,
                           float *lse, int32_t *blocks, void *stream);

/* Test hook: materialises the concatenation (Sec. 4.2) of the listed chunks
 * of one layer, in the given order, reading the pool through the same
 * address resolution the attention kernels use. k_out: device token-major
 * [sum len][H_kv][d_k]; v_out: device [sum len][H_kv][d_v] (GQA) or NULL
 * (MLA). Bit-exact copies.
 * Errors: INVALID (also more than 2^31 - 1 tokens in all), NOT_FOUND, HIP. */
pic_status pic_debug_gather(pic_store *store, const uint64_t *ids, int32_t n, int32_t layer,
                            void *k_out, void *v_out, void *stream);

/* Test hook, host only (no device work, no store): the request order the
 * planner gives a bf16 d=128 prefill call, whose row blocks (256 rows of
 * one request and kv head) are dispatched in that order, each on the first
 * free CU of its XCD. Request r has q_len[r] query tokens, self_len[r] own
 * tokens (causal, Sec. 4.1) and doc_tiles[r] 64-key tiles of linked
 * documents (Sec. 4.2); the GQA group is n_q_heads / n_kv_heads; cus and
 * xcds describe the device (workgroup ids go round-robin to the XCDs).
 * order_out: host [batch], the request at each position: heaviest first
 * (tiles x query tokens), improved by pairwise swaps when the row blocks
 * of an XCD take several rounds of its CUs. finish_out: host [2] or NULL,
 * the simulated finish time in tiles of the busiest XCD (a workgroup takes
 * its visible tiles plus 1.5) for heaviest first and for the returned
 * order; both 0 when no search runs.
 * Errors: INVALID (NULL arrays, negative lengths, n_q_heads not a multiple
 * of n_kv_heads, cus not a multiple of xcds). */
pic_status pic_debug_request_order(const int32_t *q_len, const int32_t *self_len,
                                   const int32_t *doc_tiles, int32_t batch, int32_t n_q_heads,
                                   int32_t n_kv_heads, int32_t cus, int32_t xcds,
                                   int32_t *order_out, double *finish_out);

/* Dense per-head projections around absorbed MLA link attention, for the
 * DeepSeek-V2-Lite backbone (Sec. 5.1): per head h its latent rows c (512)
 * give non-absorbed keys [W_UK[h] c | k_rope] and values W_UV[h] c, with
 * W_UK[h] and W_UV[h] 128 x 512. Absorbing W_UK into the query turns the
 * attention into the latent form pic_link_attn computes on an MLA store
 * (d_k 576, d_v 512); W_UV then maps its latent output to the 128 value dims.
 * bf16 in and out (round to nearest even), fp32 accumulation.
 * pic_mla_absorb_q: q_out[t,h,0:512] = W_UK[h]^T q[t,h,0:128] and
 *   q_out[t,h,512:576] = q[t,h,128:192] (the rope part, copied).
 *   q device [n_tokens][n_heads][192] (q_nope 128 | q_rope 64)
 *   w_uk_t device [n_heads][512][128]: W_UK[h] transposed (row j holds the
 *     128 weights of latent dim j)
 *   q_out device [n_tokens][n_heads][576]
 * pic_mla_up_v: out[t,h,0:128] = W_UV[h] o_lat[t,h,0:512].
 *   o_lat device [n_tokens][n_heads][512] (pic_link_attn's output)
 *   w_uv device [n_heads][128][512]
 *   out device [n_tokens][n_heads][128]
 * All pointers 16-byte aligned; n_heads 1..1024; n_tokens 0 does nothing.
 * Errors: INVALID, HIP. */
pic_status pic_mla_absorb_q(int32_t n_tokens, int32_t n_heads, const void *q, const void *w_uk_t,
                            void *q_out, void *stream);
pic_status pic_mla_up_v(int32_t n_tokens, int32_t n_heads, const void *o_lat, const void *w_uv,
                        void *out, void *stream);

/* Rotary positions: pairs of a head's elements are turned by an angle that
 * grows with the token's position, for the queries and keys of a layer before
 * they are put or linked (chunk caches are computed from position zero, Sec. 1),
 * and, transposed, for the gradient of that.
 *   y_a = c x_a - s x_b,  y_b = s x_a + c x_b
 *   c = magnitude cos(pos f_i),  s = magnitude sin(pos f_i);  transposed: -s
 * With i = 0 .. rot_dim/2 - 1, pair i is (rot_at + i, rot_at + rot_dim/2 + i)
 * for PIC_ROPE_HALF, (rot_at + 2i, rot_at + 2i + 1) for PIC_ROPE_INTERLEAVED; the
 * head's other elements are copied. Frequencies, g_i = theta^(-2i / rot_dim):
 *   PIC_ROPE_PLAIN   f_i = g_i
 *   PIC_ROPE_LINEAR  f_i = g_i / factor
 *   PIC_ROPE_BANDED  f_i = g_i (w + (1 - w) / factor), w = (original_len g_i / 2pi -
 *                    band_low) / (band_high - band_low) held to 0..1: pairs that
 *                    turn often within the original length are kept, slow ones
 *                    stretched (the rule of the Llama-3.1 backbone)
 *   PIC_ROPE_YARN    the same with w falling over the pair's index, 1 - w = (i - lo) /
 *                    max(hi - lo, 0.001) held to 0..1, with at(n) = rot_dim
 *                    ln(original_len / (2pi n)) / (2 ln theta), lo = max(floor(at(
 *                    turns_fast)), 0), hi = min(ceil(at(turns_slow)), rot_dim - 1)
 *                    (YaRN, used by the DeepSeek-V2-Lite backbone)
 * Angles are formed and reduced in 64 bits, products in fp32, and each output is
 * rounded once.
 * pic_rope_create: host only. dtype PIC_F32 or PIC_BF16; rot_dim even, 2..256;
 *   head_dim at most 768; magnitude 1 unless the scaling calls for another
 *   one. Fields that the scaling does not name are not read. Errors: INVALID,
 *   UNSUPPORTED, OOM.
 * pic_rope_apply: n_tensors (1..4) tensors of the same tokens in one launch.
 *   positions device int32 [n_tokens], any value.
 *   x, out device [n_tokens][n_heads][head_dim] of the handle's dtype, n_heads
 *   1..1024, token t at t * stride elements (0: dense, else at least n_heads *
 *   head_dim: slices of a fused projection). out may be x itself (same stride;
 *   the elements outside the rotated part are then not touched); buffers must not
 *   overlap otherwise. Allocates nothing: may be captured. One handle may be
 *   used by several threads at once. Errors: INVALID, HIP. */
enum { PIC_ROPE_HALF = 0, PIC_ROPE_INTERLEAVED = 1 };   /* pic_rope_desc.layout */
enum { PIC_ROPE_PLAIN = 0, PIC_ROPE_LINEAR = 1, PIC_ROPE_BANDED = 2, PIC_ROPE_YARN = 3 };
typedef struct pic_rope_desc {
  int32_t dtype;
  int32_t layout;
  int32_t head_dim;
  int32_t rot_at;
  int32_t rot_dim;
  int32_t scaling;           /* PIC_ROPE_PLAIN .. PIC_ROPE_YARN */
  double theta;
  double factor;
  double original_len;
  double band_low, band_high;
  double turns_fast, turns_slow;
  double magnitude;
} pic_rope_desc;
typedef struct pic_rope_tensor {
  const void *x;
  void *out;
  int64_t x_stride, out_stride;
  int32_t n_heads;
} pic_rope_tensor;
pic_status pic_rope_create(const pic_rope_desc *desc, pic_rope **out);
pic_status pic_rope_destroy(pic_rope *rope);
pic_status pic_rope_apply(const pic_rope *rope, int32_t n_tokens, const int32_t *positions,
                          const pic_rope_tensor *tensors, int32_t n_tensors, int32_t transposed,
                          void *stream);

/* Kernel timing for measurement. pic_prof_begin() clears and enables
 * recording of HIP events around every launch of the main attention kernel;
 * pic_prof_begin_sampled(every) around one launch in `every` (1..1000000;
 * the event pair adds a few microseconds between kernels, so sampling keeps
 * the timed steps close to an uninstrumented run); pic_prof_end() waits for
 * them, disables recording and returns the summed kernel time in
 * milliseconds, the number of timed launches and the kernel's name
 * (name_buf may be NULL). Errors: INVALID (every out of range), HIP. */
pic_status pic_prof_begin(void);
pic_status pic_prof_begin_sampled(int32_t every);
pic_status pic_prof_end(double *kernel_ms, int64_t *launches, char *name_buf, int32_t name_len);

/* Achievable peaks of this GPU, a second roofline denominator next to the
 * spec peaks (measurement helpers, not part of the method; blocking, they
 * synchronise `stream`, allocate and free a 512 KB scratch buffer).
 * pic_peak_mfma_bf16: bf16 dense matrix-core rate in TFLOP/s of `iters`
 *   rounds of four independent 32x32x16 MFMAs per wave, two waves per SIMD
 *   on every CU (iters 1..2^22; ~4096 gives a ~10 ms run).
 * pic_peak_hbm_read: HBM read rate in GB/s of one streaming pass over buf
 *   (device memory, 16-byte aligned, bytes a positive multiple of 16; use a
 *   buffer far larger than the last-level cache).
 * pic_peak_hbm_write: the same for one streaming pass of stores over buf
 *   (overwrites it). One dispatch of either moves exactly `bytes`, which
 *   also calibrates the HBM traffic counters of a profiler.
 * Errors: INVALID, HIP. */
pic_status pic_peak_mfma_bf16(int32_t iters, double *tflops, void *stream);
pic_status pic_peak_hbm_read(const void *buf, int64_t bytes, double *gbs, void *stream);
pic_status pic_peak_hbm_write(void *buf, int64_t bytes, double *gbs, void *stream);

const char *pic_status_str(pic_status status);
const char *pic_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* PIC_H */
