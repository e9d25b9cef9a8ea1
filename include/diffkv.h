/*
 * diffkv.h -- C ABI of the DiffKV decode hot path for AMD Instinct MI355X
 * (gfx950).  DiffKV: arXiv 2412.03131, "Differentiated Memory Management
 * for Large Language Models with Parallel KV Compaction".
 *
 * What the library computes
 *   A differentiated, paged KV cache: keys are kept at more bits than values
 *   (K8V4 for high-precision tokens, K4V2 for low-precision tokens, Sec. 4),
 *   each token is kept high, kept low or pruned by its significance score
 *   (Sec. 4), and every (sequence, KV head) pair -- a "table" -- keeps its own
 *   number of tokens of each kind.  Memory is managed with unified pages, a
 *   circular free page list and bidirectional page tables (Sec. 5.2); decode
 *   attention reads the compressed pages directly (Sec. 6.2).
 *
 * Conventions
 *   - All entry points are C, take plain pointers and sizes, never allocate,
 *     free or synchronise, and keep no state between calls (except the
 *     per-device scratch address of diffkv_decode_attention_noalloc).
 *   - "device" pointers point to GPU memory of the current HIP device;
 *     "host" pointers to CPU memory.  The caller owns every buffer.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     All work is enqueued on it and the call returns immediately.  Calls
 *     on one cache must be ordered on one stream; different caches are
 *     independent.
 *   - Return value: host-detectable errors (bad arguments, unsupported
 *     layout, small workspace, launch failure).  On any non-OK return
 *     nothing was enqueued (except DIFFKV_E_LAUNCH, which reports that an
 *     enqueue failed).
 *   - Device-detected conditions set sticky bits in *cache->status (device
 *     word, never cleared by the library).  The operations that can set them
 *     are all-or-nothing: when a bit is raised by a call, that call changed
 *     nothing in the cache.  The caller reads the word after a sync and
 *     recovers (e.g. releases finished sequences through compaction, then
 *     retries), and clears it.
 *   - fp16 values are passed as IEEE binary16 bit patterns (uint16_t).
 */
#ifndef DIFFKV_H
#define DIFFKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t diffkv_status;
enum {
    DIFFKV_OK = 0,
    DIFFKV_E_INVAL = 1,       /* null pointer, negative or inconsistent size       */
    DIFFKV_E_UNSUPPORTED = 2, /* layout/shape the gfx950 kernels do not implement  */
    DIFFKV_E_WORKSPACE = 3,   /* ws_bytes smaller than diffkv_workspace_size()     */
    DIFFKV_E_LAUNCH = 4,      /* a HIP launch or runtime call failed               */
    DIFFKV_E_SCRATCH = 5      /* the call needs more than the fixed scratch of
                                 diffkv_decode_attention_noalloc                   */
};

/* sticky bits of *diffkv_cache.status */
enum {
    DIFFKV_ST_OUT_OF_PAGES = 1u,   /* the free region (tail - head) was too small     */
    DIFFKV_ST_TABLE_OVERFLOW = 2u, /* a table would hold more than p_max pages        */
    DIFFKV_ST_BAD_INPUT = 4u       /* new_len disagreed with total_new / max_new      */
};

enum { DIFFKV_HIGH = 0, DIFFKV_LOW = 1 };

/*
 * Page layout (Sec. 5.2, "unified pages").  Every page has the same byte
 * stride; its precision is fixed when a table takes it.  A page of
 * precision p holds T = tokens_per_page[p] tokens in six segments, in this
 * order, each starting on a 64-byte boundary of the page:
 *   K codes   [head_dim*k_bits/128 chunks][T][16 B]: chunk c holds dims
 *             c*(128/k_bits) .. +128/k_bits-1 of one token, element e at
 *             bit e*k_bits of the 16 bytes;
 *   K meta    [T][head_dim/group] {fp16 scale, fp16 zero};
 *   V codes   [head_dim][T*v_bits/8 B]: token slot s of dim d at bit s*v_bits
 *             of the dim's row;
 *   V meta    [head_dim/group][T] {fp16 scale, fp16 zero};
 *   scores    [T] fp32 (significance score as given);
 *   positions [T] int32 (token position in its sequence).
 * Bits are little-endian within bytes.  page_bytes = the larger of the two
 * precisions' sizes.  A fresh page (one whose slot 0 is being written) is
 * cleared first, so unused slots are zero bytes.
 * Table width p_max = ceil(max_seq_len / tokens_per_page[HIGH]) + 1: one
 * more than the paper's max_len / T_high, since a partial high page and a
 * partial low page can coexist.
 */
typedef struct diffkv_layout {
    int32_t head_dim, group;
    int32_t k_bits[2], v_bits[2];      /* [HIGH], [LOW]                       */
    int32_t tokens_per_page[2];        /* [HIGH], [LOW]                       */
    int32_t max_seq_len, p_max;
    int64_t page_bytes;
    int32_t off_kcode[2], off_kmeta[2], off_vcode[2], off_vmeta[2];
    int32_t off_score[2], off_pos[2], used_bytes[2];
} diffkv_layout;

/*
 * Cache state (all device memory, all caller-owned).  Table t = b*num_kv_heads
 * + h is the bidirectional page table of sequence b, KV head h (Sec. 5.2):
 * high-precision page IDs grow from slot 0 to the right, low-precision page
 * IDs from slot p_max-1 to the left; empty slots hold -1.  Token u of a
 * section lives in slot u % T of the section's page u / T; appends add
 * tokens in position order (a generation step's removal then moves a
 * section's last token into the hole).  The free page list is a ring of
 * num_pages IDs; the free IDs are ring[head % n .. tail % n) with head/tail
 * monotone int64 counters (start pointer allocates, end pointer recycles).
 */
typedef struct diffkv_cache {
    uint8_t*  pool;          /* device [num_pages][page_bytes]                     */
    int64_t   num_pages;
    int32_t*  page_table;    /* device [num_tables][p_max]                         */
    int32_t*  pages;         /* device [num_tables][2] pages held per section      */
    int32_t*  len;           /* device [num_tables][2] tokens held per section     */
    int32_t*  seq_len;       /* device [num_seqs] tokens seen per sequence (incl.
                                pruned); the threshold form's N                   */
    int32_t*  ring;          /* device [num_pages] circular free page list         */
    int64_t*  ring_ptr;      /* device [2] {head, tail}; tail - head = free pages  */
    uint32_t* status;        /* device [1] sticky DIFFKV_ST_* bits                 */
    int32_t   num_seqs;      /* B                                                  */
    int32_t   num_kv_heads;  /* Hkv; num_tables = B * Hkv                          */
} diffkv_cache;

/* Fill *out (host) from the parameters: segment offsets, page_bytes, p_max.
 * Bits must be 1, 2, 4 or 8, head_dim*k_bits a multiple of 128,
 * T*v_bits a multiple of 8, tokens_per_page[LOW] >= tokens_per_page[HIGH].
 * DIFFKV_E_INVAL otherwise.  Any valid layout is accepted here.  The append,
 * attention and significance kernels implement head_dim 128, group 32 and
 * these (high | low) section formats (precision levels of Sec. 4 and
 * Sec. 7.2), DIFFKV_E_UNSUPPORTED otherwise:
 *   K8V4, 16 tokens | K4V2, 32 tokens   (the paper's two levels)
 *   K8V8, 16 tokens | K4V2, 32 tokens
 *   K8V2, 16 tokens | K4V1, 32 tokens
 *   K8V4, 16 tokens | K4V2, 16 tokens
 * The generation step implements the first only.  Allocation and compaction
 * accept any valid layout. */
diffkv_status diffkv_layout_init(diffkv_layout* out, int32_t head_dim, int32_t group,
                                 const int32_t k_bits[2], const int32_t v_bits[2],
                                 const int32_t tokens_per_page[2], int32_t max_seq_len);

enum {
    DIFFKV_OP_APPEND = 0,
    DIFFKV_OP_ATTENTION = 1,
    DIFFKV_OP_COMPACT = 2,
    DIFFKV_OP_ALLOC = 3,
    DIFFKV_OP_GENERATION = 4,
    DIFFKV_OP_PROMPT_SIGNIFICANCE = 5,
    DIFFKV_OP_CHUNK_ATTENTION = 6,
    DIFFKV_OP_CHUNK_SIGNIFICANCE = 7,
    DIFFKV_OP_BLOCK_ATTENTION = 8
};

/* Bytes of device workspace the operation needs (host out-parameter).
 * APPEND: num_seqs, num_kv_heads, total_new.  ATTENTION: num_seqs,
 * num_q_heads, num_splits (0 = automatic, -1 = balanced).
 * COMPACT / ALLOC / GENERATION: num_seqs*num_kv_heads tables.
 * PROMPT_SIGNIFICANCE: num_seqs, num_q_heads, total_new.
 * CHUNK_ATTENTION / CHUNK_SIGNIFICANCE / BLOCK_ATTENTION: num_seqs,
 * num_q_heads, num_kv_heads, total_new.  Unused sizes are ignored. */
diffkv_status diffkv_workspace_size(int32_t op, const diffkv_layout* layout,
                                    int32_t num_seqs, int32_t num_q_heads,
                                    int32_t num_kv_heads, int64_t total_new,
                                    int32_t num_splits, size_t* bytes);

/*
 * KV compressor (Sec. 4) + page placement (Sec. 5.2, 5.3): classes the new
 * tokens of every table, reserves the pages both sections now need with one
 * prefix-sum schedule over all tables, then quantizes and stores every kept
 * token.
 *
 *   new_len  device int32 [num_seqs]: new tokens of sequence b; their rows in
 *            k/v/score are new_off(b) .. +new_len[b]-1, new_off(b) =
 *            sum of new_len[0..b).  Must sum to total_new with every entry in
 *            [0, max_new], else DIFFKV_ST_BAD_INPUT is raised and nothing
 *            changes.
 *   k, v     device fp16 [total_new][num_kv_heads][head_dim], of any alignment
 *            an fp16 value may have (16 bytes make the loads cheapest).
 *   score    device fp32 [total_new][num_kv_heads]: significance (not NaN).
 *   quota    device int32 [num_seqs][num_kv_heads][2] = {n_high, n_low}, or
 *            NULL.  Quota form: the non-window new tokens are ranked by
 *            (score descending, position ascending; -0 == +0); the first
 *            min(n_high, avail) are high, the next min(n_low, avail - n_high')
 *            low, the rest pruned.  Threshold form (quota == NULL; Sec. 4,
 *            Algorithm 1): high iff score >= alpha_h / N, else low iff
 *            score >= alpha_l / N, else pruned, N = seq_len[b] + new_len[b]
 *            and both thresholds computed in fp32.
 *   recent_window  the last W new tokens of each sequence are high precision
 *            and outside the quotas (W >= 0).
 *
 * Quantization (Sec. 2.2) per 32-dim group of each kept K and V vector:
 *   s = fp16_rne((max - min) / (2^b - 1)) in fp32, z = min (with -0 -> +0),
 *   code = clamp(rint((x - z) / s), 0, 2^b - 1) in fp32 with the stored fp16
 *   s and z, code = 0 when s == 0; b = k_bits/v_bits of the token's class.
 * Placement: kept tokens of a section take section indices len .. in
 *   position order.  Page demand per section = ceil((len + added) / T) -
 *   pages (if positive).  Tables take their new IDs from the ring region
 *   after the demands of all lower tables, high pages first; head advances
 *   by the total.  Raises OUT_OF_PAGES / TABLE_OVERFLOW all-or-nothing.
 * Updates pool, page_table, pages, len, seq_len (+= new_len), ring_ptr[0].
 * Workspace: diffkv_workspace_size(DIFFKV_OP_APPEND, ...); it needs no
 * clearing between calls.  A call with max_new <= 1 over at most 1024 tables
 * (a decode step) runs as one launch.
 */
diffkv_status diffkv_quantize_append(const diffkv_layout* layout, const diffkv_cache* cache,
                                     int64_t total_new, int32_t max_new,
                                     const int32_t* new_len,
                                     const uint16_t* k, const uint16_t* v,
                                     const float* score, const int32_t* quota,
                                     float alpha_h, float alpha_l, int32_t recent_window,
                                     void* ws, size_t ws_bytes, void* stream);

/*
 * Decode attention over the compressed cache, Eq. (1) of Sec. 2.1, one new
 * query per sequence and query head (Sec. 6.2):
 *   out[b][hq] = sum_j softmax_j(sm_scale * q[b][hq] . k_hat_j) v_hat_j
 * over every kept token of table b*Hkv + hq/(Hq/Hkv): the high section, then
 * the low section; k_hat = s*code + z per group.  fp32 accumulation.
 *   q    device fp16 [num_seqs][num_q_heads][head_dim]
 *   out  device fp32 [num_seqs][num_q_heads][head_dim]
 *   lse  device fp32 [num_seqs][num_q_heads] (natural log of the softmax
 *        denominator incl. the max) or NULL.  An empty table gives out = 0,
 *        lse = -inf.
 *   num_splits  0 = automatic (default): no table is split when there are
 *        at least as many tables as eight-wave workgroups the device holds at
 *        once -- up to 5 query heads per KV head each workgroup takes two
 *        tables (one long, one short: ranks j and T-1-j by decreasing work)
 *        and splits its waves between them by their work; above, one
 *        workgroup per table (waves with more pages left get issue priority)
 *        -- otherwise the balanced mode.
 *        -1 = balanced: the page lists of all tables, in table order, form one
 *        list of work units (a high page 3, a 32-token low page 6, a 16-token
 *        low page 3, a table's start 50) cut into one equal
 *        share per resident workgroup -- or, where that is little work per
 *        workgroup, every table is cut into equal ranges of its own, as short as
 *        the workgroups allow; a table spread over several shares has
 *        their (max, sum, acc) states merged in page order (Sec. 6.2 sequence
 *        split).  S >= 1: each table is cut into min(S, pages) equal page
 *        ranges, merged the same way (S = 1: no split, no merge).  Results
 *        are deterministic for a given mode and device.
 *   ws   device workspace of diffkv_workspace_size(DIFFKV_OP_ATTENTION, ...)
 *        bytes (always needed: it holds the split tables' partial states and
 *        one arrival word per table, which each call tags as its own, so the
 *        workspace needs no clearing between calls).
 * num_q_heads must be a multiple of num_kv_heads, with at most 8 query heads
 * per KV head.
 * Precision: q . k_hat is exact up to fp32 summation (codes and q enter fp16
 * products exactly); each value weight p * s_v is rounded to fp16 (relative
 * 2^-11, the rounding charged at the centre code), so an output differs from
 * exact Eq. (1) by at most about 2^-12 * R plus fp32 rounding, R being the
 * largest dequantized value-group range of its table.  Any finite fp16 cache
 * is accepted: the weights never overflow fp16 (pages with a value scale above
 * 2^7 keep them <= s_v).
 */
diffkv_status diffkv_decode_attention(const diffkv_layout* layout, const diffkv_cache* cache,
                                      int32_t num_q_heads, const uint16_t* q, float sm_scale,
                                      float* out, float* lse, int32_t num_splits,
                                      void* ws, size_t ws_bytes, void* stream);

/*
 * diffkv_decode_attention without a workspace, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same arguments, minus ws / ws_bytes, and
 * the same kernels and results, bit for bit.  The arrival words and split
 * partial states go to a fixed 8 MiB array in the library's device memory, one
 * per device, held from the library's load until the process ends; its device
 * address is looked up on the first call on each device and kept (the one
 * piece of state the library keeps).  A call whose mode, as resolved on the
 * current device, needs more -- the balanced mode takes 8 B per table plus
 * (resident workgroups + tables) * (Hq/Hkv) * 520 B -- returns
 * DIFFKV_E_SCRATCH and enqueues nothing.  Nothing in the scratch needs
 * clearing between calls.  Every call on a device shares that device's array:
 * calls ordered on one stream are safe, calls that may overlap on one device
 * (unordered streams) race.  Allocates, frees and synchronizes nothing.
 */
diffkv_status diffkv_decode_attention_noalloc(const diffkv_layout* layout, const diffkv_cache* cache,
                                              int32_t num_q_heads, const uint16_t* q, float sm_scale,
                                              float* out, float* lse, int32_t num_splits, void* stream);

/*
 * Significance update of one decode step (Sec. 4: a token's significance is
 * the average of the attention scores it receives; with grouped heads the
 * scores of a KV head's query heads are combined by their maximum).  Call it
 * after diffkv_decode_attention with the same q, passing that call's lse.
 * For every kept token j of table t = b*Hkv + h at position pos_j:
 *   x_j = max over the query heads hq of KV head h of exp(logit_hq,j - lse_hq),
 *         logit = sm_scale * q[b][hq] . k_hat_j (the probability of token j
 *         in the softmax over the table's kept tokens),
 *   score_j <- score_j + (x_j - score_j) / (N - pos_j),  N = seq_len[b],
 * i.e. the mean over the N - pos_j queries (positions pos_j .. N-1) the token
 * has received, the newest being this step's.  Scores are rewritten in place
 * in the pages' score segments; nothing else changes.  fp32 arithmetic.
 *   q    device fp16 [num_seqs][num_q_heads][head_dim] (as given to attention)
 *   lse  device fp32 [num_seqs][num_q_heads] (natural log, as attention wrote it)
 * No workspace.  Same layout and group-size support as diffkv_decode_attention.
 */
diffkv_status diffkv_update_significance(const diffkv_layout* layout, const diffkv_cache* cache,
                                         int32_t num_q_heads, const uint16_t* q, float sm_scale,
                                         const float* lse, void* stream);

/*
 * Prompt-phase significance (Sec. 4): the score of every prompt token, from
 * the prompt's own queries and fp16 keys, before the prompt is appended.
 * For sequence b with N = new_len[b] prompt tokens and KV head h, token p
 * (0-based) gets
 *   score[p][h] = (1 / (N - p)) * sum_{j = p}^{N-1} max_{hq of h} P_hq[j][p],
 *   P_hq[j][.] = softmax over p' <= j of sm_scale * q[j][hq] . k[p'][h],
 * the mean of the N - p causal attention probabilities the token receives,
 * the KV head's query heads combined by their maximum per query (the score
 * diffkv_update_significance continues).  The result feeds the `score`
 * argument of diffkv_quantize_append directly (same rows, same order).
 *   new_len  device int32 [num_seqs]; rows of sequence b follow those of b-1.
 *            Lengths are clamped to [0, max_new] and rows past total_new are
 *            neither read nor scored.
 *   q        device fp16 [total_new][num_q_heads][128], 16-byte aligned
 *   k        device fp16 [total_new][num_kv_heads][128], 16-byte aligned
 *   lse      device fp32 [total_new][num_q_heads] natural-log row normalizers
 *            (as a prompt attention kernel writes them), or NULL: the call
 *            computes them in an extra pass over q and k.
 *   score    device fp32 [total_new][num_kv_heads] out
 *   ws       diffkv_workspace_size(DIFFKV_OP_PROMPT_SIGNIFICANCE, ...) bytes
 * Arithmetic: fp16 x fp16 products on the matrix cores (exact), fp32 sums,
 * fp32 softmax with exp2; probabilities below 2^-126 may come out as zero.
 * sm_scale must be positive and finite (DIFFKV_E_INVAL otherwise).
 * num_q_heads / num_kv_heads up to 8 (else DIFFKV_E_UNSUPPORTED).
 */
diffkv_status diffkv_prompt_significance(const diffkv_layout* layout, int32_t num_seqs, int64_t total_new,
                                         int32_t max_new, const int32_t* new_len, int32_t num_q_heads,
                                         int32_t num_kv_heads, const uint16_t* q, const uint16_t* k,
                                         float sm_scale, const float* lse, float* score, void* ws,
                                         size_t ws_bytes, void* stream);

/*
 * Rotary positions of queries and keys, before they reach the entry points
 * here (which all take rotated rows).  Pair i of a head's first rot_dim dims,
 *   (x[i], x[i + rot_dim/2])  DIFFKV_ROPE_HALF,
 *   (x[2i], x[2i + 1])        DIFFKV_ROPE_INTERLEAVED,
 * is turned by the angle t = pos * inv_freq[i] and scaled:
 *   a' = scale * (a cos t - b sin t),  b' = scale * (b cos t + a sin t);
 * dims rot_dim .. head_dim-1 pass unchanged.
 *   pos       device int32 [rows]: position of each row's token (any value)
 *   inv_freq  device fp32 [rot_dim/2], 16-byte aligned: radians per position
 *             (diffkv_rope_frequencies fills such a table)
 *   rot_dim   a multiple of 16 up to head_dim (DIFFKV_E_UNSUPPORTED if it is
 *             another even number)
 *   q, k      device fp16: row r, head h at q + r*q_stride + h*head_dim, so that
 *             slices of a fused projection can be passed; strides in elements,
 *             at least heads*head_dim (any value with one row).  k and k_out are
 *             NULL with num_kv_heads 0 (then only q is turned).
 *   q_out, k_out  device fp16, with strides of their own; q_out == q with
 *             the same stride turns in place, otherwise they must not overlap
 *             the inputs.
 * All row addresses 16-byte aligned, strides multiples of 8, else
 * DIFFKV_E_INVAL.  Angles are taken in 64 bits, so positions of any size keep
 * theirs; products in fp32, one rounding to fp16 (head_dim 128 only).
 */
enum { DIFFKV_ROPE_HALF = 0, DIFFKV_ROPE_INTERLEAVED = 1 };

diffkv_status diffkv_rotate(const diffkv_layout* layout, int64_t rows, const int32_t* pos,
                            const float* inv_freq, int32_t rot_dim, int32_t style, float scale,
                            int32_t num_q_heads, const uint16_t* q, int64_t q_stride,
                            uint16_t* q_out, int64_t q_out_stride,
                            int32_t num_kv_heads, const uint16_t* k, int64_t k_stride,
                            uint16_t* k_out, int64_t k_out_stride, void* stream);

/*
 * Norms of queries and keys for each head, and their rotary positions, in one
 * pass: with w the side's weights,
 *   y[d] = x[d] * w[d] / sqrt(mean of the head's x^2 + eps),
 * then y is turned as diffkv_rotate turns it (dims rot_dim .. head_dim-1 are
 * normed and pass).
 *   q_weight, k_weight  device fp32 [head_dim], 16-byte aligned, or NULL: ones
 *   eps       finite, at least the smallest normal fp32 (2^-126)
 * The other arguments, in-place calls, limits and errors as diffkv_rotate.  The
 * sum of squares, the norm and all products are fp32, with one rounding to fp16.
 */
diffkv_status diffkv_norm_rotate(const diffkv_layout* layout, int64_t rows, const int32_t* pos,
                                 const float* inv_freq, int32_t rot_dim, int32_t style, float scale,
                                 float eps, int32_t num_q_heads, const uint16_t* q, int64_t q_stride,
                                 const float* q_weight, uint16_t* q_out, int64_t q_out_stride,
                                 int32_t num_kv_heads, const uint16_t* k, int64_t k_stride,
                                 const float* k_weight, uint16_t* k_out, int64_t k_out_stride, void* stream);

/*
 * Frequencies of rotary positions, computed on the host in 64 bits:
 * f_i = base^(-2i/rot_dim), i < rot_dim/2, for contexts longer than the trained
 * ones by `factor` (>= 1):
 *   DIFFKV_ROPE_PLAIN     f_i
 *   DIFFKV_ROPE_LINEAR    f_i / factor
 *   DIFFKV_ROPE_BASE      the base becomes base * factor^(rot_dim/(rot_dim-2))
 *   DIFFKV_ROPE_BY_PARTS  f_i * (g + (1-g)/factor), g = clamp((r_i - slow)/
 *             (fast - slow), 0, 1) with r_i = trained_len * f_i / (2 pi) turns
 *             over the trained length, fast > slow >= 0 (arXiv 2309.00071), and
 *             *scale = 0.1 ln(factor) + 1.
 * *scale is 1 in the other forms.  inv_freq: host fp32 [rot_dim/2].
 * trained_len, slow and fast are read by DIFFKV_ROPE_BY_PARTS alone.
 * DIFFKV_E_INVAL: rot_dim not even and positive (above 2 for _BASE), base not
 * above 0, factor below 1, a parameter not finite, a NULL pointer.
 */
enum { DIFFKV_ROPE_PLAIN = 0, DIFFKV_ROPE_LINEAR = 1, DIFFKV_ROPE_BASE = 2, DIFFKV_ROPE_BY_PARTS = 3 };

diffkv_status diffkv_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                                      int32_t trained_len, double slow, double fast,
                                      float* inv_freq, float* scale);

/*
 * The form of a chunk's attention scores (a NULL pointer: all off).  For a
 * query of head hq at position p and a key at position c <= p:
 *   x = sm_scale * q . k;
 *   cap > 0:         x <- cap * tanh(x / cap);
 *   slopes != NULL:  x <- x - slopes[hq] * (p - c)  (device fp32 [num_q_heads]);
 *   window > 0:      the key is seen only if p - c < window.
 * cap 0 or from 1e-30 to 1e30, window >= 0, else DIFFKV_E_INVAL.
 */
typedef struct diffkv_score_form {
    float cap;
    int32_t window;
    const float* slopes;
} diffkv_score_form;

/*
 * Attention of a chunk of new tokens over the compressed cache, before the
 * chunk is appended: a prompt's next part, drafted tokens that are checked at
 * once, one decoded token, or any mixture over the sequences.  New token j of
 * sequence b has position p = seq_len[b] + j; its query of head hq attends to
 * every kept token of table b*Hkv + hq/(Hq/Hkv) (k_hat, v_hat as in
 * diffkv_decode_attention; their positions from the pages) and to the chunk's own
 * tokens 0 .. j in fp16:
 *   out[row][hq] = sum_c softmax_c(x) v_c,  x as in diffkv_score_form.
 *   new_len  device int32 [num_seqs], rows of sequence b follow those of b-1.
 *            Every entry in [0, max_new], their sum at most total_new: rows
 *            behind the last sequence's (a padded batch) are nobody's and left
 *            as they were.  Other lengths are clamped so that no row past
 *            total_new is read or written.
 *   q, k, v  device fp16: row r, head h at q + r*q_stride + h*head_dim (slices
 *            of a fused projection can be passed), 16-byte aligned, strides in
 *            elements, multiples of 8, at least heads*head_dim (any value with
 *            one row) and at most 2^24 (DIFFKV_E_UNSUPPORTED above)
 *   out      device fp16 [total_new][num_q_heads][head_dim], 16-byte aligned
 *   lse      device fp32 [total_new][num_q_heads] (natural log of the softmax
 *            denominator) or NULL
 *   ws       diffkv_workspace_size(DIFFKV_OP_CHUNK_ATTENTION, ...) bytes, no
 *            clearing needed, 16-byte aligned; calls that may overlap need one
 *            each
 * The cache is read only.  A page ID outside the pool counts no tokens, and no
 * section length leads out of the table's row: the high section ends with the
 * row, the low one where the high one begins.
 * sm_scale above 0 and at most 65536 (DIFFKV_E_INVAL otherwise).  The layouts of
 * diffkv_layout_init's list, up to 8 query heads per KV head, up to 2^22 tables
 * (DIFFKV_E_UNSUPPORTED otherwise).
 * Scores x up to 2^22 in magnitude, the slopes' part included: beyond, fp32's
 * steps are no longer small against the exponential's, and a row may come out
 * infinite or NaN.
 * Precision: q . k_hat exact up to fp32 summation, fp32 softmax statistics;
 * v_hat is rounded to fp16 (2^-11, or 2^-24 where that is more; up to twice the
 * largest fp16 it is no infinity); the weights enter in two fp16 parts (2^-22,
 * or 2^-32 of their row's largest); products are summed in fp32, and out is
 * rounded once.  That holds for every row, whatever else the call carries; the
 * order of its sums, and with it the last bits, goes by the call's lengths.
 * A NaN or infinite own key or value, or v_hat, reaches only the rows that see
 * its token.
 */
diffkv_status diffkv_chunk_attention(const diffkv_layout* layout, const diffkv_cache* cache,
                                     int64_t total_new, int32_t max_new, const int32_t* new_len,
                                     int32_t num_q_heads, const uint16_t* q, int64_t q_stride,
                                     const uint16_t* k, int64_t k_stride,
                                     const uint16_t* v, int64_t v_stride,
                                     float sm_scale, const diffkv_score_form* form,
                                     uint16_t* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Significance of a chunk (Sec. 4), after diffkv_chunk_attention with the same
 * q, k and form, before the chunk is appended.  With P the attention
 * probabilities of the chunk's n = new_len[b] queries, combined over a KV
 * head's query heads by their maximum, X_c = sum_j max_hq P_hq[j][c]:
 *   a kept token at position c:  score <- score + (X_c - n*score) / (N - c),
 *            N = seq_len[b] + n: the mean over the N - c queries it has received,
 *            in place in its page, as diffkv_update_significance does for one
 *            query;
 *   own token i:  score[row i][h] = X_i / (n - i), the mean over the queries it
 *            has received, as diffkv_prompt_significance gives it; it feeds the
 *            `score` argument of diffkv_quantize_append.
 *   lse      device fp32 [total_new][num_q_heads] as diffkv_chunk_attention
 *            wrote it
 *   score    device fp32 [total_new][num_kv_heads] out
 *   ws       diffkv_workspace_size(DIFFKV_OP_CHUNK_SIGNIFICANCE, ...) bytes
 * Tables of sequences without new tokens are left alone.  fp32 arithmetic.  A
 * probability that is NaN (a NaN key that the row sees, a NaN query) counts as 0,
 * so scores stay finite.
 * Other arguments, limits and errors as diffkv_chunk_attention.
 */
diffkv_status diffkv_chunk_significance(const diffkv_layout* layout, const diffkv_cache* cache,
                                        int64_t total_new, int32_t max_new, const int32_t* new_len,
                                        int32_t num_q_heads, const uint16_t* q, int64_t q_stride,
                                        const uint16_t* k, int64_t k_stride, float sm_scale,
                                        const diffkv_score_form* form, const float* lse, float* score,
                                        void* ws, size_t ws_bytes, void* stream);

/*
 * A uniform 8-bit cache, for layers whose tokens are not told apart by their
 * significance (sliding windows, a model's first layers): every token is kept at
 * 8 bits, in blocks of DIFFKV_BLOCK_TOKENS positions with one scale for a block's
 * keys and one for its values per KV head.  Block i of a sequence holds positions
 * 32 i .. 32 i + 31; table row b holds the IDs of sequence b's blocks, the same
 * for all KV heads.  Positions behind the last whole block are the sequence's tail,
 * fp16 rows as they were appended.  An ID outside the pool (-1) means that the block
 * is not kept: appended tokens that fill it are dropped, and attention counts
 * none there.  So a window's program gives the IDs of blocks that no row can see any
 * more to other sequences, and gives none to the blocks of a prompt that it will
 * never see.  The program assigns IDs and advances seq_len: the layers of a model
 * can share both.  A sequence may be set back within its tail (seq_len not below its
 * last whole block's end).
 * Codes: a value is code * scale.  DIFFKV_BLOCK_E4M3: e4m3 codes (four significant
 * bits, to 448), the scale a power of two; it suits keys with channels of
 * different size.  DIFFKV_BLOCK_INT8: integers from -127 to 127, the scale of
 * eight significant bits.
 * A block of a KV head, 8192 bytes: key codes [2: token / 16][8: dim / 16]
 * [16: token % 16][16: dim % 16], then value codes [4: dim / 32][4: r][16: dim % 16]
 * [2: dim / 16 % 2][8: e], e < 4 token 4 r + e, e >= 4 token 12 + 4 r + e.
 */
enum { DIFFKV_BLOCK_TOKENS = 32 };
enum { DIFFKV_BLOCK_E4M3 = 0, DIFFKV_BLOCK_INT8 = 1 };

typedef struct diffkv_block_cache {
    uint8_t*  pool;          /* device [num_blocks][num_kv_heads][8192], 16-byte aligned   */
    float*    scale;         /* device [num_blocks][num_kv_heads][2]: keys, values;
                                positive, or NaN                                     */
    int64_t   num_blocks;    /* up to INT32_MAX                                       */
    const int32_t* table;    /* device [num_seqs][ceil(max_seq_len / 32)] block IDs         */
    uint16_t* tail;          /* device fp16 [num_seqs][num_kv_heads][2][32][head_dim]: keys,
                                values of position p at p % 32; 16-byte aligned              */
    const int32_t* seq_len;  /* device [num_seqs] tokens held, up to max_seq_len             */
    uint32_t* status;        /* device [1] sticky DIFFKV_ST_* bits                     */
    int32_t   num_seqs;
    int32_t   num_kv_heads;
    int32_t   format;        /* DIFFKV_BLOCK_E4M3 or _INT8                             */
} diffkv_block_cache;

/*
 * Appends new tokens: positions seq_len[b] .. + new_len[b] - 1.  A block that they
 * fill is quantized from its tail rows and new rows and stored, if its ID is in the
 * pool; the rows behind the last whole block go to the tail.  seq_len is not
 * advanced.  What a cache holds depends on its tokens alone, not on how they were
 * cut into calls.
 * With amax the largest magnitude of a block's 32 x 128 keys (or values) of a KV head:
 *   E4M3   scale = 2^e, e the least integer with amax <= 448 * 2^e; codes are
 *          x / scale to the nearest e4m3 value, ties to the even one
 *   INT8   scale = amax / 127 rounded up to eight significant bits; codes are x / scale
 *          to the nearest integer, ties to the even one
 * exactly; scale = 1 where amax = 0.  If a value is not finite, the scale is NaN and
 * the codes are 0: every token of the block reads NaN.
 *   new_len  device int32 [num_seqs], rows of sequence b follow those of b-1.
 *            Every entry in [0, max_new], their sum at most total_new (rows behind the
 *            last sequence's are nobody's), else DIFFKV_ST_BAD_INPUT; seq_len[b] in
 *            [0, max_seq_len - new_len[b]], else DIFFKV_ST_TABLE_OVERFLOW.  A call
 *            that raises either changes nothing.
 *   k, v     device fp16: row r, head h at k + r*k_stride + h*head_dim (slices of a
 *            fused projection can be passed), 16-byte aligned, strides in elements,
 *            multiples of 8, at least heads*head_dim (any value with one row)
 * IDs of blocks that one call fills must differ.  head_dim 128, max_seq_len up to 2^30,
 * total_new up to 2^24 (DIFFKV_E_UNSUPPORTED otherwise).  No workspace.
 */
diffkv_status diffkv_block_append(const diffkv_layout* layout, const diffkv_block_cache* cache,
                                  int64_t total_new, int32_t max_new, const int32_t* new_len,
                                  const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                                  void* stream);

/*
 * Reads ranges of positions back as fp16 rows, e.g. to append them to a differentiated
 * cache, or for another sequence with the same beginning: row i of sequence b's is
 * position start[b] + i.  Stored values are code * scale rounded once to fp16 (beyond the
 * largest finite fp16: that one), tail rows come as they are.  A position that the cache does not
 * hold (outside [0, seq_len), or of a block without an ID in the pool) reads zero.
 *   start, count  device int32 [num_seqs]; rows of sequence b follow those of b-1.
 *            Counts are clamped to [0, max_count], and so that no row past
 *            total is written; rows behind the last sequence's are left as they
 *            were.
 *   k, v     device fp16 out, addressed as diffkv_block_append's inputs
 * Limits as diffkv_block_append.  No workspace; the cache is read only.
 */
diffkv_status diffkv_block_read(const diffkv_layout* layout, const diffkv_block_cache* cache, int64_t total,
                                int32_t max_count, const int32_t* start, const int32_t* count,
                                uint16_t* k, int64_t k_stride, uint16_t* v, int64_t v_stride, void* stream);

/*
 * Attention of a chunk of new tokens over a uniform cache, before the chunk is
 * appended: one token per sequence, drafted tokens, a prompt's next part, or any
 * mixture.  New token j of sequence b has position p = seq_len[b] + j; its query of
 * head hq attends to the tokens of KV head hq/(Hq/Hkv) at c <= p, the cache's
 * (code * scale), the tail's and the chunk's own in fp16:
 *   out[row][hq] = sum_c softmax_c(x) v_c,  x as in diffkv_score_form,
 * where a windowed form sees the key at c if p - c < window or c < sinks: the first
 * `sinks` tokens of a sequence stay visible (sinks >= 0; without a window it says nothing).
 * Tiles of 32 positions that no row of a sequence sees are skipped.
 *   new_len, q, k, v, out, lse, sm_scale, form  as diffkv_chunk_attention takes them
 *   ws       diffkv_workspace_size(DIFFKV_OP_BLOCK_ATTENTION, ...) bytes, no clearing
 *            needed, 16-byte aligned; calls that may overlap need one each
 *            (strides of k and v at most 2^24)
 * The cache is read only.  Up to 64 query heads per KV head, head_dim 128, total_new
 * up to 2^23, max_seq_len up to 2^30, up to 2^22 (sequence, KV head) pairs
 * (DIFFKV_E_UNSUPPORTED otherwise).  seq_len counts clamped to [0, max_seq_len].
 * Scores x up to 2^22 in magnitude, the slopes' part included.
 * Precision: codes enter the products exactly, and the weights in two fp16 parts (2^-22, or 2^-37 of
 * their row's largest, each weighed by its block's value scale); sums and softmax statistics are fp32, and out is
 * rounded once.  The order of a row's sums, and with it the last bits, goes by the
 * call's lengths.
 * A NaN or infinite key or value of a tail or chunk reaches only the rows that see its token;
 * a block whose scale is NaN, those that see one of its tokens.  Values do not reach lse.
 */
diffkv_status diffkv_block_attention(const diffkv_layout* layout, const diffkv_block_cache* cache,
                                     int64_t total_new, int32_t max_new, const int32_t* new_len,
                                     int32_t num_q_heads, const uint16_t* q, int64_t q_stride,
                                     const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                                     float sm_scale, const diffkv_score_form* form, int32_t sinks,
                                     uint16_t* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Parallel free-list compaction (Sec. 5.2 recycling, Sec. 5.3): for the
 * first num_tables tables, every live slot whose release byte is nonzero
 * gives its page back.  With one prefix sum over tables, table t writes its
 * released IDs -- in ascending slot order -- to ring[(tail + off_t + i) % n];
 * tail advances by the total.  Each table is then squeezed in place: kept
 * high IDs packed from slot 0 and kept low IDs from slot p_max-1, both in
 * their section order; vacated slots become -1.  A released page removes its
 * tokens from the section (T, or the tail page's fill; later pages shift
 * down).  Request completion = releasing every live slot of its tables.
 *   release  device uint8 [num_tables][p_max]; bytes of non-live slots are
 *            ignored.
 * Never fails on the device (released IDs always fit the ring).  p_max above
 * 8192 or more than 2^20 tables: DIFFKV_E_UNSUPPORTED.
 */
diffkv_status diffkv_compact_free_list(const diffkv_layout* layout, const diffkv_cache* cache,
                                       int32_t num_tables, const uint8_t* release,
                                       void* ws, size_t ws_bytes, void* stream);

/*
 * Page allocation alone (Sec. 5.2 allocation; the prompt phase's
 * conservative reservation of Sec. 5.3): table t appends demand[t][HIGH]
 * pages to its high side and demand[t][LOW] to its low side, reading IDs
 * from the ring region after the demands of tables 0..t-1; head advances by
 * the total.  len is unchanged (the new pages are spare until an append
 * fills them).  All-or-nothing OUT_OF_PAGES / TABLE_OVERFLOW.
 *   demand  device int32 [num_tables][2], entries >= 0.
 */
diffkv_status diffkv_alloc_pages(const diffkv_layout* layout, const diffkv_cache* cache,
                                 int32_t num_tables, const int32_t* demand,
                                 void* ws, size_t ws_bytes, void* stream);

/*
 * Generation-phase policy (Sec. 4, Algorithm 1), once per decode step, after
 * the step's diffkv_quantize_append has put the newest token of every
 * sequence into the high section (its recent window).  For table t of
 * sequence b, with N = seq_len[b] and W = recent_window:
 *   - candidate: the high token at position N - 1 - W (the one that has just
 *     left the window); a table without one is left alone;
 *   - thresholds alpha_h / N and alpha_l / N, fp32 quotients;
 *   - victim of a section: its token of lowest score (-0 == +0; ties to the
 *     lowest position) among those at positions <= N - 1 - W;
 *   - score(candidate) >= alpha_h/N: the candidate stays; the high victim
 *     moves to the low section if alpha_l/N <= its score < alpha_h/N, and is
 *     removed if its score < alpha_l/N;
 *   - alpha_l/N <= score(candidate) < alpha_h/N: the candidate moves to the
 *     low section, over the low victim's slot if that victim's score is
 *     < alpha_l/N (the victim is evicted), else at the section's end;
 *   - otherwise the candidate is removed.
 * A token leaves the high section by swap-remove: the section's last token
 * moves into its slot (bytes unchanged) and the vacated slot is cleared to
 * zero; a page emptied this way stays with the table.  A token moving to the
 * low section is re-quantized: per element s*code + z as one fp32 fma,
 * rounded to fp16 (nearest even), then quantized as diffkv_quantize_append
 * quantizes a low-precision token; its score and position are kept.
 * Appending to a full low section takes one page per table, with the
 * allocation's prefix-sum schedule over tables (ring region after the pages
 * of lower tables; head advances by the total); all-or-nothing
 * OUT_OF_PAGES / TABLE_OVERFLOW (then nothing changes).  seq_len is not
 * changed.  Sections are dense but, after a removal, no longer in position
 * order (attention does not depend on the order).
 *   recent_window  W >= 0, DIFFKV_E_INVAL otherwise.
 *   ws   device workspace of diffkv_workspace_size(DIFFKV_OP_GENERATION, ...).
 */
diffkv_status diffkv_generation_step(const diffkv_layout* layout, const diffkv_cache* cache,
                                     float alpha_h, float alpha_l, int32_t recent_window,
                                     void* ws, size_t ws_bytes, void* stream);

/* Static string for a diffkv_status value. */
const char* diffkv_status_str(diffkv_status s);

#ifdef __cplusplus
}
#endif
#endif
