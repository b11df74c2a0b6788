/*
 * cas_ops.h - kernel-level entry points of the CAS-Spec tree decoder library,
 * on caller-owned DEVICE buffers.
 *
 * These expose single kernels of the forward of cas.h so that each can be
 * checked against a CPU definition on identical inputs, and timed alone.
 * All pointers are device pointers (except where noted) owned by the caller;
 * `stream` is a hipStream_t (NULL = the null stream).  Every call is
 * asynchronous on that stream and returns CAS_ERR_ARG / CAS_ERR_UNSUPPORTED
 * for shapes it does not handle, CAS_ERR_DEVICE if the launch fails.
 */
#ifndef CAS_OPS_H
#define CAS_OPS_H

#include "cas.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CAS_W_F32 = 0, CAS_W_BF16 = 1, CAS_W_I8 = 2, CAS_W_I4 = 3 } cas_wtype;
typedef enum {
    CAS_EPI_STORE = 0,   /* out[t*ldo + n] = y (float32) */
    CAS_EPI_RESID = 1,   /* out[t*ldo + n] += y (float32 residual stream) */
    CAS_EPI_RAW_I32 = 2  /* out[t*ldo + n] = integer accumulator (int32; int8 and int4 only) */
} cas_epi;

/*
 * Linear layer y[t][n] = sum_k X[t][k] W[n][k] for t < T, n < N (the weight
 * streaming GEMM of every projection and the LM head).
 *   W: [N][K] row-major, element type wtype (float32, bf16 bits, int8; for
 *      CAS_W_I4 int8 codes in [-7, 7], which the library packs to 4 bits)
 *   X: [T][K] row-major, same element type as W (int8 codes for CAS_W_I4)
 *   xs, ws: for CAS_W_I8 / CAS_W_I4 the per-row activation scales [T] and
 *           per-output channel weight scales [N]; y = (float(acc) * xs[t]) * ws[n]
 *           (ignored for the other types; unused with CAS_EPI_RAW_I32)
 *   work: device scratch of at least cas_op_gemm_work_bytes(...) bytes; the
 *         operands are first rearranged there into the fragment-tiled layout
 *         the kernel streams (the layout the library keeps its weights in)
 * Limits: N multiple of 16, K multiple of 16, 1 <= T <= 128.
 * Accumulation: fp32 (float32, bf16 inputs), exact int32 (int8 and int4
 * inputs; the W4A4 form of activation quantisation, Sec. 4.1 and App. C, runs
 * its int4 codes on the int8 MFMA).  One-row calls (T = 1) with N >= 8192
 * and bf16 or int8 weights run the GEMV-style tiles the library uses for
 * one-node drafts (VALU dot products per lane, the four k-group lanes of a
 * row summed at the end), other calls the MFMA tiles.
 */
size_t cas_op_gemm_work_bytes(int32_t wtype, int32_t N, int32_t K, int32_t T);
cas_status cas_op_gemm(int32_t wtype, const void* W, const void* X, int32_t N, int32_t K, int32_t T,
                       const float* xs, const float* ws, int32_t epi, void* out, int32_t ldo,
                       void* work, size_t work_bytes, void* stream);

/*
 * Per-row symmetric int8 quantisation of activations (App. C, activation
 * quantisation; one row per token): s[t] = max_k |x[t][k]| / 127 (fp32),
 * q[t][k] = clamp(round-half-even(x[t][k] / s[t]), -127, 127); a zero row
 * gives s = 0, q = 0.  x: [T][K] of type atype (CAS_W_F32 or CAS_W_BF16).
 */
cas_status cas_op_quant_rows(int32_t atype, const void* x, int32_t T, int32_t K,
                             int8_t* q, float* s, void* stream);
/* The same rule with codes in [-qmax, qmax]: qmax 127 (int8, as above) or 7
 * (int4 codes of the W4A4 draft, one per int8 byte): s[t] = amax / qmax. */
cas_status cas_op_quant_rows_q(int32_t atype, const void* x, int32_t T, int32_t K, int32_t qmax,
                               int8_t* q, float* s, void* stream);

/* Per-output-channel int8 copy of W [N][K] (same rule, one row per output
 * channel), through the library's tiled weight layout: q [N][K] row-major,
 * s [N].  wtype: CAS_W_F32 or CAS_W_BF16; N and K multiples of 16; work:
 * device scratch of cas_op_quant_weight_work_bytes(...) bytes. */
size_t cas_op_quant_weight_work_bytes(int32_t wtype, int32_t N, int32_t K);
cas_status cas_op_quant_weight(int32_t wtype, const void* W, int32_t N, int32_t K,
                               int8_t* q, float* s, void* work, size_t work_bytes, void* stream);
/* Per-output-channel int4 copy of W (s[n] = amax / 7, codes in [-7, 7]),
 * through the library's tiled weights and its packed 4-bit layout, returned
 * unpacked: q [N][K] row-major int8 codes, s [N].  Same arguments, limits and
 * work size as cas_op_quant_weight. */
cas_status cas_op_quant_weight_i4(int32_t wtype, const void* W, int32_t N, int32_t K,
                                  int8_t* q, float* s, void* work, size_t work_bytes, void* stream);

/*
 * Tree-masked attention of one layer (bf16 storage, fp32 softmax):
 *   q:   [T][n_heads][head_dim] bf16 (after RoPE)
 *   k:   [n_kv_heads][ctx_cap][head_dim] bf16 keys (row-major)
 *   v:   [n_kv_heads][ctx_cap][head_dim] bf16 values (row-major)
 *   anc: [T][2] 64-bit ancestor-or-self masks over the round's nodes
 *        (bit j = node j, whose slot is Lc + j)
 *   out: [T][n_heads*head_dim] bf16
 * Query row t sees slots [0, Lc) and the slots Lc + j of the nodes j set in
 * anc[t]; n_tree nodes exist (Lc + n_tree <= ctx_cap, n_tree <= 128;
 * ctx_cap a multiple of 32).  head_dim 64 or 128; T <= 128.  work: device
 * scratch of cas_op_attention_work_bytes(...) bytes (the keys and values are
 * first copied there into the library's cache layout).
 */
cas_status cas_op_attention(const void* q, const void* k, const void* v, int32_t ctx_cap,
                            int32_t Lc, int32_t n_tree, int32_t T, int32_t n_heads,
                            int32_t n_kv_heads, int32_t head_dim, const uint64_t* anc,
                            void* out, void* work, size_t work_bytes, void* stream);
size_t cas_op_attention_work_bytes(int32_t Lc, int32_t n_tree, int32_t T, int32_t n_heads,
                                   int32_t head_dim, int32_t n_kv_heads, int32_t ctx_cap);

/*
 * cas_op_attention for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same arguments, kernels and results, without `work`.  The scratch (the
 * key and value copies in the library's cache layout, the step parameters
 * and the KV-split partials) is a device array of the library of
 * cas_op_attention_noalloc_max_bytes() bytes (64 MiB), one per GPU, held
 * until the process ends.  Calls whose cas_op_attention_work_bytes(...)
 * exceeds it return CAS_ERR_CAPACITY and do nothing.  Nothing is allocated:
 * no hipMalloc, hipFree or allocating library call.  The calling thread's
 * current device must be the device of `stream`.  All calls on one GPU
 * share its array: calls that overlap in time on one GPU (other threads or
 * streams) race; the call returns after its kernels have finished, so calls
 * made one after another from one thread do not.  Every byte of the array a
 * call reads is written by that call first.
 */
size_t cas_op_attention_noalloc_max_bytes(void);
cas_status cas_op_attention_noalloc(const void* q, const void* k, const void* v, int32_t ctx_cap, int32_t Lc,
                                    int32_t n_tree, int32_t T, int32_t n_heads, int32_t n_kv_heads,
                                    int32_t head_dim, const uint64_t* anc, void* out, void* stream);

/*
 * The fused quantisers of the forward, each run alone.  Activation
 * quantisation (Sec. 4.1; App. C) is applied by the forward inside three
 * kernels rather than by a separate pass; these entry points run exactly
 * those kernels, so their codes can be compared bit for bit with the row
 * quantiser's rule (cas_op_quant_rows_q) on identical inputs.
 *
 * RMSNorm of the residual rows, optionally straight to per-token codes (the
 * input of the QKV and gate/up projections of a quantised draft):
 *   h:      [T][d] fp32 residual rows (device).  With nparts > 0 the rows
 *           first take the pending split-K sums: h += parts[0] + ... +
 *           parts[nparts-1], summed in that order, stored back to h
 *   gain:   [d] fp32 gains; eps inside the square root (eps >= 0)
 *   parts:  [nparts][T][d] fp32 (nparts in [0, 8])
 *   qmax:   0: out receives the normalised rows [T][d] in the model type
 *           (atype CAS_W_BF16: bf16 bits rounded to nearest even; CAS_W_F32:
 *           fp32); 127 or 7: q [T][d] receives the codes and qs [T] the
 *           scales of those normalised (rounded) rows, s = amax / qmax,
 *           q = clamp(rne(x / s), -qmax, qmax), zero rows s = 0, q = 0
 *   work:   device scratch of cas_op_rmsnorm_work_bytes(...) bytes (the
 *           kernel's tiled output before it is written back row-major)
 * Limits: 1 <= T <= 128, d a multiple of 16, d <= 16384.
 */
size_t cas_op_rmsnorm_work_bytes(int32_t atype, int32_t T, int32_t d, int32_t qmax);
cas_status cas_op_rmsnorm(int32_t atype, float* h, const float* gain, int32_t T, int32_t d, float eps,
                          const float* parts, int32_t nparts, int32_t qmax, void* out, int8_t* q, float* qs,
                          void* work, size_t work_bytes, void* stream);

/*
 * Merge of the attention's KV-split partial states (the second kernel of
 * the tree attention of a bf16 model), optionally straight to the O
 * projection's per-token codes (the merge-and-quantise kernel of quantised
 * drafts):
 *   part_o:  [S][n_heads][T][head_dim] fp32: split s's unnormalised sum of
 *            2^(x_j - m) v_j over its keys j, where x_j is the score in base-2
 *            units (q.k_j / sqrt(head_dim) * log2(e))
 *   part_ml: [S][n_heads][T][2] fp32: (m, l) = the split's largest x_j and
 *            its sum of 2^(x_j - m)
 *   The merged row is sum_s 2^(m_s - M) part_o_s / sum_s 2^(m_s - M) l_s with
 *   M the running maximum, merged in split order, rounded to bf16.
 *   qmax 0: out [T][n_heads*head_dim] bf16 bits; 127 or 7: q [T][n_heads*
 *   head_dim] codes and qs [T] scales of those bf16 rows (row quantiser rule)
 *   work: device scratch of cas_op_attn_merge_work_bytes(...) bytes
 * Limits: S in [1, 64], 1 <= T <= 128, head_dim 64 or 128,
 * n_heads * head_dim <= 16384.
 */
size_t cas_op_attn_merge_work_bytes(int32_t T, int32_t n_heads, int32_t head_dim, int32_t qmax);
cas_status cas_op_attn_merge(const float* part_o, const float* part_ml, int32_t S, int32_t T, int32_t n_heads,
                             int32_t head_dim, int32_t qmax, uint16_t* out, int8_t* q, float* qs, void* work,
                             size_t work_bytes, void* stream);

/*
 * Split-K residual projection that quantises its bf16 input on load (the O
 * and down projections of one-node quantised drafts on bf16 models): every
 * workgroup takes the row's amax over the whole row, writes the codes of its
 * own K range by the row quantiser's rule (s = amax / qmax) and runs the
 * integer GEMM on them.
 *   wtype:  CAS_W_I8 (W: codes in [-127, 127], qmax 127) or CAS_W_I4 (W:
 *           codes in [-7, 7], packed to 4 bits by the library, qmax 7)
 *   W [N][K] row-major codes, ws [N] per-output-channel weight scales,
 *   x [T][K] bf16 bits (T = 1)
 *   parts:  [splits][T][N] fp32: split k's dequantised sums over its K range,
 *           (fp32(acc_k) * s) * ws[n]; splits = cas_op_gemm_qx_splits(...)
 *           (0: the shape does not take this form)
 *   work:   device scratch of cas_op_gemm_qx_work_bytes(...) bytes
 */
int32_t cas_op_gemm_qx_splits(int32_t wtype, int32_t N, int32_t K, int32_t T);
size_t cas_op_gemm_qx_work_bytes(int32_t wtype, int32_t N, int32_t K, int32_t T);
cas_status cas_op_gemm_qx(int32_t wtype, const int8_t* W, const float* ws, const uint16_t* x, int32_t N, int32_t K,
                          int32_t T, int32_t qmax, float* parts, void* work, size_t work_bytes, void* stream);

/*
 * The 4-bit KV cache (App. C: activation quantisation of the "(partial) KV
 * cache"): rows appended to it, attended and read back by the three calls
 * below.  Keys and values are microscaled floats (OCP MX, E2M1 elements): 32
 * consecutive elements x of a token's head row share the scale 2^e, e =
 * max(floor(log2 max|x|) - 2, -125), held as the byte e + 127, and an element
 * is the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} to x / 2^e (codes 0-7, sign
 * in bit 3; ties to the even code; saturating at 6).  A block that holds a NaN
 * or an infinity has the scale byte 255 and reads as NaN.  Every value held is
 * exact in bf16.
 *   kv4: cas_op_kv4_bytes(...) bytes, 16-byte aligned: [n_kv_heads][ctx_cap /
 *        32] records of 34 * head_dim bytes for 32 slots, in this order (hd =
 *        head_dim, w = 512 / hd, the last index fastest):
 *          16 hd  key codes [2 s][4 g][4 i][4 j][hd/32 u][4 c]: elements d =
 *                 g hd/4 + 8u + 2c (low four bits) and d + 1 of slot 8i + 4s + j
 *          16 hd  value codes [hd/64 m][4 g][hd/32 b][w r][2 n][8 j]: elements
 *                 d = 32b + w (4m + 2n) + r (low four bits) and d + w of slot 8g + j
 *             hd  key scales [hd/32 b][4 i][4 j][2 s] (slot 8i + 4s + j)
 *             hd  value scales [hd/32 b][32 slots]
 *        Nothing outside the records matters to a later call, so a cache may be
 *        copied, saved and cut at record boundaries; slots never appended may
 *        hold anything.
 * Limits: head_dim 64 or 128; ctx_cap a multiple of 32, at most 1048576;
 * n_kv_heads at most 65535.
 */
size_t cas_op_kv4_bytes(int32_t n_kv_heads, int32_t head_dim, int32_t ctx_cap);

/*
 * Append T tokens' keys and values: quantise them into slots slot0 ..
 * slot0 + T - 1 (of every kv head).  Other slots' bytes are not touched.
 *   k, v:  bf16 rows of n_kv_heads * head_dim elements, ldk and ldv elements
 *          apart (at least that many: rows of a wider product can be passed in
 *          place).  Rows that start at multiples of 16 bytes load fastest
 *   rope_cos, rope_sin: NULL (the keys are stored as they are), or [n_pos]
 *          [head_dim/2] fp32, 16-byte aligned: the keys are rotated first,
 *          pairs (i, i + head_dim/2) as in cas.h, the exact rotated value
 *          rounded once to fp32 and quantised from there
 *   pos:   [T] positions (device), or NULL: row t's position is slot0 + t.  A
 *          position outside [0, n_pos) stores that row's keys as NaN.  Not
 *          read without a rotation
 * 1 <= T, 0 <= slot0, slot0 + T <= ctx_cap.
 */
cas_status cas_op_kv4_append(const void* k, const void* v, int64_t ldk, int64_t ldv, int32_t T, int32_t slot0,
                             const int32_t* pos, const float* rope_cos, const float* rope_sin, int32_t n_pos,
                             int32_t n_kv_heads, int32_t head_dim, void* kv4, int32_t ctx_cap, void* stream);

/* The values that slots slot0 .. slot0 + n - 1 hold, as bf16: k, v
 * [n_kv_heads][n][head_dim], 16-byte aligned. */
cas_status cas_op_kv4_read(const void* kv4, int32_t ctx_cap, int32_t slot0, int32_t n, int32_t n_kv_heads,
                           int32_t head_dim, void* k, void* v, void* stream);

/*
 * Tree-masked attention over a cache whose first n4 slots are held in 4 bits:
 * the rule, q, anc and out of cas_op_attention, with fp32 softmax.
 *   n4:    slots [0, n4) are read from kv4, the others from k, v.  A multiple
 *          of 32, or Lc + n_tree (every slot in 4 bits, the round's too)
 *   k, v:  bf16 [n_kv_heads][kv_cap][head_dim], row j holding slot n4 + j,
 *          kv_cap >= Lc + n_tree - n4 (NULL where no slot needs them)
 *   attn_sink, attn_window: as in cas_draft_opts (0: every committed slot)
 *   q, k, v and out are 16-byte aligned
 * Slots and rows that a row does not see never reach it, whatever they hold.
 * A row that sees no slot gives zeros; one that sees a key that is not finite
 * gives NaN, and one that sees such a value NaN at its element.
 * Probabilities are rounded to bf16 for the product with the values (each by
 * at most 2^-8 of itself; cas_op_attention, over slots read back, by 2^-16).
 * The result does not depend on earlier calls or on timing; it may depend in
 * the last bits on T.
 * 1 <= T <= 128, 1 <= n_tree <= 128, 0 <= Lc, Lc + n_tree <= 1048576, n4 <=
 * ctx_cap (the bf16 rows need no record), n_heads <= 4096.
 * work: device scratch of cas_op_attention_kv4_work_bytes(...) bytes (0: none
 * is needed, work may be NULL), 16-byte aligned, used by one call at a time.
 */
size_t cas_op_attention_kv4_work_bytes(int32_t Lc, int32_t n_tree, int32_t T, int32_t n_heads, int32_t n_kv_heads,
                                       int32_t head_dim, int32_t attn_sink, int32_t attn_window);
cas_status cas_op_attention_kv4(const void* q, const void* kv4, int32_t ctx_cap, int32_t n4, const void* k,
                                const void* v, int32_t kv_cap, int32_t Lc, int32_t n_tree, int32_t T,
                                int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t attn_sink,
                                int32_t attn_window, const uint64_t* anc, void* out, void* work, size_t work_bytes,
                                void* stream);

/*
 * The paged KV cache: the new rows of several sequences appended to pages of a
 * common pool, with their rotation, and attention of those rows over the
 * sequences' pages.  One cas_paged describes the cache of a layer and the batch
 * of a step; both calls take it (a host struct, read during the call; its
 * arrays are on the device and are read by the kernels, so that a captured call
 * replays with the lengths and pages that they hold then).
 *   pages:     cas_op_paged_bytes(...) bytes, 16-byte aligned: bf16 [n_pages][2]
 *              [n_kv_heads][page_size * head_dim], keys then values.  A head's
 *              run is page_size / 32 tiles of 32 slots, the last index fastest:
 *                keys    [2 h][hd/32 u][4 g][4 i][4 j][8 e]: slot 8i + 4h + j,
 *                        element g hd/4 + 8u + e
 *                values  [hd/16 m][4 g][16 r][8 e]: slot 8g + e, element 16m + r
 *   table:     [n_seqs][table_len] page numbers; slot s of sequence b is slot
 *              s % page_size of page table[b][s / page_size].  Entries past a
 *              sequence's slots are not read.  Sequences may share pages
 *   seq_start: [n_seqs + 1], not decreasing: sequence b's rows are the rows
 *              seq_start[b] .. seq_start[b + 1] - 1 of the call (none, or not
 *              rows of the call: it takes no part).  Where it decreases some
 *              rows may be left out; nothing outside the buffers is touched
 *   ctx_len:   [n_seqs] committed slots
 *   nodes:     NULL, or [n_seqs] slots of the sequence's round behind the
 *              committed ones, appended by earlier calls.  Row i of sequence b
 *              lies in slot ctx_len[b] + nodes[b] + i
 *   n_rows:    rows of the calls' tensors; rows behind the last sequence's are
 *              not read and not written
 *   max_rows:  rows of the longest sequence as far as the caller knows (0: may
 *              be all): a hint by which a kernel is chosen, results are right
 *              whatever it says
 * A sequence whose slots do not fit its table row stores nothing, and its
 * attention rows are NaN; so are rows that see a slot of a page outside [0,
 * n_pages), and such a page is not written.
 * Limits: head_dim 64 or 128; page_size a power of two from 32 to 4096;
 * table_len * page_size at most 1048576; n_kv_heads at most 4096; n_seqs at most
 * 65536; n_rows * n_heads / n_kv_heads below 2^24; CAS_ERR_UNSUPPORTED where a
 * call would take more than 2^32 - 1 threads.
 */
typedef struct {
    void* pages;
    int32_t n_pages, page_size, n_kv_heads, head_dim;
    const int32_t* table;
    int32_t table_len, n_seqs;
    const int32_t* seq_start;
    const int32_t* ctx_len;
    const int32_t* nodes;
    int32_t n_rows, max_rows;
} cas_paged;
size_t cas_op_paged_bytes(int32_t n_pages, int32_t page_size, int32_t n_kv_heads, int32_t head_dim);

/*
 * Write the rows' keys and values into their slots, and their queries to q_out.
 * Other slots' bytes are not touched; two rows given the same slot (through
 * shared pages) leave either.
 *   k, v:  bf16 rows of n_kv_heads * head_dim elements, ldk and ldv elements
 *          apart (at least that many: rows of a fused product in place)
 *   q, q_out: NULL, or bf16 rows of n_heads * head_dim elements, ldq apart, and
 *          [n_rows][n_heads][head_dim], 16-byte aligned.  q_out may be q (then
 *          ldq = n_heads * head_dim)
 *   rope_cos, rope_sin: NULL (nothing is rotated), or [n_pos][head_dim/2] fp32,
 *          16-byte aligned: keys and queries are rotated, pairs (i, i +
 *          head_dim/2) as in cas.h, in fp32, and rounded to bf16 once
 *   pos:   [n_rows] positions, or NULL: a row's position is its slot.  A
 *          position outside [0, n_pos) gives a key and query of NaN
 */
cas_status cas_op_paged_append(const cas_paged* cache, const void* q, int64_t ldq, int32_t n_heads, const void* k,
                               int64_t ldk, const void* v, int64_t ldv, const int32_t* pos, const float* rope_cos,
                               const float* rope_sin, int32_t n_pos, void* q_out, void* stream);

/*
 * Attention of the rows over their sequences' slots (fp32 softmax, scale 1 /
 * sqrt(head_dim)).
 *   q:    bf16 [n_rows][n_heads][head_dim]; out: bf16 [n_rows][n_heads * head_dim]
 *   anc:  NULL: causal, a row sees the slots up to its own; or [n_rows][2]
 *         ancestor-or-self masks: a row sees the committed slots, and slot
 *         ctx_len + j where bit j of its mask is set (nodes + rows of a sequence
 *         at most 128, else its rows are NaN)
 *   attn_sink, attn_window: attn_window > 0 limits the slots before a causal
 *         row's own, or a tree row's committed slots, to the first attn_sink and
 *         the last attn_window ones (0: all)
 * Slots and rows that a row does not see never reach it, whatever they hold.  A
 * row that sees no slot gives zeros; one with a score of NaN or +infinity gives
 * NaN, and one that sees a value that is not finite no finite one at its element.
 * A score of -infinity has no weight.
 * Probabilities are rounded for the product with the values, each by at most 2^-16
 * of itself where max_rows (0: n_rows) times n_heads / n_kv_heads is at most 32 (as
 * in cas_op_attention), and by 2^-8, to bf16, where it is more.  The result does
 * not depend on earlier calls or on timing; it may depend in the last bits on the
 * batch.
 * n_heads <= 4096.  work: device scratch of cas_op_attention_paged_work_bytes
 * (...) bytes (0: none is needed, work may be NULL), 16-byte aligned, used by
 * one call at a time.  The size rests on the struct's numbers, not on its arrays.
 */
size_t cas_op_attention_paged_work_bytes(const cas_paged* cache, int32_t n_heads);
cas_status cas_op_attention_paged(const cas_paged* cache, const void* q, int32_t n_heads, const uint64_t* anc,
                                  int32_t attn_sink, int32_t attn_window, void* out, void* work, size_t work_bytes,
                                  void* stream);

/*
 * Log probabilities of given tokens, entropy and top alternatives of rows of
 * logits, under the distribution p = softmax(scale * x) (natural logarithms):
 *   ltype:   CAS_W_F32 or CAS_W_BF16; logits: n rows of V elements, ld (>= V)
 *            elements apart
 *   tokens:  [n][m] token ids; logp [n][m] fp32: log p of each, NaN for an id
 *            outside [0, V) (m may be 0)
 *   entropy: NULL, or [n] fp32: - sum p log p
 *   K:       0 to 32; top_ids [n][K] int32 and top_logp [n][K] fp32: the tokens
 *            of highest logit (decreasing, the lower id on ties; id -1 and
 *            -infinity past the row's finite entries)
 * A logit of -infinity has probability 0.  A row that holds a NaN or +infinity,
 * or nothing but -infinity, has no distribution: NaN, and ids -1.
 * scale: > 0 (1 / temperature), its product with log2(e) finite.  V at most 1048576, n at most
 * 2097152.  Sums in fp32.
 * work: device scratch of cas_op_logprobs_work_bytes(...) bytes (no less for
 * more rows or a larger K), 16-byte aligned, used by one call at a time.
 */
size_t cas_op_logprobs_work_bytes(int32_t n, int32_t V, int32_t K);
cas_status cas_op_logprobs(int32_t ltype, const void* logits, int64_t ld, int32_t n, int32_t V, float scale,
                           const int32_t* tokens, int32_t m, float* logp, float* entropy, int32_t K, int32_t* top_ids,
                           float* top_logp, void* work, size_t work_bytes, void* stream);

/*
 * How a prefill block of T rows (129 to 2048) runs a linear layer; host only.
 *   wtype:  CAS_W_F32 or CAS_W_BF16; W [N][K]
 *   resid:  1 for the O and down projections (added to the residual stream)
 *   info:   weight rows and activation rows of a workgroup's block, the K
 *           ranges summed apart, and 1 if each of them has workgroups of its own
 */
cas_status cas_op_prefill_block(int32_t wtype, int32_t N, int32_t K, int32_t T, int32_t resid, int32_t info[4]);

/* Plain device copy kernel (16-byte vector loads and stores): the reference
 * traffic for calibrating HBM byte counters.  bytes must be a multiple of 16. */
cas_status cas_op_copy(void* dst, const void* src, size_t bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CAS_OPS_H */
