/* libecco -- the compressed KV cache in pages: C ABI.
 *
 * A serving program holds the keys and values of all its sequences in one pool of pages, and a table per sequence says which
 * pages are its own, in order.  Blocks and meta words are those of ecco.h (two-chain format), as are the conventions: statuses,
 * streams, ownership, the order in which arguments are checked, FP16 as uint16_t.
 *
 *   pool        n_pages pages of page_tokens tokens, page_tokens a power of two from 16 to 1024
 *               k_blocks, v_blocks  device, [n_pages][H][page_tokens] blocks of 64 bytes, 64-byte aligned
 *               k_meta, v_meta      device, [n_pages][H][page_tokens] uint32
 *   page_table  device, [B][max_pages] int32: entry i of a sequence is the page that holds its tokens i * page_tokens and on.
 *               Entries behind a sequence's last page may be anything.
 *   slot        page * page_tokens + token of the page.  n_pages * page_tokens and max_pages * page_tokens are at most 2^31 - 1.
 *   rows        the new tokens of a step, sequence by sequence: sequence b has the rows q_start[b] .. q_start[b + 1] - 1.
 * Contents of device memory are never trusted with an address: pages outside the pool are neither written nor read.  Calls are launched on the
 * calling thread's current device, which must hold the tensors (and, where there are models, the models).
 */
#ifndef ECCO_PAGED_H
#define ECCO_PAGED_H

#include "ecco.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Gives every sequence the pages for its new tokens and says where each of them goes.
 *   seq_len, new_len  device, [B] int32: tokens that the sequence holds already, and new ones of this step (negative: none)
 *   page_table        in and out: the entries ceil(seq_len / page_tokens) .. ceil((seq_len + new_len) / page_tokens) - 1 are written
 *   free_pages        device, [n_pages] int32: a stack of the pages that nobody holds
 *   free_count        device, one int32: how many there are (taken as 0..n_pages);  free_left  device, one int32: how many are left;
 *                     the two may be one address
 *   n_tokens          rows of the step;  q_start  device, [B + 1] int32 out;  kv_len  device, [B] int32 out
 *   slots             device, [n_tokens] int32 out: the slot of every row, -1 for rows that have none
 * Pages come off the top of the stack (free_pages[count - 1] first), sequence by sequence.  A sequence is not served -- no page
 * taken, no entry written, its slots -1, its kv_len 0 -- if not all of its rows lie below n_tokens, if it needs more than max_pages, or
 * if the pages that it and the sequences before it need are more than there are (one that needs none is served all the same).
 * Otherwise kv_len = seq_len + new_len.  q_start is the running sum of new_len, at most n_tokens; rows from q_start[B] on get slot -1.
 * Apart from free_left, which may be free_count, outputs must not overlap inputs.  Behind the step, lengths are advanced to the larger of seq_len and
 * kv_len, element by element: a sequence that was not served then keeps its length, with it its pages and what their tokens hold, and may be
 * offered the same tokens again.  (kv_len alone would make it 0 tokens long, and its pages nobody's.)
 * Errors: EINVAL (null), ESHAPE (B, max_pages, n_pages <= 0, n_tokens < 0, page_tokens, sizes over 2^31 - 1), EALIGN (4 bytes), EINVAL (kv_len is
 * seq_len or new_len), EHIP.  With n_tokens == 0 slots may be null. */
int ecco_kv_pages_take(const int32_t* seq_len, const int32_t* new_len, int B, int page_tokens, int max_pages, int32_t* page_table,
                       const int32_t* free_pages, const int32_t* free_count, int32_t* free_left, int n_pages,
                       int n_tokens, int32_t* q_start, int32_t* kv_len, int32_t* slots, void* stream);

/* Puts the pages back that sequences no longer need: of a sequence that goes from seq_len to keep_len tokens (0: it is done) the
 * entries ceil(keep_len / page_tokens) .. ceil(seq_len / page_tokens) - 1, sequence by sequence, onto the stack.  keep_len is taken as
 * 0..seq_len.  Entries that are no pages of the pool, or behind max_pages, are left out, and so is what would exceed n_pages.
 * page_table is not changed.  Arguments and errors as above; free_pages is written from free_pages[count] on.
 * Nothing counts who holds a page: one that is released twice -- by two sequences that share it, or by one in two calls -- is on the stack
 * twice and will be given to two sequences.  A program that lets sequences share pages counts their holders itself, and leaves a shared
 * page out with a keep_len behind it until the last one ends. */
int ecco_kv_pages_release(const int32_t* seq_len, const int32_t* keep_len, int B, int page_tokens, int max_pages, const int32_t* page_table,
                          int32_t* free_pages, const int32_t* free_count, int32_t* free_left, int n_pages, void* stream);

/* ecco_kv_append for any number of new tokens per sequence: row i of the keys and values goes to slots[i], every head.
 *   k_new, v_new   device, 4-byte aligned: row i at k_new + i * k_stride, its H x 128 FP16 values one behind the other; the strides are
 *                  even and at least H * 128, so that the rows may lie in the output of a projection fused over queries, keys and values
 *   slots          device, [n_tokens] int32; a row whose slot is not one of the pool's writes nothing.  Rows must not share a slot.
 * n_tokens == 0 is a no-op.  Pattern selection as ecco_encode, or as ecco_encode_minmax.
 * Errors: EINVAL, ESHAPE (sizes, strides, n_tokens * H over 2^31 - 1), EALIGN, EHIP. */
int ecco_kv_append_paged(const ecco_model* mk, const ecco_model* mv, const uint16_t* k_new, const uint16_t* v_new, int64_t k_stride, int64_t v_stride,
                         void* k_blocks, uint32_t* k_meta, void* v_blocks, uint32_t* v_meta,
                         const int32_t* slots, int n_tokens, int H, int n_pages, int page_tokens, void* stream);
int ecco_kv_append_paged_minmax(const ecco_model* mk, const ecco_model* mv, const uint16_t* k_new, const uint16_t* v_new, int64_t k_stride, int64_t v_stride,
                                void* k_blocks, uint32_t* k_meta, void* v_blocks, uint32_t* v_meta,
                                const int32_t* slots, int n_tokens, int H, int n_pages, int page_tokens, void* stream);

/* Attention of a step's new tokens over their sequences' pages (append first: a token sees itself).  With n rows and kv = kv_len[b]
 * tokens, row i of sequence b stands at position kv - n + i and sees the tokens 0 .. kv - n + i; scores q.K_t / sqrt(128), softmax, sum of
 * p_t V_t.  Rows before position 0, and rows that see no page of the pool, are zeros; a token whose page is none of the pool's is
 * not seen.  Slots behind kv may be uninitialised, rows behind the last sequence's are neither read nor written.
 *   q          device, 16-byte aligned: row i at q + i * q_stride, [Hq][128] FP16; q_stride a multiple of 8, at least Hq * 128
 *   out        device, [n_tokens][Hq][128], 16-byte aligned, FP32, or FP16 if out_half is 1
 *   page_table, q_start, kv_len   as ecco_kv_pages_take leaves them;  Hq % Hkv == 0, Hq / Hkv <= 16
 *   max_new, max_kv, total_kv     at least the most rows of a sequence, the most tokens of one, and the tokens of all of them together:
 *              they size the launches and the workspace.  Where the device's lengths exceed them, rows of out are left
 *              unwritten or see too little; nothing out of range is touched.
 *   workspace  device, 256-byte aligned, workspace_bytes >= ecco_kv_attend_paged_workspace(...) of the same sizes on the models' device,
 *              contents irrelevant before and after.  Calls that share one must not overlap; null if 0 bytes are asked for.
 * Sequences with few rows per key/value head (n * Hq / Hkv up to 32; beside longer ones, a token) are decoded on the way into the products; those with
 * more are decoded into the workspace, as operands of the matrix cores, and then read by all their rows.  The softmax's sums are FP32; its weights
 * enter the second product as two FP16 numbers (22 bits), or as one (11 bits) where out is FP16 and the sequence has many rows.  They are scaled so that
 * the largest is at FP16's top: whatever its size, a weight is off by 2^-40 of the largest at the most (few rows) or 2^-36 (many), or by its last bit.  The
 * same call gives the same bits; other bounds may cut the sums elsewhere.
 * A query that is not finite makes its own outputs NaN (zeros, if all its scores are minus infinity), and no others.
 * A block with a scale that is not finite (never written by the encoder) makes all rows of its sequence unspecified.
 * The workspace never shrinks when n_tokens, B, max_new, max_kv or total_kv grows: one for a program's largest step serves all of them.  What it
 * holds where max_new * Hq / Hkv is above 32 are mainly operands, 512 bytes per token and key/value head -- of min(total_kv, s * max_kv) tokens, s being the sequences
 * that may have more rows than a token: min(B, n_tokens / 2), also where most of them bring a token each -- and up to 34 MB of parts (256 compute units).
 * Where that is too much, a step's chunks and its single tokens can be two calls, each with the table's, q_start's and kv_len's entries of its own sequences and
 * their bounds, over the same q and out.
 * With fewer rows it is parts alone: at most 520 bytes for each of 32 rows, and of twice the compute units and one per sequence and head, if there are
 * fewer of these than compute units; 0 for sequences of up to 256 tokens.
 * Errors: EINVAL (also a workspace too small), ESHAPE, EALIGN, EHIP.  n_tokens == 0 is a no-op, also with 0 sequences and bounds of 0; with rows
 * all of these are at least 1. */
size_t ecco_kv_attend_paged_workspace(int device, int n_tokens, int B, int Hq, int Hkv, int max_new, int max_kv, int64_t total_kv);
int ecco_kv_attend_paged(const ecco_model* mk, const ecco_model* mv, const uint16_t* q, int64_t q_stride,
                         const void* k_blocks, const uint32_t* k_meta, const void* v_blocks, const uint32_t* v_meta,
                         const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len,
                         int n_tokens, int B, int Hq, int Hkv, int n_pages, int page_tokens, int max_pages,
                         int max_new, int max_kv, int64_t total_kv, void* workspace, size_t workspace_bytes,
                         void* out, int out_half, void* stream);

#ifdef __cplusplus
}
#endif
#endif
