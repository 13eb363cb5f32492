/* C ABI of the paged cache of keys and values in 4 bits, and of the attention over it, on gfx950 (MI355X).
 *
 * A cache is one buffer of bytes [pages][heads][page_size][d + d/16] (device, 16-byte aligned): page_size a power of two
 * from 16 to 65536, d 64 or 128.  A slot is page * page_size + place in the page.  For one head, the 16 tokens
 * from a place that divides by 16 have their 16 * (d + d/16) bytes together:
 *     8d   codes of the keys    [token][channel / 2]
 *     8d   codes of the values  [token / 4][channel / (d/16)][token % 4][channel % (d/16) / 2]
 *     d/2  scales of the keys   [token][channel / 32]
 *     d/2  scales of the values [token / 4][channel / 32][token % 4]
 * A byte of codes holds an even channel in its low half, the next channel in its high half.  A code is a sign (8) and an index
 * into 0, 0.5, 1, 1.5, 2, 3, 4, 6; a byte b of scales stands for 2^(b - 127), 255 for NaN.  The cache holds no state
 * beside these bytes: a copy of a page is a page.
 *
 * 32 channels of a token share a scale: with M their largest magnitude, 2^e is the power of two for which
 * M / 2^e lies in (3.5, 7], e limited to -23 .. 13; each x / 2^e is rounded to the nearest code, ties to the even index, and magnitudes over 6 become 6.
 * So a value is off by at most 1/5 of M where 2^-21.2 <= M <= 57344, and every value of the cache is exact in both binary16 and
 * bfloat16.  Larger values become 49152.  32 channels that hold an infinity or a NaN become NaN.
 *
 * General rules (those of attn.h): device pointers are the caller's, nothing is allocated, cleared or waited for, calls are asynchronous
 * on `stream` and may be recorded into a graph; KV4_OK or a negative error comes back.  On KV4_EINVAL and KV4_EUNSUPPORTED nothing has been
 * enqueued.  After KV4_ELAUNCH the first of kv4_attn's two kernels may have been: its memory is in use until the
 * stream has run, and what it writes is undefined.  No C++ exception crosses this boundary.  dtype: KV4_F16 or KV4_BF16 for all 16-bit elements of a call.
 * Indices (slots, positions, tables, lengths) are read on the device and may change between replays of a graph.
 */
#ifndef PAPER_2403_16863_AMD_KV4_H
#define PAPER_2403_16863_AMD_KV4_H

#ifdef __cplusplus
extern "C" {
#endif

enum { KV4_F16 = 0, KV4_BF16 = 1 };

enum {
    KV4_OK = 0,
    KV4_EINVAL = -1,       /* null, misaligned or overlapping pointer, bad size, stride, dtype or scale */
    KV4_EUNSUPPORTED = -2, /* head_dim other than 64 or 128; sizes beyond the limits below */
    KV4_ELAUNCH = -3       /* the HIP runtime refused a launch */
};

/* Appends: for every token t with 0 <= slots[t] < pages * page_size and every head, k[t] rotated by its position and v[t] go into the
 * cache's slot.  Other tokens (padding) are left out; no other byte of the cache is touched.  The slots of one call
 * have to differ: of two tokens with one slot, parts of both may be held there.
 *
 *  k, v      : device, elements of `dtype`: token t, head h at t * token_stride + h * head_stride (strides in elements, multiples of
 *              8, k's and v's own), d contiguous; 16-byte aligned.
 *  slots     : device, int32 [T].
 *  cos, sin  : device, fp32 [rows, d/2], 16-byte aligned, or both null: no rotation.  positions: device, int32 [T]; a
 *              position outside 0 .. rows-1 makes the key NaN.  Pair i of a head, channels i and i + d/2 (interleaved != 0: 2i and 2i + 1):
 *                  (a, b) -> (a c - b s, b c + a s)
 *              in fp32, each product and each sum rounded, and from there to 4 bits: the codes are the same as
 *              from these elementary operations.
 *  Limits (KV4_EUNSUPPORTED): T * heads * d < 2^36 (T rounded up to a multiple of 16), pages * page_size <= 2^31 - 1. */
int kv4_append(const void* k, long long k_token_stride, long long k_head_stride, const void* v, long long v_token_stride,
               long long v_head_stride, void* cache, const int* slots, const float* cos, const float* sin, const int* positions,
               int rows, int interleaved, int T, int heads, int d, int pages, int page_size, int dtype, void* stream);

/* The values that the cache holds in the given slots: k, v (device, [T, heads, d] contiguous, 16-byte aligned) <- slot slots[t]
 * of every head, exact in `dtype`; zeros for a slot outside the cache.  Either of k and v may be null; they overlap neither each other
 * nor the cache. */
int kv4_read(const void* cache, const int* slots, void* k, void* v, int T, int heads, int d, int pages, int page_size, int dtype,
             void* stream);

/* Attention over the cache.  Sequence b has lens[b] keys, key j in page tables[b * width + j / page_size], and the queries
 * cu_q[b] .. cu_q[b + 1] - 1 of q; query head a uses the cache's head a / (H / heads).  For query i of n of a sequence with L keys, over the visible
 * keys j (all; causal != 0: j <= L - n + i, so that the last query sees the last key):
 *     x_j = scale * q . k_j,   lse = ln sum_j exp(x_j),   out = sum_j exp(x_j - lse) v_j
 * A row that sees no key gets out = 0 and lse = -infinity.
 *
 *  q, out : device, [T, H, d] contiguous, 16-byte aligned; lse: device, fp32 [T, H].  out, lse and the workspace overlap nothing.  Rows of q before cu_q[0]
 *           and from cu_q[B] on belong to nobody: their out and lse stay as they are.
 *  tables : device, int32 [B, width].  Only the entries of pages that hold keys below lens[b] are read; keys of an entry outside
 *           0 .. pages-1 are not seen.  lens: device, int32 [B]; counts above width * page_size are taken as that, negative ones as 0.
 *  cu_q   : device, int32 [B + 1], not decreasing, within 0 .. T, no sequence with more than max_q queries (what exceeds
 *           that is not computed); or null: T / B queries for every sequence, T a multiple of B.
 *  max_q  : the largest number of queries of a sequence (cu_q null: T / B); an upper bound will do, but costs workgroups.
 *  workspace : device, 16-byte aligned, kv4_attn_workspace bytes (8 T H, and 9 to 69 MB whatever the sequences), any contents, not used by anybody else until the call's
 *           kernels have run; null or fewer bytes: each workgroup goes over all keys of its rows, which is slower for few
 *           long sequences or unequal ones.
 *  Limits (KV4_EUNSUPPORTED): pages * page_size <= 2^31 - 1, pages * heads * page_size < 2^36, width * page_size <= 2^31 - 2^16, T * H <= 2^31 - 1, H / heads * max_q <= 2^30,
 *           B <= 65535, fewer than 2^23 workgroups (16 to 256 rows of a sequence and head each), and these times width * page_size / 32 below 2^31 where
 *           there is a use for a workspace.
 *
 * Accuracy: products of 16-bit values and of the cache's values in fp32 (bfloat16 queries become binary16 relative to the row's largest: elements
 * below 2^-17 of it lose bits, below 2^-25 all), the probabilities are rounded to binary16 before the second product, and out once at the end.
 * |out - exact| <= u |out| + 2^-11 sum_j p_j |v_j| + 2^-32 max_j p_j sum_j |v_j| + small fp32 terms, u = 2^-11 or 2^-8 (binary16 has steps of
 * 2^-24, and the largest p_j is held as 2^7 or more).  The order of all sums is fixed by the arguments and the contents of lens and cu_q: results do
 * not change from run to run.
 * NaN: a query with a NaN or an infinity has NaN rows, and so has one that sees a key with a NaN; rows with a score beyond 2^126, and bfloat16 rows whose largest
 * element times |scale| passes 2^141, may be NaN.  A NaN among the values that a row
 * sees makes the 32 channels NaN that it stands in, and may make the whole row NaN; it never enters a row that does not see it. */
int kv4_attn(const void* q, const void* cache, const int* tables, const int* lens, const int* cu_q, void* out, float* lse, int T,
             int B, int H, int heads, int d, int pages, int page_size, int width, int max_q, int causal, float scale, int dtype,
             void* workspace, long long workspace_bytes, void* stream);

/* The bytes of scratch memory that kv4_attn has a use for (0: none); negative: the error that the call would give. */
long long kv4_attn_workspace(int T, int B, int H, int heads, int d, int page_size, int width, int max_q);

const char* kv4_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif
