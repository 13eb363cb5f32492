/* C ABI of the norms of queries and keys with the position rotation, forward and backward, on gfx950 (MI355X): what stands between a
 * layer's projections and attn_fwd (attn.h), or the cache and its attention (kv4.h).
 *
 * For every token and head, x in R^d, with the tensor's weight w (none: n = x) and the cosines c and sines s of the
 * token's position:
 *     r = (mean_i x_i^2 + eps)^(-1/2),   n = r x w,
 *     pair p, channels (i, j) = (p, p + d/2), interleaved != 0: (2p, 2p + 1):   y_i = n_i c_p - n_j s_p,   y_j = n_j c_p + n_i s_p
 * in fp32, rounded once (squares too: a head with values beyond 1e18 has r = 0, and with eps = 0 one of values below 1e-19 has r = infinity).  Backward, from dy: with g the gradient turned back, h = g w:
 *     dw = sum over tokens and heads of g r x,      dx = r (h - r x mean_i(h_i r x_i)),      without a weight dx = g.
 *
 * General rules (those of attn.h): device pointers are the caller's, nothing is allocated, cleared or waited for, calls are asynchronous
 * on `stream` and may be recorded into a graph; QK_OK or a negative error comes back.  On QK_EINVAL and QK_EUNSUPPORTED nothing has been
 * enqueued.  After QK_ELAUNCH the first of qk_norm_rope_bwd's two kernels may have been: its memory is in use until the
 * stream has run, and what it writes is undefined.  No C++ exception crosses this boundary.
 */
#ifndef PAPER_2403_16863_AMD_QK_ROPE_H
#define PAPER_2403_16863_AMD_QK_ROPE_H

#ifdef __cplusplus
extern "C" {
#endif

enum { QK_F16 = 0, QK_BF16 = 1 };

enum {
    QK_OK = 0,
    QK_EINVAL = -1,       /* null or misaligned pointer, an output over another tensor, bad size, stride, dtype or eps, no workspace */
    QK_EUNSUPPORTED = -2, /* head_dim other than 64 or 128; B * N * heads beyond 2^31 - 1 */
    QK_ELAUNCH = -3       /* the HIP runtime refused a launch */
};

/* A tensor of heads: token n of sequence b, head h at data + b * batch_stride + n * token_stride + h * head_stride (in elements), its d
 * channels on end.  data is aligned to 16 bytes and the strides divide by 8 (a stride of a size of 1 is not looked at), so
 * slices of a joint projection and both [B,N,H,d] and [B,H,N,d] will do; what is
 * written has no stride of 0.  data null: the tensor is left out. */
typedef struct {
    void* data;
    long long batch_stride, token_stride, head_stride;
} qk_heads;

/* q_out, k_out <- norm and rotation of q, k (either pair may be left out).
 *  q, q_out : H heads; k, k_out: Hkv heads; elements of `dtype`.  An output may be its input's own memory with
 *             the same strides; otherwise outputs overlap nothing.
 *  q_weight, k_weight : device, [d], 16-byte aligned, fp32 (weight_f32 != 0) or `dtype`; null: no norm for that tensor.
 *  cos, sin : device, fp32 [rows, d/2], 16-byte aligned.  positions: device, int32 [B, N]; a position outside 0 .. rows-1 makes
 *             the token's outputs (backward: gradients) NaN.
 *  eps      : >= 0 and finite. */
int qk_norm_rope(const qk_heads* q, const qk_heads* k, const qk_heads* q_out, const qk_heads* k_out, const void* q_weight,
                 const void* k_weight, int weight_f32, const float* cos, const float* sin, const int* positions, int rows, float eps,
                 int interleaved, int B, int N, int H, int Hkv, int d, int dtype, void* stream);

/* dq, dk, dq_weight, dk_weight <- gradients, from dq_out, dk_out and the forward's q, k.  A tensor without a weight needs no q (k)
 * and has no weight gradient.
 *  dq_weight, dk_weight : device, fp32 [d], written (not added to); one for each weight.
 *  workspace : needed where there is a weight: device, 16-byte aligned, qk_norm_rope_bwd_workspace bytes, any contents, not used by
 *              anybody else until the call's kernels have run.
 * dq may be dq_out's own memory with the same strides.  The order of all sums is fixed by the sizes: results do not change from run to run. */
int qk_norm_rope_bwd(const qk_heads* dq_out, const qk_heads* dk_out, const qk_heads* q, const qk_heads* k, const qk_heads* dq,
                     const qk_heads* dk, const void* q_weight, const void* k_weight, int weight_f32, float* dq_weight,
                     float* dk_weight, const float* cos, const float* sin, const int* positions, int rows, float eps, int interleaved,
                     int B, int N, int H, int Hkv, int d, int dtype, void* workspace, long long workspace_bytes, void* stream);

/* Bytes for B sequences of N tokens; negative: the error that the call would give. */
long long qk_norm_rope_bwd_workspace(int B, int N, int H, int Hkv, int d);

const char* qk_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif
