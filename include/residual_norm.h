/* C ABI of the norms behind a block and ahead of the next with the residual stream's update between them, forward and backward, on
 * gfx950 (MI355X).
 *
 * For every token, with the block's result h, the stream x and the channels' vectors in R^C:
 *     u = post_weight h r(h)   (without a post_weight: u = h),
 *     y = alpha x + gate u     (without a gate: 1; without h: y = x),
 *     z = pre_weight y r(y),                          r(v) = (mean_i v_i^2 + eps)^(-1/2)
 * in fp32; y and z are rounded once each, z from the unrounded y.  Backward, from the gradients dy and dz of both (dy: what comes back along the stream):
 *     D = dy + r (p - n mean_i(p_i n_i))     with r = r(y), n = y r, p = dz pre_weight,
 *     dx = alpha D,   dgate = sum over the gate's tokens of D u,   dpre_weight = sum over all tokens of dz n,
 *     g = D gate, without a post_weight dh = g; else with r = r(h), n = h r, p = g post_weight:
 *     dh = r (p - n mean_i(p_i n_i)),   dpost_weight = sum over all tokens of g n.
 * (Squares are fp32: a token with values beyond 1e18 has r = 0, and with eps = 0 one of values below 1e-19 has r = infinity.)
 *
 * General rules (those of attn.h): device pointers are the caller's, nothing is allocated, cleared or waited for, calls are asynchronous
 * on `stream` and may be recorded into a graph; NORM_OK or a negative error comes back.  On NORM_EINVAL and NORM_EUNSUPPORTED nothing has been
 * enqueued.  After NORM_ELAUNCH the first of residual_norm_bwd's two kernels may have been: its memory is in use until the
 * stream has run, and what it writes is undefined.  No C++ exception crosses this boundary.
 */
#ifndef PAPER_2403_16863_AMD_RESIDUAL_NORM_H
#define PAPER_2403_16863_AMD_RESIDUAL_NORM_H

#ifdef __cplusplus
extern "C" {
#endif

enum { NORM_F16 = 0, NORM_BF16 = 1 };

enum {
    NORM_OK = 0,
    NORM_EINVAL = -1,       /* null or misaligned pointer, an output over another tensor, bad size, stride, dtype, alpha or eps, no workspace */
    NORM_EUNSUPPORTED = -2, /* C no multiple of 8 or beyond 16384; more than 2^31 - 1 tokens */
    NORM_ELAUNCH = -3       /* the HIP runtime refused a launch */
};

/* A tensor of tokens: token n of sequence b at data + b * batch_stride + n * token_stride (in elements), its C channels on end.  data is aligned to 16 bytes
 * and the strides divide by 8 (a stride of a size of 1 is not looked at).  The tokens of what is written do not overlap each other.  data null: left out. */
typedef struct {
    void* data;
    long long batch_stride, token_stride;
} norm_tokens;

/* The vectors of a call. */
typedef struct {
    const void* gate;          /* [C], or with gate_stride > 0 a row of C for each sequence, gate_stride elements apart (a multiple of 8, at least C); null: none */
    long long gate_stride;
    int gate_f32;              /* fp32, else `dtype` */
    const void* post_weight;   /* [C] or null */
    const void* pre_weight;    /* [C], goes with z and dz */
    int weight_f32;            /* both weights are fp32, else `dtype` */
    float alpha, eps;          /* finite; eps >= 0 */
} norm_vectors;                /* all pointers 16-byte aligned, device */

/* y, z <- as above.  x is needed.  h left out: y = x, no gate, post_weight or alpha other than 1, and y is left out too.  y or z may be left out, not both.
 * An output may be an input's own memory with the same strides (y that of x, for one); otherwise outputs overlap nothing. */
int residual_norm(const norm_tokens* x, const norm_tokens* h, const norm_tokens* y, const norm_tokens* z, const norm_vectors* vectors, int B,
                  int N, int C, int dtype, void* stream);

/* dx, dh and the vectors' gradients, from dy and dz (one may be left out) and the forward's y (needed with dz; without h it is x) and h (needed with a gate or
 * post_weight).
 *  dx, dh : either may be left out, but not both; dh needs alpha's, the gate's and the weights' values as the forward had them.
 *  dgate  : fp32, [C] or, with a gate_stride, [B, C] on end;  dpost_weight, dpre_weight: fp32 [C]; 16-byte aligned, written, not added to.  Each may be
 *           null; one whose vector (or dz) is left out has to be.
 *  workspace : device, 16-byte aligned, residual_norm_bwd_workspace bytes where one of the three is asked for, any contents, not used by anybody
 *              else until the call's kernels have run.
 * An output may be an input's own memory with the same strides (dx that of dy, for one).  The order of all sums is fixed by the sizes: results do not
 * change from run to run. */
int residual_norm_bwd(const norm_tokens* dy, const norm_tokens* dz, const norm_tokens* y, const norm_tokens* h, const norm_tokens* dx,
                      const norm_tokens* dh, const norm_vectors* vectors, float* dgate, float* dpost_weight, float* dpre_weight, int B, int N,
                      int C, int dtype, void* workspace, long long workspace_bytes, void* stream);

/* Bytes for B sequences of N tokens; by_sequence: the gate is one for each sequence.  Negative: the error that the call would give. */
long long residual_norm_bwd_workspace(int B, int N, int C, int by_sequence);

const char* norm_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif
