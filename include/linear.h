/* C ABI of the matrix product with bias, activation and residual in its epilogue, and its backward pass, on gfx950 (MI355X): what a
 * model's linear layers are (gemm_lrelu.h has the product with a leaky ReLU alone).
 *
 *     pre = x w + bias,      out = act(pre) + residual           x [M, K], w [K, N], bias [N], the others [M, N]
 *     act: none, relu max(z, 0), silu z / (1 + e^-z), gelu z (1 + erf(z / sqrt 2)) / 2,
 *          gelu_tanh z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2
 * and from out's gradient dy, with dz = dy act'(pre) (relu'(0) = 0):
 *     dx = dz w^T,   dw = x^T dz,   dbias = sum over rows of dz.           (The residual's gradient is dy itself.)
 * Elements are 16 bits, binary16 or bfloat16, the same for all matrices; products are summed in fp32, the epilogue is fp32, and
 * out and pre are rounded once, to nearest even.  The activation is of the unrounded pre.  Where there is an activation, dz is rounded to the matrices' type ahead of
 * both products, which read it several times (binary16: a dz below 2^-14 loses digits, and one beyond 65504 is infinite); dbias adds the unrounded dz in fp32.
 *
 * General rules (those of attn.h): device pointers are the caller's, nothing is allocated, cleared or waited for, calls are asynchronous
 * on `stream` and may be recorded into a graph; LINEAR_OK or a negative error comes back.  On LINEAR_EINVAL and LINEAR_EUNSUPPORTED nothing has
 * been enqueued.  After LINEAR_ELAUNCH earlier kernels of the call may have been: its memory is in use until the stream has run, and what
 * it writes is undefined.  No C++ exception crosses this boundary.  The order of all sums is fixed by the sizes, the layouts of w and dw and whether there is a
 * workspace: results do not change from run to run.
 */
#ifndef PAPER_2403_16863_AMD_LINEAR_H
#define PAPER_2403_16863_AMD_LINEAR_H

#ifdef __cplusplus
extern "C" {
#endif

enum { LINEAR_F16 = 0, LINEAR_BF16 = 1 };

enum { LINEAR_NONE = 0, LINEAR_RELU = 1, LINEAR_SILU = 2, LINEAR_GELU = 3, LINEAR_GELU_TANH = 4 };

enum {
    LINEAR_OK = 0,
    LINEAR_EINVAL = -1,       /* null, misaligned or overlapping pointer, bad size, stride, dtype or activation */
    LINEAR_EUNSUPPORTED = -2, /* N, K or a stride beyond 2^22, M beyond 2^30, more tiles than a launch holds */
    LINEAR_ELAUNCH = -3,      /* the HIP runtime refused a launch */
    LINEAR_ENOMEM = -4        /* gemm_linear_bwd without a workspace of the bytes that it needs; nothing has been enqueued */
};

/* A matrix: row r begins at data + r * stride (in elements), its columns lie on end.  data is aligned to 16 bytes, stride divides by 8 and is no
 * less than a row (the stride of a single row is not looked at).  Slices of the columns of a wider matrix will do.  data null: left out. */
typedef struct {
    void* data;
    long long stride;
} linear_rows;

/* out, pre <- as above.
 *  M >= 1 (any); N, K : multiples of 8, from 8 on.
 *  w        : w_rows_of_n == 0: K rows of N; else N rows of K, one for each output.
 *  bias     : [N], 16-byte aligned, fp32 (bias_f32 != 0) or `dtype`, or null.
 *  residual : may be left out, and may be out's own memory with the same stride.  pre: may be left out (null too).
 *  out and pre overlap nothing else.
 *  workspace: device, 16-byte aligned, any contents, not used by anybody else until the call's kernels have run.  With gemm_linear_workspace bytes
 *             (0: none wanted) few tiles split a long K among them; null or fewer: they do not. */
int gemm_linear(const linear_rows* x, const linear_rows* w, int w_rows_of_n, const void* bias, int bias_f32, const linear_rows* residual,
                const linear_rows* pre, const linear_rows* out, int activation, int M, int N, int K, int dtype, void* workspace,
                long long workspace_bytes, void* stream);

/* The same for callers that take the memory call by call, with one look at the sizes: `scratch` is called at most once, with `owner` and the
 * bytes, after the other arguments have been checked and only where there are any.  It returns memory as above or null (none), and must not throw. */
typedef void* (*linear_scratch_fn)(void* owner, long long bytes);
int gemm_linear_with(const linear_rows* x, const linear_rows* w, int w_rows_of_n, const void* bias, int bias_f32, const linear_rows* residual,
                     const linear_rows* pre, const linear_rows* out, int activation, int M, int N, int K, int dtype, linear_scratch_fn scratch,
                     void* owner, void* stream);

/* Bytes that the sizes ask for (at most 64 MiB); negative: the error that the call would give. */
long long gemm_linear_workspace(int M, int N, int K, int w_rows_of_n);

/* dx, dw, dbias <- gradients; each may be left out, not all three.
 *  pre : the forward's, needed with an activation (and not looked at without one).
 *  x   : needed for dw.  w: needed for dx.  dw has a layout of its own (dw_rows_of_n), as w has.
 *  dbias : fp32 [N], 16-byte aligned, written (not added to).
 *  dx, dw and dbias overlap nothing.
 *  workspace : gemm_linear_bwd_workspace bytes for the gradients that are given; null or fewer are refused (LINEAR_ENOMEM) unless it is 0. */
int gemm_linear_bwd(const linear_rows* dy, const linear_rows* x, const linear_rows* w, int w_rows_of_n, const linear_rows* pre,
                    const linear_rows* dx, const linear_rows* dw, int dw_rows_of_n, float* dbias, int activation, int M, int N, int K,
                    int dtype, void* workspace, long long workspace_bytes, void* stream);

int gemm_linear_bwd_with(const linear_rows* dy, const linear_rows* x, const linear_rows* w, int w_rows_of_n, const linear_rows* pre,
                         const linear_rows* dx, const linear_rows* dw, int dw_rows_of_n, float* dbias, int activation, int M, int N, int K,
                         int dtype, linear_scratch_fn scratch, void* owner, void* stream);

/* dx, dw, dbias: whether that gradient is asked for. */
long long gemm_linear_bwd_workspace(int M, int N, int K, int w_rows_of_n, int dw_rows_of_n, int activation, int dx, int dw, int dbias);

/* One product c [M, N] = a b on tile `tile` in [0, linear_num_tiles()) with k in `ranges` parts: for tests and measurement of what the
 * calls above choose from.  layout 0: a is M rows of K, b K rows of N (both of the forward's forms begin with it);  1: b is N rows of K;  2: a is K rows of
 * M, b K rows of N (the weight's gradient, K any).  ranges > 1: workspace of ranges * M * N floats. */
int linear_product(const linear_rows* a, const linear_rows* b, int layout, const linear_rows* c, int M, int N, int K, int dtype, int tile,
                   int ranges, void* workspace, long long workspace_bytes, void* stream);
int linear_num_tiles(void);
/* What the calls choose for a product (host logic): its tile, and the ranges of k where there is a workspace. */
int linear_choice(int M, int N, int K, int layout, int* tile, int* ranges);

const char* linear_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif
