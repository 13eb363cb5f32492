// Host side of the linear layers' products (include/linear.h): checks, choice of the tile, launches; and the small kernels around
// the products of linear_kernel.h: the joining of parts, and the activation's backward step.
#include "../../include/linear.h"

#include <limits.h>

#include "linear_tiles.h"
#include "memory_check.h"

namespace linear {

// C from the parts of the ranges of k, in range order, with the epilogue; a thread for eight consecutive elements.
template <class T>
__global__ __launch_bounds__(64) void join_kernel(const float* parts, Args p, int ranges, unsigned chunks) {
    const unsigned i = blockIdx.x * 64 + threadIdx.x;
    if (i >= chunks) return;
    const unsigned row = (unsigned)p.N / 8, m = i / row, n = (i - m * row) * 8;
    float bias[8];
    load_bias<T, 8>(p.e, (int)n, true, bias);
    const u32x4 residual = load_residual<8>(p.e, (int)m, (int)n, true);
    const f32x4* src = reinterpret_cast<const f32x4*>(parts) + (size_t)i * 2;
    f32x4 x = src[0], y = src[1];
#pragma unroll 4
    for (int r = 1; r < ranges; ++r) {
        src += (size_t)chunks * 2;
        x += src[0];
        y += src[1];
    }
    float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    finish<T, 8>(p.e, (uint16_t*)p.out, p.ldo, (int)m, (int)n, v, bias, residual);
}

// dz = dy act'(pre), rounded, and the rows' sums for dbias, in one pass over dy and pre: memory binds.  A workgroup has 256 / lanes rows of `lanes` vectors of 8
// columns (a power of two, 64 at most) and goes through a chunk of the rows; its sums meet in LDS in a fixed order.
// dz is held in the matrices' 16 bits: products of 32 bits run at a fifteenth of the rate, and dz in two parts of 16 bits would be both products twice.
// The gradients' error against 64 bits is 1.4 times that of the result's own rounding for it (2.3e-3 in bfloat16, 2.9e-4 in binary16).
struct SlopeArgs {
    const uint16_t *dy, *pre;
    uint16_t* dz;
    float* sums;  // [chunk][N] (one chunk: dbias itself), or null
    long long lddy, ldpre;
    int M, N, rows, lanes, act;
};

template <class T>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a) {
    __shared__ float part[256 * 9];
    const int lane = threadIdx.x % a.lanes, at = threadIdx.x / a.lanes, step = 256 / a.lanes;
    const int n = (blockIdx.x * a.lanes + lane) * 8;
    const long long first = (long long)blockIdx.y * a.rows, end = min((long long)a.M, first + a.rows);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (n < a.N) {
        const uint16_t *dy = a.dy + n, *pre = a.pre + n;
        constexpr int AT_ONCE = 2;  // rows whose loads are in flight together
        for (long long m0 = first + at; m0 < end; m0 += AT_ONCE * step) {
            u32x4 gr[AT_ONCE], vr[AT_ONCE];
#pragma unroll
            for (int r = 0; r < AT_ONCE; ++r) {
                const long long m = m0 + r * step;
                gr[r] = vr[r] = u32x4{0, 0, 0, 0};
                if (m < end) gr[r] = *(const u32x4*)(dy + m * a.lddy);
                if (m < end && a.act) vr[r] = *(const u32x4*)(pre + m * a.ldpre);
            }
#pragma unroll
            for (int r = 0; r < AT_ONCE; ++r) {
                const long long m = m0 + r * step;
                float g[8], v[8];
                unpack<T, 8>(gr[r], g);
                if (a.act) {
                    unpack<T, 8>(vr[r], v);
                    act_slope8(v, g, a.act);
                    if (a.dz && m < end) *(u32x4*)(a.dz + m * a.N + n) = pack<T, 8>(g);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += g[i];
            }
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[threadIdx.x * 9 + i] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.lanes * 8; c += 256) {
        float t = 0;
        for (int r = 0; r < step; ++r) t += part[(r * a.lanes + c / 8) * 9 + c % 8];
        const int column = blockIdx.x * a.lanes * 8 + c;
        if (column < a.N) a.sums[(size_t)blockIdx.y * a.N + column] = t;
    }
}

// dbias from the chunks' sums: 32 columns a workgroup, 32 threads to a column, so that 128 chunks are four loads to a thread.
__global__ __launch_bounds__(1024) void bias_kernel(const float* sums, int chunks, int N, float* dbias) {
    __shared__ float part[1024];
    const int c = blockIdx.x * 32 + threadIdx.x % 32;
    float t = 0;
    if (c < N) {
#pragma unroll 4
        for (int i = threadIdx.x / 32; i < chunks; i += 32) t += sums[(size_t)i * N + c];
    }
    part[threadIdx.x] = t;
#pragma unroll
    for (int n = 512; n >= 32; n /= 2) {
        __syncthreads();
        if (threadIdx.x < n) part[threadIdx.x] += part[threadIdx.x + n];
    }
    if (threadIdx.x < 32 && c < N) dbias[c] = part[threadIdx.x];
}

// ---- choice of the tile.  With n tiles on the busiest of the 256 units, and f of the units' n rounds filled, a product takes about
//     ceil(K / kstage) * max(ceil(n / occ) * alone, n * full) * (1 + load * f) * (1 + off_a) * (1 + off_b) * (1 + tokens) * (1 + by_k) + n * ends + base + MB of C * out    (us)
// (load: what the units take from each other; off_a, off_b: where rows of A, of B do not all begin on a line of 128 bytes; tokens, by_k: where A, B lie by rows of k, and are read
// by the transposing reads, and in short pieces of a row by narrow tiles; ends: prologue and epilogue of a tile; out: the result's way to memory) and in ranges of k, whose MB of C are those of all parts in 32 bits,
// a second launch and their reading in addition.  Fitted to the times of 12437 drawn products, M 1 .. 8192, N, K 8 .. 16384 and up to 3e11 multiplications, in the three
// layouts, each on the tiles that could be its best and up to ten numbers of ranges, three sets of buffers in turn.  The standard deviation of time over model is 9 to 13 % by
// tile; what the model chooses takes 2.0 % longer than the best that was measured (geometric mean; 12 % in the worst twentieth).  Each tile but the 64 x 64, without
// which it is 4 %, is worth up to 1.4 % of that mean, and 10 to 15 % in its own range (779 x 1408 x 3904: 96 x 64 tiles on eight waves 17.6 us, the next best 21.0; 4 rows, 8192 -> 2048, k
// along both: 16 x 16 tiles 8.5, the next best 10.4).
// Tiles of 64 x 128, 32 x 64 with k split four ways and 16 x 128 were built and gave nothing, and neither did rings of one stage more, up to the whole LDS.
struct Shape {
    int bm, bn, bk, wk, threads, occ;
    float alone, full, load, ends, off_a, off_b, tokens, base, out, by_k;
};
template <int I>
constexpr Shape shape(float alone, float full, float load, float ends, float off_a, float off_b, float tokens, float base, float out, float by_k) {
    using T = TileOf<I>;
    return {T::BM, T::BN, T::BK, T::WK, T::WM * T::WN * T::WK * 64, T::OCC, alone, full, load, ends, off_a, off_b, tokens, base, out, by_k};
}
static constexpr Shape kShapes[kTiles] = {
    shape<0>(0.338f, 0.109f, 1.643f, 1.297f, 0.012f, 0.117f, 0.062f, 2.175f, 0.220f, 0.371f),
    shape<1>(0.294f, 0.168f, 1.984f, 0.775f, 0.008f, 0.226f, 0.050f, 2.447f, 0.411f, 0.103f),
    shape<2>(0.203f, 0.204f, 1.249f, 0.357f, 0.025f, 0.092f, -0.054f, 2.817f, 0.181f, 0.125f),
    shape<3>(0.171f, 0.195f, 0.342f, 0.036f, 0.052f, 0.048f, -0.043f, 2.946f, 0.207f, 0.042f),
    shape<4>(0.231f, 0.110f, 0.916f, 1.495f, 0.069f, 0.106f, 0.034f, 2.179f, 0.315f, 0.131f),
    shape<5>(0.296f, 0.144f, 0.779f, 1.804f, 0.047f, 0.081f, 0.169f, 2.175f, 0.321f, 0.085f),
    shape<6>(0.227f, 0.202f, 0.589f, 0.000f, 0.085f, 0.065f, 0.024f, 3.299f, 0.250f, 0.031f),
    shape<7>(0.325f, 0.176f, 0.660f, 0.803f, 0.065f, 0.024f, 0.065f, 3.026f, 0.251f, -0.048f),
    shape<8>(0.382f, 0.293f, 0.680f, 0.545f, 0.074f, 0.032f, 0.017f, 2.967f, 0.143f, -0.010f),
    shape<9>(0.496f, 0.496f, 0.367f, 2.551f, 0.112f, 0.017f, 0.031f, 2.094f, 0.127f, -0.022f),
    shape<10>(0.602f, 0.573f, 0.455f, 3.706f, 0.077f, 0.011f, 0.009f, 1.500f, 0.092f, -0.047f),
    shape<11>(0.769f, 0.003f, 0.495f, 4.676f, 0.063f, -0.001f, -0.006f, 1.500f, 0.058f, -0.032f),
    shape<12>(0.980f, 0.145f, 0.449f, 5.520f, 0.055f, -0.007f, 0.005f, 1.500f, 0.002f, 0.009f),
    shape<13>(0.229f, 0.190f, 1.636f, 0.504f, 0.039f, 0.080f, 0.068f, 2.534f, 0.082f, 0.246f),
    shape<14>(0.226f, 0.028f, 1.295f, 1.450f, -0.011f, 0.076f, 0.156f, 1.847f, 0.189f, 0.800f)};

constexpr long long kUnits = 256, kPartBytes = 64ll << 20;
constexpr int kMostRanges = 32;

struct Plan {
    int tile, ranges, kc;
    long long bytes;  // of the parts
};

static long long tiles_of(const Shape& s, int M, int N) { return (long long)(1 + (M - 1) / s.bm) * (1 + (N - 1) / s.bn); }
static bool fits(const Shape& s, int M, int N, int ranges) { return tiles_of(s, M, N) * ranges * s.threads <= (long long)UINT_MAX; }

static Plan plan_of(int tile, int M, int N, int K, int ranges) {
    const Shape& s = kShapes[tile];
    const int step = s.bk * s.wk;
    const int kc = (int)(((long long)K + ranges - 1) / ranges + step - 1) / step * step;
    ranges = (int)(((long long)K + kc - 1) / kc);
    return {tile, ranges, kc, ranges > 1 ? 4ll * ranges * M * N : 0};
}

static float time_of(const Shape& s, long long tiles, int M, int N, const Plan& p, int K, float factor) {
    const bool parts = p.ranges > 1;
    tiles *= p.ranges;
    const int n = (int)((tiles + kUnits - 1) / kUnits), stages = (int)(((parts ? p.kc : K) + s.bk * s.wk - 1) / (s.bk * s.wk));
    const float alone = (float)((n + s.occ - 1) / s.occ) * s.alone, full = (float)n * s.full, filled = (float)tiles / ((float)n * kUnits);
    const float us = (float)stages * (alone > full ? alone : full) * (1.f + s.load * filled) * factor + (float)n * s.ends + s.base;
    const float mb = 1e-6f * (float)M * (float)N;
    return parts ? us + 2.13f + 4.f * (float)p.ranges * mb * (0.44f + s.out) : us + 2.f * mb * s.out;
}

static Plan choose(int M, int N, int K, int layout, bool memory) {
    Plan best = {-1, 1, K, 0};
    float best_us = 0;
    const bool off_a = (layout == TOKENS ? M : K) % 64, off_b = (layout == ROWS_N ? K : N) % 64;
    for (int t = 0; t < kTiles; ++t) {
        const Shape& s = kShapes[t];
        if (!fits(s, M, N, 1)) continue;
        const long long tiles = tiles_of(s, M, N);
        const float factor = (off_a ? 1.f + s.off_a : 1.f) * (off_b ? 1.f + s.off_b : 1.f) * (layout == TOKENS ? 1.f + s.tokens : 1.f) * (layout != ROWS_N ? 1.f + s.by_k : 1.f);
        for (int r : {1, 2, 3, 4, 6, 8, 12, 16, 24, kMostRanges}) {
            if (r > 1 && (!memory || tiles * r > kUnits * s.occ || (long long)r * 128 > K)) break;
            const Plan p = r > 1 ? plan_of(t, M, N, K, r) : Plan{t, 1, K, 0};
            if (p.ranges != r || p.bytes > kPartBytes) continue;
            const float us = time_of(s, tiles, M, N, p, K, factor);
            if (best.tile < 0 || us < best_us) best = p, best_us = us;
        }
    }
    return best;
}

static const void* kernel_of(int layout, int dtype, int tile, bool parts) {
    if (layout == ROWS) return dtype ? product_of<ROWS, true>(tile, parts) : product_of<ROWS, false>(tile, parts);
    if (layout == ROWS_N) return dtype ? product_of<ROWS_N, true>(tile, parts) : product_of<ROWS_N, false>(tile, parts);
    return dtype ? product_of<TOKENS, true>(tile, parts) : product_of<TOKENS, false>(tile, parts);
}

static int launch(const void* fn, dim3 grid, int threads, void** args, void* stream) {
    if (hipLaunchKernel(fn, grid, dim3(threads), args, 0, (hipStream_t)stream) == hipSuccess) return LINEAR_OK;
    (void)hipGetLastError();
    return LINEAR_ELAUNCH;
}

static int run(const Plan& plan, int layout, int dtype, Args a, void* workspace, void* stream) {
    const Shape& s = kShapes[plan.tile];
    const bool parts = plan.ranges > 1;
    Args product = a;
    product.kc = plan.kc;
    if (parts) product.out = (char*)workspace;
    void* args[] = {&product};
    const int rc = launch(kernel_of(layout, dtype, plan.tile, parts), dim3((unsigned)(tiles_of(s, a.M, a.N) * plan.ranges)), s.threads, args, stream);
    if (rc || !parts) return rc;
    const float* from = (const float*)workspace;
    int ranges = plan.ranges;
    unsigned chunks = (unsigned)((long long)a.M * a.N / 8);
    void* join[] = {&from, &a, &ranges, &chunks};
    return launch(dtype ? (const void*)join_kernel<BF16> : (const void*)join_kernel<F16>, dim3((chunks + 63) / 64), 64, join, stream);
}

// ---- checks
constexpr int kMost = 1 << 22, kMostRows = 1 << 30;

static bool given(const linear_rows* t) { return t && t->data; }

static int check_sizes(int M, int N, int K, int dtype, int activation) {
    if (M < 1 || N < 8 || K < 8 || N % 8 || K % 8 || (dtype != LINEAR_F16 && dtype != LINEAR_BF16) || activation < LINEAR_NONE ||
        activation > LINEAR_GELU_TANH)
        return LINEAR_EINVAL;
    return M > kMostRows || N > kMost || K > kMost ? LINEAR_EUNSUPPORTED : LINEAR_OK;
}

static int check_matrix(const linear_rows* t, int rows, int columns) {
    if (!given(t) || (uintptr_t)t->data % 16) return LINEAR_EINVAL;
    if (rows == 1) return LINEAR_OK;
    if (t->stride % 8 || t->stride < columns) return LINEAR_EINVAL;
    return t->stride > kMost ? LINEAR_EUNSUPPORTED : LINEAR_OK;
}

static int stride_of(const linear_rows* t, int rows, int columns) { return rows > 1 ? (int)t->stride : columns; }
static Rows2D block(const linear_rows* t, int rows, int columns) { return {given(t) ? t->data : nullptr, rows, columns, given(t) ? t->stride : 0}; }
static Rows2D vector_of(const void* p, long long bytes) { return {p, 1, bytes / 2, 0}; }

// Scratch memory of a call: the caller's, or asked for by the call once it knows how much.
struct Memory {
    void* given;
    long long bytes;
    linear_scratch_fn ask;
    void* owner;
    void* take(long long need) const { return ask ? ask(owner, need) : bytes >= need ? given : nullptr; }
};

static long long up(long long bytes) { return (bytes + 255) / 256 * 256; }

// Workgroups of the activation's backward step: 1024 where there are rows enough for them to have two passes each.  Up to four passes of rows are one chunk,
// whose sums are dbias: that spares a launch.
struct SlopeGrid {
    int lanes, blocks, rows, chunks;
};
static SlopeGrid slope_grid(int M, int N) {
    SlopeGrid g;
    g.lanes = 1;
    while (g.lanes < 64 && g.lanes * 8 < N) g.lanes *= 2;
    g.blocks = (N + g.lanes * 8 - 1) / (g.lanes * 8);
    const int pass = 256 / g.lanes;
    const long long most = (M + 2ll * pass - 1) / (2 * pass), want = g.blocks >= 1024 ? 1 : 1024 / g.blocks;
    const long long chunks = want < most ? want : most;
    const long long rows = M / chunks, whole = rows > pass ? 2ll * pass : pass;  // (a thread's two rows at once, where it has as many)
    g.rows = (int)(rows < whole ? whole : rows / whole * whole);
    if (M <= 4 * pass) g.rows = 4 * pass;
    g.chunks = (int)(((long long)M + g.rows - 1) / g.rows);
    return g;
}

struct Backward {
    Plan dx, dw;
    SlopeGrid slope;
    int dx_layout;
    long long dz, sums, parts;  // bytes
    long long total() const { return dz + sums + parts; }
};
// dx = dz w^T: of a weight of K rows both operands have the products' index, N, along their rows.  dw: the tokens are the index; the
// product is dw itself or, of N rows, its transpose.
static Backward backward_of(int M, int N, int K, int w_rows_of_n, int dw_rows_of_n, int activation, bool dx, bool dw, bool dbias) {
    Backward b = {};
    b.slope = slope_grid(M, N);
    b.dx_layout = w_rows_of_n ? ROWS : ROWS_N;
    if (dx) b.dx = choose(M, K, N, b.dx_layout, true);
    if (dw) b.dw = dw_rows_of_n ? choose(N, K, M, TOKENS, true) : choose(K, N, M, TOKENS, true);
    b.dz = activation && (dx || dw) ? up(2ll * M * N) : 0;
    b.sums = dbias && b.slope.chunks > 1 ? up(4ll * b.slope.chunks * N) : 0;
    b.parts = b.dx.bytes > b.dw.bytes ? b.dx.bytes : b.dw.bytes;
    return b;
}

static int forward(const linear_rows* x, const linear_rows* w, int w_rows_of_n, const void* bias, int bias_f32, const linear_rows* residual,
                   const linear_rows* pre, const linear_rows* out, int activation, int M, int N, int K, int dtype, const Memory& memory, void* stream) {
    if (const int rc = check_sizes(M, N, K, dtype, activation)) return rc;
    const int wr = w_rows_of_n ? N : K, wc = w_rows_of_n ? K : N;
    if (const int rc = check_matrix(x, M, K)) return rc;
    if (const int rc = check_matrix(w, wr, wc)) return rc;
    if (const int rc = check_matrix(out, M, N)) return rc;
    if (given(residual))
        if (const int rc = check_matrix(residual, M, N)) return rc;
    if (given(pre))
        if (const int rc = check_matrix(pre, M, N)) return rc;
    if ((uintptr_t)bias % 16 || (uintptr_t)memory.given % 16) return LINEAR_EINVAL;
    const Rows2D xs = block(x, M, K), ws = block(w, wr, wc), bs = vector_of(bias, (long long)N * (bias_f32 ? 4 : 2)), rs = block(residual, M, N);
    const Rows2D os = block(out, M, N), ps = block(pre, M, N);
    const bool in_place = given(residual) && residual->data == out->data && (M == 1 || residual->stride == out->stride);
    if (rows_meet(os, xs) || rows_meet(os, ws) || rows_meet(os, bs) || (!in_place && rows_meet(os, rs)) || rows_meet(os, ps)) return LINEAR_EINVAL;
    if (rows_meet(ps, xs) || rows_meet(ps, ws) || rows_meet(ps, bs) || rows_meet(ps, rs)) return LINEAR_EINVAL;
    const int layout = w_rows_of_n ? ROWS_N : ROWS;
    Plan plan = choose(M, N, K, layout, true);
    if (plan.tile < 0) return LINEAR_EUNSUPPORTED;
    void* const workspace = plan.bytes ? memory.take(plan.bytes) : nullptr;
    if (plan.bytes) {
        if (!workspace) {
            plan = choose(M, N, K, layout, false);
        } else {
            const Rows2D mine = vector_of(workspace, plan.bytes);
            for (const Rows2D& t : {xs, ws, bs, rs, os, ps})
                if (rows_meet(mine, t)) return LINEAR_EINVAL;
        }
    }
    Args a = {};
    a.a = (const char*)x->data, a.b = (const char*)w->data, a.out = (char*)out->data, a.M = M, a.N = N, a.K = K;
    a.lda = stride_of(x, M, K), a.ldb = stride_of(w, wr, wc), a.ldo = stride_of(out, M, N);
    a.e.bias = bias, a.e.bias_f32 = bias_f32, a.e.act = activation;
    if (given(residual)) a.e.residual = (const uint16_t*)residual->data, a.e.ldr = stride_of(residual, M, N);
    if (given(pre)) {
        a.e.pre = (uint16_t*)pre->data, a.e.ldp = stride_of(pre, M, N);
        a.e.pre_lines = (uintptr_t)pre->data % 128 == 0 && a.e.ldp % 64 == 0;
    }
    return run(plan, layout, dtype, a, workspace, stream);
}

static int backward(const linear_rows* dy, const linear_rows* x, const linear_rows* w, int w_rows_of_n, const linear_rows* pre,
                    const linear_rows* dx, const linear_rows* dw, int dw_rows_of_n, float* dbias, int activation, int M, int N, int K,
                    int dtype, const Memory& memory, void* stream) {
    if (const int rc = check_sizes(M, N, K, dtype, activation)) return rc;
    const bool want_x = given(dx), want_w = given(dw);
    if (!want_x && !want_w && !dbias) return LINEAR_EINVAL;
    const int wr = w_rows_of_n ? N : K, wc = w_rows_of_n ? K : N, dwr = dw_rows_of_n ? N : K, dwc = dw_rows_of_n ? K : N;
    if (const int rc = check_matrix(dy, M, N)) return rc;
    if (activation)
        if (const int rc = check_matrix(pre, M, N)) return rc;
    if (want_x) {
        if (const int rc = check_matrix(w, wr, wc)) return rc;
        if (const int rc = check_matrix(dx, M, K)) return rc;
    }
    if (want_w) {
        if (const int rc = check_matrix(x, M, K)) return rc;
        if (const int rc = check_matrix(dw, dwr, dwc)) return rc;
    }
    if ((uintptr_t)dbias % 16 || (uintptr_t)memory.given % 16) return LINEAR_EINVAL;
    const Backward b = backward_of(M, N, K, w_rows_of_n, dw_rows_of_n, activation, want_x, want_w, dbias);
    if (b.dx.tile < 0 || b.dw.tile < 0 || (long long)b.slope.blocks * b.slope.chunks * 256 > (long long)UINT_MAX || b.slope.chunks > 65535)
        return LINEAR_EUNSUPPORTED;
    const Rows2D in[] = {block(dy, M, N), activation ? block(pre, M, N) : Rows2D{}, want_w ? block(x, M, K) : Rows2D{},
                         want_x ? block(w, wr, wc) : Rows2D{}};
    const Rows2D out[] = {want_x ? block(dx, M, K) : Rows2D{}, want_w ? block(dw, dwr, dwc) : Rows2D{}, vector_of(dbias, 4ll * N)};
    for (int i = 0; i < 3; ++i) {
        for (const Rows2D& t : in)
            if (rows_meet(out[i], t)) return LINEAR_EINVAL;
        for (int j = 0; j < i; ++j)
            if (rows_meet(out[i], out[j])) return LINEAR_EINVAL;
    }
    void* const workspace = b.total() ? memory.take(b.total()) : nullptr;
    if (b.total()) {
        if (!workspace) return LINEAR_ENOMEM;
        const Rows2D mine = vector_of(workspace, b.total());
        for (const Rows2D& t : in)
            if (rows_meet(mine, t)) return LINEAR_EINVAL;
        for (const Rows2D& t : out)
            if (rows_meet(mine, t)) return LINEAR_EINVAL;
    }
    char* const dz = (char*)workspace;
    float* const sums = (float*)(dz + b.dz);
    void* const parts = dz + b.dz + b.sums;
    if (b.dz || dbias) {
        SlopeArgs s = {};
        s.dy = (const uint16_t*)dy->data, s.lddy = stride_of(dy, M, N), s.M = M, s.N = N, s.rows = b.slope.rows, s.lanes = b.slope.lanes, s.act = activation;
        s.pre = s.dy;
        if (activation) s.pre = (const uint16_t*)pre->data, s.ldpre = stride_of(pre, M, N);
        if (b.dz) s.dz = (uint16_t*)dz;
        if (dbias) s.sums = b.sums ? sums : dbias;
        void* args[] = {&s};
        if (const int rc = launch(dtype ? (const void*)slope_kernel<BF16> : (const void*)slope_kernel<F16>, dim3(b.slope.blocks, b.slope.chunks), 256, args, stream))
            return rc;
        if (b.sums) {
            const float* from = sums;
            int chunks = b.slope.chunks;
            void* list[] = {&from, &chunks, &N, &dbias};
            if (const int rc = launch((const void*)bias_kernel, dim3((N + 31) / 32), 1024, list, stream)) return rc;
        }
    }
    const char* const g = b.dz ? dz : (const char*)dy->data;
    const int ldg = b.dz ? N : stride_of(dy, M, N);
    if (want_x) {
        Args a = {};
        a.a = g, a.lda = ldg, a.b = (const char*)w->data, a.ldb = stride_of(w, wr, wc), a.out = (char*)dx->data, a.ldo = stride_of(dx, M, K);
        a.M = M, a.N = K, a.K = N;
        if (const int rc = run(b.dx, b.dx_layout, dtype, a, parts, stream)) return rc;
    }
    if (want_w) {
        Args a = {};
        a.a = (const char*)x->data, a.lda = stride_of(x, M, K), a.b = g, a.ldb = ldg, a.M = K, a.N = N, a.K = M;
        if (dw_rows_of_n) a.b = (const char*)x->data, a.ldb = stride_of(x, M, K), a.a = g, a.lda = ldg, a.M = N, a.N = K;
        a.out = (char*)dw->data, a.ldo = stride_of(dw, dwr, dwc);
        if (const int rc = run(b.dw, TOKENS, dtype, a, parts, stream)) return rc;
    }
    return LINEAR_OK;
}

}  // namespace linear

extern "C" {

long long gemm_linear_workspace(int M, int N, int K, int w_rows_of_n) {
    using namespace linear;
    if (const int rc = check_sizes(M, N, K, LINEAR_F16, LINEAR_NONE)) return rc;
    const Plan p = choose(M, N, K, w_rows_of_n ? ROWS_N : ROWS, true);
    return p.tile < 0 ? LINEAR_EUNSUPPORTED : p.bytes;
}

int gemm_linear(const linear_rows* x, const linear_rows* w, int w_rows_of_n, const void* bias, int bias_f32, const linear_rows* residual,
                const linear_rows* pre, const linear_rows* out, int activation, int M, int N, int K, int dtype, void* workspace,
                long long workspace_bytes, void* stream) {
    return linear::forward(x, w, w_rows_of_n, bias, bias_f32, residual, pre, out, activation, M, N, K, dtype, {workspace, workspace_bytes, nullptr, nullptr},
                           stream);
}

int gemm_linear_with(const linear_rows* x, const linear_rows* w, int w_rows_of_n, const void* bias, int bias_f32, const linear_rows* residual,
                     const linear_rows* pre, const linear_rows* out, int activation, int M, int N, int K, int dtype, linear_scratch_fn scratch,
                     void* owner, void* stream) {
    return linear::forward(x, w, w_rows_of_n, bias, bias_f32, residual, pre, out, activation, M, N, K, dtype, {nullptr, 0, scratch, owner}, stream);
}

long long gemm_linear_bwd_workspace(int M, int N, int K, int w_rows_of_n, int dw_rows_of_n, int activation, int dx, int dw, int dbias) {
    using namespace linear;
    if (const int rc = check_sizes(M, N, K, LINEAR_F16, activation)) return rc;
    if (!dx && !dw && !dbias) return LINEAR_EINVAL;
    const Backward b = backward_of(M, N, K, w_rows_of_n, dw_rows_of_n, activation, dx, dw, dbias);
    return b.dx.tile < 0 || b.dw.tile < 0 ? LINEAR_EUNSUPPORTED : b.total();
}

int gemm_linear_bwd(const linear_rows* dy, const linear_rows* x, const linear_rows* w, int w_rows_of_n, const linear_rows* pre,
                    const linear_rows* dx, const linear_rows* dw, int dw_rows_of_n, float* dbias, int activation, int M, int N, int K,
                    int dtype, void* workspace, long long workspace_bytes, void* stream) {
    return linear::backward(dy, x, w, w_rows_of_n, pre, dx, dw, dw_rows_of_n, dbias, activation, M, N, K, dtype,
                            {workspace, workspace_bytes, nullptr, nullptr}, stream);
}

int gemm_linear_bwd_with(const linear_rows* dy, const linear_rows* x, const linear_rows* w, int w_rows_of_n, const linear_rows* pre,
                         const linear_rows* dx, const linear_rows* dw, int dw_rows_of_n, float* dbias, int activation, int M, int N, int K,
                         int dtype, linear_scratch_fn scratch, void* owner, void* stream) {
    return linear::backward(dy, x, w, w_rows_of_n, pre, dx, dw, dw_rows_of_n, dbias, activation, M, N, K, dtype, {nullptr, 0, scratch, owner}, stream);
}

int linear_num_tiles(void) { return linear::kTiles; }

int linear_choice(int M, int N, int K, int layout, int* tile, int* ranges) {
    using namespace linear;
    if (M < 1 || N < 8 || K < 1 || N % 8 || layout < ROWS || layout > TOKENS || !tile || !ranges || (layout == TOKENS ? M % 8 : K % 8)) return LINEAR_EINVAL;
    if (N > kMost || (layout == TOKENS ? M > kMost || K > kMostRows : K > kMost || M > kMostRows)) return LINEAR_EUNSUPPORTED;
    const Plan p = choose(M, N, K, layout, true);
    if (p.tile < 0) return LINEAR_EUNSUPPORTED;
    *tile = p.tile, *ranges = p.ranges;
    return LINEAR_OK;
}

int linear_product(const linear_rows* a, const linear_rows* b, int layout, const linear_rows* c, int M, int N, int K, int dtype, int tile,
                   int ranges, void* workspace, long long workspace_bytes, void* stream) {
    using namespace linear;
    int chosen, most;
    if (const int rc = linear_choice(M, N, K, layout, &chosen, &most)) return rc;
    if ((dtype != LINEAR_F16 && dtype != LINEAR_BF16) || tile < 0 || tile >= kTiles || ranges < 1 || ranges > kMostRanges || (uintptr_t)workspace % 16)
        return LINEAR_EINVAL;
    const int ar = layout == TOKENS ? K : M, ac = layout == TOKENS ? M : K, br = layout == ROWS_N ? N : K, bc = layout == ROWS_N ? K : N;
    if (const int rc = check_matrix(a, ar, ac)) return rc;
    if (const int rc = check_matrix(b, br, bc)) return rc;
    if (const int rc = check_matrix(c, M, N)) return rc;
    const Plan plan = plan_of(tile, M, N, K, ranges);
    if (!fits(kShapes[tile], M, N, plan.ranges) || (plan.bytes && (long long)M * N / 8 > INT_MAX)) return LINEAR_EUNSUPPORTED;
    if (plan.bytes && (!workspace || workspace_bytes < plan.bytes)) return LINEAR_EINVAL;
    const Rows2D cs = block(c, M, N), mine = plan.bytes ? vector_of(workspace, plan.bytes) : Rows2D{};
    for (const Rows2D& t : {block(a, ar, ac), block(b, br, bc)})
        if (rows_meet(cs, t) || rows_meet(mine, t)) return LINEAR_EINVAL;
    if (rows_meet(mine, cs)) return LINEAR_EINVAL;
    Args p = {};
    p.a = (const char*)a->data, p.b = (const char*)b->data, p.out = (char*)c->data, p.M = M, p.N = N, p.K = K;
    p.lda = stride_of(a, ar, ac), p.ldb = stride_of(b, br, bc), p.ldo = stride_of(c, M, N);
    return run(plan, layout, dtype, p, workspace, stream);
}

const char* linear_strerror(int code) {
    switch (code) {
        case LINEAR_OK: return "ok";
        case LINEAR_EINVAL: return "invalid argument";
        case LINEAR_EUNSUPPORTED: return "unsupported size";
        case LINEAR_ENOMEM: return "no workspace, or too small a one";
        case LINEAR_ELAUNCH: return "the HIP runtime refused the launch";
        default: return "unknown error";
    }
}

}  // extern "C"
