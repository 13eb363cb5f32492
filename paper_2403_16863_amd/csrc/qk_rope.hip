// Norms of queries and keys with the rotation in the same pass, forward and backward (include/qk_rope.h has the formulas).
//
// Everything is read once and written once, so memory binds.  d / 16 lanes share a vector (one token's head), each with 8 channels of
// the lower and 8 of the upper half (neighbouring pairs: 16 on end): loads and stores of 16 bytes, a rotation's pairs in one lane, the sum of
// squares in 3 (d = 64: 2) exchanges.  A workgroup takes 8 tokens and goes through heads: a lane keeps its token's 8 cosines and sines
// in registers for all of them (read for each head they would be twice the bytes of the head), and 8 tokens of one head are 2 KB on end where the output is head-major.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/qk_rope.h"
#include "kv4_format.h"

namespace qk {

using kv4::load8;
using kv4::load8f;
using kv4::pack2;

struct Tensor {
    const uint16_t *x, *dy;  // dy: backward only
    uint16_t* y;             // forward: the output; backward: dx
    long long xs[3], dys[3], ys[3];
    const void* w;
    int heads;
};

struct Args {
    Tensor t[2];
    const float *cos, *sin;
    const int* positions;
    float* ws;  // [block][2][d] sums for the weights
    long long tokens;
    int N, rows, interleaved, weight_f32, head_step, blocks_y;
    float eps;
};

constexpr int kTokens = 8;

template <int D, bool BF>
__device__ __forceinline__ void weights(const Args& a, const void* w, int lo, int hi, float* out) {
    if (a.weight_f32) {
        load8f((const float*)w + lo, out);
        load8f((const float*)w + hi, out + 8);
    } else {
        load8<BF>((const uint16_t*)w + lo, out);
        load8<BF>((const uint16_t*)w + hi, out + 8);
    }
}

template <bool BF>
__device__ __forceinline__ void store8(uint16_t* p, const float* x) {
    *(uint4*)p = {pack2<BF>(x[0], x[1]), pack2<BF>(x[2], x[3]), pack2<BF>(x[4], x[5]), pack2<BF>(x[6], x[7])};
}

template <int L>
__device__ __forceinline__ float vector_sum(float x) {
#pragma unroll
    for (int d = 1; d < L; d *= 2) x += __shfl_xor(x, d);
    return x;
}

template <int D, bool BF, bool BACK, bool PAIRS>
__global__ __launch_bounds__(256, 4) void rope_kernel(Args a) {
    constexpr int L = D / 16, SLOTS = 256 / L, PHASES = SLOTS / kTokens, PARTS = 256 / D;
    __shared__ float sums[BACK ? SLOTS * (D + 4) : 1], parts[BACK ? 256 : 1];
    const int l = threadIdx.x % L, slot = threadIdx.x / L, phase = slot / kTokens;
    const int lo = PAIRS ? 16 * l : 8 * l, hi = PAIRS ? lo + 8 : lo + D / 2;
    const int by = blockIdx.x % a.blocks_y, bx = blockIdx.x / a.blocks_y, step = gridDim.x / a.blocks_y;
    const int h0 = by * a.head_step, h1 = min(h0 + a.head_step, a.t[0].heads + a.t[1].heads);

    // One tensor after the other: the weight and its gradient's sums take 32 registers, not 64.
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const Tensor& T = a.t[z];
        const int from = z ? max(0, h0 - a.t[0].heads) : h0, to = z ? h1 - a.t[0].heads : min(h1, T.heads);
        float* const out = BACK && a.ws ? a.ws + ((long long)blockIdx.x * 2 + z) * D : nullptr;
        if (from >= to) {  // none of this tensor's heads here
            if (BACK && out && threadIdx.x < D) out[threadIdx.x] = 0;
            continue;
        }
        float w[16], dw[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = 1, dw[i] = 0;
        if (T.w) weights<D, BF>(a, T.w, lo, hi, w);
        for (long long first = (long long)bx * kTokens; first < a.tokens; first += (long long)step * kTokens) {
            const long long token = first + slot % kTokens;
            if (token >= a.tokens) break;  // no later tile has one for this lane; the lanes of a vector leave together
            const long long b = token / a.N, n = token % a.N;
            float c[8], s[8];
            const int at = a.positions[token];
            if ((unsigned)at < (unsigned)a.rows) {
                load8f(a.cos + (long long)at * (D / 2) + 8 * l, c);
                load8f(a.sin + (long long)at * (D / 2) + 8 * l, s);
            } else {
                for (int i = 0; i < 8; ++i) c[i] = s[i] = __uint_as_float(0x7fc00000u);
            }
            const uint16_t* x = T.x + b * T.xs[0] + n * T.xs[1];
            const uint16_t* dy = T.dy + b * T.dys[0] + n * T.dys[1];
            uint16_t* y = T.y + b * T.ys[0] + n * T.ys[1];
            for (int h = from + phase; h < to; h += PHASES) {
                float v[16], g[16], r = 1;
                if (!BACK || T.w) {
                    load8<BF>(x + h * T.xs[2] + lo, v);
                    load8<BF>(x + h * T.xs[2] + hi, v + 8);
                }
                if (BACK) {
                    load8<BF>(dy + h * T.dys[2] + lo, g);
                    load8<BF>(dy + h * T.dys[2] + hi, g + 8);
                }
                if (T.w) {
                    float sq = 0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) sq = fmaf(v[i], v[i], sq);
                    r = __builtin_amdgcn_rsqf(fmaf(vector_sum<L>(sq), 1.f / D, a.eps));
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] *= r;
                }
                if (!BACK) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int p = PAIRS ? 2 * i : i, q = PAIRS ? 2 * i + 1 : i + 8;
                        const float m = v[p] * w[p], k = v[q] * w[q];
                        v[p] = m * c[i] - k * s[i];
                        v[q] = k * c[i] + m * s[i];
                    }
                    store8<BF>(y + h * T.ys[2] + lo, v);
                    store8<BF>(y + h * T.ys[2] + hi, v + 8);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int p = PAIRS ? 2 * i : i, q = PAIRS ? 2 * i + 1 : i + 8;
                        const float m = g[p] * c[i] + g[q] * s[i];
                        g[q] = g[q] * c[i] - g[p] * s[i];
                        g[p] = m;
                    }
                    if (T.w) {
                        float dot = 0;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            dw[i] = fmaf(g[i], v[i], dw[i]);
                            g[i] *= w[i];
                            dot = fmaf(g[i], v[i], dot);
                        }
                        dot = vector_sum<L>(dot) * (1.f / D);
#pragma unroll
                        for (int i = 0; i < 16; ++i) g[i] = r * fmaf(-v[i], dot, g[i]);
                    }
                    store8<BF>(y + h * T.ys[2] + lo, g);
                    store8<BF>(y + h * T.ys[2] + hi, g + 8);
                }
            }
        }
        if (!BACK || !out) continue;
        // The lanes' sums meet in LDS, and 256 / D threads add a column's.
        float* mine = sums + slot * (D + 4);
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            *(float4*)(mine + lo + i) = {dw[i], dw[i + 1], dw[i + 2], dw[i + 3]};
            *(float4*)(mine + hi + i) = {dw[i + 8], dw[i + 9], dw[i + 10], dw[i + 11]};
        }
        __syncthreads();
        const int c = threadIdx.x % D, part = threadIdx.x / D;
        float sum = 0;
#pragma unroll 8
        for (int i = 0; i < SLOTS / PARTS; ++i) sum += sums[(part * (SLOTS / PARTS) + i) * (D + 4) + c];
        parts[threadIdx.x] = sum;
        __syncthreads();
        if (threadIdx.x < D) {
            for (int i = 1; i < PARTS; ++i) sum += parts[i * D + threadIdx.x];
            out[threadIdx.x] = sum;
        }
        __syncthreads();  // the next tensor's sums take the place of these
    }
}

// The weights' gradients from the blocks' sums: 8 columns a workgroup, 128 threads to a column, so that 1024 blocks are eight
// loads to a thread (with 32 threads to a column the chain of loads took 11.8 us).
__global__ __launch_bounds__(1024) void weight_sum_kernel(const float* ws, int blocks, int d, float* dq_weight, float* dk_weight) {
    __shared__ float part[1024];
    const int c = blockIdx.x * 8 + threadIdx.x % 8;
    float t = 0;
#pragma unroll 8
    for (int i = threadIdx.x / 8; i < blocks; i += 128) t += ws[(long long)i * 2 * d + c];
    part[threadIdx.x] = t;
#pragma unroll
    for (int n = 512; n >= 8; n /= 2) {
        __syncthreads();
        if (threadIdx.x < n) part[threadIdx.x] += part[threadIdx.x + n];
    }
    if (threadIdx.x >= 8) return;
    float* to = c < d ? dq_weight : dk_weight;
    if (to) to[c % d] = part[threadIdx.x];
}

struct Grid {
    int x, y, head_step;
};

// Token tiles, and the heads cut into as many pieces as it takes to have 1024 workgroups (four on each of 256 units; backward 512, whose sums are fewer to
// add: 3 x 1001 tokens of 24 heads, d = 64, 14.6 us against 15.6), none smaller than one round of the workgroup's phases; at most 2048 workgroups where their sums have to be added up.
Grid grid_of(long long tokens, int heads, int d, bool back) {
    const long long tiles = (tokens + kTokens - 1) / kTokens;
    const int phases = 256 / (d / 16) / kTokens, most = (heads + phases - 1) / phases;
    Grid g;
    const int enough = back ? 512 : 1024;
    const int want = tiles >= enough ? 1 : (int)((enough + tiles - 1) / tiles);
    const int pieces = want < most ? want : most;
    g.head_step = ((heads + pieces - 1) / pieces + phases - 1) / phases * phases;
    g.y = (heads + g.head_step - 1) / g.head_step;
    const long long limit = back ? 2048 / g.y : INT_MAX / 256 / g.y;
    g.x = (int)(tiles < limit ? tiles : limit < 1 ? 1 : limit);
    return g;
}

int check_tensor(const qk_heads* t, int B, int N, int heads, bool written) {
    if ((uintptr_t)t->data % 16) return QK_EINVAL;
    if (written && ((B > 1 && !t->batch_stride) || (N > 1 && !t->token_stride) || (heads > 1 && !t->head_stride))) return QK_EINVAL;
    if ((B > 1 && t->batch_stride % 8) || (N > 1 && t->token_stride % 8) || (heads > 1 && t->head_stride % 8)) return QK_EINVAL;
    return QK_OK;
}

int check(int B, int N, int H, int Hkv, int d) {
    if (B < 1 || N < 1 || H < 0 || Hkv < 0 || H + (long long)Hkv < 1) return QK_EINVAL;
    if (d != 64 && d != 128) return QK_EUNSUPPORTED;
    return (long long)H + Hkv > INT_MAX || (long long)B * N > INT_MAX / ((long long)H + Hkv) ? QK_EUNSUPPORTED : QK_OK;
}

bool given(const qk_heads* t) { return t && t->data; }

// An output that begins where another tensor does writes what other workgroups still read, or write.  Its own input's memory (`own`) with the
// same strides is left to it: a lane reads a vector before it writes it.
bool meets(const qk_heads* out, const qk_heads* other, bool own, int B, int N, int heads) {
    if (!given(out) || !given(other) || out->data != other->data) return false;
    return !own || (B > 1 && out->batch_stride != other->batch_stride) || (N > 1 && out->token_stride != other->token_stride) ||
           (heads > 1 && out->head_stride != other->head_stride);
}

void strides(const qk_heads* t, long long* s) { s[0] = t->batch_stride, s[1] = t->token_stride, s[2] = t->head_stride; }

template <bool BACK>
const void* kernel(int d, int dtype, int pairs) {
    if (d == 128) {
        if (dtype) return pairs ? (const void*)rope_kernel<128, true, BACK, true> : (const void*)rope_kernel<128, true, BACK, false>;
        return pairs ? (const void*)rope_kernel<128, false, BACK, true> : (const void*)rope_kernel<128, false, BACK, false>;
    }
    if (dtype) return pairs ? (const void*)rope_kernel<64, true, BACK, true> : (const void*)rope_kernel<64, true, BACK, false>;
    return pairs ? (const void*)rope_kernel<64, false, BACK, true> : (const void*)rope_kernel<64, false, BACK, false>;
}

}  // namespace qk

extern "C" {

int qk_norm_rope(const qk_heads* q, const qk_heads* k, const qk_heads* q_out, const qk_heads* k_out, const void* q_weight,
                 const void* k_weight, int weight_f32, const float* cos, const float* sin, const int* positions, int rows, float eps,
                 int interleaved, int B, int N, int H, int Hkv, int d, int dtype, void* stream) {
    using namespace qk;
    if (given(q) != given(q_out) || given(k) != given(k_out)) return QK_EINVAL;
    if (!given(q)) H = 0;
    if (!given(k)) Hkv = 0;
    if (!cos || !sin || !positions || rows < 1 || (dtype != QK_F16 && dtype != QK_BF16) || !(eps >= 0) || !isfinite(eps)) return QK_EINVAL;
    if ((uintptr_t)cos % 16 || (uintptr_t)sin % 16 || (uintptr_t)positions % 4 || (uintptr_t)q_weight % 16 || (uintptr_t)k_weight % 16) return QK_EINVAL;
    if (const int rc = check(B, N, H, Hkv, d)) return rc;
    Args a = {};
    const qk_heads* in[2] = {q, k};
    const qk_heads* out[2] = {q_out, k_out};
    const void* w[2] = {q_weight, k_weight};
    const int heads[2] = {H, Hkv};
    for (int z = 0; z < 2; ++z) {
        if (!heads[z]) continue;
        if (check_tensor(in[z], B, N, heads[z], false) || check_tensor(out[z], B, N, heads[z], true)) return QK_EINVAL;
        a.t[z].x = (const uint16_t*)in[z]->data, a.t[z].y = (uint16_t*)out[z]->data, a.t[z].w = w[z], a.t[z].heads = heads[z];
        strides(in[z], a.t[z].xs), strides(out[z], a.t[z].ys);
    }
    for (int z = 0; z < 2; ++z)
        for (int y = 0; y < 2; ++y)
            if (heads[z] && heads[y] && meets(out[z], in[y], z == y, B, N, heads[z])) return QK_EINVAL;
    if (H && Hkv && meets(q_out, k_out, false, B, N, H)) return QK_EINVAL;
    const Grid g = grid_of((long long)B * N, H + Hkv, d, false);
    a.cos = cos, a.sin = sin, a.positions = positions, a.tokens = (long long)B * N, a.N = N, a.rows = rows, a.interleaved = interleaved;
    a.weight_f32 = weight_f32, a.head_step = g.head_step, a.blocks_y = g.y, a.eps = eps;
    void* list[] = {&a};
    if (hipLaunchKernel(kernel<false>(d, dtype, interleaved), dim3((unsigned)g.x * g.y), dim3(256), list, 0, (hipStream_t)stream) != hipSuccess) {
        (void)hipGetLastError();
        return QK_ELAUNCH;
    }
    return QK_OK;
}

long long qk_norm_rope_bwd_workspace(int B, int N, int H, int Hkv, int d) {
    using namespace qk;
    if (const int rc = check(B, N, H, Hkv, d)) return rc;
    const Grid g = grid_of((long long)B * N, H + Hkv, d, true);
    return (long long)g.x * g.y * 2 * d * 4;
}

int qk_norm_rope_bwd(const qk_heads* dq_out, const qk_heads* dk_out, const qk_heads* q, const qk_heads* k, const qk_heads* dq,
                     const qk_heads* dk, const void* q_weight, const void* k_weight, int weight_f32, float* dq_weight,
                     float* dk_weight, const float* cos, const float* sin, const int* positions, int rows, float eps, int interleaved,
                     int B, int N, int H, int Hkv, int d, int dtype, void* workspace, long long workspace_bytes, void* stream) {
    using namespace qk;
    if (given(dq_out) != given(dq) || given(dk_out) != given(dk)) return QK_EINVAL;
    if (!given(dq)) H = 0, q_weight = nullptr, dq_weight = nullptr;
    if (!given(dk)) Hkv = 0, k_weight = nullptr, dk_weight = nullptr;
    if (!cos || !sin || !positions || rows < 1 || (dtype != QK_F16 && dtype != QK_BF16) || !(eps >= 0) || !isfinite(eps)) return QK_EINVAL;
    if ((uintptr_t)cos % 16 || (uintptr_t)sin % 16 || (uintptr_t)positions % 4 || (uintptr_t)q_weight % 16 || (uintptr_t)k_weight % 16) return QK_EINVAL;
    if (!q_weight != !dq_weight || !k_weight != !dk_weight || (uintptr_t)dq_weight % 4 || (uintptr_t)dk_weight % 4) return QK_EINVAL;
    if (const int rc = check(B, N, H, Hkv, d)) return rc;
    const Grid g = grid_of((long long)B * N, H + Hkv, d, true);
    const bool sums = q_weight || k_weight;
    if (sums && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < (long long)g.x * g.y * 2 * d * 4)) return QK_EINVAL;
    Args a = {};
    const qk_heads* x[2] = {q, k};
    const qk_heads* dy[2] = {dq_out, dk_out};
    const qk_heads* dx[2] = {dq, dk};
    const void* w[2] = {q_weight, k_weight};
    const int heads[2] = {H, Hkv};
    for (int z = 0; z < 2; ++z) {
        if (!heads[z]) continue;
        if (w[z] && !given(x[z])) return QK_EINVAL;
        if (check_tensor(dy[z], B, N, heads[z], false) || check_tensor(dx[z], B, N, heads[z], true) || (w[z] && check_tensor(x[z], B, N, heads[z], false)))
            return QK_EINVAL;
        if (w[z]) a.t[z].x = (const uint16_t*)x[z]->data, strides(x[z], a.t[z].xs);
        a.t[z].dy = (const uint16_t*)dy[z]->data, a.t[z].y = (uint16_t*)dx[z]->data, a.t[z].w = w[z], a.t[z].heads = heads[z];
        strides(dy[z], a.t[z].dys), strides(dx[z], a.t[z].ys);
    }
    for (int z = 0; z < 2; ++z)
        for (int y = 0; y < 2; ++y)
            if (heads[z] && heads[y] && (meets(dx[z], dy[y], z == y, B, N, heads[z]) || (w[y] && meets(dx[z], x[y], z == y, B, N, heads[z])))) return QK_EINVAL;
    if (H && Hkv && meets(dq, dk, false, B, N, H)) return QK_EINVAL;
    a.cos = cos, a.sin = sin, a.positions = positions, a.ws = sums ? (float*)workspace : nullptr, a.tokens = (long long)B * N, a.N = N;
    a.rows = rows, a.interleaved = interleaved, a.weight_f32 = weight_f32, a.head_step = g.head_step, a.blocks_y = g.y, a.eps = eps;
    void* list[] = {&a};
    const float* ws = a.ws;
    int blocks = g.x * g.y;
    void* sum_list[] = {&ws, &blocks, &d, &dq_weight, &dk_weight};
    if (hipLaunchKernel(kernel<true>(d, dtype, interleaved), dim3((unsigned)blocks), dim3(256), list, 0, (hipStream_t)stream) != hipSuccess ||
        (sums && hipLaunchKernel((const void*)weight_sum_kernel, dim3((unsigned)d / 4), dim3(1024), sum_list, 0, (hipStream_t)stream) != hipSuccess)) {
        (void)hipGetLastError();
        return QK_ELAUNCH;
    }
    return QK_OK;
}

const char* qk_strerror(int code) {
    switch (code) {
        case QK_OK: return "ok";
        case QK_EINVAL: return "invalid argument";
        case QK_EUNSUPPORTED: return "unsupported size";
        case QK_ELAUNCH: return "the HIP runtime refused the launch";
        default: return "unknown error";
    }
}

}  // extern "C"
