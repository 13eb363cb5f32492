// The norms behind a block and ahead of the next with the residual stream's update between them, forward and backward
// (include/residual_norm.h has the formulas).
//
// Everything is read once and written once, so memory binds.  W waves share a token, a lane holding V vectors of 8 channels in registers
// from the loads to the stores, and a workgroup goes through a run of tokens with the products of its vectors (gate times post_weight, which is
// all that either direction needs of the two, and pre_weight) in registers.  A token's sums meet in LDS: forward, the stream's
// mean square needs the first norm's, two meetings; backward, all sums of the inputs alone meet at once (both mean squares and sum dz pre_weight y) and
// sum D gate post_weight h second.  Two buffers in turn, so a meeting is one barrier.
//
// Backward, the vectors' gradients need two sums over tokens, kept in registers: S1 = sum D h r(h), by sequence where the gate is, and
// S2 = sum dz y r(y).  dgate = post_weight S1, dpost_weight = sum over sequences of gate S1, dpre_weight = S2.  Workgroups write theirs, and a second kernel adds them in order.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/residual_norm.h"
#include "kv4_format.h"
#include "memory_check.h"
#include "turns.h"

namespace stream_norm {

using kv4::load8f;
using kv4::pack2;
using kv4::values_of;

struct Tokens {
    char* data;
    long long bs, ts;  // bytes
};

struct Args {
    Tokens x, h, y, z, dy, dz, dx, dh;
    const void *gate, *post, *pre;
    long long gate_stride;  // elements; 0: one for all
    int gate_f32, weight_f32;
    float* sums;            // backward: [workgroup][2][C], what dpost_weight (a shared gate: S1) and dpre_weight are added from, or null
    float* units;           // backward, gate by sequence: [unit][C] S1, or with one unit a sequence dgate itself; or null
    // Units of work: `runs` of `length` tokens on end (the sequences, where a backward pass has a gate for each; else one run of all) in `chunks` of `rows`.
    int N, C, runs, length, chunks, rows;
    float alpha, eps;
};

template <bool BF>
__device__ __forceinline__ void load_vector(const void* p, int f32, long long at, float* v) {
    if (f32) load8f((const float*)p + at, v);
    else kv4::load8<BF>((const uint16_t*)p + at, v);
}

template <bool BF>
__device__ __forceinline__ uint4 pack8(const float* x) {
    return {pack2<BF>(x[0], x[1]), pack2<BF>(x[2], x[3]), pack2<BF>(x[4], x[5]), pack2<BF>(x[6], x[7])};
}

template <int CONTROL>
__device__ __forceinline__ float dpp(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CONTROL, 0xf, 0xf, false));
}
// Over the 64 lanes, the same in each: neighbours, pairs, the halves of 8, of 16, then across.
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp<0xb1>(x);
    x += dpp<0x4e>(x);
    x += dpp<0x141>(x);
    x += dpp<0x140>(x);
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    return x;
}

// Sums over a token's W waves; `at`: 0 and 1 in turn.
template <int W, int K>
__device__ __forceinline__ void token_sums(float (&s)[K], float* meeting, int at, int group) {
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = wave_sum(s[k]);
    if (W == 1) return;
    const int wave = threadIdx.x / 64 % W;
    float* const mine = meeting + (at * 8 + group) * (W * 4);
    if (threadIdx.x % 64 == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) mine[wave * 4 + k] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float t = mine[k];
#pragma unroll
        for (int w = 1; w < W; ++w) t += mine[w * 4 + k];
        s[k] = t;
    }
}

// Tokens of a workgroup: eight waves' (forward on 2 x 4096 x 4096: 52.5 us with eight waves to a workgroup, 55.2 with four).
template <int W>
struct Block {
    static constexpr int groups = W <= 4 ? 8 / W : 1, threads = W * 64 * groups;
};

// A lane's vectors of 8 channels: v * 64 W + lane of the token's lanes.
template <bool BF, int W, int V>
__global__ __launch_bounds__(Block<W>::threads) void forward_kernel(Args a) {
    constexpr int G = Block<W>::groups;
    __shared__ float meeting[W > 1 ? 2 * 8 * W * 4 : 1];
    const int group = threadIdx.x / (64 * W), lane = threadIdx.x % (64 * W);
    int c[V];
    bool in[V];
#pragma unroll
    for (int v = 0; v < V; ++v) c[v] = (v * 64 * W + lane) * 8, in[v] = c[v] < a.C;
    float gp[V][8], pre[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) gp[v][i] = 1, pre[v][i] = 0;
        if (in[v] && a.z.data) load_vector<BF>(a.pre, a.weight_f32, c[v], pre[v]);
    }
    int have = -1;  // the sequence whose gate is in gp
    const float mean = 1.f / (float)a.C;
    int at = 0;
    const long long first = (long long)blockIdx.x * a.rows;
    const long long end = min((long long)a.length, first + a.rows);
    for (long long r = first; r < end; r += G) {
        const bool there = r + group < end;
        const unsigned token = (unsigned)(there ? r + group : r), b = token / (unsigned)a.N, n = token - b * (unsigned)a.N;
        uint4 xr[V], hr[V];
        const char* const xp = a.x.data + b * a.x.bs + n * a.x.ts;
        const char* const hp = a.h.data + b * a.h.bs + n * a.h.ts;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            xr[v] = hr[v] = uint4{0, 0, 0, 0};
            if (!in[v] || !there) continue;
            xr[v] = *(const uint4*)(xp + c[v] * 2);
            if (a.h.data) hr[v] = *(const uint4*)(hp + c[v] * 2);
        }
        float y[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) values_of<BF>(xr[v], y[v]);
        if (a.h.data) {
            if ((a.gate || a.post) && have != (a.gate_stride ? (int)b : 0)) {
                have = a.gate_stride ? (int)b : 0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (!in[v]) continue;
                    float p[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) gp[v][i] = 1;
                    if (a.gate) load_vector<BF>(a.gate, a.gate_f32, have * a.gate_stride + c[v], gp[v]);
                    if (!a.post) continue;
                    load_vector<BF>(a.post, a.weight_f32, c[v], p);
#pragma unroll
                    for (int i = 0; i < 8; ++i) gp[v][i] *= p[i];
                }
            }
            float h[V][8], s[1] = {0}, rh = 1;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                values_of<BF>(hr[v], h[v]);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0] = fmaf(h[v][i], h[v][i], s[0]);
            }
            if (a.post) {
                token_sums<W>(s, meeting, at, group);
                at ^= 1;
                rh = __builtin_amdgcn_rsqf(fmaf(s[0], mean, a.eps));
            }
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[v][i] = fmaf(a.alpha, y[v][i], gp[v][i] * (h[v][i] * rh));
        }
        if (a.y.data && there) {
            char* const yp = a.y.data + b * a.y.bs + n * a.y.ts;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (in[v]) *(uint4*)(yp + c[v] * 2) = pack8<BF>(y[v]);
        }
        if (!a.z.data) continue;
        float s[1] = {0};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] = fmaf(y[v][i], in[v] ? y[v][i] : 0.f, s[0]);
        token_sums<W>(s, meeting, at, group);
        at ^= 1;
        if (!there) continue;
        const float r2 = __builtin_amdgcn_rsqf(fmaf(s[0], mean, a.eps));
        char* const zp = a.z.data + b * a.z.bs + n * a.z.ts;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!in[v]) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[v][i] = pre[v][i] * (y[v][i] * r2);
            *(uint4*)(zp + c[v] * 2) = pack8<BF>(y[v]);
        }
    }
}

template <bool BF, int W, int V>
__global__ __launch_bounds__(Block<W>::threads) void backward_kernel(Args a) {
    constexpr int G = Block<W>::groups, LANES = 64 * W;
    __shared__ float meeting[W > 1 ? 2 * 8 * W * 4 : 1];
    __shared__ __attribute__((aligned(16))) float joined[G > 1 ? (G - 1) * LANES * V * 8 : 1];
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    int c[V];
    bool in[V];
#pragma unroll
    for (int v = 0; v < V; ++v) c[v] = (v * LANES + lane) * 8, in[v] = c[v] < a.C;
    float gp[V][8], pre[V][8], s1[V][8], s2[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) gp[v][i] = 1, pre[v][i] = s1[v][i] = s2[v][i] = 0;
        if (in[v] && a.dz.data) load_vector<BF>(a.pre, a.weight_f32, c[v], pre[v]);
    }
    // The groups' sums, added in group order, to group 0's registers.
    auto join = [&](float (&s)[V][8]) __attribute__((always_inline)) {
        if (G == 1) return;
        __syncthreads();
        if (group) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; i += 4)
                    *(float4*)&joined[(((group - 1) * V + v) * LANES + lane) * 8 + i] = {s[v][i], s[v][i + 1], s[v][i + 2], s[v][i + 3]};
        }
        __syncthreads();
        if (!group) {
            for (int g = 1; g < G; ++g)
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[v][i] += joined[(((g - 1) * V + v) * LANES + lane) * 8 + i];
        }
    };
    auto store = [&](float* to, const float* s) __attribute__((always_inline)) {
        ((float4*)to)[0] = {s[0], s[1], s[2], s[3]};
        ((float4*)to)[1] = {s[4], s[5], s[6], s[7]};
    };
    const bool by_sequence = a.gate && a.gate_stride;
    const float mean = 1.f / (float)a.C;
    int at = 0;
    float* const sums = a.sums ? a.sums + (long long)blockIdx.x * 2 * a.C : nullptr;
    for (Turns turn = {blockIdx.x, gridDim.x, (unsigned)a.runs * (unsigned)a.chunks}; turn.left(); turn.next()) {
        const int unit = (int)turn.at, run = unit / a.chunks;
        const long long base = (long long)run * a.length, first = (long long)(unit - run * a.chunks) * a.rows;
        const long long end = min((long long)a.length, first + a.rows);
        if (unit == (int)blockIdx.x || by_sequence) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!in[v]) continue;
                float p[8];
                if (a.gate) load_vector<BF>(a.gate, a.gate_f32, (by_sequence ? run * a.gate_stride : 0) + c[v], gp[v]);
                if (!a.post) continue;
                load_vector<BF>(a.post, a.weight_f32, c[v], p);
#pragma unroll
                for (int i = 0; i < 8; ++i) gp[v][i] = a.gate ? gp[v][i] * p[i] : p[i];
            }
        }
        for (long long r = first; r < end; r += G) {
            const bool there = r + group < end;
            const unsigned token = (unsigned)(base + (there ? r + group : r)), b = token / (unsigned)a.N, n = token - b * (unsigned)a.N;
            auto row = [&](const Tokens& t) __attribute__((always_inline)) { return t.data + b * t.bs + n * t.ts; };
            uint4 yr[V], hr[V], dyr[V], dzr[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                yr[v] = hr[v] = dyr[v] = dzr[v] = uint4{0, 0, 0, 0};
                if (!in[v] || !there) continue;
                if (a.dz.data) yr[v] = *(const uint4*)(row(a.y) + c[v] * 2), dzr[v] = *(const uint4*)(row(a.dz) + c[v] * 2);
                if (a.dy.data) dyr[v] = *(const uint4*)(row(a.dy) + c[v] * 2);
                if (a.h.data) hr[v] = *(const uint4*)(row(a.h) + c[v] * 2);
            }
            float D[V][8], r1 = 1;
#pragma unroll
            for (int v = 0; v < V; ++v) values_of<BF>(dyr[v], D[v]);
            if (a.dz.data || a.post) {
                float s[3] = {0, 0, 0};
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float y[8], dz[8], h[8];
                    values_of<BF>(yr[v], y), values_of<BF>(dzr[v], dz), values_of<BF>(hr[v], h);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        s[0] = fmaf(y[i], y[i], s[0]);
                        s[1] = fmaf(dz[i] * pre[v][i], y[i], s[1]);
                        s[2] = fmaf(h[i], h[i], s[2]);
                    }
                }
                token_sums<W>(s, meeting, at, group);
                at ^= 1;
                if (a.post) r1 = __builtin_amdgcn_rsqf(fmaf(s[2], mean, a.eps));
                if (a.dz.data) {
                    const float r2 = __builtin_amdgcn_rsqf(fmaf(s[0], mean, a.eps)), m = s[1] * r2 * mean;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float y[8], dz[8];
                        values_of<BF>(yr[v], y), values_of<BF>(dzr[v], dz);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float n2 = y[i] * r2;
                            if (there) s2[v][i] = fmaf(dz[i], n2, s2[v][i]);
                            D[v][i] = fmaf(r2, fmaf(-n2, m, dz[i] * pre[v][i]), D[v][i]);
                        }
                    }
                }
            }
            if (a.dx.data && there) {
                char* const to = row(a.dx);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float t[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[i] = a.alpha * D[v][i];
                    if (in[v]) *(uint4*)(to + c[v] * 2) = pack8<BF>(t);
                }
            }
            float s[1] = {0};
            if (a.h.data) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float h[8];
                    values_of<BF>(hr[v], h);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float n1 = h[i] * r1;
                        if (there) s1[v][i] = fmaf(D[v][i], n1, s1[v][i]);
                        D[v][i] *= gp[v][i];  // from here on the gradient of n1 (without a post_weight of h)
                        if (in[v]) s[0] = fmaf(D[v][i], n1, s[0]);
                    }
                }
            }
            if (!a.dh.data) continue;
            if (a.post) {
                token_sums<W>(s, meeting, at, group);
                at ^= 1;
            }
            if (!there) continue;
            const float m = s[0] * mean;
            char* const to = row(a.dh);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!in[v]) continue;
                if (a.post) {
                    float h[8];
                    values_of<BF>(hr[v], h);
#pragma unroll
                    for (int i = 0; i < 8; ++i) D[v][i] = r1 * fmaf(-(h[i] * r1), m, D[v][i]);
                }
                *(uint4*)(to + c[v] * 2) = pack8<BF>(D[v]);
            }
        }
        if (!by_sequence || (!a.units && !sums)) continue;
        join(s1);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!group && in[v]) {
                float t[8];
                if (sums) {  // (this lane's own earlier sum)
                    float g[8];
                    load_vector<BF>(a.gate, a.gate_f32, run * a.gate_stride + c[v], g);
                    if (unit == (int)blockIdx.x) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) t[i] = 0;
                    } else {
                        load8f(sums + c[v], t);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[i] = fmaf(g[i], s1[v][i], t[i]);
                    store(sums + c[v], t);
                }
                if (a.units) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[i] = 1;
                    if (a.chunks == 1 && a.post) load_vector<BF>(a.post, a.weight_f32, c[v], t);
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[i] *= s1[v][i];
                    store(a.units + (long long)unit * a.C + c[v], t);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) s1[v][i] = 0;
        }
    }
    if (!sums) return;
    if (!by_sequence) join(s1);
    join(s2);
    if (group) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!in[v]) continue;
        if (!by_sequence) store(sums + c[v], s1[v]);
        store(sums + a.C + c[v], s2[v]);
    }
}

// The vectors' gradients from the workgroups' sums: 32 columns a workgroup, 32 threads to a column.  blockIdx.y 0: dpost_weight (shared gate: and dgate),
// 1: dpre_weight, from 2 on: dgate of a sequence.
struct SumArgs {
    const float *sums, *units;
    const void *gate, *post;
    float *dgate, *dpost, *dpre;
    int gate_f32, weight_f32, blocks, chunks, C, by_sequence;
};

template <bool BF>
__device__ __forceinline__ float value_of(const void* p, int f32, int at) {
    if (f32) return ((const float*)p)[at];
    const unsigned w = ((const uint16_t*)p)[at];
    float x[8];
    values_of<BF>(uint4{w, 0, 0, 0}, x);
    return x[0];
}

template <bool BF>
__global__ __launch_bounds__(1024) void vector_sum_kernel(SumArgs a) {
    __shared__ float part[1024];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, job = blockIdx.y;
    const bool units = job >= 2;
    const int count = units ? a.chunks : a.blocks;
    const long long step = units ? a.C : 2ll * a.C;
    const float* const from = units ? a.units + (long long)(job - 2) * a.chunks * a.C : a.sums + (long long)job * a.C;
    float t = 0;
    if (c < a.C) {
#pragma unroll 8
        for (int i = threadIdx.x / 32; i < count; i += 32) t += from[i * step + c];
    }
    part[threadIdx.x] = t;
#pragma unroll
    for (int n = 512; n >= 32; n /= 2) {
        __syncthreads();
        if (threadIdx.x < n) part[threadIdx.x] += part[threadIdx.x + n];
    }
    if (threadIdx.x >= 32 || c >= a.C) return;
    t = part[threadIdx.x];
    if (job == 1) {
        if (a.dpre) a.dpre[c] = t;
    } else if (units) {
        a.dgate[(long long)(job - 2) * a.C + c] = a.post ? t * value_of<BF>(a.post, a.weight_f32, c) : t;
    } else {
        if (a.dpost) a.dpost[c] = a.by_sequence || !a.gate ? t : t * value_of<BF>(a.gate, a.gate_f32, c);
        if (a.dgate && !a.by_sequence) a.dgate[c] = a.post ? t * value_of<BF>(a.post, a.weight_f32, c) : t;
    }
}

// ---- host side
struct Kernel {
    int most, waves[2];  // channels; waves of a token, forward and backward
    const void *forward[2], *backward[2];
};
template <int W, int V, int WB = W, int VB = V>
static constexpr Kernel kernel_of() {
    static_assert(W * V == WB * VB, "as many channels both ways");
    return {512 * W * V, {W, WB}, {(const void*)forward_kernel<false, W, V>, (const void*)forward_kernel<true, W, V>},
            {(const void*)backward_kernel<false, WB, VB>, (const void*)backward_kernel<true, WB, VB>}};
}
// One vector a lane up to 4096 channels: a backward pass is then 100 to 115 registers and four waves to a SIMD.  With more channels on fewer waves, and two waves to a
// SIMD, it was 27.0 against 20.0 us on 3 x 1001 x 1152 (three vectors a lane), 50.3 against 41.7 on 2 x 4096 x 1536, 28.9 against 28.0 on 2 x 2048 x 2048 (two), and the
// same on 2 x 4096 x 4096; on 2 x 2048 x 8192 sixteen waves with one vector each 110 against 98.5 on eight with two.  Beyond 8192 channels the backward pass spills (163 us for
// 2048 x 12288 on eight waves, 210 on sixteen; forward 56 and 51).
static const Kernel kKernels[] = {kernel_of<1, 1>(), kernel_of<2, 1>(), kernel_of<3, 1>(), kernel_of<4, 1>(), kernel_of<8, 1>(), kernel_of<8, 2>(), kernel_of<16, 2, 8, 4>()};

static const Kernel& choose(int C) {
    int i = 0;
    while (kKernels[i].most < C) ++i;
    return kKernels[i];
}
static int groups_of(int waves) { return waves <= 4 ? 8 / waves : 1; }

static bool given(const norm_tokens* t) { return t && t->data; }

static int check_sizes(int B, int N, int C) {
    if (B < 1 || N < 1 || C < 1) return NORM_EINVAL;
    return C % 8 || C > 16384 || (long long)B * N > INT_MAX ? NORM_EUNSUPPORTED : NORM_OK;
}

// The strides that count; those of sizes of 1 are 0.
static long long batch_stride(const norm_tokens* t, int B) { return B > 1 ? t->batch_stride : 0; }
static long long token_stride(const norm_tokens* t, int N) { return N > 1 ? t->token_stride : 0; }

static int check_tokens(const norm_tokens* t, int B, int N, int C, bool written) {
    if (!given(t)) return NORM_OK;
    const long long bs = batch_stride(t, B), ts = token_stride(t, N);
    if ((uintptr_t)t->data % 16 || bs % 8 || ts % 8 || bs < 0 || ts < 0 || bs > (1ll << 59) / B || ts > (1ll << 59) / N) return NORM_EINVAL;
    if (!written) return NORM_OK;
    // tokens lie apart: the smaller stride steps over the channels, the larger one over all that the smaller one reaches
    if (B > 1 && N > 1) {
        const bool inner = ts <= bs;  // tokens inside sequences
        return (inner ? ts : bs) < C || (inner ? bs : ts) < (inner ? ts * (N - 1ll) : bs * (B - 1ll)) + C ? NORM_EINVAL : NORM_OK;
    }
    return (B > 1 && bs < C) || (N > 1 && ts < C) ? NORM_EINVAL : NORM_OK;
}

// Whether an output meets another tensor other than token by token in place.
static bool tokens_meet(const norm_tokens* out, const norm_tokens* other, bool in_place, int B, int N, int C) {
    if (!given(out) || !given(other)) return false;
    const long long bs = batch_stride(out, B), ts = token_stride(out, N), obs = batch_stride(other, B), ots = token_stride(other, N);
    const bool alike = bs == obs && ts == ots;
    if (in_place && alike && out->data == other->data) return false;
    const unsigned long long bytes = 2ull * (bs * (B - 1ll) + ts * (N - 1ll) + C), others = 2ull * (obs * (B - 1ll) + ots * (N - 1ll) + C);
    if (!bytes_meet(out->data, bytes, other->data, others)) return false;
    // side by side in the rows of a wider tensor: with the same strides, one a multiple of the other
    const long long small = !ts || (bs && bs < ts) ? bs : ts, large = small == ts ? bs : ts;
    if (!alike || !small || large % small) return true;
    return columns_meet(out->data, C, other->data, C, small);
}

static bool vector_meets(const norm_tokens* out, const void* p, unsigned long long bytes, int B, int N, int C) {
    if (!given(out) || !p) return false;
    return bytes_meet(out->data, 2ull * (batch_stride(out, B) * (B - 1ll) + token_stride(out, N) * (N - 1ll) + C), p, bytes);
}

static Tokens tokens(const norm_tokens* t, int B, int N) {
    return given(t) ? Tokens{(char*)t->data, 2 * batch_stride(t, B), 2 * token_stride(t, N)} : Tokens{nullptr, 0, 0};
}

static int check_vectors(const norm_vectors* v, int B, int C, int dtype) {
    if (!v || (dtype != NORM_F16 && dtype != NORM_BF16) || !isfinite(v->alpha) || !isfinite(v->eps) || v->eps < 0) return NORM_EINVAL;
    if ((uintptr_t)v->gate % 16 || (uintptr_t)v->post_weight % 16 || (uintptr_t)v->pre_weight % 16) return NORM_EINVAL;
    if (v->gate && (v->gate_stride < 0 || v->gate_stride % 8 || (v->gate_stride && v->gate_stride < C) || v->gate_stride > (1ll << 59) / B)) return NORM_EINVAL;
    return NORM_OK;
}
static bool by_sequence(const norm_vectors* v) { return v->gate && v->gate_stride; }
static unsigned long long gate_bytes(const norm_vectors* v, int B, int C) {
    return (by_sequence(v) ? v->gate_stride * (B - 1ull) + C : (unsigned long long)C) * (v->gate_f32 ? 4 : 2);
}

static int launch(const void* fn, dim3 grid, int threads, void* args, void* stream) {
    void* list[] = {args};
    if (hipLaunchKernel(fn, grid, dim3(threads), list, 0, (hipStream_t)stream) == hipSuccess) return NORM_OK;
    (void)hipGetLastError();
    return NORM_ELAUNCH;
}

// Units of a backward pass: as many workgroups as the card holds at once, and no more, for each has sums to be added (half as many, up to 4096 channels: 108.6 against
// 97.8 us on 2 x 4096 x 4096; 768 in place of 512 21.8 against 18.0 on 3 x 1001 x 1152).
struct Units {
    int runs, length, chunks, rows, blocks;
};
static Units units_of(int B, int N, int C, bool sequences) {
    const Kernel& k = choose(C);
    const int groups = groups_of(k.waves[1]);
    Units u;
    u.runs = sequences ? B : 1;
    u.length = sequences ? N : B * N;
    const int limit = k.most > 4096 ? 256 : 512, each = u.runs >= limit ? 1 : limit / u.runs;
    const long long most = ((long long)u.length + groups - 1) / groups, chunks = each < most ? each : most;
    u.rows = (int)((u.length + chunks - 1) / chunks + groups - 1) / groups * groups;
    u.chunks = (int)(((long long)u.length + u.rows - 1) / u.rows);
    const long long units = (long long)u.runs * u.chunks;
    u.blocks = (int)(units < limit ? units : limit);
    return u;
}

}  // namespace stream_norm

extern "C" {

int residual_norm(const norm_tokens* x, const norm_tokens* h, const norm_tokens* y, const norm_tokens* z, const norm_vectors* vectors, int B,
                  int N, int C, int dtype, void* stream) {
    using namespace stream_norm;
    if (const int rc = check_sizes(B, N, C)) return rc;
    if (const int rc = check_vectors(vectors, B, C, dtype)) return rc;
    const norm_vectors& v = *vectors;
    if (!given(x) || (!given(y) && !given(z)) || given(z) != (v.pre_weight != nullptr)) return NORM_EINVAL;
    if (!given(h) && (given(y) || v.gate || v.post_weight || v.alpha != 1.f)) return NORM_EINVAL;
    if (check_tokens(x, B, N, C, false) || check_tokens(h, B, N, C, false) || check_tokens(y, B, N, C, true) || check_tokens(z, B, N, C, true)) return NORM_EINVAL;
    const unsigned long long wide = (v.weight_f32 ? 4ull : 2ull) * C;
    for (const norm_tokens* out : {y, z})
        if (tokens_meet(out, x, true, B, N, C) || tokens_meet(out, h, true, B, N, C) || vector_meets(out, v.gate, v.gate ? gate_bytes(&v, B, C) : 0, B, N, C) ||
            vector_meets(out, v.post_weight, wide, B, N, C) || vector_meets(out, v.pre_weight, wide, B, N, C))
            return NORM_EINVAL;
    if (tokens_meet(y, z, false, B, N, C)) return NORM_EINVAL;
    const Kernel& k = choose(C);
    const int groups = groups_of(k.waves[0]);
    Args a = {};
    a.x = tokens(x, B, N), a.h = tokens(h, B, N), a.y = tokens(y, B, N), a.z = tokens(z, B, N);
    a.gate = v.gate, a.gate_stride = v.gate ? v.gate_stride : 0, a.gate_f32 = v.gate_f32, a.post = v.post_weight, a.pre = v.pre_weight, a.weight_f32 = v.weight_f32;
    a.N = N, a.C = C, a.runs = 1, a.length = B * N, a.alpha = v.alpha, a.eps = v.eps;
    // workgroups of one round each up to 2048, then longer runs of tokens
    const long long rounds = ((long long)a.length + groups - 1) / groups, blocks = rounds < 2048 ? rounds : 2048;
    a.rows = (int)((rounds + blocks - 1) / blocks) * groups;
    a.chunks = (int)(((long long)a.length + a.rows - 1) / a.rows);
    return launch(k.forward[dtype], dim3(a.chunks), 64 * k.waves[0] * groups, &a, stream);
}

long long residual_norm_bwd_workspace(int B, int N, int C, int sequences) {
    using namespace stream_norm;
    if (const int rc = check_sizes(B, N, C)) return rc;
    const Units u = units_of(B, N, C, sequences);
    return 4ll * C * (2ll * u.blocks + (sequences && u.chunks > 1 ? (long long)u.runs * u.chunks : 0));
}

int residual_norm_bwd(const norm_tokens* dy, const norm_tokens* dz, const norm_tokens* y, const norm_tokens* h, const norm_tokens* dx,
                      const norm_tokens* dh, const norm_vectors* vectors, float* dgate, float* dpost_weight, float* dpre_weight, int B, int N,
                      int C, int dtype, void* workspace, long long workspace_bytes, void* stream) {
    using namespace stream_norm;
    if (const int rc = check_sizes(B, N, C)) return rc;
    if (const int rc = check_vectors(vectors, B, C, dtype)) return rc;
    const norm_vectors& v = *vectors;
    const bool need_h = v.gate || v.post_weight, sequences = by_sequence(&v);
    if ((!given(dy) && !given(dz)) || (!given(dx) && !given(dh)) || given(dz) != (v.pre_weight != nullptr) || (given(dz) && !given(y)) || (need_h && !given(h)))
        return NORM_EINVAL;
    if ((dgate && !v.gate) || (dpost_weight && !v.post_weight) || (dpre_weight && !v.pre_weight)) return NORM_EINVAL;
    const norm_tokens* in[] = {dy, dz, given(dz) ? y : nullptr, need_h ? h : nullptr};
    for (const norm_tokens* t : in)
        if (check_tokens(t, B, N, C, false)) return NORM_EINVAL;
    if (check_tokens(dx, B, N, C, true) || check_tokens(dh, B, N, C, true)) return NORM_EINVAL;
    if ((uintptr_t)dgate % 16 || (uintptr_t)dpost_weight % 16 || (uintptr_t)dpre_weight % 16 || (uintptr_t)workspace % 16) return NORM_EINVAL;
    const Units u = units_of(B, N, C, sequences);
    const bool any = dgate || dpost_weight || dpre_weight;
    const long long need = any ? residual_norm_bwd_workspace(B, N, C, sequences) : 0;
    if (need && (!workspace || workspace_bytes < need)) return NORM_EINVAL;
    const unsigned long long wide = (v.weight_f32 ? 4ull : 2ull) * C;
    const struct { const void* p; unsigned long long bytes; bool written; } vectors_of[] = {
        {v.gate, v.gate ? gate_bytes(&v, B, C) : 0, false}, {v.post_weight, wide, false}, {v.pre_weight, wide, false},
        {dgate, 4ull * C * (sequences ? B : 1), true}, {dpost_weight, 4ull * C, true}, {dpre_weight, 4ull * C, true},
        {need ? workspace : nullptr, (unsigned long long)need, true}};
    for (const norm_tokens* out : {dx, dh}) {
        for (const norm_tokens* t : in)
            if (tokens_meet(out, t, true, B, N, C)) return NORM_EINVAL;
        for (const auto& t : vectors_of)
            if (vector_meets(out, t.p, t.bytes, B, N, C)) return NORM_EINVAL;
    }
    if (tokens_meet(dx, dh, false, B, N, C)) return NORM_EINVAL;
    for (int i = 3; i < 7; ++i) {
        for (int j = 0; j < i; ++j)
            if (bytes_meet(vectors_of[i].p, vectors_of[i].bytes, vectors_of[j].p, vectors_of[j].bytes)) return NORM_EINVAL;
        for (const norm_tokens* t : in)
            if (vector_meets(t, vectors_of[i].p, vectors_of[i].bytes, B, N, C)) return NORM_EINVAL;
    }
    const Kernel& k = choose(C);
    Args a = {};
    a.dy = tokens(dy, B, N), a.dz = tokens(dz, B, N), a.dx = tokens(dx, B, N), a.dh = tokens(dh, B, N);
    if (given(dz)) a.y = tokens(y, B, N);
    if (need_h) a.h = tokens(h, B, N);
    a.gate = v.gate, a.gate_stride = v.gate ? v.gate_stride : 0, a.gate_f32 = v.gate_f32, a.post = v.post_weight, a.pre = v.pre_weight, a.weight_f32 = v.weight_f32;
    a.N = N, a.C = C, a.runs = u.runs, a.length = u.length, a.chunks = u.chunks, a.rows = u.rows, a.alpha = v.alpha, a.eps = v.eps;
    if (any) a.sums = (float*)workspace;
    float* const units = sequences && u.chunks > 1 ? (float*)workspace + 2ll * u.blocks * C : nullptr;
    if (sequences && dgate) a.units = units ? units : dgate;
    if (const int rc = launch(k.backward[dtype], dim3(u.blocks), 64 * k.waves[1] * groups_of(k.waves[1]), &a, stream)) return rc;
    if (!any) return NORM_OK;
    SumArgs s = {(float*)workspace, units, v.gate, v.post_weight, dgate, dpost_weight, dpre_weight, v.gate_f32, v.weight_f32, u.blocks, u.chunks, C, sequences};
    const int jobs = units && dgate ? 2 + B : 2;
    return launch(dtype ? (const void*)vector_sum_kernel<true> : (const void*)vector_sum_kernel<false>, dim3((C + 31) / 32, jobs), 1024, &s, stream);
}

const char* norm_strerror(int code) {
    switch (code) {
        case NORM_OK: return "ok";
        case NORM_EINVAL: return "invalid argument";
        case NORM_EUNSUPPORTED: return "unsupported size";
        case NORM_ELAUNCH: return "the HIP runtime refused the launch";
        default: return "unknown error";
    }
}

}  // extern "C"
