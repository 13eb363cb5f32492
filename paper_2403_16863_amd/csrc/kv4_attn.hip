// Attention over the paged 4-bit cache (include/kv4.h has the operation and the format).
//
// A workgroup takes RB = 16 NT rows (query i and head of the group: row = i * group + head) of one sequence and one head of the
// cache over a run of keys, and goes once over them with the running maximum and sum of the softmax.  Its four waves take
// turns at tiles of 32 keys, each with statistics and an output of its own; they meet at the end.  Tiles stay in
// registers: a lane's 16 bytes of key codes are one token's block of 32 channels under one scale, which is also what the
// 16 x 16 x 32 MFMA wants as rows of its first operand once the channels are taken in this order on both sides; the conversion
// instruction takes two codes and their scale to two binary16 values, exactly, at the rate of any other vector instruction.
//     S^T (16 tokens x 16 rows) = K Q^T:  lane l has row l % 16 of Q and tokens 4 (l / 16) .. + 3
//     O^T (16 channels x 16 rows) += V^T P^T: the second operand is P as S^T leaves it, so lane l's tokens are 4 (l / 16) .. + 3 of
//     each of two groups of 16, and the cache holds the values in quads of tokens for that reason.
// All values of the cache are exact in binary16, so one kernel serves both types: bfloat16 queries become binary16 relative to
// the power of two of their row's largest element.
//
// The keys of all sequences are dealt on the device, from the lengths that the launch finds in memory (a captured launch meets new ones
// at every replay): `plan` picks the tiles of a run so that all runs together are about `target`, and a second kernel joins the runs of a row.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/kv4.h"
#include "kv4_format.h"

namespace kv4 {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const uint16_t* q;
    const uint8_t* cache;
    const int *tables, *lens, *cu_q;
    uint16_t* out;
    float* lse;
    float* ws;  // partial outputs, then maxima and sums; null: no runs, each workgroup takes all keys
    int T, B, H, heads, group, pages, page_shift, width, max_q, causal;
    float scale_l2;  // scale * log2(e)
    int target;      // runs that the launch is to be cut into
};

constexpr int kTile = 32;     // keys of a step of one wave
constexpr int kMinTiles = 4;  // a run's tiles at least: one for each wave
constexpr float kRaise = 8;   // scores (in powers of two) by which a row may pass its reference before that is raised: P < 2^8 in binary16

struct Sequence {
    int len, q0, nq;
};

__device__ __forceinline__ Sequence sequence(const AttnArgs& a, int b) {
    Sequence s;
    s.len = min(max(a.lens[b], 0), a.width << a.page_shift);
    if (a.cu_q) {
        s.q0 = min(max(a.cu_q[b], 0), a.T);
        s.nq = min(min(max(a.cu_q[b + 1], s.q0), a.T) - s.q0, a.max_q);
    } else {
        s.nq = a.max_q;
        s.q0 = b * s.nq;
    }
    return s;
}

// The same for a sequence that all lanes share: what follows from it stays in scalar registers.
__device__ __forceinline__ Sequence shared_sequence(const AttnArgs& a, int b) {
    Sequence s = sequence(a, b);
    s.len = __builtin_amdgcn_readfirstlane(s.len), s.q0 = __builtin_amdgcn_readfirstlane(s.q0), s.nq = __builtin_amdgcn_readfirstlane(s.nq);
    return s;
}

__device__ __forceinline__ int wave_sum_scan(int x) {  // inclusive prefix sum over the 64 lanes
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

template <int RB>
__device__ __forceinline__ int blocks_of(const AttnArgs& a, const Sequence& s) {
    return (s.nq * a.group + RB - 1) / RB;
}
__device__ __forceinline__ int tiles_of(const Sequence& s) { return (s.len + kTile - 1) / kTile; }
__device__ __forceinline__ int runs_of(int tiles, int run) { return max(1, (tiles + run - 1) / run); }

// Tiles of a run: all (sequence, row block, head) together make about `target` runs, none shorter than kMinTiles.
template <int RB>
__device__ __forceinline__ int plan(const AttnArgs& a) {
    if (!a.ws) return INT_MAX / 2;  // no runs
    const int lane = threadIdx.x & 63;
    long long all = 0;
    for (int b = lane; b < a.B; b += 64) {
        const Sequence s = sequence(a, b);
        all += (long long)tiles_of(s) * blocks_of<RB>(a, s);
    }
#pragma unroll
    for (int d = 32; d; d /= 2) all += __shfl_xor(all, d);
    return (int)max((long long)kMinTiles, (all * a.heads + a.target - 1) / a.target);
}

// The sequence that item `id` of the launch belongs to, and the id of that sequence's first item; false: there is no such item.
template <int RB>
__device__ __forceinline__ bool find_item(const AttnArgs& a, int run, long long id, int& b, long long& first) {
    const int lane = threadIdx.x & 63;
    long long before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int n = 0;
        if (b0 + lane < a.B) {
            const Sequence s = sequence(a, b0 + lane);
            n = s.nq ? runs_of(tiles_of(s), run) * blocks_of<RB>(a, s) * a.heads : 0;
        }
        const int upto = wave_sum_scan(n);
        const unsigned long long past = __ballot(before + upto > id);
        if (past) {
            const int l = __ffsll(past) - 1;
            b = b0 + l;
            first = before + __shfl(upto, l) - __shfl(n, l);
            return true;
        }
        before += __shfl(upto, 63);
    }
    return false;
}

// Of sequence b alone: the id of its first item.
template <int RB>
__device__ __forceinline__ long long first_item(const AttnArgs& a, int run, int b) {
    const int lane = threadIdx.x & 63;
    long long n = 0;
    for (int i = lane; i < b; i += 64) {
        const Sequence s = sequence(a, i);
        n += s.nq ? runs_of(tiles_of(s), run) * blocks_of<RB>(a, s) * a.heads : 0;
    }
#pragma unroll
    for (int d = 32; d; d /= 2) n += __shfl_xor(n, d);
    return n;
}

// Keys that row `row` of a sequence sees: those below the result.
__device__ __forceinline__ int keys_of(const AttnArgs& a, const Sequence& s, int row) {
    return a.causal ? max(0, s.len - s.nq + row / a.group + 1) : s.len;
}

// One tile's bytes of one lane: [group of 16 tokens][words].
template <int D>
struct Raw {
    unsigned k[2][D / 32], v[2][D / 32];
    unsigned ks[2], vs[2];
};

// Indices that the launch only reads, through the scalar cache.
typedef const int __attribute__((address_space(4))) * const_ints;

template <int D, int NT, int NW, bool BF>
__global__ __launch_bounds__(64 * NW, NW / 4 * (NT == 1 ? 4 : NT == 2 ? 2 : 1)) void attn_kernel(AttnArgs a) {
    constexpr int RB = 16 * NT, KS = D / 32, CT = D / 16, W = D / 32;
    __shared__ float joined[NW / 2][CT * NT][64 * 4];
    __shared__ float stats[NW][RB][2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;

    const int run = __builtin_amdgcn_readfirstlane(plan<RB>(a));
    int b = 0;
    long long first = 0;
    const long long id = blockIdx.x;
    if (!find_item<RB>(a, run, id, b, first)) return;
    b = __builtin_amdgcn_readfirstlane(b);
    const Sequence s = shared_sequence(a, b);
    const int rbs = blocks_of<RB>(a, s);
    int rest = __builtin_amdgcn_readfirstlane((int)(id - first));
    const int h = rest % a.heads;
    rest /= a.heads;
    const int rb = rest % rbs, r = rest / rbs;
    const int rows = s.nq * a.group, row0 = rb * RB;
    const int most = keys_of(a, s, min(row0 + RB, rows) - 1), least = keys_of(a, s, row0);  // over the block's rows
    const int tiles = (most + kTile - 1) / kTile, runs = runs_of(tiles, run);
    if (r >= runs) return;  // these rows see fewer keys than the sequence has
    const int t0 = r * run, t1 = min(tiles, t0 + run);

    const const_ints table = (const_ints)(uintptr_t)(a.tables + (long long)b * a.width);
    const int groups_page = 1 << (a.page_shift - 4);
    // Group g's (16 tokens') page; groups behind the last one stand for that one (their keys are masked).
    const int last_group = max(0, (most + 15) / 16 - 1);
    auto page_of = [&](int g) { return table[min(g, last_group) >> (a.page_shift - 4)]; };
    auto group_at = [&](int g, int page) {
        const int p = (unsigned)page < (unsigned)a.pages ? page : 0;
        return a.cache + (((long long)p * a.heads + h) * groups_page + (min(g, last_group) & (groups_page - 1))) * Group<D>::bytes;
    };
    Raw<D> raw;
    auto fetch_k = [&](const uint8_t* at, int i) {
        const unsigned* k = (const unsigned*)(at + col * (D / 2) + quad * (D / 8));
#pragma unroll
        for (int w = 0; w < W; ++w) raw.k[i][w] = k[w];
        raw.ks[i] = at[Group<D>::k_scales + col * (D / 32) + quad * (D / 4) / 32];
    };
    auto fetch_v = [&](const uint8_t* at, int i) {
        const unsigned* v = (const unsigned*)(at + Group<D>::v_codes + quad * (2 * D) + col * (D / 8));
#pragma unroll
        for (int w = 0; w < W; ++w) raw.v[i][w] = v[w];
        raw.vs[i] = *(const unsigned*)(at + Group<D>::v_scales + quad * (D / 8) + col * (D / 16) / 32 * 4);
    };
    // The first tile's bytes, and the pages of the second, are under way before the queries are asked for.
    int t = t0 + wave, pages[2] = {-1, -1}, ahead[2] = {-1, -1};
    if (t < t1) {
        for (int i = 0; i < 2; ++i) pages[i] = page_of(2 * t + i), ahead[i] = page_of(2 * (t + NW) + i);
        for (int i = 0; i < 2; ++i) fetch_k(group_at(2 * t + i, pages[i]), i);
        for (int i = 0; i < 2; ++i) fetch_v(group_at(2 * t + i, pages[i]), i);
    }

    // Queries: row col of tile n, channels quad * D/4 + 8 ks .. + 7.
    f16x8 q[NT][KS];
    float factor[NT];  // scores to powers of two
    int limit[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 16 * n + col;
        const bool there = row < rows;
        limit[n] = there ? keys_of(a, s, row) : 0;
        const long long at = ((long long)(s.q0 + (there ? row / a.group : 0)) * a.H + h * a.group + (there ? row % a.group : 0)) * D + quad * (D / 4);
        factor[n] = a.scale_l2;
        float x[KS][8], top = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            load8<BF>(a.q + at + 8 * k, x[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[k][i]));
        }
        int e = 0;
        if (BF) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (top > 0 && top < INFINITY) e = ilogbf(top);
            factor[n] *= ldexpf(1.f, e);
        }
        if (top == INFINITY) x[0][0] = __uint_as_float(0x7fc00000u);  // an infinity among the scores would hide where all of them are -inf
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[n][k][i] = (_Float16)(BF ? ldexpf(x[k][i], -e) : x[k][i]);
    }

    f32x4 o[NT][CT];
    float m[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = -INFINITY, l[n] = 0;
#pragma unroll
        for (int c = 0; c < CT; ++c) o[n][c] = {0, 0, 0, 0};
    }

    for (; t < t1; t += NW) {
        const bool there[2] = {(unsigned)pages[0] < (unsigned)a.pages, (unsigned)pages[1] < (unsigned)a.pages};
        const bool masked = (t + 1) * kTile > least || !there[0] || !there[1];

        float x[NT][8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x4 acc[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n] = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const uint4 w = values8<false>(raw.k[i][k], raw.ks[i] << 23);
                const f16x8 f = __builtin_bit_cast(f16x8, w);
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, q[n][k], acc[n], 0, 0, 0);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[n][4 * i + j] = acc[n][j] * factor[n];
        }
        // The next tile's keys take the registers of this one's (behind the run's end: the last group's once more).
        const uint8_t* next[2];
        for (int i = 0; i < 2; ++i) {
            pages[i] = ahead[i];
            next[i] = group_at(2 * (t + NW) + i, pages[i]);
            fetch_k(next[i], i);
            ahead[i] = page_of(2 * (t + 2 * NW) + i);
        }
        if (masked) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = t * kTile + 16 * i + 4 * quad + j;
                    // Values that some row of the block does not see must not reach it as 0 * NaN: a NaN among them goes into the
                    // scores of the rows that do see it, and the codes that nobody sees are cleared with it.
                    const unsigned byte = raw.vs[i] << (24 - 8 * j) >> 24;
                    const unsigned long long bad = __ballot(byte == 255u);
                    const bool nan = (bad >> (16 * quad) & 0xffffu) != 0;
                    const bool dead = nan || key >= most || !there[i];
                    if (dead) {
                        if (D == 128) raw.v[i][j % W] = 0;
                        else raw.v[i][j / 2] &= j % 2 ? 0xffffu : 0xffff0000u;
                        raw.vs[i] = (raw.vs[i] & ~(0xffu << (8 * j))) | 127u << (8 * j);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if (key >= limit[n] || !there[i]) x[n][4 * i + j] = -INFINITY;
                        else if (nan) x[n][4 * i + j] = __uint_as_float(0x7fc00000u);
                    }
                }
        }
        f16x8 p[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = x[n][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) top = fmaxf(top, x[n][j]);
            if (__any(top > m[n] + kRaise)) {  // all four lanes of a row take the same reference
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float to = fmaxf(m[n], top);
                const float by = to == m[n] ? 1.f : __builtin_amdgcn_exp2f(m[n] - to);
                m[n] = to;
                l[n] *= by;
#pragma unroll
                for (int c = 0; c < CT; ++c) o[n][c] *= by;
            }
            const float ref = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = __builtin_amdgcn_exp2f(x[n][j] - ref);
                l[n] += e;
                p[n][j] = (_Float16)e;
            }
        }
        // Values: pairs of channels of one token become pairs of tokens of one channel.
        unsigned sc[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            sc[i][0] = raw.vs[i] << 23, sc[i][1] = raw.vs[i] << 15, sc[i][2] = raw.vs[i] << 7, sc[i][3] = raw.vs[i] >> 1;
        }
        auto channels = [&](auto SEL) {
            constexpr int c = decltype(SEL)::value;  // channels 2c and 2c + 1 of the lane's run
            unsigned two[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if constexpr (D == 128) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) two[i][j] = values2<false, c>(raw.v[i][j % W], sc[i][j]);
                } else {
                    two[i][0] = values2<false, c>(raw.v[i][0], sc[i][0]);
                    two[i][1] = values2<false, 2 + c>(raw.v[i][0], sc[i][1]);
                    two[i][2] = values2<false, c>(raw.v[i][1], sc[i][2]);
                    two[i][3] = values2<false, 2 + c>(raw.v[i][1], sc[i][3]);
                }
            }
            uint4 even, odd;
            even.x = __builtin_amdgcn_perm(two[0][1], two[0][0], 0x05040100u), odd.x = __builtin_amdgcn_perm(two[0][1], two[0][0], 0x07060302u);
            even.y = __builtin_amdgcn_perm(two[0][3], two[0][2], 0x05040100u), odd.y = __builtin_amdgcn_perm(two[0][3], two[0][2], 0x07060302u);
            even.z = __builtin_amdgcn_perm(two[1][1], two[1][0], 0x05040100u), odd.z = __builtin_amdgcn_perm(two[1][1], two[1][0], 0x07060302u);
            even.w = __builtin_amdgcn_perm(two[1][3], two[1][2], 0x05040100u), odd.w = __builtin_amdgcn_perm(two[1][3], two[1][2], 0x07060302u);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                o[n][2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, even), p[n], o[n][2 * c], 0, 0, 0);
                o[n][2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, odd), p[n], o[n][2 * c + 1], 0, 0, 0);
            }
            if (NT == 1) __builtin_amdgcn_sched_barrier(0);  // a few channels at a time: all of them at once would not fit 128 registers
        };
        channels(std::integral_constant<int, 0>());
        channels(std::integral_constant<int, 1>());
        if constexpr (D == 128) {
            channels(std::integral_constant<int, 2>());
            channels(std::integral_constant<int, 3>());
        }
        for (int i = 0; i < 2; ++i) fetch_v(next[i], i);
    }

    // The waves meet: a common reference for each row, then the upper half's outputs go to the lower half, until one is left.
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (quad == 0) stats[wave][16 * n + col][0] = m[n], stats[wave][16 * n + col][1] = l[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float top = -INFINITY, sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, stats[w][16 * n + col][0]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += stats[w][16 * n + col][1] * __builtin_amdgcn_exp2f(stats[w][16 * n + col][0] - ref);
        const float by = __builtin_amdgcn_exp2f(m[n] - ref);
        m[n] = top, l[n] = sum;
#pragma unroll
        for (int c = 0; c < CT; ++c) o[n][c] *= by;
    }
#pragma unroll
    for (int half = NW / 2; half; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < CT; ++c) *(f32x4*)&joined[wave - half][n * CT + c][4 * lane] = o[n][c];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < CT; ++c) o[n][c] += *(const f32x4*)&joined[wave][n * CT + c][4 * lane];
        if (half > 1) __syncthreads();
    }
    if (wave) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 16 * n + col;
        if (row >= rows) continue;
        if (runs == 1) {
            const float by = l[n] == 0.f ? 0.f : 1.f / l[n];
            const long long vec = (long long)(s.q0 + row / a.group) * a.H + h * a.group + row % a.group;
            if (quad == 0) a.lse[vec] = l[n] == 0.f ? -INFINITY : (m[n] + __builtin_amdgcn_logf(l[n])) * 0.6931471805599453f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unsigned w[CT / 2];
#pragma unroll
                for (int c = 0; c < CT / 2; ++c) w[c] = pack2<BF>(o[n][2 * c][j] * by, o[n][2 * c + 1][j] * by);
                unsigned* to = (unsigned*)(a.out + vec * D + (4 * quad + j) * CT);
#pragma unroll
                for (int c = 0; c < CT / 2; ++c) to[c] = w[c];
            }
        } else {
            float* to = a.ws + ((id * RB) + 16 * n + col) * (D + 2);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < CT; ++c) to[(4 * quad + j) * CT + c] = o[n][c][j];
            if (quad == 0) to[D] = m[n], to[D + 1] = l[n];
        }
    }
}

// WAVES waves join the runs of one row (query, head): a lane has one run's maximum and sum, then the weighted outputs are added, eight runs'
// loads at a time (one run after another took 75 us for rows of 128 runs).
template <int D, int RB, bool BF, int WAVES>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a) {
    constexpr int C = D / 64;
    __shared__ float part[WAVES > 1 ? 4 : 1][D + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = wave % WAVES;
    const long long vec = (long long)blockIdx.x * (4 / WAVES) + wave / WAVES;
    if (vec >= (long long)a.T * a.H) return;
    const int t = (int)(vec / a.H), head = (int)(vec % a.H), h = head / a.group;
    int b;
    if (a.cu_q) {  // the sequence with cu_q[b] <= t < cu_q[b + 1]
        int upto = 0;
        for (int i = lane; i < a.B; i += 64) upto += a.cu_q[i + 1] <= t;
#pragma unroll
        for (int d = 32; d; d /= 2) upto += __shfl_xor(upto, d);
        b = __builtin_amdgcn_readfirstlane(upto);
        if (b >= a.B || t < a.cu_q[b]) return;
    } else {
        b = t / a.max_q;
    }
    const int run = __builtin_amdgcn_readfirstlane(plan<RB>(a));
    const Sequence s = shared_sequence(a, b);
    if (t - s.q0 >= s.nq) return;
    const int row = (t - s.q0) * a.group + head % a.group, rb = row / RB, rows = s.nq * a.group;
    const int most = keys_of(a, s, min((rb + 1) * RB, rows) - 1);
    const int runs = runs_of((most + kTile - 1) / kTile, run);
    if (runs == 1) return;
    const int rbs = blocks_of<RB>(a, s);
    const long long id = first_item<RB>(a, run, b) + (long long)rb * a.heads + h, step = (long long)rbs * a.heads * RB * (D + 2);
    const float* from = a.ws + (id * RB + row % RB) * (D + 2);
    // Lane l has run r0 + WAVES l: its reference is raised for 64 runs at a time.
    float top = -INFINITY, sum = 0, o[C] = {};
    for (int r0 = mine; r0 < runs; r0 += 64 * WAVES) {
        const int r = r0 + WAVES * lane;
        float m = -INFINITY, l = 0;
        if (r < runs) m = from[r * step + D], l = from[r * step + D + 1];
        float to = m;
#pragma unroll
        for (int d = 32; d; d /= 2) to = fmaxf(to, __shfl_xor(to, d));
        to = fmaxf(to, top);
        const float ref = to == -INFINITY ? 0.f : to, by = __builtin_amdgcn_exp2f(top - ref);
        const float weight = __builtin_amdgcn_exp2f(m - ref);
        top = to;
        sum = sum * by + weight * l;  // each lane's own runs
        for (int i = 0; i < C; ++i) o[i] *= by;
        const int n = min(64, (runs - r0 + WAVES - 1) / WAVES);
        for (int k = 0; k < n; k += 8) {
            float x[8][C];
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int i = 0; i < C; ++i) x[u][i] = from[(r0 + WAVES * min(k + u, n - 1)) * step + lane * C + i];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float w = __shfl(weight, min(k + u, n - 1));
#pragma unroll
                for (int i = 0; i < C; ++i)
                    if (k + u < n) o[i] += x[u][i] * w;
            }
        }
    }
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if constexpr (WAVES > 1) {
#pragma unroll
        for (int i = 0; i < C; ++i) part[wave][lane * C + i] = o[i];
        if (lane == 0) part[wave][D] = top, part[wave][D + 1] = sum;
        __syncthreads();
        if (wave) return;
        top = -INFINITY;
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, part[w][D]);
        const float ref = top == -INFINITY ? 0.f : top;
        sum = 0;
        for (int i = 0; i < C; ++i) o[i] = 0;
        for (int w = 0; w < WAVES; ++w) {
            const float by = __builtin_amdgcn_exp2f(part[w][D] - ref);
            sum += part[w][D + 1] * by;
            for (int i = 0; i < C; ++i) o[i] += part[w][lane * C + i] * by;
        }
    }
    const float by = sum == 0.f ? 0.f : 1.f / sum;
    if (lane == 0) a.lse[vec] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    if (D == 128) {
        *(unsigned*)(a.out + vec * D + 2 * lane) = pack2<BF>(o[0] * by, o[C - 1] * by);
    } else {
        a.out[vec * D + lane] = (uint16_t)pack2<BF>(o[0] * by, 0.f);
    }
}

struct Choice {
    int nt, nw, target;
    long long blocks, bytes;
};

constexpr int kShort = 2048;   // keys
constexpr int kTarget = 1024;  // runs of a launch: four workgroups on each of 256 units

Choice choose(int B, int heads, int group, int d, long long cap, int max_q) {
    const long long rows = (long long)group * max_q;
    Choice c;
    c.nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    c.target = kTarget;
    const long long rbs = (rows + 16 * c.nt - 1) / (16 * c.nt), alone = B * rbs * heads;
    // Sequences that cannot be long are not cut: 16 waves go over up to four tiles each, and there is nothing to join.
    const bool one = cap <= kShort;
    c.nw = one && c.nt == 1 ? 16 : 4;
    c.blocks = one ? alone : alone + c.target;
    c.bytes = one ? 0 : c.blocks * 16 * c.nt * (d + 2) * 4;
    return c;
}

int check_sizes(int B, int H, int heads, int d, int page_size, int width, int max_q) {
    if (B < 1 || heads < 1 || H < heads || H % heads || width < 1 || max_q < 1) return KV4_EINVAL;
    if (page_size < 16 || page_size > 65536 || (page_size & (page_size - 1))) return KV4_EINVAL;
    if (d != 64 && d != 128) return KV4_EUNSUPPORTED;
    if ((long long)width * page_size > INT_MAX || (long long)(H / heads) * max_q > 1 << 30 || B > 65535) return KV4_EUNSUPPORTED;
    return choose(B, heads, H / heads, d, (long long)width * page_size, max_q).blocks >= 1 << 23 ? KV4_EUNSUPPORTED : KV4_OK;
}

template <int D, bool BF>
int launch_attn(const Choice& c, AttnArgs& a, void* stream) {
    const void* fn = c.nw == 16  ? (const void*)attn_kernel<D, 1, 16, BF>
                     : c.nt == 1 ? (const void*)attn_kernel<D, 1, 4, BF>
                     : c.nt == 2 ? (const void*)attn_kernel<D, 2, 4, BF>
                                 : (const void*)attn_kernel<D, 4, 4, BF>;
    // Rows enough to fill the units get a wave each, fewer ones a workgroup: those are the rows with many runs.
    const long long rows = (long long)a.T * a.H;
    const bool many = rows >= 4096;
    const void* join = c.nt == 1   ? (many ? (const void*)join_kernel<D, 16, BF, 1> : (const void*)join_kernel<D, 16, BF, 4>)
                       : c.nt == 2 ? (many ? (const void*)join_kernel<D, 32, BF, 1> : (const void*)join_kernel<D, 32, BF, 4>)
                                   : (many ? (const void*)join_kernel<D, 64, BF, 1> : (const void*)join_kernel<D, 64, BF, 4>);
    void* list[] = {&a};
    if (hipLaunchKernel(fn, dim3((unsigned)c.blocks), dim3(64 * c.nw), list, 0, (hipStream_t)stream) != hipSuccess ||
        (a.ws && hipLaunchKernel(join, dim3((unsigned)(many ? (rows + 3) / 4 : rows)), dim3(256), list, 0, (hipStream_t)stream) != hipSuccess)) {
        (void)hipGetLastError();
        return KV4_ELAUNCH;
    }
    return KV4_OK;
}

bool overlap(const void* a, long long an, const void* b, long long bn) {
    return (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}

}  // namespace kv4

extern "C" {

int kv4_attn(const void* q, const void* cache, const int* tables, const int* lens, const int* cu_q, void* out, float* lse, int T,
             int B, int H, int heads, int d, int pages, int page_size, int width, int max_q, int causal, float scale, int dtype,
             void* workspace, long long workspace_bytes, void* stream) {
    using namespace kv4;
    if (!q || !cache || !tables || !lens || !out || !lse || T < 0 || pages < 1) return KV4_EINVAL;
    if ((uintptr_t)q % 16 || (uintptr_t)cache % 16 || (uintptr_t)out % 16 || (uintptr_t)workspace % 16) return KV4_EINVAL;
    if ((uintptr_t)tables % 4 || (uintptr_t)lens % 4 || (uintptr_t)cu_q % 4 || (uintptr_t)lse % 4) return KV4_EINVAL;
    if ((dtype != KV4_F16 && dtype != KV4_BF16) || !isfinite(scale)) return KV4_EINVAL;
    if (T == 0 && B >= 1) return KV4_OK;
    if (!cu_q && (B < 1 || T % B || max_q != T / B)) return KV4_EINVAL;
    if (const int rc = check_sizes(B, H, heads, d, page_size, width, max_q)) return rc;
    if ((long long)pages * page_size > INT_MAX || (long long)T * H > INT_MAX) return KV4_EUNSUPPORTED;
    const long long bytes = (long long)T * H * d * 2;
    if (overlap(q, bytes, out, bytes) || overlap(lse, (long long)T * H * 4, out, bytes)) return KV4_EINVAL;
    const Choice c = choose(B, heads, H / heads, d, (long long)width * page_size, max_q);
    const bool cut = c.bytes && workspace && workspace_bytes >= c.bytes;
    AttnArgs a = {(const uint16_t*)q, (const uint8_t*)cache, tables, lens, cu_q, (uint16_t*)out, lse, cut ? (float*)workspace : nullptr,
                  T, B, H, heads, H / heads, pages, __builtin_ctz(page_size), width, max_q, causal, scale * 1.4426950408889634f, c.target};
    if (d == 128) return dtype ? launch_attn<128, true>(c, a, stream) : launch_attn<128, false>(c, a, stream);
    return dtype ? launch_attn<64, true>(c, a, stream) : launch_attn<64, false>(c, a, stream);
}

long long kv4_attn_workspace(int B, int H, int heads, int d, int page_size, int width, int max_q) {
    using namespace kv4;
    if (const int rc = check_sizes(B, H, heads, d, page_size, width, max_q)) return rc;
    return choose(B, heads, H / heads, d, (long long)width * page_size, max_q).bytes;
}

}  // extern "C"
