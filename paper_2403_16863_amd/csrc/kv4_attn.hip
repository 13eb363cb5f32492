// Attention over the paged 4-bit cache (include/kv4.h has the operation and the format).
//
// Rows (query i and head of the group: row = i * group + head) of one sequence and one head of the cache share its keys, and a workgroup
// goes once over a run of them with the running maximum and sum of the softmax.  There are two forms.
//
// Up to 32 rows (`segment`): 16 or 32 rows a workgroup, whose waves take turns at tiles of 32 keys, each with statistics and an
// output of its own; they meet at the end.  Tiles stay in registers: a lane's 16 bytes of key codes are one token's block of 32 channels under one
// scale, which is also what the 16 x 16 x 32 MFMA wants as rows of its first operand once the channels are taken in this order on both
// sides; the conversion instruction takes two codes and their scale to two binary16 values, exactly, at the rate of any other vector
// instruction (2.1 ns a wave on each of four units).
//     S^T (16 tokens x 16 rows) = K Q^T:  lane l has row l % 16 of Q and tokens 4 (l / 16) .. + 3
//     O^T (16 channels x 16 rows) += V^T P^T: the second operand is P as S^T leaves it, so lane l's tokens are 4 (l / 16) .. + 3 of
//     each of two groups of 16, and the cache holds the values in quads of tokens for that reason.
// Memory binds long calls: the loop reads 6.3 TB/s (64 sequences of up to 8192 keys); a launch's beginnings, ends and second kernel are the rest.
// More rows (`wide_segment`): 128 or 256 a workgroup, tiles of 64 keys converted once into LDS, the next tile's scores multiplied during this one's
// softmax.  The card's power binds it (1050 to 1100 TFLOP/s, by the card, for 2048 queries behind 14336 keys, 32 heads on 8, d = 128): its matrix instructions run at 2500
// TFLOP/s on constant data, on random data at 1700, and at 1390 with a read of LDS, an exponential and four more vector instructions to each.
//
// All values of the cache are exact in binary16, so one kernel serves both types: bfloat16 queries become binary16 relative to
// the power of two of their row's largest element.  (The MFMA that takes the codes and scales themselves, with the queries as
// sums of e4m3 terms, has sums that are off by 4e-5 of sum |q k|: too far for scores.)
//
// The keys of all sequences are dealt on the device, from the lengths that the launch finds in memory (a captured launch meets new ones
// at every replay).  A segment is a sequence, a block of rows and a head; all segments' tiles on end are cut into ranges of one length, one for
// each workgroup, wherever that falls, so that workgroups end together however unequal the sequences are; a second
// kernel joins the pieces of a row.  Where no sequence is long, workgroups take whole segments instead.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/kv4.h"
#include "kv4_format.h"

namespace kv4 {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct AttnArgs {
    const uint16_t* q;
    const uint8_t* cache;
    const int *tables, *lens, *cu_q;
    uint16_t* out;
    float* lse;
    int2* heads_ws;  // of each row: its first piece's row in ws, its pieces; null: no scratch memory, whole segments only
    float* ws;       // pieces' rows: output, maximum, sum
    int T, B, H, heads, group, pages, page_shift, width, max_q, causal;
    float scale_l2;  // scale * log2(e)
    int target;      // ranges that a launch is cut into at most
};

constexpr int kTile = 32;    // keys of a step of one wave
// A row's reference lies kRoom powers of two below its largest score when it was last raised, and is raised when a score passes it by more than
// kRaise: P, in binary16, is 2^7 for the largest key and below 2^15 for any, so that what is rounded in steps of 2^-24 (P below 2^-14) is 21 powers of
// two below the largest key's (with kRoom = 0, 14: many keys that far below a few could lose all they add up to).
constexpr float kRaise = 15, kRoom = 7;

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

// Inclusive prefix sum over the 64 lanes, in the rows of 16 first.
__device__ __forceinline__ int prefix_sum(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

template <int RB>
__device__ __forceinline__ int blocks_of(const AttnArgs& a, const Sequence& s) {
    return (s.nq * a.group + RB - 1) / RB;
}
// Positions of a segment: F::begin and then its tiles; one without keys has its rows to write and counts as one tile.
template <class F>
__device__ __forceinline__ int positions_of(const Sequence& s) { return F::begin + max(1, (s.len + F::tile - 1) / F::tile); }

// Where a workgroup begins.
struct Start {
    int range;   // tiles of a range; 0: whole segments
    int b;       // the sequence
    int first;   // position of its first segment
    int total;   // positions of all
    Sequence s;
};

template <class F>
__device__ __forceinline__ bool start_of(const AttnArgs& a, int id, Start& at) {
    const int lane = threadIdx.x & 63;
    int all = 0, longest = 0, segments = 0, tiles = 0;
    Sequence s = {};
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        segments = tiles = 0;
        if (b0 + lane < a.B) {
            s = sequence(a, b0 + lane);
            segments = blocks_of<F::rows>(a, s) * a.heads;
            tiles = segments ? positions_of<F>(s) : 0;
        }
        all += segments * tiles;
        longest = max(longest, tiles);
    }
    const bool whole = !a.ws || !__any(longest > F::begin + F::whole);
    const int W = __builtin_amdgcn_readlane(prefix_sum(all), 63);
    at.range = whole ? 0 : max(F::least, (W + a.target - 1) / a.target);
    if (!whole && id >= a.target) return false;
    const int pos = whole ? id : id * at.range;
    at.first = 0;
    if (whole && a.B > 1 && a.B <= 64) {
        // Layer by layer: the last row blocks of all sequences, which see the most keys, then those before them.
        const int blocks = segments / a.heads;
        auto before = [&](int layer) { return __builtin_amdgcn_readlane(prefix_sum(min(blocks, layer)), 63) * a.heads; };
        int layer = 0, most = (a.max_q * a.group + F::rows - 1) / F::rows;
        if (id >= before(most)) return false;
        while (most - layer > 1) {  // before(layer) <= id < before(most)
            const int mid = (layer + most) / 2;
            (before(mid) <= id ? layer : most) = mid;
        }
        const int k = (id - before(layer)) / a.heads;
        const unsigned long long in = __ballot(blocks > layer);
        const int mine = __builtin_amdgcn_mbcnt_hi((unsigned)(in >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)in, 0));
        const int l = __builtin_ctzll(__ballot(blocks > layer && mine == k));
        at.b = l;
        at.first = id - (layer * a.heads + (id - before(layer)) % a.heads);
        at.s = {__builtin_amdgcn_readlane(s.len, l), __builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.nq, l)};
        return true;
    }
    for (int b0 = 0;; b0 += 64) {
        if (a.B > 64) {
            if (b0 >= a.B) return false;
            segments = tiles = 0;
            if (b0 + lane < a.B) {
                s = sequence(a, b0 + lane);
                segments = blocks_of<F::rows>(a, s) * a.heads;
                tiles = segments ? positions_of<F>(s) : 0;
            }
        }
        const int mine = whole ? segments : segments * tiles;
        const int upto = prefix_sum(mine);
        const unsigned long long past = __ballot(at.first + upto > pos);
        if (past) {
            const int l = __builtin_ctzll(past);
            at.b = b0 + l;
            at.first += __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l);
            at.total = whole ? pos + 1 : W;
            at.s = {__builtin_amdgcn_readlane(s.len, l), __builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.nq, l)};
            return true;
        }
        if (a.B <= 64) return false;
        at.first += __builtin_amdgcn_readlane(upto, 63);
    }
}

// Keys that row `row` of a sequence sees: those below the result.
__device__ __forceinline__ int keys_of(const AttnArgs& a, const Sequence& s, int row) {
    return a.causal ? max(0, s.len - s.nq + row / a.group + 1) : s.len;
}

// A row's scores are products of its queries, turned by the scale's sign (and zero: the largest score is found before the factor) and, in bfloat16, relative
// to 2^e, times a factor.  `top` is the row's largest magnitude.  Where 2^e of the row would take the factor out of range, the queries stay 14 powers of two
// larger; a factor below every normal number would make -infinity, a key that is not seen, a NaN, and no score that it makes differs from 0.
struct Scale {
    float factor, turn;
    int e;
};
template <bool BF>
__device__ __forceinline__ Scale scale_of(const AttnArgs& a, float top) {
    Scale s = {a.scale_l2 == 0 ? 1.f : fabsf(a.scale_l2), a.scale_l2 < 0 ? -1.f : a.scale_l2 > 0 ? 1.f : 0.f, 0};
    if (BF && top > 0 && top < INFINITY) {
        s.e = ilogbf(top);
        if (!(ldexpf(s.factor, s.e) < INFINITY)) s.e -= 14;
        s.factor = ldexpf(s.factor, s.e);
    }
    s.factor = s.factor < INFINITY ? fmaxf(s.factor, 0x1p-126f) : __uint_as_float(0x7fc00000u);
    return s;
}

// The exponentials' arguments x * factor - reference are single operations, which is right while the reference, a rounded product, is within
// half of the product itself.  From 2^22 on the products are rounded first, as the reference was: otherwise the largest key's exponential
// would be 0 or infinite, whichever way the rounding went.
constexpr float kFar = 0x1p22f;
__device__ __forceinline__ bool is_far(float ref) { return __any(fabsf(ref) > kFar && fabsf(ref) < INFINITY); }
__device__ __forceinline__ float rounded_product(float x, float factor) {
#pragma clang fp contract(off)
    return x * factor;
}

// One tile's bytes of one lane: [group of 16 tokens][words].
template <int D>
struct Raw {
    unsigned k[2][D / 32], v[2][D / 32];
    unsigned ks[2], vs[2];
};

// Indices that the launch only reads, through the scalar cache.
typedef const int __attribute__((address_space(4))) * const_ints;

template <int D, int NT, int NW>
struct Shared {
    float joined[NW][16 * NT][D + 4], stats[NW][16 * NT][2];
};

// Tiles t0 .. t1 - 1 of one segment: row block rb and head h of sequence b.  `pieces` workgroups have a part of it, and this one's goes
// to `slot` if there are several: a range has one piece at most that its segment begins with (slot 2 id + 1), its last, and one at
// most that it does not (slot 2 id), its first.
template <int D, int NT, int NW, bool BF>
__device__ __forceinline__ void segment(const AttnArgs& a, const Sequence& s, int b, int h, int rb, int t0, int t1, int most, int pieces, int slot,
                                        Shared<D, NT, NW>& lds) {
    constexpr int RB = 16 * NT, KS = D / 32, CT = D / 16, W = D / 32;
    auto& joined = lds.joined;
    auto& stats = lds.stats;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned col = lane & 15, quad = lane >> 4;
    const int rows = s.nq * a.group, row0 = rb * RB, least = keys_of(a, s, row0);
    const bool first = t0 == 0;
    if (most == 0) t1 = 0;

    const const_ints table = (const_ints)(uintptr_t)(a.tables + (long long)b * a.width);
    const int groups_page = 1 << (a.page_shift - 4);
    // Group g's (16 tokens') page; groups behind the last one stand for that one (their keys are masked).  All groups are fewer than 2^32.
    const int last_group = max(0, (most + 15) / 16 - 1);
    auto page_of = [&](int g) { return table[min(g, last_group) >> (a.page_shift - 4)]; };
    auto group_at = [&](int g, int page) {
        const int p = (unsigned)page < (unsigned)a.pages ? page : 0;
        return a.cache + (unsigned long long)(((unsigned)p * a.heads + h) * groups_page + (min(g, last_group) & (groups_page - 1))) * Group<D>::bytes;
    };
    // A lane's places in a group, unsigned so that they are 32-bit offsets to a scalar address.
    const unsigned k_off = col * (D / 2) + quad * (D / 8), ks_off = Group<D>::k_scales + col * (D / 32) + quad * (D / 4) / 32;
    const unsigned v_off = Group<D>::v_codes + quad * (2 * D) + col * (D / 8), vs_off = Group<D>::v_scales + quad * (D / 8) + col * (D / 16) / 32 * 4;
    Raw<D> raw;
    auto fetch_k = [&](const uint8_t* at, int i) {
        const unsigned* k = (const unsigned*)(at + k_off);
#pragma unroll
        for (int w = 0; w < W; ++w) raw.k[i][w] = k[w];
        raw.ks[i] = at[ks_off];
    };
    auto fetch_v = [&](const uint8_t* at, int i) {
        const unsigned* v = (const unsigned*)(at + v_off);
#pragma unroll
        for (int w = 0; w < W; ++w) raw.v[i][w] = v[w];
        raw.vs[i] = *(const unsigned*)(at + vs_off);
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
        float x[KS][8], top = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            load8<BF>(a.q + at + 8 * k, x[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[k][i]));
        }
        if (BF) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
        }
        const Scale scale = scale_of<BF>(a, top);
        factor[n] = scale.factor;
        if (top == INFINITY) x[0][0] = __uint_as_float(0x7fc00000u);  // an infinity among the scores would hide where all of them are -inf
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[n][k][i] = (_Float16)(scale.turn * (BF ? ldexpf(x[k][i], -scale.e) : x[k][i]));
    }

    f32x4 o[NT][CT];
    float m[NT], l[NT];
    bool far = false;  // of any row of the wave
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
            if (NT == 1) __builtin_amdgcn_sched_barrier(0);
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
                for (int j = 0; j < 4; ++j) x[n][4 * i + j] = acc[n][j];
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
            unsigned nan = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // Codes that no row sees are cleared, with their scales: what lies there may be anything.
                const int key = t * kTile + 16 * i + 4 * quad, live = there[i] ? most - key : 0;  // of the lane's four tokens
                const unsigned keep = live >= 4 ? ~0u : live <= 0 ? 0u : (1u << (8 * live)) - 1;
                raw.vs[i] = (raw.vs[i] & keep) | (0x7f7f7f7fu & ~keep);
                if (D == 128) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) raw.v[i][j % W] = j < live ? raw.v[i][j % W] : 0;
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) raw.v[i][j] &= (2 * j < live ? 0xffffu : 0u) | (2 * j + 1 < live ? 0xffff0000u : 0u);
                }
                nan |= ((raw.vs[i] & 0x7f7f7f7fu) + 0x01010101u) & raw.vs[i] & 0x80808080u;  // bytes of 255
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[n][4 * i + j] = key + j < limit[n] && there[i] ? x[n][4 * i + j] : -INFINITY;
            }
            if (__builtin_expect(__any(nan != 0), 0)) {
                // A NaN among values that some rows see and others do not must not reach the others as 0 * NaN: it goes into the scores
                // of the rows that see it.
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const bool mine = (raw.vs[i] >> (8 * j) & 255u) == 255u;
                        const bool token = (__ballot(mine) >> (16 * quad) & 0xffffu) != 0;
                        if (mine) raw.vs[i] &= ~(0x80u << (8 * j));
                        if (D == 128) raw.v[i][j % W] = mine ? 0 : raw.v[i][j % W];
                        else raw.v[i][j / 2] &= mine ? (j % 2 ? 0xffffu : 0xffff0000u) : ~0u;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (token && t * kTile + 16 * i + 4 * quad + j < limit[n]) x[n][4 * i + j] = __uint_as_float(0x7fc00000u);
                    }
            }
        }
        f16x8 p[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = x[n][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) top = fmaxf(top, x[n][j]);
            top *= factor[n];
            if (__any(top - m[n] > kRaise)) {  // all four lanes of a row take the same reference
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float to = fmaxf(m[n], top - kRoom);
                far = far || is_far(to);
                const float by = to == m[n] ? 1.f : __builtin_amdgcn_exp2f(m[n] - to);
                m[n] = to;
                l[n] *= by;
#pragma unroll
                for (int c = 0; c < CT; ++c) o[n][c] *= by;
            }
            const float ref = m[n] == -INFINITY ? 0.f : m[n];
            float f = factor[n];
            if (__builtin_expect(far, 0)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[n][j] = rounded_product(x[n][j], f);
                f = 1;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = __builtin_amdgcn_exp2f(fmaf(x[n][j], f, -ref));
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

    // The waves meet in LDS, all of them once: [wave][row][channel], rows 4 words apart in the banks.  Then a thread has two channels of a
    // row and adds the waves' in their order.  (Outputs handed on from half of the waves to the other half until one is left took 16 waves 6 us.)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (quad == 0) stats[wave][16 * n + col][0] = m[n], stats[wave][16 * n + col][1] = l[n];
        float* to = joined[wave][16 * n + col] + 4 * quad * CT;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < CT; c += 4) *(f32x4*)(to + j * CT + c) = f32x4{o[n][c][j], o[n][c + 1][j], o[n][c + 2][j], o[n][c + 3][j]};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < RB * (D / 2); i += 64 * NW) {
        const int at = i / (D / 2), c = 2 * (i % (D / 2)), row = row0 + at;
        if (row >= rows) break;
        float top = -INFINITY, sum = 0, x = 0, y = 0;
#pragma unroll 4
        for (int w = 0; w < NW; ++w) top = fmaxf(top, stats[w][at][0]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll 4
        for (int w = 0; w < NW; ++w) {
            const float by = __builtin_amdgcn_exp2f(stats[w][at][0] - ref);
            sum += stats[w][at][1] * by;
            x += joined[w][at][c] * by;
            y += joined[w][at][c + 1] * by;
        }
        const long long vec = (long long)(s.q0 + row / a.group) * a.H + h * a.group + row % a.group;
        if (a.ws && c == 0 && first) a.heads_ws[vec] = int2{slot * RB + at, pieces};
        if (pieces == 1) {
            const float by = sum == 0.f ? 0.f : 1.f / sum;
            if (c == 0) a.lse[vec] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
            *(unsigned*)(a.out + vec * D + c) = pack2<BF>(x * by, y * by);
        } else {
            float* to = a.ws + (long long)(slot * RB + at) * (D + 2);
            to[c] = x, to[c + 1] = y;
            if (c == 0) to[D] = top, to[D + 1] = sum;
        }
    }
}

// Many rows: a wave has 32 rows, all waves go over the same tiles of 64 keys, and the converted tile lies in LDS, in the order in which
// the 32 x 32 x 16 MFMA takes its first operand, so that 16 bytes of a lane are one read.  A tile is converted once for the workgroup's
// rows, from bytes that were asked for a tile ahead, the keys two tiles ahead of their softmax and the values one: while a tile's
// exponentials run, the next one's scores are multiplied between them (one after the other: 2048 queries behind as many keys 55 us, so 52).
//     S^T (32 tokens x 32 rows) = K Q^T:  lane l has row l % 32 of Q, register v token 8 (v / 4) + 4 (l / 32) + v % 4
//     O^T (32 channels x 32 rows) += V^T P^T: P as S^T leaves it, so half l / 32 has tokens 4 (l / 32) .. + 3 and 8 + 4 (l / 32) .. + 3 of 16
// A row's output stays in one wave (of each group).
constexpr int kWideTile = 64;

template <int D>
struct WideTiles {
    uint4 k[2][2 * (D / 16) * 64], v[2][4 * (D / 32) * 64];  // [buffer][32 tokens][16 channels][lane], [buffer][16 tokens][32 channels][lane]
    unsigned flags[2][4];  // of 16 tokens: whose values hold a NaN, and (bit 16) whether their page is outside the cache
};
template <int D, int G>
struct WideShared {
    WideTiles<D> of[G];
};

// G = 2: two groups of NW waves take turns at the tiles of the same rows, whole segments only.
template <int D, int NW, int G, bool BF>
__device__ __forceinline__ void wide_segment(const AttnArgs& a, const Sequence& s, int b, int h, int rb, int t0, int t1, int most, int pieces,
                                             int slot, WideShared<D, G>& shared) {
    constexpr int RB = 32 * NW, KS = D / 16, CT = D / 32, W = D / 32, RUN = D / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % NW);
    const int turn = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / NW);
    WideTiles<D>& lds = shared.of[turn];
    const unsigned col = lane & 31, half = lane >> 5, c16 = lane & 15, quad = lane >> 4;
    const int rows = s.nq * a.group, row0 = rb * RB + 32 * wave, row = row0 + (int)col;
    const bool first = t0 == 0, mine = row < rows;
    if (most == 0) t1 = 0;
    // The wave's own rows: keys that its first row sees, and its last one.
    const int least = row0 < rows ? keys_of(a, s, row0) : 0, top_key = row0 < rows ? keys_of(a, s, min(row0 + 32, rows) - 1) : 0;
    const int limit = mine ? keys_of(a, s, row) : 0;

    const const_ints table = (const_ints)(uintptr_t)(a.tables + (long long)b * a.width);
    const int groups_page = 1 << (a.page_shift - 4), last_group = max(0, (most + 15) / 16 - 1);
    auto page_of = [&](int g) { return table[min(g, last_group) >> (a.page_shift - 4)]; };
    auto group_at = [&](int g, int page) {
        const int p = (unsigned)page < (unsigned)a.pages ? page : 0;
        return a.cache + (unsigned long long)(((unsigned)p * a.heads + h) * groups_page + (min(g, last_group) & (groups_page - 1))) * Group<D>::bytes;
    };
    // Groups of 16 tokens are shared out: with eight waves four convert keys and four values, with four a wave does both of its group.
    const int mine_g = wave & 3;
    const bool keys = NW == 4 || wave < 4, vals = NW == 4 || wave >= 4;
    unsigned rk[W], rv[W], rks = 0, rvs = 0;
    const unsigned k_off = c16 * (D / 2) + quad * (D / 8), ks_off = Group<D>::k_scales + c16 * (D / 32) + quad * (D / 4) / 32;
    const unsigned v_off = Group<D>::v_codes + quad * (2 * D) + c16 * (D / 8), vs_off = Group<D>::v_scales + quad * (D / 8) + c16 * (D / 16) / 32 * 4;
    auto fetch_k = [&](const uint8_t* at) {
        if (!keys) return;
        const unsigned* k = (const unsigned*)(at + k_off);
#pragma unroll
        for (int w = 0; w < W; ++w) rk[w] = k[w];
        rks = at[ks_off];
    };
    auto fetch_v = [&](const uint8_t* at) {
        if (!vals) return;
        const unsigned* v = (const unsigned*)(at + v_off);
#pragma unroll
        for (int w = 0; w < W; ++w) rv[w] = v[w];
        rvs = *(const unsigned*)(at + vs_off);
    };
    auto put_k = [&](int t) {  // the lane's token and D/4 channels from quad * D/4
        if (!keys) return;
        uint4* to = lds.k[t / G & 1] + ((mine_g >> 1) * KS * 64 + (mine_g & 1) * 16 + c16);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const unsigned piece = quad * W + w;  // 8 channels: half piece % 2 of 16
            to[(piece >> 1) * 64 + (piece & 1) * 32] = values8<false>(rk[w], rks << 23);
        }
    };
    auto put_v = [&](int t, int page) {
        if (!vals) return;
        const int buf = t / G & 1, key = t * kWideTile + 16 * mine_g + 4 * (int)quad;
        const bool there = (unsigned)page < (unsigned)a.pages;
        if (!there || t * kWideTile + 16 * mine_g + 16 > most) {
            const int live = there ? most - key : 0;
            const unsigned keep = live >= 4 ? ~0u : live <= 0 ? 0u : (1u << (8 * live)) - 1;
            rvs = (rvs & keep) | (0x7f7f7f7fu & ~keep);
#pragma unroll
            for (int w = 0; w < W; ++w)
                rv[w] = D == 128 ? (w < live ? rv[w] : 0) : rv[w] & ((2 * w < live ? 0xffffu : 0u) | (2 * w + 1 < live ? 0xffff0000u : 0u));
        }
        // A NaN must reach the rows that see its token and no other: it goes into their scores, and its codes are cleared.
        unsigned flags = there ? 0 : 1u << 16;
        if (__builtin_expect(__any((((rvs & 0x7f7f7f7fu) + 0x01010101u) & rvs & 0x80808080u) != 0), 0)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool bad = (rvs >> (8 * j) & 255u) == 255u;
                const unsigned long long all = __ballot(bad);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (all >> (16 * q) & 0xffffu) flags |= 1u << (4 * q + j);
                if (bad) rvs &= ~(0x80u << (8 * j));
                if (D == 128) rv[j % W] = bad ? 0 : rv[j % W];
                else rv[j / 2] &= bad ? (j % 2 ? 0xffffu : 0xffff0000u) : ~0u;
            }
        }
        if (lane == 0) lds.flags[buf][mine_g] = flags;
        const unsigned sc[4] = {rvs << 23, rvs << 15, rvs << 7, rvs >> 1};
        // Four tokens of a channel are 8 bytes: half quad % 2, the lower or upper 8 bytes of the lane's 16 by quad / 2.
        uint2* to = (uint2*)lds.v[buf] + (mine_g * CT * 64 + (quad & 1) * 32 + c16) * 2 + (quad >> 1);
        auto channels = [&](auto SEL) {
            constexpr int c = decltype(SEL)::value;
            unsigned two[4];
            if constexpr (D == 128) {
#pragma unroll
                for (int j = 0; j < 4; ++j) two[j] = values2<false, c>(rv[j % W], sc[j]);
            } else {
                two[0] = values2<false, c>(rv[0], sc[0]), two[1] = values2<false, 2 + c>(rv[0], sc[1]);
                two[2] = values2<false, c>(rv[1], sc[2]), two[3] = values2<false, 2 + c>(rv[1], sc[3]);
            }
            to[c * 128] = uint2{__builtin_amdgcn_perm(two[1], two[0], 0x05040100u), __builtin_amdgcn_perm(two[3], two[2], 0x05040100u)};
            to[c * 128 + 32] = uint2{__builtin_amdgcn_perm(two[1], two[0], 0x07060302u), __builtin_amdgcn_perm(two[3], two[2], 0x07060302u)};
        };
        channels(std::integral_constant<int, 0>());
        channels(std::integral_constant<int, 1>());
        if constexpr (D == 128) {
            channels(std::integral_constant<int, 2>());
            channels(std::integral_constant<int, 3>());
        }
    };

    const int t00 = t0 + turn;
    int pages[3] = {-1, -1, -1};  // of the wave's tokens in the tiles t + G, t + 2 G and t + 3 G
    int ahead = -1;
    if (t0 < t1) {
        for (int i = 0; i < 3; ++i) pages[i] = page_of(4 * (t00 + G * i) + mine_g);
        ahead = page_of(4 * (t00 + 3 * G) + mine_g);
        fetch_k(group_at(4 * t00 + mine_g, pages[0]));
        fetch_v(group_at(4 * t00 + mine_g, pages[0]));
    }

    // Queries: the lane's row, channels 16 ks + 8 half .. + 7.
    f16x8 q[KS];
    float factor;
    {
        const long long at = ((long long)(s.q0 + (mine ? row / a.group : 0)) * a.H + h * a.group + (mine ? row % a.group : 0)) * D + 8 * half;
        float top = 0;
        uint4 raw[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            raw[k] = *(const uint4*)(a.q + at + 16 * k);
            float x[8];
            values_of<BF>(raw[k], x);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
        }
        if (BF) top = fmaxf(top, __shfl_xor(top, 32));
        const Scale scale = scale_of<BF>(a, top);
        factor = scale.factor;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            float x[8];
            values_of<BF>(raw[k], x);
            if (k == 0 && top == INFINITY) x[0] = __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int i = 0; i < 8; ++i) q[k][i] = (_Float16)(scale.turn * (BF ? ldexpf(x[i], -scale.e) : x[i]));
        }
    }
    f32x16 o[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[c][v] = 0;
    float m = -INFINITY, l = 0;
    bool far = false;  // as in `segment`

    // A step's products in their order: the next tile's scores (32 tokens s % 2, 16 channels s / 2) for s = 0, 1, .. and, from the first eight
    // exponentials on, this tile's outputs between them.
    struct Product {
        bool score;
        int i, k;  // score: half of the tile, channels; output: 16 tokens, tile of channels
    };
    constexpr int L = D / 16, kProducts = 2 * KS + 4 * CT, kAhead = 4;  // L products to 8 exponentials
    constexpr auto product = [](int n) constexpr -> Product {
        if (n < L) return {true, n % 2, n / 2};
        if (n < 3 * L) {
            const int g = n / L, r = n % L, s = L + (g - 1) * (L / 2) + r / 2;
            return r % 2 ? Product{true, s % 2, s / 2} : Product{false, g - 1, r / 2};
        }
        return {false, 2 + (n - 3 * L) / CT, (n - 3 * L) % CT};
    };
    auto operand = [&](int n, int t) {
        const Product p = product(n);
        return p.score ? lds.k[(t / G + 1) & 1][(p.i * KS + p.k) * 64 + lane] : lds.v[t / G & 1][(p.i * CT + p.k) * 64 + lane];
    };
    const uint8_t* at_v = a.cache;  // the bytes whose keys were fetched last: the next values to fetch
    f32x16 xs[2][2];  // scores of the tile and of the next
    if (t0 < t1) {
        put_k(t00);
        put_v(t00, pages[0]);
        fetch_k(group_at(4 * (t00 + G) + mine_g, pages[1]));
        fetch_v(group_at(4 * (t00 + G) + mine_g, pages[1]));
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int v = 0; v < 16; ++v) xs[0][i][v] = 0;
#pragma unroll
            for (int k = 0; k < KS; ++k)
                xs[0][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, lds.k[t00 / G & 1][(i * KS + k) * 64 + lane]), q[k], xs[0][i], 0, 0, 0);
        }
        put_k(t00 + G);
        at_v = group_at(4 * (t00 + 2 * G) + mine_g, pages[2]);
        fetch_k(at_v);
        pages[0] = pages[1], pages[1] = pages[2], pages[2] = ahead;
        ahead = page_of(4 * (t00 + 4 * G) + mine_g);
    }
    // One tile: its scores are in x, and the next one's go to y (behind the last: of whatever lies there, for nobody).
    auto step = [&](int t, f32x16 (&x)[2], f32x16 (&y)[2]) {
        __syncthreads();  // keys of tile t + G and values of tile t are there, and nobody reads keys of t or values of t - G any more
        const int buf = t / G & 1;
        const uint4 flags = *(const uint4*)lds.flags[buf];
        uint4 op[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) op[n] = operand(n, t);
        if (t + G < t1) {
            put_v(t + G, pages[0]);
            put_k(t + 2 * G);
            fetch_v(at_v);
            at_v = group_at(4 * (t + 3 * G) + mine_g, pages[2]);
            fetch_k(at_v);
            pages[0] = pages[1], pages[1] = pages[2], pages[2] = ahead;
            ahead = page_of(4 * (t + 5 * G) + mine_g);
        }
        if (t * kWideTile >= top_key) return;
        if ((t + 1) * kWideTile > least) {
            const int seen = limit - t * kWideTile - 4 * (int)half;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) x[i][v] = 32 * i + 8 * (v / 4) + v % 4 < seen ? x[i][v] : -INFINITY;
        }
        auto largest = [&] {
            float top = x[0][0];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) top = fmaxf(top, x[i][v]);
            return top;
        };
        float top = largest();
        const unsigned any = __builtin_amdgcn_readfirstlane(flags.x | flags.y | flags.z | flags.w);
        if (__builtin_expect(any != 0, 0)) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int in = 8 * (v / 4) + v % 4;  // token of the 32, less 4 half
                    const unsigned f = lds.flags[buf][2 * i + in / 16];
                    const bool seen = t * kWideTile + 32 * i + in + 4 * (int)half < limit;
                    x[i][v] = f >> 16 ? -INFINITY : f >> (in % 16 + 4 * half) & 1 && seen ? __uint_as_float(0x7fc00000u) : x[i][v];
                }
            top = largest();
        }
        top *= factor;
        if (__any(top - m > kRaise)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = fmaxf(m, top - kRoom);
            far = far || is_far(to);
            const float by = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= by;
#pragma unroll
            for (int c = 0; c < CT; ++c) o[c] *= by;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float f = factor;
        if (__builtin_expect(far, 0)) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) x[i][v] = rounded_product(x[i][v], f);
            f = 1;
        }
        f16x8 p[4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) y[i][v] = 0;
        auto multiply = [&](int n) {
            const Product w = product(n);
            const f16x8 with = __builtin_bit_cast(f16x8, op[n % kAhead]);
            if (w.score) y[w.i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(with, q[w.k], y[w.i], 0, 0, 0);
            else o[w.k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(with, p[w.i], o[w.k], 0, 0, 0);
            if (n + kAhead < kProducts) op[n % kAhead] = operand(n + kAhead, t);
        };
        int n = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (j * L / 8 * 8 == j * L && (j < 24 || j * L / 8 % 2 == 0)) multiply(n++);
            const float e = __builtin_amdgcn_exp2f(fmaf(x[j / 16][j % 16], f, -ref));
            l += e;
            p[j / 8][j % 8] = (_Float16)e;
        }
#pragma unroll
        for (int i = 0; i < CT; ++i) multiply(n++);
    };
    for (int t = t00; t - turn < t1; t += G) {  // as many steps in both groups: behind t1 nobody has a key
        step(t, xs[0], xs[1]);
        if ((t += G) - turn >= t1) break;
        step(t, xs[1], xs[0]);
    }

    l += __shfl_xor(l, 32);
    if constexpr (G == 2) {  // the second group's rows go to the first through LDS
        constexpr int n = 16 * CT + 2;
        static_assert(sizeof(shared) >= NW * n * 64 * sizeof(float), "room for the rows of a group");
        float* const at = (float*)&shared + wave * n * 64 + lane;
        __syncthreads();
        if (turn) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int v = 0; v < 16; ++v) at[(16 * c + v) * 64] = o[c][v];
            at[(n - 2) * 64] = m, at[(n - 1) * 64] = l;
        }
        __syncthreads();
        if (turn) return;
        const float other = at[(n - 2) * 64], top = fmaxf(m, other), ref = top == -INFINITY ? 0.f : top;
        const float by = __builtin_amdgcn_exp2f(m - ref), add = __builtin_amdgcn_exp2f(other - ref);
        m = top;
        l = l * by + at[(n - 1) * 64] * add;
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[c][v] = o[c][v] * by + at[(16 * c + v) * 64] * add;
    }
    if (!mine) return;
    const long long vec = (long long)(s.q0 + row / a.group) * a.H + h * a.group + row % a.group;
    const int at = slot * RB + 32 * wave + (int)col;
    if (a.ws && half == 0 && first) a.heads_ws[vec] = int2{at, pieces};
    const float by = l == 0.f ? 0.f : 1.f / l;
    if (half == 0) {
        if (pieces == 1) a.lse[vec] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        else a.ws[(long long)at * (D + 2) + D] = m, a.ws[(long long)at * (D + 2) + D + 1] = l;
    }
    // Row 16 i + r of channel tile c is channel 2 c + i of run r: a lane has all channels of its runs.
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int channel = (8 * u + 4 * (int)half + r) * RUN;
            if (pieces == 1) {
                unsigned w[CT];
#pragma unroll
                for (int c = 0; c < CT; ++c) w[c] = pack2<BF>(o[c][4 * u + r] * by, o[c][8 + 4 * u + r] * by);
                unsigned* to = (unsigned*)(a.out + vec * D + channel);
#pragma unroll
                for (int c = 0; c < CT; ++c) to[c] = w[c];
            } else {
                float* to = a.ws + (long long)at * (D + 2) + channel;
#pragma unroll
                for (int c = 0; c < CT; ++c) to[2 * c] = o[c][4 * u + r], to[2 * c + 1] = o[c][8 + 4 * u + r];
            }
        }
}

// The two forms of a segment: NT tiles of 16 rows with the keys shared out to NW waves, or 32 rows to each of NW waves in G groups.  In tiles: `begin`, what
// it costs a workgroup to begin and end a segment (about 5 us; 0, 4, 8, 16 tiles: 64 sequences of up to 8192 keys 75.4, 72.7, 71.7, 72.0 us, 8 of up to
// 4000 18.6, 15.6, 14.8, 14.8); `least`, the shortest range; `whole`, up to which a segment is left whole if no other is longer.
template <int D, int NT, int NW, bool BF>
struct Narrow {
    static constexpr int rows = 16 * NT, tile = kTile, waves_simd = NT == 1 ? 4 : 2, threads = 64 * NW;
    static constexpr int begin = 8, least = 16, whole = 48;
    typedef Shared<D, NT, NW> Lds;
    template <class... A>
    static __device__ __forceinline__ void run(A&&... x) { segment<D, NT, NW, BF>(x...); }
};
template <int D, int NW, int G, bool BF>
struct Wide {
    static constexpr int rows = 32 * NW, tile = kWideTile, waves_simd = 2, threads = 64 * NW * G;
    static constexpr int begin = 2, least = 4, whole = 32;
    typedef WideShared<D, G> Lds;
    template <class... A>
    static __device__ __forceinline__ void run(A&&... x) { wide_segment<D, NW, G, BF>(x...); }
};

template <class F>
__global__ __launch_bounds__(F::threads, F::waves_simd) void attn_kernel(AttnArgs a) {
    constexpr int RB = F::rows;
    __shared__ typename F::Lds lds;
    const int id = blockIdx.x;
    Start at;
    if (!start_of<F>(a, id, at)) return;
    Sequence s = at.s;
    int b = at.b, of = positions_of<F>(s), segments = blocks_of<RB>(a, s) * a.heads;
    int seg = id - at.first, w0 = 0, left = of;  // a whole segment
    if (at.range) {
        const int pos = id * at.range;
        seg = (pos - at.first) / of;
        w0 = pos - at.first - seg * of;
        left = min(at.range, at.total - pos);
    }
    for (;;) {
        const int w1 = min(of, w0 + left), rb = segments / a.heads - 1 - seg / a.heads;  // the last rows, which see the most, first
        // The keys that the row block's last row sees may be fewer than the sequence has.
        const int most = keys_of(a, s, min((rb + 1) * RB, s.nq * a.group) - 1), tiles = max(1, (most + F::tile - 1) / F::tile);
        int pieces = 1;
        if (at.range) {
            const int from = at.first + seg * of + F::begin;
            pieces = (from + tiles - 1) / at.range - from / at.range + 1;
        }
        const int t0 = max(0, w0 - F::begin), t1 = min(tiles, w1 - F::begin);
        if (t0 < t1) F::run(a, s, b, seg % a.heads, rb, t0, t1, most, pieces, 2 * id + (t0 == 0), lds);
        left -= w1 - w0;
        if (left <= 0) return;
        __syncthreads();  // the next segment takes this one's place in LDS
        w0 = 0;
        if (++seg < segments) continue;
        at.first += segments * of, seg = 0;
        do {  // positions are left, so a sequence with rows is (unless somebody writes the lengths meanwhile)
            if (++b >= a.B) return;
            s = shared_sequence(a, b);
            segments = blocks_of<RB>(a, s) * a.heads;
        } while (!segments);
        of = positions_of<F>(s);
    }
}

// WAVES waves join the pieces of one row (query, head): a lane has one piece's maximum and sum, then the weighted outputs are added, eight pieces'
// loads at a time (one after another took 75 us for rows of 128).
template <int D, int RB, bool BF, int WAVES>
__global__ __launch_bounds__(WAVES > 4 ? 64 * WAVES : 256) void join_kernel(AttnArgs a) {
    constexpr int C = D / 64, ROWS = WAVES > 4 ? 1 : 4 / WAVES;  // of a workgroup
    __shared__ float part[WAVES][D + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = wave % WAVES;
    const long long vec = (long long)blockIdx.x * ROWS + wave / WAVES;
    if (vec >= (long long)a.T * a.H) return;
    const int t = (int)(vec / a.H);
    const int2 mine_at = a.heads_ws[vec];  // for a row of nobody: anything
    if (a.cu_q) {  // whether the row is somebody's: the sequence is the one with cu_q[b] <= t < cu_q[b + 1]
        int q0, end;
        if (a.B < 64) {
            const int from = a.cu_q[min(lane, a.B)];
            const int b = __popcll(__ballot(lane > 0 && lane <= a.B && from <= t));
            if (b >= a.B) return;
            q0 = __builtin_amdgcn_readlane(from, b), end = __builtin_amdgcn_readlane(from, b + 1);
        } else {
            int upto = 0;
            for (int i = lane; i < a.B; i += 64) upto += a.cu_q[i + 1] <= t;
            const int b = __builtin_amdgcn_readlane(prefix_sum(upto), 63);
            if (b >= a.B) return;
            q0 = a.cu_q[b], end = a.cu_q[b + 1];
        }
        q0 = min(max(q0, 0), a.T);  // as in `sequence`
        if (t < q0 || t - q0 >= min(min(max(end, q0), a.T) - q0, a.max_q)) return;
    }
    const int runs = __builtin_amdgcn_readfirstlane(mine_at.y);
    if (runs == 1) return;
    // The first piece's row, an odd slot's; the next ranges' pieces are in even slots.
    const float* head = a.ws + (long long)__builtin_amdgcn_readfirstlane(mine_at.x) * (D + 2);
    constexpr long long step = 2 * RB * (D + 2);
    auto piece = [&](int r) { return head + r * step - (r ? RB * (D + 2) : 0); };
    // Lane l has piece r0 + WAVES l: its reference is raised for 64 pieces at a time.
    float top = -INFINITY, sum = 0, o[C] = {};
    for (int r0 = mine; r0 < runs; r0 += 64 * WAVES) {
        const int r = r0 + WAVES * lane;
        float m = -INFINITY, l = 0;
        if (r < runs) m = piece(r)[D], l = piece(r)[D + 1];
        const int n = min(64, (runs - r0 + WAVES - 1) / WAVES);
        float x[8][C];
        auto fetch = [&](int k) {
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int i = 0; i < C; ++i) x[u][i] = piece(r0 + WAVES * min(k + u, n - 1))[lane * C + i];
        };
        fetch(0);  // under way together with the maxima
        float to = m;
#pragma unroll
        for (int d = 32; d; d /= 2) to = fmaxf(to, __shfl_xor(to, d));
        to = fmaxf(to, top);
        const float ref = to == -INFINITY ? 0.f : to, by = __builtin_amdgcn_exp2f(top - ref);
        const float weight = __builtin_amdgcn_exp2f(m - ref);
        top = to;
        sum = sum * by + weight * l;  // each lane's own pieces
        for (int i = 0; i < C; ++i) o[i] *= by;
        for (int k = 0; k < n; k += 8) {
            if (k) fetch(k);
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
    int wide, nt, nw, groups, rows, target;  // wide: 32 rows a wave, `groups` of nw waves; otherwise nt tiles of 16 rows
    long long segments, blocks, slots, bytes;
};

// Both sides of the choices, in us (bfloat16, d = 128, 32 heads on 8 unless said; forms timed in turn on one card):
//  * rows from 33 on in the wide form, not four tiles of 16 rows a wave: 40 rows over four caches of up to 20000 keys 39 against 58, 64 over the
//    same 31 against 53.  Up to 32 in two tiles of 16: 24 rows over 16 caches of up to 6000 keys 26.4 against 31.0, 32 rows, d = 64, 21.4 against 24.4.
//  * kRanges: 768, 1024, 1536, 2048 ranges: 64 sequences of up to 8192 keys 70, 72, 76, 75; two of up to 131072 36.5, 37.6, 43, 44; but with 3/4 of the ranges, so
//    of the units, the other forms take 5 to 21 % longer (the chunk below 582 against 481).  Eight waves a workgroup and half the ranges: 72.5 and 36.7.
//    Forms of which two workgroups fill a unit, 1024 and 512: 24 rows over 16 caches of up to 6000 keys 33.7, 26.4, 32 rows, d = 64, 25.8, 21.4.
//  * kMany: 256 rows a workgroup instead of 128 halve the conversions, but twice as many rows begin and end together: 2048 queries behind 14336 keys
//    515 against 485, 300 behind 12000, 16 heads on 4, d = 64, 59 against 58 (1200 rows), 150 behind 12000 83 against 84 (600 rows); caches of 2048 keys, which
//    are not cut, 51 against 61.
//  * kPaired: one prompt of 1500, 12 heads on 4, d = 64, 22.7 against 26.6, eight times 100 queries over 2000 keys 37.6 against 43.8 (256 row blocks), three prompts of
//    1500 (432) 29.7 against 29.0, two of 32 heads (752) 66 against 55.  Of 200 keys, four tiles, 11.6 against 10.6: from 512 on.
//  * kShort: caches of 1500 keys cut all the same: 64 sequences 23 against 19, one of 1003 keys 11.5 against 10.7 with its 16 waves, one prompt 32 against 23, three 55 against 29.
constexpr int kShort = 2048;   // keys up to which nothing is cut
constexpr int kMany = 1024;    // rows of a sequence and head from which 256 of them share a tile's conversion
constexpr int kPaired = 256;   // row blocks up to which two groups of waves share one: a workgroup to each unit
constexpr int kRanges = 1024;  // four workgroups of 128 registers on each of 256 units; of the other forms two, and half the ranges

Choice choose(long long T, int B, int H, int heads, int d, long long cap, int max_q) {
    const long long rows = (long long)(H / heads) * max_q;
    Choice c;
    c.wide = rows > 32;
    c.nt = rows <= 16 ? 1 : 2;
    c.nw = c.wide && cap > kShort && rows >= kMany ? 8 : 4;
    c.rows = c.wide ? 32 * c.nw : 16 * c.nt;
    c.target = c.nw == 8 ? kRanges / 4 : c.wide || c.nt == 2 ? kRanges / 2 : kRanges;
    const long long alone = c.segments = B * ((rows + c.rows - 1) / c.rows) * heads;
    // Segments that fill the launch by themselves stay whole, and so do those that cannot be long: if they are few, 16 waves take one,
    // up to four tiles each.
    // The joining kernel has up to 16 waves for each row of q, somebody's or not, and threads of a launch are counted in 32 bits.
    const bool whole = cap <= kShort || alone >= 4 * c.target || T * H >= 1 << 22;
    if (c.nt == 1 && cap <= kShort && alone <= 256) c.nw = 16;
    c.groups = c.wide && cap <= kShort && cap >= 512 && alone <= kPaired ? 2 : 1;
    c.blocks = whole || alone > c.target ? alone : c.target;
    c.slots = 2 * c.target;
    c.bytes = whole ? 0 : (T * H * 8 + 15) / 16 * 16 + c.slots * c.rows * (d + 2) * 4;
    return c;
}

int check_sizes(long long T, int B, int H, int heads, int d, int page_size, int width, int max_q) {
    if (T < 0 || B < 1 || heads < 1 || H < heads || H % heads || width < 1 || max_q < 1) return KV4_EINVAL;
    if (page_size < 16 || page_size > 65536 || (page_size & (page_size - 1))) return KV4_EINVAL;
    if (d != 64 && d != 128) return KV4_EUNSUPPORTED;
    const long long cap = (long long)width * page_size, rows = (long long)(H / heads) * max_q;
    if (cap > INT_MAX - 65535 || rows > 1 << 30 || B > 65535 || T * H > INT_MAX) return KV4_EUNSUPPORTED;
    // The refusal below, for the largest row blocks and in numbers that do not wrap around.
    if ((double)B * (double)((rows + 255) / 256) * heads >= 1 << 23) return KV4_EUNSUPPORTED;
    const Choice c = choose(T, B, H, heads, d, cap, max_q);
    // Positions and rows of pieces are counted in 32 bits, and so are keys up to the end of the last tile.
    return c.blocks >= 1 << 23 || (c.bytes && (double)(c.blocks + c.target) * (double)(cap / kTile + 32) > INT_MAX) ? KV4_EUNSUPPORTED : KV4_OK;
}

template <int D, bool BF>
int launch_attn(const Choice& c, AttnArgs& a, void* stream) {
    const void* fn = c.nw == 8   ? (const void*)attn_kernel<Wide<D, 8, 1, BF>>
                     : c.groups == 2 ? (const void*)attn_kernel<Wide<D, 4, 2, BF>>
                     : c.wide    ? (const void*)attn_kernel<Wide<D, 4, 1, BF>>
                     : c.nw == 16 ? (const void*)attn_kernel<Narrow<D, 1, 16, BF>>
                     : c.nt == 1  ? (const void*)attn_kernel<Narrow<D, 1, 4, BF>>
                                  : (const void*)attn_kernel<Narrow<D, 2, 4, BF>>;
    // A wave takes eight pieces at a time.  A launch's ranges, shared out to its segments, say how many a row has on the average.
    const long long rows = (long long)a.T * a.H, pieces = c.target / c.segments;
    const int waves = pieces <= 4 ? 1 : pieces <= 32 ? 4 : 16;
    auto join_of = [&](auto RB) {
        constexpr int rb = decltype(RB)::value;
        return waves == 1 ? (const void*)join_kernel<D, rb, BF, 1> : waves == 4 ? (const void*)join_kernel<D, rb, BF, 4> : (const void*)join_kernel<D, rb, BF, 16>;
    };
    const void* join = c.rows == 16   ? join_of(std::integral_constant<int, 16>())
                       : c.rows == 32 ? join_of(std::integral_constant<int, 32>())
                       : c.rows == 128 ? join_of(std::integral_constant<int, 128>())
                                       : join_of(std::integral_constant<int, 256>());
    void* list[] = {&a};
    if (hipLaunchKernel(fn, dim3((unsigned)c.blocks), dim3(64 * c.nw * c.groups), list, 0, (hipStream_t)stream) != hipSuccess ||
        (a.ws && hipLaunchKernel(join, dim3((unsigned)(waves == 1 ? (rows + 3) / 4 : rows)), dim3(waves == 16 ? 1024 : 256), list, 0, (hipStream_t)stream) != hipSuccess)) {
        (void)hipGetLastError();
        return KV4_ELAUNCH;
    }
    return KV4_OK;
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
    if ((dtype != KV4_F16 && dtype != KV4_BF16) || !isfinite(scale * 1.4426950408889634f)) return KV4_EINVAL;
    if (T == 0 && B >= 1) return KV4_OK;
    if (!cu_q && (B < 1 || T % B || max_q != T / B)) return KV4_EINVAL;
    if (const int rc = check_sizes(T, B, H, heads, d, page_size, width, max_q)) return rc;
    if ((long long)pages * page_size > INT_MAX || (long long)pages * heads * (page_size / 16) > UINT_MAX) return KV4_EUNSUPPORTED;
    const long long bytes = (long long)T * H * d * 2;
    const long long held = (long long)pages * heads * page_size * (d + d / 16);
    const long long lse_bytes = (long long)T * H * 4;
    if (overlap(q, bytes, out, bytes) || overlap(lse, lse_bytes, out, bytes) || overlap(cache, held, out, bytes)) return KV4_EINVAL;
    if (overlap(q, bytes, lse, lse_bytes) || overlap(cache, held, lse, lse_bytes)) return KV4_EINVAL;
    const Choice c = choose(T, B, H, heads, d, (long long)width * page_size, max_q);
    const bool cut = c.bytes && workspace && workspace_bytes >= c.bytes;
    if (cut && (overlap(q, bytes, workspace, c.bytes) || overlap(out, bytes, workspace, c.bytes) || overlap(lse, lse_bytes, workspace, c.bytes) ||
                overlap(cache, held, workspace, c.bytes)))
        return KV4_EINVAL;
    AttnArgs a = {(const uint16_t*)q, (const uint8_t*)cache, tables, lens, cu_q, (uint16_t*)out, lse, cut ? (int2*)workspace : nullptr,
                  cut ? (float*)((char*)workspace + c.bytes - c.slots * c.rows * (d + 2) * 4) : nullptr, T, B, H,
                  heads, H / heads, pages, __builtin_ctz(page_size), width, max_q, causal, scale * 1.4426950408889634f, c.target};
    if (d == 128) return dtype ? launch_attn<128, true>(c, a, stream) : launch_attn<128, false>(c, a, stream);
    return dtype ? launch_attn<64, true>(c, a, stream) : launch_attn<64, false>(c, a, stream);
}

long long kv4_attn_workspace(int T, int B, int H, int heads, int d, int page_size, int width, int max_q) {
    using namespace kv4;
    if (const int rc = check_sizes(T, B, H, heads, d, page_size, width, max_q)) return rc;
    return choose(T, B, H, heads, d, (long long)width * page_size, max_q).bytes;
}

}  // extern "C"
