// Matrix products in three layouts with bias, activation and residual in the epilogue, for gfx950 (MI355X): the kernel behind
// gemm_linear and the two products of gemm_linear_bwd (include/linear.h has the formulas).
//
// C[m, n] = sum_k A(m, k) B(k, n).  Either operand lies by rows of its own index with k along them (A of every product but the weight's
// gradient, a weight [N, K]) or by rows of k (a weight [K, N], both operands of the weight's gradient, whose k are the tokens).
//
//  * 16x16x32 MFMA, transposed product C^T += B^T A^T: a lane of the accumulator holds four consecutive n of one row of C.  Fragments of
//    an operand with k along its rows are 16-byte reads of LDS, those of one by rows of k two transposing reads: the two operands are
//    symmetric, so all layouts run one loop.
//  * A ring of NB stages of BK values of k in LDS, filled by direct global -> LDS buffer loads, NB - 1 stages ahead of the products.  A
//    stage is BK / 32 steps; each step multiplies the fragments that were read one step ago and reads the next step's, and the one barrier of a
//    stage stands ahead of its last step, where all of its fragments are in registers.  Loads go out between the products: with
//    two stages in the step behind the barrier, else spread from there to the next one.
//  * BK = 64: rows of 64 k are whole lines of 128 bytes.
//  * Workgroups of WK groups of waves split the k of a tile among them, each with a ring of its own, and sum in LDS in group order; a group
//    of one wave needs no barrier.  For few rows, where the weight's bytes are all that counts, such groups keep most of LDS in flight.
#pragma once
#include "gemm_kernel.h"

namespace linear {

using attn::u32x2;
using attn::u32x4;
using gemm::lds_address;
using gemm::lds_s16x4_ptr;
typedef float f32x4 __attribute__((ext_vector_type(4)));

enum { NONE = 0, RELU = 1, SILU = 2, GELU = 3, GELU_TANH = 4 };

struct F16 {
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(attn::f16x8, a), __builtin_bit_cast(attn::f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack2(float a, float b) { return attn::F16::pack2(a, b); }
    static __device__ __forceinline__ void unpack2(unsigned w, float* x) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const h2 h = __builtin_bit_cast(h2, w);
        x[0] = (float)h[0], x[1] = (float)h[1];
    }
};
struct BF16 {
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(attn::bf16x8, a), __builtin_bit_cast(attn::bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack2(float a, float b) { return attn::BF16::pack2(a, b); }
    static __device__ __forceinline__ void unpack2(unsigned w, float* x) { x[0] = __uint_as_float(w << 16), x[1] = __uint_as_float(w & 0xffff0000u); }
};

template <class T>
__device__ __forceinline__ void unpack8(u32x4 w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) T::unpack2(w[i], x + 2 * i);
}
template <class T>
__device__ __forceinline__ u32x4 pack8(const float* x) {
    return u32x4{T::pack2(x[0], x[1]), T::pack2(x[2], x[3]), T::pack2(x[4], x[5]), T::pack2(x[6], x[7])};
}

// The activations of eight values.  In 32 bits with the hardware's exponential (2^x) and reciprocal, each good to a step or so: the results
// are rounded to 16 bits.  z = -inf gives NaN in silu and both gelu, -inf times 0, as their formulas do.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)); }
// Twice the argument of the tanh form.  tanh(u / 2) = 2 sigmoid(u) - 1, so the form is z sigmoid(u): one exponential, and no
// difference of near values where the result is small.
__device__ __forceinline__ float tanh_argument(float z) { return 1.5957691216057308f * z * fmaf(0.044715f * z, z, 1.f); }
// The normal distribution's integral from -inf to z, and in *density its density.  With x = |z| / sqrt 2 and t = 1 / (1 + 0.38 x), e^(x^2) erfc(x) is a
// polynomial in t (Hastings' form) to 2e-6 of itself, its coefficients fitted to the least relative error over 0 .. 20: the tail
// keeps its digits for negative z, where 1 + erf loses them, at a third of the library function's instructions.
__device__ __forceinline__ float normal(float z, float* density) {
    const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f), t = __builtin_amdgcn_rcpf(fmaf(0.26870057685088805f, fabsf(z), 1.f));
    float y = fmaf(-0.1221754432f, t, 0.325358889f);
    y = fmaf(y, t, -0.05603825632f);
    y = fmaf(y, t, 0.2388010393f);
    y = fmaf(y, t, 0.1836745718f);
    y = fmaf(y, t, 0.2160605577f);
    y = fmaf(y, t, 0.2143203926f);
    const float tail = 0.5f * e * (y * t);
    *density = 0.3989422804014327f * e;
    return z < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ void act8(float* v, int kind) {
    if (kind == RELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
    } else if (kind == SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= sigmoid(v[i]);
    } else if (kind == GELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float density;
            v[i] *= normal(v[i], &density);
        }
    } else if (kind == GELU_TANH) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= sigmoid(tanh_argument(v[i]));
    }
}

// g <- g act'(v)
__device__ __forceinline__ void act_slope8(const float* v, float* g, int kind) {
    if (kind == RELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = v[i] > 0.f ? g[i] : v[i] <= 0.f ? 0.f : v[i];
    } else if (kind == SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = sigmoid(v[i]);
            g[i] *= p * fmaf(v[i], 1.f - p, 1.f);
        }
    } else if (kind == GELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float density;
            const float p = normal(v[i], &density);
            g[i] *= fmaf(v[i], density, p);
        }
    } else if (kind == GELU_TANH) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = sigmoid(tanh_argument(v[i]));
            g[i] *= p * fmaf(1.5957691216057308f * v[i] * (1.f - p), fmaf(3.f * 0.044715f * v[i], v[i], 1.f), 1.f);
        }
    }
}

template <int BM_, int BN_, int BK_, int WM_, int WN_, int WK_, int NB_, int OCC_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_;  // tile of C of one workgroup
    static constexpr int BK = BK_;            // k extent of one stage: 32 or 64
    static constexpr int WM = WM_, WN = WN_;  // its waves, as a grid over that tile
    static constexpr int WK = WK_;            // groups of WM x WN waves that split k between them
    static constexpr int NB = NB_;            // stages of a ring
    static constexpr int OCC = OCC_;          // workgroups per compute unit
};

// Size of the buffer descriptors and, as a lane's offset, the mark of a chunk outside the matrix: real offsets stay below it (checked by the host).
constexpr unsigned kBufferSize = 0x80000000u;

struct Epilogue {
    const void* bias;        // [N] or null
    const uint16_t* residual;  // or null
    uint16_t* pre;           // or null
    int ldr, ldp, bias_f32, act;
};

struct Args {
    const char *a, *b;
    char* out;               // C, or the ranges' parts, [range][M][N] floats
    int M, N, K, lda, ldb, ldo;
    int kc;                  // values of k of a range (PARTS)
    Epilogue e;
};

// Eight consecutive values of one row of C: bias, activation, residual, one rounding.
template <class T>
__device__ __forceinline__ void finish8(const Epilogue& e, uint16_t* out, int ldo, int m, int n, float* v) {
    if (e.bias) {
        float b[8];
        if (e.bias_f32) {
            const float4 lo = ((const float4*)((const float*)e.bias + n))[0], hi = ((const float4*)((const float*)e.bias + n))[1];
            b[0] = lo.x, b[1] = lo.y, b[2] = lo.z, b[3] = lo.w, b[4] = hi.x, b[5] = hi.y, b[6] = hi.z, b[7] = hi.w;
        } else {
            unpack8<T>(*(const u32x4*)((const uint16_t*)e.bias + n), b);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += b[i];
    }
    if (e.pre) *(u32x4*)(e.pre + (size_t)m * e.ldp + n) = pack8<T>(v);
    act8(v, e.act);
    if (e.residual) {
        float r[8];
        unpack8<T>(*(const u32x4*)(e.residual + (size_t)m * e.ldr + n), r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    *(u32x4*)(out + (size_t)m * ldo + n) = pack8<T>(v);
}

// One operand's piece of a stage: R rows (m or n) of BK values of k, or BK rows of R values.
template <bool ALONG, int R, int BK, int NW>
struct Piece {
    static constexpr int BYTES = R * BK * 2, LOADS = BYTES / 1024 / NW, CHUNKS = ALONG ? BK / 8 : R / 8;  // (chunks of 16 bytes of a row)
    static_assert(LOADS * 1024 * NW == BYTES, "whole load instructions per wave");
    static constexpr int SLOTS = R / 16;
    // Where a row's chunks lie.  k along: the chunk is XOR-ed with a code of the row that puts 16 rows' reads of one chunk into all
    // banks.  Else 32-byte slots of 16 columns: the transposing read takes 4 rows x 32 bytes per 16 lanes, and two such groups, 8
    // rows apart, per clock.
    static __device__ __forceinline__ int code(int row) {
        if (ALONG) return gemm::a_code<CHUNKS>(row);
        const int hi = (row >> 3) & 1;
        return SLOTS % 8 == 0 ? ((row & 3) | (hi << 2)) : SLOTS % 4 == 0 ? (((row >> 1) & 1) | (hi << 1)) : SLOTS == 2 ? hi : 0;
    }
    unsigned voff[LOADS];
    int k[LOADS];       // k of the lane's chunk inside a stage
    const char* p;
    __device__ __forceinline__ void init(const char* base, int ld, int first, int end, int k0, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int ci = (wave * LOADS + i) * 64 + lane, row = ci / CHUNKS, pos = ci % CHUNKS;
            if (ALONG) {
                k[i] = (pos ^ code(row)) * 8;
                voff[i] = first + row < end ? (unsigned)row * (unsigned)(ld * 2) + (unsigned)(k[i] * 2) : kBufferSize;
            } else {
                const int col = ((((pos >> 1) ^ code(row)) << 1) | (pos & 1)) * 8;
                k[i] = row;
                voff[i] = first + col < end ? (unsigned)row * (unsigned)(ld * 2) + (unsigned)(col * 2) : kBufferSize;
            }
        }
        p = base + (ALONG ? (size_t)first * ld * 2 + (size_t)k0 * 2 : (size_t)first * 2 + (size_t)k0 * ld * 2);
    }
    __device__ __forceinline__ void clip(int left) {  // values of k that are left
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (k[i] >= left) voff[i] = kBufferSize;
    }
    __device__ __forceinline__ void advance(int step, int ld) { p += ALONG ? (size_t)step * 2 : (size_t)step * ld * 2; }
    // A lane's address for fragments of 16 rows (columns) from `at` on, k from 32 j on.
    static __device__ __forceinline__ unsigned address(int at, int j, int lane) {
        if (ALONG) return (at + (lane & 15)) * (BK * 2) + (((j * 4 + (lane >> 4)) ^ code(lane & 15)) * 16);
        const int i16 = lane & 15, row = 8 * (lane >> 4) + (i16 >> 2);
        return (row + 32 * j) * (R * 2) + (((at >> 4) ^ code(row)) * 32) + (i16 & 3) * 8;
    }
    static __device__ __forceinline__ u32x4 read(unsigned at) {
        if constexpr (ALONG) {
            typedef const u32x4 __attribute__((address_space(3))) * lds_u32x4_ptr;
            return *(lds_u32x4_ptr)(unsigned long)at;
        } else {
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(unsigned long)at));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(unsigned long)(at + 4 * R * 2)));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

template <class T, class TL, bool A_ALONG, bool B_ALONG, bool PARTS>
__global__ __launch_bounds__(TL::WM * TL::WN * TL::WK * 64, (TL::OCC * TL::WM * TL::WN * TL::WK + 3) / 4) void product_kernel(Args p) {
    constexpr int BM = TL::BM, BN = TL::BN, WM = TL::WM, WN = TL::WN, WK = TL::WK, NB = TL::NB, BK = TL::BK, KS = BK / 32;
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    using PA = Piece<A_ALONG, BM, BK, NW>;
    using PB = Piece<B_ALONG, BN, BK, NW>;
    constexpr int LA = PA::LOADS, LB = PB::LOADS, LPS = LA + LB;
    constexpr int RING = NB * (PA::BYTES + PB::BYTES);
    static_assert(NT % 2 == 0, "C is stored in pairs of 16-column tiles");
    static_assert(NB >= 2 && (NB - 1) * LPS <= 63, "the counted waits must fit s_waitcnt's field");
    static_assert(WK == 1 || RING >= BM * BN * 4, "a ring also holds its group's partial sums");
    static_assert(WK * RING <= 160 * 1024, "LDS of a compute unit");

    __shared__ __attribute__((aligned(256))) u32x4 smem[WK * RING / 16];
    char* const smem_b = reinterpret_cast<char*>(smem);

    const int lane = threadIdx.x & 63;
    const int wave_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wk = wave_wg / NW, wave = wave_wg % NW;
    const unsigned lds_a = lds_address(smem_b) + wk * RING, lds_b = lds_a + NB * PA::BYTES;
    const int wm = wave / WN, wn = wave % WN;
    const int M = p.M, N = p.N;
    const int ntm = 1 + (M - 1) / BM, ntn = 1 + (N - 1) / BN;
    int tm, tn, range = 0, k0 = 0, K1 = p.K;  // (K1: end of the k range)
    if constexpr (PARTS) {
        const int tiles = ntm * ntn;
        range = (int)blockIdx.x / tiles;
        gemm::tile_of_block((int)blockIdx.x - range * tiles, ntm, ntn, tm, tn);
        k0 = range * p.kc;
        K1 = min(p.K, k0 + p.kc);
    } else {
        gemm::tile_of_block((int)blockIdx.x, ntm, ntn, tm, tn);
    }
    const int m0 = tm * BM, n0 = tn * BN;
    const int nkt = (K1 - k0 + WK * BK - 1) / (WK * BK);  // a group's k: every WK-th stage
    constexpr int step = WK * BK;
    k0 += wk * BK;

    PA pa;
    PB pb;
    pa.init(p.a, p.lda, m0, M, k0, wave, lane);
    pb.init(p.b, p.ldb, n0, N, k0, wave, lane);
    int left = K1 - k0;  // values of k behind the first of the next stage to be requested
    u32x4 ra, rb;
    auto next_stage = [&](int t) __attribute__((always_inline)) {
        if (left < BK) pa.clip(left), pb.clip(left);  // the last, partial stage: chunks past the end deliver zeros on both sides
        const unsigned size = t < nkt ? kBufferSize : 0u;
        ra = attn::buffer_resource(pa.p, size), rb = attn::buffer_resource(pb.p, size);
        pa.advance(step, p.lda), pb.advance(step, p.ldb);
        left -= step;
    };
    unsigned lbuf = 0;  // buffer of the stage being requested
    auto issue = [&](auto l_c) __attribute__((always_inline)) {
        constexpr int l = decltype(l_c)::value;
        if constexpr (l < LA) attn::buffer_to_lds_16(ra, pa.voff[l], lds_a + lbuf * PA::BYTES + (wave * LA + l) * 1024);
        else attn::buffer_to_lds_16(rb, pb.voff[l - LA], lds_b + lbuf * PB::BYTES + (wave * LB + l - LA) * 1024);
    };

    // k along the rows: one address for each step, fragments 16 rows apart; by rows of k: one for each fragment, steps 32 rows apart
    unsigned a_base[A_ALONG ? KS : MT], b_base[B_ALONG ? KS : NT];
#pragma unroll
    for (int i = 0; i < (A_ALONG ? KS : MT); ++i) a_base[i] = lds_a + (A_ALONG ? PA::address(wm * TM, i, lane) : PA::address(wm * TM + 16 * i, 0, lane));
#pragma unroll
    for (int i = 0; i < (B_ALONG ? KS : NT); ++i) b_base[i] = lds_b + (B_ALONG ? PB::address(wn * TN, i, lane) : PB::address(wn * TN + 16 * i, 0, lane));
    auto read_a = [&](int mt, int j, unsigned buf) __attribute__((always_inline)) -> u32x4 {
        return PA::read(buf * PA::BYTES + (A_ALONG ? a_base[j] + mt * 16 * (BK * 2) : a_base[mt] + j * 32 * (BM * 2)));
    };
    auto read_b = [&](int nt, int j, unsigned buf) __attribute__((always_inline)) -> u32x4 {
        return PB::read(buf * PB::BYTES + (B_ALONG ? b_base[j] + nt * 16 * (BK * 2) : b_base[nt] + j * 32 * (BN * 2)));
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};

    // The loads l = 0 .. LPS-1 of a stage go out one by one between the MFMAs, from the step behind the barrier on and through the steps
    // ahead of the next one; load l behind MFMA number slot(l).
    constexpr int FIRST = NB == 2 ? 0 : KS == 1 ? MT * NT / 2 : MT * NT / 4, SPAN = (NB == 2 ? 1 : KS) * MT * NT;
    auto slot = [](int l) constexpr { return FIRST + l * (SPAN - FIRST) / LPS; };
    auto first_loads = [=]() constexpr { int n = 0; for (int l = 0; l < LPS; ++l) n += slot(l) < MT * NT; return n; };
#pragma unroll
    for (int t = 0; t < NB; ++t) {
        next_stage(t);
        lbuf = t;
        attn::static_for<LPS>([&](auto l_c) __attribute__((always_inline)) {
            if (t < NB - 1 || slot(decltype(l_c)::value) < MT * NT) issue(l_c);
        });
    }
    u32x4 fa[2][MT], fb[2][NT];
    auto meet = []() __attribute__((always_inline)) { if constexpr (NW > 1) asm volatile("s_barrier" ::: "memory"); };
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 2) * LPS + first_loads()) : "memory");
    meet();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) fb[0][nt] = read_b(nt, 0, 0);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) fa[0][mt] = read_a(mt, 0, 0);

    unsigned buf = 0;  // t % NB
    auto stage = [&](auto par_c, int t) __attribute__((always_inline)) {
        const unsigned nbuf = buf + 1 == NB ? 0 : buf + 1;
        attn::static_for<KS>([&](auto j_c) __attribute__((always_inline)) {
            constexpr int j = decltype(j_c)::value, P = (decltype(par_c)::value + j) & 1, Q = P ^ 1;
            constexpr bool LAST = j == KS - 1;
            constexpr int nj = LAST ? 0 : j + 1;
            const unsigned rbuf = LAST ? nbuf : buf;
            if constexpr (LAST) {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NB - 2) * LPS) : "memory");
                meet();
                next_stage(t + NB);
                lbuf = buf;
            }
            attn::static_for<MT * NT>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value, mt = i / NT, nt = i % NT;
                acc[mt][nt] = T::mfma(fb[P][nt], fa[P][mt], acc[mt][nt]);
                // fragment reads spread over the first half of the step, loads over the second
                constexpr int R = MT + NT, STEPS = MT * NT / 2 > R ? R : (MT * NT + 1) / 2;
                attn::static_for<R>([&](auto r_c) __attribute__((always_inline)) {
                    constexpr int q = decltype(r_c)::value;
                    if constexpr (i == q * STEPS / R) {
                        if constexpr (q < NT) fb[Q][q] = read_b(q, nj, rbuf);
                        else fa[Q][q - NT] = read_a(q - NT, nj, rbuf);
                    }
                });
                attn::static_for<LPS>([&](auto l_c) __attribute__((always_inline)) {
                    if constexpr (slot(decltype(l_c)::value) == (LAST ? 0 : j + 1) * MT * NT + i) issue(l_c);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        buf = nbuf;
    };
    if constexpr (KS % 2 == 0) {
        for (int t = 0; t < nkt; ++t) stage(std::integral_constant<int, 0>{}, t);
    } else {
        for (int t = 0; t < nkt; t += 2) {
            stage(std::integral_constant<int, 0>{}, t);
            stage(std::integral_constant<int, 1>{}, t + 1);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (stages past the end were requested empty)

    // ---- a lane holds n = 4g .. 4g+3 of one row of each 16 x 16 tile; exchanged between the odd and even 16-lane groups of two
    // neighbouring tiles it has eight consecutive n.
    const int g = lane >> 4;
    auto store_pair = [&](int mt, int nt, f32x4 x, f32x4 y) __attribute__((always_inline)) {
        const int m = m0 + wm * TM + mt * 16 + (lane & 15);
        if constexpr (PARTS) {
            const int n = n0 + wn * TN + nt * 16 + g * 4;
            float* const row = (float*)p.out + ((size_t)range * M + m) * N;
            if (m < M && n < N) *(f32x4*)(row + n) = x;
            if (m < M && n + 16 < N) *(f32x4*)(row + n + 16) = y;
            return;
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[i]), __float_as_uint(y[i]), false, false);
            v[i] = __uint_as_float(s[0]), v[4 + i] = __uint_as_float(s[1]);
        }
        const int n = n0 + wn * TN + nt * 16 + (g & 1) * 16 + (g >> 1) * 8;
        if (m < M && n < N) finish8<T>(p.e, (uint16_t*)p.out, p.ldo, m, n, v);
    };
    if constexpr (WK == 1) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; nt += 2) store_pair(mt, nt, acc[mt][nt], acc[mt][nt + 1]);
    } else {
        constexpr int PAIRS = MT * NT / 2;
        if constexpr (NW > 1) __syncthreads();  // the ring is shared by the group's waves
        f32x4* const mine = reinterpret_cast<f32x4*>(smem_b + wk * RING + wave * (TM * TN * 4)) + lane;
#pragma unroll
        for (int i = 0; i < MT * NT; ++i) mine[i * 64] = acc[i / NT][i % NT];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < (PAIRS + WK - 1) / WK; ++q) {
            const int pr = q * WK + wk;
            if (PAIRS % WK != 0 && pr >= PAIRS) break;
            f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const f32x4* part = reinterpret_cast<const f32x4*>(smem_b + w * RING + wave * (TM * TN * 4)) + lane;
                x += part[2 * pr * 64];
                y += part[(2 * pr + 1) * 64];
            }
            store_pair(pr / (NT / 2), pr % (NT / 2) * 2, x, y);
        }
    }
}

}  // namespace linear
