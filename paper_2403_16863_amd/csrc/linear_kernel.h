// Matrix products in three layouts with bias, activation and residual in the epilogue, for gfx950 (MI355X): the kernel behind
// gemm_linear and the two products of gemm_linear_bwd (include/linear.h has the formulas).
//
// C[m, n] = sum_k A(m, k) B(k, n).  Either operand lies by rows of its own index with k along them (A of every product but the weight's
// gradient, a weight [N, K]) or by rows of k (a weight [K, N], both operands of the weight's gradient, whose k are the tokens).
//
//  * 16x16x32 MFMA, transposed product C^T += B^T A^T: a lane of the accumulator holds four consecutive n of one row of C.  Fragments of
//    an operand with k along its rows are 16-byte reads of LDS, those of one by rows of k two transposing reads: the two operands are
//    symmetric, so all layouts run one loop.
//  * A ring of NB stages of BK values of k in LDS, filled by direct global -> LDS buffer loads.  A stage is two steps; each multiplies the fragments that
//    were read one step ago and reads the next step's, with the stage's loads and barriers between the products (where, is said at FREED and LANDED).
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

// The activations of a lane's values.  In 32 bits with the hardware's exponential (2^x) and reciprocal, each good to a step or so: the results
// are rounded to 16 bits.  z = -inf gives NaN in silu and both gelu, -inf times 0, as their formulas do.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)); }
// sigmoid(2 v) of the tanh form's argument v = sqrt(2 / pi) (z + 0.044715 z^3): tanh v = 2 sigmoid(2 v) - 1, so the form is z times it: one
// exponential, and no difference of near values where the result is small.  (The constants times -log2 e.)
__device__ __forceinline__ float sigmoid_of_cubic(float z) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * fmaf(z * z, -0.10294324f, -2.3022082f)));
}
// The normal distribution's integral from -inf to z, and in *density its density.  With x = |z| / sqrt 2 and t = 1 / (1 + 0.44 x), e^(x^2) erfc(x) is a
// polynomial in t (Hastings' form) to 5e-7 of itself, its coefficients fitted to the least relative error over 0 .. 20: the tail
// keeps its digits for negative z, where 1 + erf loses them, at a third of the library function's instructions.
__device__ __forceinline__ float normal(float z, float* density) {
    const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f), t = __builtin_amdgcn_rcpf(fmaf(0.31112698372208092f, fabsf(z), 1.f));
    float y = fmaf(0.06935601595f, t, -0.2710227993f);
    y = fmaf(y, t, 0.2862967791f);
    y = fmaf(y, t, -0.01209306972f);
    y = fmaf(y, t, 0.2123377131f);
    y = fmaf(y, t, 0.2181195787f);
    y = fmaf(y, t, 0.2487810698f);
    y = fmaf(y, t, 0.2482244134f);
    const float tail = 0.5f * e * (y * t);
    *density = 0.3989422804014327f * e;
    return z < 0.f ? tail : 1.f - tail;
}

template <int W>
__device__ __forceinline__ void activate(float* v, int kind) {
    if (kind == RELU) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
    } else if (kind == SILU) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= sigmoid(v[i]);
    } else if (kind == GELU) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            float density;
            v[i] *= normal(v[i], &density);
        }
    } else if (kind == GELU_TANH) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= sigmoid_of_cubic(v[i]);
    }
}

// Beyond 10^4 the smooth activations' slopes are 0 and 1 to all digits, and their terms, whose products would be infinity times 0, are formed there.  NaN stays.
__device__ __forceinline__ float within(float v) { return v > 1e4f ? 1e4f : v < -1e4f ? -1e4f : v; }

// g <- g act'(v)
__device__ __forceinline__ void act_slope8(const float* values, float* g, int kind) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = kind == RELU ? values[i] : within(values[i]);
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
            const float p = sigmoid_of_cubic(v[i]);
            g[i] *= p * fmaf(1.5957691216057308f * v[i] * (1.f - p), fmaf(3.f * 0.044715f * v[i], v[i], 1.f), 1.f);
        }
    }
}

template <int BM_, int BN_, int BK_, int WM_, int WN_, int WK_, int NB_, int OCC_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_;  // tile of C of one workgroup
    static constexpr int BK = BK_;            // k extent of one stage
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
    // Rows of pre begin on lines of 128 bytes: it is stored past the caches, for the backward pass reads it later (4096 x 16384 x 4096 437 -> 428 us; off the
    // lines the parts of a line would go out by themselves, 7782 x 10248 x 648 236 us in place of 165).
    int pre_lines;
};

struct Args {
    const char *a, *b;
    char* out;               // C, or the ranges' parts, [range][M][N] floats
    int M, N, K, lda, ldb, ldo;
    int kc;                  // values of k of a range (PARTS)
    Epilogue e;
};

// What the epilogue reads for W = 8 or 4 consecutive columns of a row.  All of it is asked for ahead of the first store, behind which the compiler, which
// does not know that they do not meet, would keep it: a load's time for each store.
template <int W>
using Packed = std::conditional_t<W == 8, u32x4, u32x2>;
template <class T, int W>
__device__ __forceinline__ void unpack(Packed<W> w, float* x) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) T::unpack2(w[i], x + 2 * i);
}
template <class T, int W>
__device__ __forceinline__ Packed<W> pack(const float* x) {
    Packed<W> w;
#pragma unroll
    for (int i = 0; i < W / 2; ++i) w[i] = T::pack2(x[2 * i], x[2 * i + 1]);
    return w;
}
template <class T, int W>
__device__ __forceinline__ void load_bias(const Epilogue& e, int n, bool in, float* b) {
    if (in && e.bias && e.bias_f32) {
#pragma unroll
        for (int i = 0; i < W; i += 4) *(f32x4*)(b + i) = *(const f32x4*)((const float*)e.bias + n + i);
    } else if (in && e.bias) {
        unpack<T, W>(*(const Packed<W>*)((const uint16_t*)e.bias + n), b);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) b[i] = 0;
    }
}
template <int W>
__device__ __forceinline__ Packed<W> load_residual(const Epilogue& e, int m, int n, bool in) {
    return in && e.residual ? *(const Packed<W>*)(e.residual + (size_t)m * e.ldr + n) : Packed<W>(0);
}

// Consecutive values of one row of C: bias, activation, residual, one rounding.
template <class T, int W>
__device__ __forceinline__ void finish(const Epilogue& e, uint16_t* out, int ldo, int m, int n, float* v, const float* bias, Packed<W> residual) {
    if (e.bias) {  // (a sum without one keeps the sign of a zero)
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += bias[i];
    }
    if (e.pre) {
        Packed<W>* const to = (Packed<W>*)(e.pre + (size_t)m * e.ldp + n);
        if (e.pre_lines) __builtin_nontemporal_store(pack<T, W>(v), to);
        else *to = pack<T, W>(v);
    }
    activate<W>(v, e.act);
    if (e.residual) {
        float r[W];
        unpack<T, W>(residual, r);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += r[i];
    }
    *(Packed<W>*)(out + (size_t)m * ldo + n) = pack<T, W>(v);
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
        return SLOTS % 8 == 0 ? ((row & 3) | (hi << 2)) : SLOTS % 4 == 0 ? (((row >> 1) & 1) | (hi << 1)) : SLOTS % 2 == 0 ? hi : 0;
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
    // The fragment `offset` bytes (a constant) behind a lane's address.
    static __device__ __forceinline__ u32x4 read(unsigned at, int offset) {
        typedef const char __attribute__((address_space(3))) * lds_char_ptr;
        const lds_char_ptr p = (lds_char_ptr)(unsigned long)at + offset;
        if constexpr (ALONG) {
            typedef const u32x4 __attribute__((address_space(3))) * lds_u32x4_ptr;
            return *(lds_u32x4_ptr)p;
        } else {
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)p));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(p + 4 * R * 2)));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

// 16 bytes a lane from global memory to LDS, OFFSET bytes behind `lds`.
template <int OFFSET>
__device__ __forceinline__ void buffer_to_lds(u32x4 rsrc, unsigned voff, unsigned lds) {
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds), "n"(OFFSET) : "memory", "m0", "scc");
}

template <class T, class TL, bool A_ALONG, bool B_ALONG, bool PARTS>
__global__ __launch_bounds__(TL::WM * TL::WN * TL::WK * 64, (TL::OCC * TL::WM * TL::WN * TL::WK + 3) / 4) void product_kernel(Args p) {
    constexpr int BM = TL::BM, BN = TL::BN, WM = TL::WM, WN = TL::WN, WK = TL::WK, NB = TL::NB, BK = TL::BK, KS = BK / 32;
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 16, NT = TN / 16;
    using PA = Piece<A_ALONG, BM, BK, NW>;
    using PB = Piece<B_ALONG, BN, BK, NW>;
    constexpr int LA = PA::LOADS, LB = PB::LOADS, LPS = LA + LB;
    constexpr int RING = NB * (PA::BYTES + PB::BYTES);
    static_assert(KS == 2, "fragments of a stage's two steps take turns");
    constexpr int TOGETHER = NT % 2 ? 1 : 2, WIDE = 4 * TOGETHER;  // 16-column tiles whose values a lane stores at once, and how many those are
    static_assert(NT == 1 || TOGETHER == 2, "C is stored in pairs of 16-column tiles, or it is one");
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
        if (left < BK) {  // the last, partial stage: chunks past the end deliver zeros on both sides
            asm volatile("");  // (a branch: as selections the clipping would cost every stage)
            pa.clip(left), pb.clip(left);
        }
        const unsigned size = t < nkt ? kBufferSize : 0u;
        ra = attn::buffer_resource(pa.p, size), rb = attn::buffer_resource(pb.p, size);
        pa.advance(step, p.lda), pb.advance(step, p.ldb);
        left -= step;
    };
    unsigned load_a = lds_a + wave * (LA * 1024), load_b = lds_b + wave * (LB * 1024);  // where the stage being requested goes
    auto issue = [&](auto l_c) __attribute__((always_inline)) {
        constexpr int l = decltype(l_c)::value;
        if constexpr (l < LA) buffer_to_lds<l * 1024>(ra, pa.voff[l], load_a);
        else buffer_to_lds<(l - LA) * 1024>(rb, pb.voff[l - LA], load_b);
    };

    // k along the rows: one address for each step, fragments 16 rows apart; by rows of k: one for each fragment, steps 32 rows apart.  They follow
    // the stage whose fragments are read, so that everything else of an address is a constant of the instruction.
    constexpr int NBA = A_ALONG ? KS : MT, NBB = B_ALONG ? KS : NT;
    unsigned a_base[NBA], b_base[NBB];
#pragma unroll
    for (int i = 0; i < NBA; ++i) a_base[i] = lds_a + (A_ALONG ? PA::address(wm * TM, i, lane) : PA::address(wm * TM + 16 * i, 0, lane));
#pragma unroll
    for (int i = 0; i < NBB; ++i) b_base[i] = lds_b + (B_ALONG ? PB::address(wn * TN, i, lane) : PB::address(wn * TN + 16 * i, 0, lane));
    auto read_a = [&](int mt, int j) __attribute__((always_inline)) -> u32x4 {
        return PA::read(a_base[A_ALONG ? j : mt], A_ALONG ? mt * 16 * (BK * 2) : j * 32 * (BM * 2));
    };
    auto read_b = [&](int nt, int j) __attribute__((always_inline)) -> u32x4 {
        return PB::read(b_base[B_ALONG ? j : nt], B_ALONG ? nt * 16 * (BK * 2) : j * 32 * (BN * 2));
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};

    // A stage is 2 S products, S to a step; where its other work goes, in products from its first:
    //   0 ..      the second step's fragments are read
    //   FREED     all of the stage's fragments are in registers, in all waves: its buffer takes the loads of stage t + NB from here on, load l at slot(l)
    //   LANDED    the loads of stage t + 1 are there, of all waves; its first step's fragments are read
    // With three buffers and more both are one barrier, ahead of the second step.  With two the loads have to go out and land within the stage between two such
    // barriers, and half of that is the time that 64 KB take to come; a barrier of its own for each gives them longer, from FREED to the next stage's LANDED.
    // (256 x 256 tiles, bfloat16, us, with one barrier / with two and the reads among a quarter of a step / five eighths, as here: 4096 x 16384 x 4096 with k along both
    // 430 / 417 / 404, the other layouts 435 / 427 / 410 and 435 / 435 / 416; reads in a lump meet those of the unit's other waves.  The vendor's library takes
    // 360, 412 and 485.  Four waves of 128 x 128 read a third less and take 414 to 425.)
    constexpr int S = MT * NT, R = MT + NT, READS = NB == 2 ? S * 5 / 8 : S / 2 > R ? R : (S + 1) / 2;  // (products among which a step's fragments are read)
    constexpr int FREED = NB == 2 ? S * 6 / 8 : S, LANDED = NB == 2 ? S + S * 3 / 8 : S;
    constexpr int FIRST = NB == 2 ? FREED : S + S / 4, SPAN = NB == 2 ? S * 10 / 8 : 2 * S - S / 4;
    auto slot = [](int l) constexpr { return FIRST + l * SPAN / LPS; };
    auto before = [=](int at) constexpr { int n = 0; for (int l = 0; l < LPS; ++l) n += slot(l) < at; return n; };
    static_assert(FREED > (R - 1) * READS / R && LANDED + READS <= 2 * S, "a step's fragments are read before their buffer is freed, and within a stage");
    static_assert(NB > 2 || FIRST + SPAN <= 2 * S, "with two buffers a stage's loads go out within one");
#pragma unroll
    for (int t = 0; t < NB; ++t) {
        next_stage(t);
        attn::static_for<LPS>([&](auto l_c) __attribute__((always_inline)) {
            if (NB == 2 || t < NB - 1 || slot(decltype(l_c)::value) < 2 * S) issue(l_c);
        });
        if (t < NB - 1) load_a += PA::BYTES, load_b += PB::BYTES;
    }
    u32x4 fa[2][MT], fb[2][NT];
    auto meet = []() __attribute__((always_inline)) { if constexpr (NW > 1) asm volatile("s_barrier" ::: "memory"); };
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NB == 2 ? LPS : (NB - 2) * LPS + before(2 * S)) : "memory");
    meet();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) fb[0][nt] = read_b(nt, 0);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) fa[0][mt] = read_a(mt, 0);

    unsigned buf = 0;  // t % NB
    for (int t = 0; t < nkt; ++t) {
        const unsigned nbuf = buf + 1 == NB ? 0 : buf + 1;
        attn::static_for<2 * S>([&](auto at_c) __attribute__((always_inline)) {
            constexpr int at = decltype(at_c)::value, P = at / S, i = at % S, mt = i / NT, nt = i % NT;
            if constexpr (at == FREED && NB == 2) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                meet();
            }
            if constexpr (at == LANDED) {
                if constexpr (NB == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(before(LANDED)) : "memory");
                else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NB - 2) * LPS) : "memory");
                meet();
                const unsigned on_a = nbuf ? PA::BYTES : -(NB - 1) * PA::BYTES, on_b = nbuf ? PB::BYTES : -(NB - 1) * PB::BYTES;
#pragma unroll
                for (int n = 0; n < NBA; ++n) a_base[n] += on_a;
#pragma unroll
                for (int n = 0; n < NBB; ++n) b_base[n] += on_b;
            }
            if constexpr (at == FREED) {
                next_stage(t + NB);
                load_a = lds_a + wave * (LA * 1024) + buf * PA::BYTES, load_b = lds_b + wave * (LB * 1024) + buf * PB::BYTES;
            }
            acc[mt][nt] = T::mfma(fb[P][nt], fa[P][mt], acc[mt][nt]);
            attn::static_for<R>([&](auto r_c) __attribute__((always_inline)) {
                constexpr int q = decltype(r_c)::value, when = q * READS / R;
                if constexpr (at == when || at == LANDED + when) {
                    if constexpr (q < NT) fb[at == when][q] = read_b(q, at == when);
                    else fa[at == when][q - NT] = read_a(q - NT, at == when);
                }
            });
            attn::static_for<LPS>([&](auto l_c) __attribute__((always_inline)) {
                if constexpr (slot(decltype(l_c)::value) % (2 * S) == at) issue(l_c);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        buf = nbuf;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (stages past the end were requested empty)

    // ---- a lane holds n = 4g .. 4g+3 of one row of each 16 x 16 tile; exchanged between the odd and even 16-lane groups of two
    // neighbouring tiles it has eight consecutive n.
    const int g = lane >> 4;
    auto row_of = [&](int mt) __attribute__((always_inline)) { return m0 + wm * TM + mt * 16 + (lane & 15); };
    auto column_of = [&](int nt) __attribute__((always_inline)) {
        return n0 + wn * TN + nt * 16 + (PARTS || TOGETHER == 1 ? g * 4 : (g & 1) * 16 + (g >> 1) * 8);
    };
    auto store = [&](int mt, int nt, f32x4 x, f32x4 y, const float* bias, Packed<WIDE> residual) __attribute__((always_inline)) {
        const int m = row_of(mt), n = column_of(nt);
        if constexpr (PARTS) {
            float* const row = (float*)p.out + ((size_t)range * M + m) * N;
            if (m < M && n < N) *(f32x4*)(row + n) = x;
            if (TOGETHER == 2 && m < M && n + 16 < N) *(f32x4*)(row + n + 16) = y;
            return;
        }
        float v[WIDE];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TOGETHER == 2) {
                const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[i]), __float_as_uint(y[i]), false, false);
                v[i] = __uint_as_float(s[0]), v[4 + i] = __uint_as_float(s[1]);
            } else {
                v[i] = x[i];
            }
        }
        if (m < M && n < N) finish<T, WIDE>(p.e, (uint16_t*)p.out, p.ldo, m, n, v, bias, residual);
    };
    constexpr int ACROSS = NT / TOGETHER, STORES = MT * ACROSS;
    if constexpr (WK == 1) {
        float bias[ACROSS][WIDE];
        Packed<WIDE> residual[MT][ACROSS];
        if constexpr (!PARTS) {
#pragma unroll
            for (int q = 0; q < ACROSS; ++q) {
                const int n = column_of(TOGETHER * q);
                load_bias<T, WIDE>(p.e, n, n < N, bias[q]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) residual[mt][q] = load_residual<WIDE>(p.e, row_of(mt), n, n < N && row_of(mt) < M);
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; nt += TOGETHER) store(mt, nt, acc[mt][nt], acc[mt][nt + TOGETHER - 1], bias[nt / TOGETHER], residual[mt][nt / TOGETHER]);
    } else {
        constexpr int MINE = (STORES + WK - 1) / WK;
        if constexpr (NW > 1) __syncthreads();  // the ring is shared by the group's waves
        f32x4* const mine = reinterpret_cast<f32x4*>(smem_b + wk * RING + wave * (TM * TN * 4)) + lane;
#pragma unroll
        for (int i = 0; i < MT * NT; ++i) mine[i * 64] = acc[i / NT][i % NT];
        float bias[MINE][WIDE];
        Packed<WIDE> residual[MINE];
        if constexpr (!PARTS) {
#pragma unroll
            for (int q = 0; q < MINE; ++q) {
                const int at = q * WK + wk, m = row_of(at / ACROSS), n = column_of(at % ACROSS * TOGETHER);
                load_bias<T, WIDE>(p.e, n, at < STORES && n < N, bias[q]);
                residual[q] = load_residual<WIDE>(p.e, m, n, at < STORES && n < N && m < M);
            }
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < MINE; ++q) {
            const int at = q * WK + wk;
            if (STORES % WK != 0 && at >= STORES) break;
            f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const f32x4* part = reinterpret_cast<const f32x4*>(smem_b + w * RING + wave * (TM * TN * 4)) + lane;
                x += part[TOGETHER * at * 64];
                if (TOGETHER == 2) y += part[(2 * at + 1) * 64];
            }
            store(at / ACROSS, at % ACROSS * TOGETHER, x, y, bias[q], residual[q]);
        }
    }
}

}  // namespace linear
