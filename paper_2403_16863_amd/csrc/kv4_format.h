// The 4-bit cache's bytes (include/kv4.h) as the kernels see them, and small conversions.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kv4 {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Whether an bytes at a and bn at b meet.
inline bool overlap(const void* a, long long an, const void* b, long long bn) {
    return (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}

// 16 tokens of one head.
template <int D>
struct Group {
    static constexpr int v_codes = 8 * D, k_scales = 16 * D, v_scales = 16 * D + D / 2, bytes = 17 * D;
};

template <class T>
__device__ __forceinline__ unsigned bits_of(T x) {
    static_assert(sizeof(T) == 4, "a word");
    return __builtin_bit_cast(unsigned, x);
}

// Eight 16-bit elements as floats.
template <bool BF>
__device__ __forceinline__ void values_of(uint4 w, float* x) {
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        } else {
            const f16x2 h = __builtin_bit_cast(f16x2, u[i]);
            x[2 * i] = (float)h[0];
            x[2 * i + 1] = (float)h[1];
        }
    }
}

template <bool BF>
__device__ __forceinline__ void load8(const uint16_t* p, float* x) {
    values_of<BF>(*(const uint4*)p, x);
}

__device__ __forceinline__ void load8f(const float* p, float* x) {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

template <bool BF>
__device__ __forceinline__ unsigned pack2(float a, float b) {
    if (BF) {
        const bf16x2 h = {(__bf16)a, (__bf16)b};
        return bits_of(h);
    }
    const f16x2 h = {(_Float16)a, (_Float16)b};
    return bits_of(h);
}

// Two codes (byte SEL of `codes`) times a scale, given as a word whose bits 23 to 30 are the scale's byte: the conversion
// looks at no other bit, and gives NaN where they are all ones (checked on hardware for all codes).
template <bool BF, int SEL>
__device__ __forceinline__ unsigned values2(unsigned codes, unsigned scale) {
    if (BF) return bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __uint_as_float(scale), SEL));
    return bits_of(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, __uint_as_float(scale), SEL));
}

template <bool BF>
__device__ __forceinline__ uint4 values8(unsigned codes, unsigned scale) {
    return {values2<BF, 0>(codes, scale), values2<BF, 1>(codes, scale), values2<BF, 2>(codes, scale), values2<BF, 3>(codes, scale)};
}

}  // namespace kv4
