// Appending to the 4-bit cache and reading it back (include/kv4.h has the format).
//
// Both move bytes: a token's head comes as 4d bytes and stays as d + d/16.  d / 16 lanes share a head's vector, each with
// 8 channels of the lower and 8 of the upper half, so that a rotation's pairs (i, i + d/2) meet in one lane without an exchange, a
// load is 16 bytes, and the four lanes of a block of 32 find its largest value in two steps.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/kv4.h"
#include "kv4_format.h"

namespace kv4 {

struct AppendArgs {
    const uint16_t *k, *v;
    long long k_token, k_head, v_token, v_head;
    uint8_t* cache;
    const int* slots;
    const float *cos, *sin;
    const int* positions;
    int rows, interleaved, T, heads, slots_all, page_shift;
};

// Vector `vec` of a launch is a token and a head: 16 tokens of one head follow each other, so that the lanes of a wave write (and read) a cache's
// block of 16 tokens together where the tokens have neighbouring slots (heads first: 16384 tokens of 8 heads, d = 64, appended in 15.0 us, so in 11.8).
// False behind the last token of a block of 16 that is not full.
__device__ __forceinline__ bool vector_of(long long vec, int T, int heads, int& t, int& h) {
    const long long block = vec >> 4;
    t = (int)(block / heads) * 16 + (int)(vec & 15), h = (int)(block % heads);
    return t < T;
}

// The scale byte and (as a float's exponent) the scale of a block whose largest magnitude is `top`: the carry out of the mantissa
// raises the exponent where top > 1.75 * 2^n.  A NaN or an infinity in the block gives 255.
__device__ __forceinline__ unsigned scale_byte(float top) {
    const unsigned bits = __float_as_uint(top);
    const int e = (int)((bits + 0x1fffffu) >> 23) - 2;
    return bits >= 0x7f800000u ? 255u : (unsigned)min(max(e, 104), 140);
}

// fmaxf would drop a NaN: magnitudes are compared as integers, where NaN is above infinity.
__device__ __forceinline__ float larger(float a, float b) {
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
}

__device__ __forceinline__ float top_of(const float* x, int n) {
    float t = 0;
    for (int i = 0; i < n; ++i) t = larger(t, fabsf(x[i]));
    return t;
}

// Eight values to four bytes of codes: the conversion rounds to nearest even and limits to 6, as the format asks.
__device__ __forceinline__ unsigned codes_of(const float* x, unsigned byte) {
    if (byte == 255u) return 0;
    const float scale = __uint_as_float(byte << 23);
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    return w;
}

template <int D, bool BF>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
#pragma clang fp contract(off)  // each product of the rotation is rounded: the codes are those of the elementary operations
    constexpr int L = D / 16;
    const long long vec = ((long long)blockIdx.x * 256 + threadIdx.x) / L;
    const int l = threadIdx.x % L;
    int t, h;
    if (!vector_of(vec, a.T, a.heads, t, h)) return;  // whole vectors: the lanes that meet below leave together
    const int slot = a.slots[t];
    if ((unsigned)slot >= (unsigned)a.slots_all) return;
    const uint16_t* pk = a.k + t * a.k_token + h * a.k_head;
    const uint16_t* pv = a.v + t * a.v_token + h * a.v_head;
    const bool pairs = a.interleaved != 0;
    const int lo = pairs ? 16 * l : 8 * l, hi = pairs ? lo + 8 : lo + D / 2;
    float k[16], v[16];
    load8<BF>(pk + lo, k);
    load8<BF>(pk + hi, k + 8);
    load8<BF>(pv + 8 * l, v);
    load8<BF>(pv + D / 2 + 8 * l, v + 8);
    if (a.cos) {
        const int at = a.positions[t];
        float c[8], s[8];
        if ((unsigned)at < (unsigned)a.rows) {
            load8f(a.cos + (long long)at * (D / 2) + 8 * l, c);
            load8f(a.sin + (long long)at * (D / 2) + 8 * l, s);
        } else {
            for (int i = 0; i < 8; ++i) c[i] = s[i] = __uint_as_float(0x7fc00000u);
        }
        for (int i = 0; i < 8; ++i) {
            const int x = pairs ? 2 * i : i, y = pairs ? 2 * i + 1 : i + 8;
            const float p = k[x], q = k[y];
            k[x] = p * c[i] - q * s[i];
            k[y] = q * c[i] + p * s[i];
        }
    }
    float k0 = top_of(k, 8), k1 = top_of(k + 8, 8), v0 = top_of(v, 8), v1 = top_of(v + 8, 8);
    if (pairs) {  // 16 channels on end: two lanes to a block
        k0 = larger(k0, k1);
        k0 = k1 = larger(k0, __shfl_xor(k0, 1));
    } else {
        k0 = larger(k0, __shfl_xor(k0, 1));
        k0 = larger(k0, __shfl_xor(k0, 2));
        k1 = larger(k1, __shfl_xor(k1, 1));
        k1 = larger(k1, __shfl_xor(k1, 2));
    }
    v0 = larger(v0, __shfl_xor(v0, 1));
    v0 = larger(v0, __shfl_xor(v0, 2));
    v1 = larger(v1, __shfl_xor(v1, 1));
    v1 = larger(v1, __shfl_xor(v1, 2));
    const unsigned bk0 = scale_byte(k0), bk1 = scale_byte(k1), bv0 = scale_byte(v0), bv1 = scale_byte(v1);

    const int page = slot >> a.page_shift, place = slot & ((1 << a.page_shift) - 1), tok = place & 15;
    uint8_t* g = a.cache + (((long long)page * a.heads + h) * (1 << (a.page_shift - 4)) + (place >> 4)) * Group<D>::bytes;
    unsigned* kc = (unsigned*)(g + tok * (D / 2));
    kc[lo / 8] = codes_of(k, bk0);
    kc[hi / 8] = codes_of(k + 8, bk1);
    uint8_t* vc = g + Group<D>::v_codes + (tok >> 2) * (2 * D) + (tok & 3) * (D / 32);
    const unsigned w0 = codes_of(v, bv0), w1 = codes_of(v + 8, bv1);
    if (D == 128) {
        *(unsigned*)(vc + l * 16) = w0;
        *(unsigned*)(vc + (8 + l) * 16) = w1;
    } else {
        *(uint16_t*)(vc + (2 * l) * 8) = (uint16_t)w0;
        *(uint16_t*)(vc + (2 * l + 1) * 8) = (uint16_t)(w0 >> 16);
        *(uint16_t*)(vc + (8 + 2 * l) * 8) = (uint16_t)w1;
        *(uint16_t*)(vc + (9 + 2 * l) * 8) = (uint16_t)(w1 >> 16);
    }
    uint8_t* ks = g + Group<D>::k_scales + tok * (D / 32);
    uint8_t* vs = g + Group<D>::v_scales + (tok >> 2) * (D / 8) + (tok & 3);
    if (pairs) {
        if ((l & 1) == 0) ks[l / 2] = (uint8_t)bk0;
    } else if ((l & 3) == 0) {
        ks[l / 4] = (uint8_t)bk0;
        ks[D / 64 + l / 4] = (uint8_t)bk1;
    }
    if ((l & 3) == 0) {
        vs[(l / 4) * 4] = (uint8_t)bv0;
        vs[(D / 64 + l / 4) * 4] = (uint8_t)bv1;
    }
}

struct ReadArgs {
    const uint8_t* cache;
    const int* slots;
    uint16_t *k, *v;
    int T, heads, slots_all, page_shift;
};

// Lane l of a vector has channels 16 l .. 16 l + 15 of keys and values: 8 bytes of codes each, under one scale.
template <int D, bool BF>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
    constexpr int L = D / 16;
    const long long vec = ((long long)blockIdx.x * 256 + threadIdx.x) / L;
    const int l = threadIdx.x % L;
    int t, h;
    if (!vector_of(vec, a.T, a.heads, t, h)) return;
    const int slot = a.slots[t];
    uint2 kc = {0, 0}, vc = {0, 0};
    unsigned kb = 127, vb = 127;
    if ((unsigned)slot < (unsigned)a.slots_all) {
        const int page = slot >> a.page_shift, place = slot & ((1 << a.page_shift) - 1), tok = place & 15;
        const uint8_t* g = a.cache + (((long long)page * a.heads + h) * (1 << (a.page_shift - 4)) + (place >> 4)) * Group<D>::bytes;
        if (a.k) {
            kc = *(const uint2*)(g + tok * (D / 2) + 8 * l);
            kb = g[Group<D>::k_scales + tok * (D / 32) + l / 2];
        }
        if (a.v) {
            const uint8_t* p = g + Group<D>::v_codes + (tok >> 2) * (2 * D) + (tok & 3) * (D / 32);
            if (D == 128) {
                vc.x = *(const unsigned*)(p + (2 * l) * 16);
                vc.y = *(const unsigned*)(p + (2 * l + 1) * 16);
            } else {
                const uint16_t* r = (const uint16_t*)(p + (4 * l) * 8);
                vc.x = r[0] | (unsigned)r[4] << 16;
                vc.y = r[8] | (unsigned)r[12] << 16;
            }
            vb = g[Group<D>::v_scales + (tok >> 2) * (D / 8) + (l / 2) * 4 + (tok & 3)];
        }
    }
    const long long at = ((long long)t * a.heads + h) * D + 16 * l;
    if (a.k) {
        *(uint4*)(a.k + at) = values8<BF>(kc.x, kb << 23);
        *(uint4*)(a.k + at + 8) = values8<BF>(kc.y, kb << 23);
    }
    if (a.v) {
        *(uint4*)(a.v + at) = values8<BF>(vc.x, vb << 23);
        *(uint4*)(a.v + at + 8) = values8<BF>(vc.y, vb << 23);
    }
}

int check_cache(const void* cache, int heads, int d, int pages, int page_size) {
    if (!cache || (uintptr_t)cache % 16 || heads < 1 || pages < 1) return KV4_EINVAL;
    if (page_size < 16 || page_size > 65536 || (page_size & (page_size - 1))) return KV4_EINVAL;
    if (d != 64 && d != 128) return KV4_EUNSUPPORTED;
    return (long long)pages * page_size > INT_MAX ? KV4_EUNSUPPORTED : KV4_OK;
}

// Threads of a launch are counted in 32 bits.
bool too_many(long long T, int heads, int d) { return (double)((T + 15) / 16 * 16) * heads * (d / 16) > 0xffffff00LL; }

int launch(const void* fn, unsigned grid, void* args, void* stream) {
    void* list[] = {args};
    if (hipLaunchKernel(fn, dim3(grid), dim3(256), list, 0, (hipStream_t)stream) != hipSuccess) {
        (void)hipGetLastError();
        return KV4_ELAUNCH;
    }
    return KV4_OK;
}

}  // namespace kv4

extern "C" {

int kv4_append(const void* k, long long k_token_stride, long long k_head_stride, const void* v, long long v_token_stride,
               long long v_head_stride, void* cache, const int* slots, const float* cos, const float* sin, const int* positions,
               int rows, int interleaved, int T, int heads, int d, int pages, int page_size, int dtype, void* stream) {
    using namespace kv4;
    if (!k || !v || !slots || T < 0 || (dtype != KV4_F16 && dtype != KV4_BF16)) return KV4_EINVAL;
    if ((uintptr_t)k % 16 || (uintptr_t)v % 16 || (uintptr_t)slots % 4 || (uintptr_t)positions % 4) return KV4_EINVAL;
    if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 8) return KV4_EINVAL;
    if (!cos != !sin || (cos && (!positions || rows < 1 || (uintptr_t)cos % 16 || (uintptr_t)sin % 16))) return KV4_EINVAL;
    if (const int rc = check_cache(cache, heads, d, pages, page_size)) return rc;
    if (too_many(T, heads, d)) return KV4_EUNSUPPORTED;
    if (T == 0) return KV4_OK;
    AppendArgs a = {(const uint16_t*)k, (const uint16_t*)v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, (uint8_t*)cache,
                    slots, cos, sin, positions, rows, interleaved, T, heads, pages * page_size, __builtin_ctz(page_size)};
    const unsigned grid = (unsigned)((((long long)T + 15) / 16 * 16 * heads * (d / 16) + 255) / 256);
    const void* fn = d == 128 ? (dtype ? (const void*)append_kernel<128, true> : (const void*)append_kernel<128, false>)
                              : (dtype ? (const void*)append_kernel<64, true> : (const void*)append_kernel<64, false>);
    return launch(fn, grid, &a, stream);
}

int kv4_read(const void* cache, const int* slots, void* k, void* v, int T, int heads, int d, int pages, int page_size, int dtype,
             void* stream) {
    using namespace kv4;
    if ((!k && !v) || !slots || T < 0 || (dtype != KV4_F16 && dtype != KV4_BF16)) return KV4_EINVAL;
    if ((uintptr_t)k % 16 || (uintptr_t)v % 16 || (uintptr_t)slots % 4) return KV4_EINVAL;
    if (const int rc = check_cache(cache, heads, d, pages, page_size)) return rc;
    if (too_many(T, heads, d)) return KV4_EUNSUPPORTED;
    if (T == 0) return KV4_OK;
    const long long bytes = (long long)T * heads * d * 2;
    const long long held = (long long)std::min((double)pages * page_size * heads * (d + d / 16), 0x1p60);  // no cache is that large
    if ((k && v && overlap(k, bytes, v, bytes)) || (k && overlap(k, bytes, cache, held)) || (v && overlap(v, bytes, cache, held))) return KV4_EINVAL;
    ReadArgs a = {(const uint8_t*)cache, slots, (uint16_t*)k, (uint16_t*)v, T, heads, pages * page_size, __builtin_ctz(page_size)};
    const unsigned grid = (unsigned)((((long long)T + 15) / 16 * 16 * heads * (d / 16) + 255) / 256);
    const void* fn = d == 128 ? (dtype ? (const void*)read_kernel<128, true> : (const void*)read_kernel<128, false>)
                              : (dtype ? (const void*)read_kernel<64, true> : (const void*)read_kernel<64, false>);
    return launch(fn, grid, &a, stream);
}

const char* kv4_strerror(int code) {
    switch (code) {
        case KV4_OK: return "ok";
        case KV4_EINVAL: return "invalid argument";
        case KV4_EUNSUPPORTED: return "unsupported size";
        case KV4_ELAUNCH: return "the HIP runtime refused the launch";
        default: return "unknown error";
    }
}

}  // extern "C"
