// Device helpers of the 8-bit cache (pe_q8.cu, pe_evict.cu): e4m3 codes with
// one power-of-two scale for each (layer, page, kv-head), for K and for V.
//
// With a the largest magnitude of a page's valid tokens, the exponent e is the
// least integer with a <= 448 * 2^e (448 = the largest e4m3 number), at least
// -126, and -126 where a = 0; code = e4m3(x * 2^-e), nearest, ties to even;
// value = code * 2^e.  (e is at most 119, so that every value is a finite bf16:
// magnitudes past 1.75 * 2^127 become that.)  A power of two costs a floating format no precision, makes
// both scalings exact, and makes quantising a page again from its values change
// only what falls below 2^-14 of its largest.
//
// e4m3 has no infinity.  A token whose K or V holds an infinity or NaN for a
// kv-head is held as K codes NaN and V codes 0 there: every query row that sees
// the key gets NaN, and because V never holds NaN, a masked key's weight 0 times
// its V is 0.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "pe_internal.h"

namespace pe {

constexpr uint32_t kQ8NanWord = 0x7f7f7f7fu;   // four NaN codes
constexpr uint32_t kBf16NanPair = 0x7fc07fc0u;

__device__ __forceinline__ float pow2i(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// The scale exponent of a page whose largest magnitude has the bf16 bits a (finite, sign cleared).
__device__ __forceinline__ int q8_exponent(uint32_t a)
{
    // a = (1 + m / 128) 2^(E - 127): 448 * 2^e = 1.75 * 2^(e + 8), so e + 8 = E - 127, one more when m > 96
    const int e = static_cast<int>(a >> 7) - 135 + ((a & 0x7fu) > 96u ? 1 : 0);
    return e < -126 ? -126 : (e > 119 ? 119 : e);
}

// The same from a magnitude in 32 bits.
__device__ __forceinline__ int q8_exponent_f32(float a)
{
    const uint32_t w = __float_as_uint(a);
    const int e = static_cast<int>(w >> 23) - 135 + ((w & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -126 ? -126 : (e > 119 ? 119 : e);
}

// two codes, low byte first
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t codes)
{
    const __half2_raw hr =
        __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes & 0xffffu), __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2 *>(&hr));
}

// two codes times s, as a bf16 pair
__device__ __forceinline__ uint32_t q8_pair_to_bf16(uint32_t codes, float s)
{
    const float2 f = e4m3x2_to_float2(codes);
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * s, f.y * s);
    return *reinterpret_cast<const uint32_t *>(&b);
}

// eight codes times s as eight bf16 (exact while the scaled value is a normal bf16)
__device__ __forceinline__ uint4 q8_to_bf16(uint2 c, float s)
{
    return make_uint4(q8_pair_to_bf16(c.x, s), q8_pair_to_bf16(c.x >> 16, s), q8_pair_to_bf16(c.y, s),
                      q8_pair_to_bf16(c.y >> 16, s));
}

// eight codes times s in 32 bits
__device__ __forceinline__ void q8_to_float(uint2 c, float s, float (&y)[8])
{
    const uint32_t w[4] = {c.x, c.x >> 16, c.y, c.y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = e4m3x2_to_float2(w[i]);
        y[2 * i] = f.x * s;
        y[2 * i + 1] = f.y * s;
    }
}

// eight floats times s, rounded to codes
__device__ __forceinline__ uint2 q8_from_float(const float (&y)[8], float s)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(y[2 * i] * s, y[2 * i + 1] * s), __NV_SATFINITE, __NV_E4M3));
    return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

// a bf16 pair times s, rounded to two codes
__device__ __forceinline__ uint32_t q8_pair_from_bf16(uint32_t w, float s)
{
    const float2 f = make_float2(__uint_as_float(w << 16) * s, __uint_as_float(w & 0xffff0000u) * s);
    return static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3));
}

__device__ __forceinline__ uint2 q8_from_bf16(uint4 v, float s)
{
    return make_uint2(q8_pair_from_bf16(v.x, s) | (q8_pair_from_bf16(v.y, s) << 16),
                      q8_pair_from_bf16(v.z, s) | (q8_pair_from_bf16(v.w, s) << 16));
}

// the largest of sixteen codes' magnitudes, as a code
__device__ __forceinline__ uint32_t codes_absmax(uint4 c)
{
    constexpr uint32_t kAbs = 0x7f7f7f7fu;
    uint32_t m = __vmaxu4(__vmaxu4(c.x & kAbs, c.y & kAbs), __vmaxu4(c.z & kAbs, c.w & kAbs));
    m = __vmaxu4(m, m >> 16);
    return max(m & 0xffu, m >> 8 & 0xffu);
}

// sixteen codes times 2^k, rounded (every one that is not zero stays within 448)
__device__ __forceinline__ uint4 rescale_codes(uint4 c, int k)
{
    const float s = pow2i(max(-100, min(100, k)));
    uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const float2 a = e4m3x2_to_float2(w[x]), b = e4m3x2_to_float2(w[x] >> 16);
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a.x * s, a.y * s), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(b.x * s, b.y * s), __NV_SATFINITE, __NV_E4M3);
        w[x] = lo | hi << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// the largest magnitude of eight bf16, as bits; an infinity or NaN gives 0x7f80 or more
__device__ __forceinline__ uint32_t bf16x8_absmax(uint4 v)
{
    constexpr uint32_t kAbs = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & kAbs, v.y & kAbs), __vmaxu2(v.z & kAbs, v.w & kAbs));
    return max(m & 0xffffu, m >> 16);
}

// Threads that share one page of one kv-head, and the chunks of eight values each holds of K and of V: all of
// a page (up to 128 x 128) sits in registers between the maximum and the rounding.
__host__ __device__ constexpr int q8_unit_threads(int page_elems)
{
    return page_elems / 64 < 32 ? 32 : (page_elems / 64 > 256 ? 256 : page_elems / 64);
}
__host__ __device__ constexpr int q8_unit_chunks(int page_elems) { return page_elems / 8 / q8_unit_threads(page_elems); }

constexpr int kLogQ8Block = 8, kQ8Block = 1 << kLogQ8Block;

// Quantises one page of one kv-head.  Thread t of `threads` holds chunks c = i * threads + t (row c / CPR, eight
// columns from 8 (c % CPR)): rows [0, n_rows) are valid; load(row, col8, k, v) gives their bf16 values.  Rows below
// `old` are the page's own, held with exponents (ke0, ve0): where an exponent stays, so do their codes.  Every
// thread of the block calls this (pages wider than a warp meet at the block's barrier), `on` or not.
template <int CPR, int NC, typename Load>
__device__ __forceinline__ void q8_write_page(bool on, int t, int threads, int n_rows, int old, int ke0, int ve0,
                                              uint8_t *k_dst, uint8_t *v_dst, int8_t *exps, uint32_t *s_max, const Load &load)
{
    uint4 k[NC], v[NC];
    uint32_t bad = 0, km = 0, vm = 0;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = i * threads + t;
        const int row = c / CPR;
        k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (on && row < n_rows) load(row, c % CPR, k[i], v[i]);
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const uint32_t ka = bf16x8_absmax(k[i]), va = bf16x8_absmax(v[i]);
        // a row is CPR lanes of one warp
        const uint32_t any = __ballot_sync(0xffffffffu, ka >= 0x7f80u || va >= 0x7f80u);
        if ((any >> (lane / CPR * CPR)) & ((1u << CPR) - 1)) {
            bad |= 1u << i;
        } else {
            km = max(km, ka);
            vm = max(vm, va);
        }
    }
    uint32_t m = (km << 16) | vm;
    km = __reduce_max_sync(0xffffffffu, m >> 16);
    vm = __reduce_max_sync(0xffffffffu, m & 0xffffu);
    if (threads > 32) {  // uniform over the block
        const int warp = threadIdx.x >> 5;
        if (lane == 0) s_max[warp] = (km << 16) | vm;
        __syncthreads();
        const int w0 = (threadIdx.x / threads) * (threads >> 5);
        for (int w = w0; w < w0 + (threads >> 5); ++w) {
            km = max(km, s_max[w] >> 16);
            vm = max(vm, s_max[w] & 0xffffu);
        }
    }
    if (!on) return;
    const int ke = q8_exponent(km), ve = q8_exponent(vm);
    const float ks = pow2i(-ke), vs = pow2i(-ve);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = i * threads + t;
        if (c / CPR >= n_rows) continue;
        uint2 kc = q8_from_bf16(k[i], ks), vc = q8_from_bf16(v[i], vs);
        if (bad >> i & 1u) {
            kc = make_uint2(kQ8NanWord, kQ8NanWord);
            vc = make_uint2(0u, 0u);
        }
        if (c / CPR >= old || ke != ke0) reinterpret_cast<uint2 *>(k_dst)[c] = kc;
        if (c / CPR >= old || ve != ve0) reinterpret_cast<uint2 *>(v_dst)[c] = vc;
    }
    if (t == 0) *reinterpret_cast<char2 *>(exps) = make_char2(static_cast<char>(ke), static_cast<char>(ve));
}

// The same with K in 32 bits: load(row, col8, float (&k)[8], uint4 &v).
template <int CPR, int NC, typename Load>
__device__ __forceinline__ void q8_write_page_f32(bool on, int t, int threads, int n_rows, int old, int ke0, int ve0,
                                                  uint8_t *k_dst, uint8_t *v_dst, int8_t *exps, uint32_t *s_max, const Load &load)
{
    float k[NC][8];
    uint4 v[NC];
    uint32_t bad = 0, vm = 0;
    float kmax = 0.f;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = i * threads + t;
#pragma unroll
        for (int x = 0; x < 8; ++x) k[i][x] = 0.f;
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (on && c / CPR < n_rows) load(c / CPR, c % CPR, k[i], v[i]);
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        // (as bits: an infinity or NaN is 0x7f800000 or more)
        uint32_t ka = 0;
#pragma unroll
        for (int x = 0; x < 8; ++x) ka = max(ka, __float_as_uint(k[i][x]) & 0x7fffffffu);
        const uint32_t va = bf16x8_absmax(v[i]);
        const uint32_t any = __ballot_sync(0xffffffffu, ka >= 0x7f800000u || va >= 0x7f80u);
        if ((any >> (lane / CPR * CPR)) & ((1u << CPR) - 1)) {
            bad |= 1u << i;
        } else {
            kmax = fmaxf(kmax, __uint_as_float(ka));
            vm = max(vm, va);
        }
    }
    // An exponent is monotone in the magnitude: the page's is the largest of the threads' (biased, a byte each).
    const uint32_t ke_t = static_cast<uint32_t>(q8_exponent_f32(kmax) + 127), ve_t = static_cast<uint32_t>(q8_exponent(vm) + 127);
    uint32_t km = __reduce_max_sync(0xffffffffu, ke_t);
    vm = __reduce_max_sync(0xffffffffu, ve_t);
    if (threads > 32) {  // uniform over the block
        const int warp = threadIdx.x >> 5;
        __syncthreads();
        if (lane == 0) s_max[warp] = (km << 16) | vm;
        __syncthreads();
        const int w0 = (threadIdx.x / threads) * (threads >> 5);
        for (int w = w0; w < w0 + (threads >> 5); ++w) {
            km = max(km, s_max[w] >> 16);
            vm = max(vm, s_max[w] & 0xffffu);
        }
    }
    if (!on) return;
    const int ke = static_cast<int>(km) - 127, ve = static_cast<int>(vm) - 127;
    const float ks = pow2i(-ke), vs = pow2i(-ve);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = i * threads + t;
        if (c / CPR >= n_rows) continue;
        uint2 kc = q8_from_float(k[i], ks), vc = q8_from_bf16(v[i], vs);
        if (bad >> i & 1u) {
            kc = make_uint2(kQ8NanWord, kQ8NanWord);
            vc = make_uint2(0u, 0u);
        }
        if (c / CPR >= old || ke != ke0) reinterpret_cast<uint2 *>(k_dst)[c] = kc;
        if (c / CPR >= old || ve != ve0) reinterpret_cast<uint2 *>(v_dst)[c] = vc;
    }
    if (t == 0) *reinterpret_cast<char2 *>(exps) = make_char2(static_cast<char>(ke), static_cast<char>(ve));
}

}  // namespace pe
