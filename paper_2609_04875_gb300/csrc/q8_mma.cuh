// What the tcgen05 kernels on e4m3 codes share (pe_q8_attn.cu, pe_weights.cu).
#pragma once

#include "dev_common.cuh"
#include "q8.cuh"

namespace pe {

// kind::f8f6f4: e4m3 A and B (format 0), fp32 D; the fields are those of kind::f16
__host__ __device__ constexpr uint32_t idesc_e4m3_f32(int M, int N, bool mn_major)
{
    return (1u << 4) | ((mn_major ? 3u : 0u) << 15) | (static_cast<uint32_t>(N >> 3) << 17) |
           (static_cast<uint32_t>(M >> 4) << 24);
}

// wait_bar_warp (dev_common.cuh) that looks at the clock and the abort flag once in kQ8Spins tries (reading the clock
// takes longer than a try), out of line but for its first try: the kernel's code has to stay in the instruction cache.
constexpr uint32_t kQ8Spins = 64;
static __device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int *abort, int32_t *status)
{
    bool ok = false;
    uint64_t t0 = 0;
    for (uint32_t n = 1; !ok; ++n) {
        ok = ptx::mbar_try_wait(bar, parity);
        if (ok || (n & (kQ8Spins - 1))) continue;
        if (*abort) break;
        const uint64_t now = ptx::globaltimer();
        if (n == kQ8Spins) t0 = now;
        if (now - t0 > kWaitNs) {
            *abort = 1;
            atomicCAS(status, 0, kStatusWaitTimeout);
            break;
        }
    }
    return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ bool wait_spin(uint32_t bar, uint32_t parity, const WaitCtx &w)
{
    if (__all_sync(0xffffffffu, ptx::mbar_try_wait(bar, parity))) return true;
    return wait_slow(bar, parity, w.abort, w.status);
}

__device__ __forceinline__ void mma_e4m3_warp(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                              uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// smem_desc_sw128, or the same for 64-byte rows (64-byte swizzle) where HD = 64
template <int HD>
__device__ __forceinline__ uint64_t row_desc(uint32_t addr, uint32_t lbo_bytes)
{
    const uint64_t d = ptx::smem_desc_sw128(addr, lbo_bytes, 8 * HD);
    return HD == 128 ? d : (d & ~(7ull << 61)) | (4ull << 61);
}

__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t ra, rb, rd;
    asm("mov.b64 %0, {%1, %2};" : "=l"(ra) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(rb) : "f"(b.x), "f"(b.y));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(rd) : "l"(ra), "l"(rb));
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(rd));
    return d;
}

// byte offset of 16-byte chunk c of row r in a tile of HD-byte rows
template <int HD>
__device__ __forceinline__ int row_chunk(int r, int c)
{
    return HD == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}

// Eight bf16 of q times s in two e4m3 parts, the second of what the first leaves over, times `up`.
__device__ __forceinline__ void q8_split(uint4 v, float s, float up, uint2 &hi, uint2 &low)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t a[4], b[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const float2 f = make_float2(__uint_as_float(w[x] << 16) * s, __uint_as_float(w[x] & 0xffff0000u) * s);
        a[x] = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
        const float2 h = e4m3x2_to_float2(a[x]);
        b[x] = __nv_cvt_float2_to_fp8x2(make_float2((f.x - h.x) * up, (f.y - h.y) * up), __NV_SATFINITE, __NV_E4M3);
    }
    hi = make_uint2(a[0] | a[1] << 16, a[2] | a[3] << 16);
    low = make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
}

}  // namespace pe
