// Device helpers of differential attention's kernels (pe_diff.cu, pe_diff_many.cu).
#pragma once

#include "dev_common.cuh"

namespace pe {

constexpr float kDiffSumLimit = 1.8446744e19f;  // 2^64: larger tile sums move a row's reference (pe_attn.cu)

// A taker's pieces, one after another: every role walks them alike.
template <typename Shape>
struct DiffWalk {
    const DiffParams &p;
    int u, t, u1, t1;  // next piece, end of the stretch
    int taker;
    int si, pair, map, block, t0, n, slot;
    __device__ __forceinline__ DiffWalk(const DiffParams &p_, int cta) : p(p_), taker(cta), map(0)
    {
        u = p.start[cta].u;
        t = p.start[cta].t;
        u1 = p.start[cta + 1].u;
        t1 = p.start[cta + 1].t;
    }
    // The next piece with tiles [t0, t0 + n), or false.
    __device__ __forceinline__ bool next()
    {
        while (u < u1 || (u == u1 && t < t1)) {
            int lo = 0, hi = p.n_seqs - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (p.seqs[mid].unit0 <= u) lo = mid; else hi = mid - 1;
            }
            si = lo;
            const int local = u - p.seqs[si].unit0;
            block = local % p.seqs[si].n_blocks;
            pair = local / p.seqs[si].n_blocks;
            if (Shape::kMaps == 2) {
                map = pair & 1;
                pair >>= 1;
            }
            slot = u + taker;
            t0 = t;
            n = (u == u1 ? t1 : diff_tiles<Shape>(p.seqs[si], p.group, block)) - t;
            ++u;
            t = 0;
            if (n > 0) return true;
        }
        return false;
    }
};

// ---------------------------------------------------------------- merge
// The taker whose stretch holds the unit's first tile: the last one that begins at or before it.
__device__ __forceinline__ int diff_first_taker(const DiffParams &p, int u)
{
    int lo = 0, hi = p.n_takers - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.start[mid].u < u || (p.start[mid].u == u && p.start[mid].t == 0)) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ bool diff_takes_nothing(const DiffParams &p, int c)
{
    return p.start[c].u == p.start[c + 1].u && p.start[c].t == p.start[c + 1].t;
}

// A partial row's columns 4 lane .. + 3 of every 128.
template <int HD>
__device__ __forceinline__ void diff_load(const float *row, int lane, float4 (&y)[2 * HD / 128])
{
#pragma unroll
    for (int v = 0; v < 2 * HD / 128; ++v) y[v] = __ldcg(reinterpret_cast<const float4 *>(row) + v * 32 + lane);
}

// Pieces of one row and map: o = sum 2^(lse - m) O, l = sum 2^(lse - m).
template <int HD>
struct DiffMerge {
    float m = -INFINITY, l = 0.f;
    float4 o[2 * HD / 128];
    __device__ __forceinline__ DiffMerge()
    {
#pragma unroll
        for (int v = 0; v < 2 * HD / 128; ++v) o[v] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ void add(float lse, const float4 (&y)[2 * HD / 128])
    {
        if (lse == -INFINITY) return;  // (no key seen; its row may hold anything)
        const float mn = fmaxf(m, lse);
        const float f = m == -INFINITY ? 0.f : ex2(m - mn), g = ex2(lse - mn);  // (NaN where lse is)
        m = mn;
        l = l * f + g;
#pragma unroll
        for (int v = 0; v < 2 * HD / 128; ++v)
            o[v] = make_float4(o[v].x * f + y[v].x * g, o[v].y * f + y[v].y * g, o[v].z * f + y[v].z * g, o[v].w * f + y[v].w * g);
    }
};

template <int HD>
__device__ __forceinline__ void diff_axpy(float g, const float4 (&z)[2 * HD / 128], bool on, float4 (&y)[2 * HD / 128])
{
    if (!on) return;
#pragma unroll
    for (int v = 0; v < 2 * HD / 128; ++v)
        y[v] = make_float4(y[v].x + g * z[v].x, y[v].y + g * z[v].y, y[v].z + g * z[v].z, y[v].w + g * z[v].w);
}

// The norm over a head's 2d columns, held by a warp, and the output row.
template <int HD>
__device__ __forceinline__ void diff_finish(const DiffParams &p, int64_t out_row, int lane, float4 (&y)[2 * HD / 128])
{
    constexpr int V4 = 2 * HD / 128;
    if (p.gain) {
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < V4; ++v) sum += y[v].x * y[v].x + y[v].y * y[v].y + y[v].z * y[v].z + y[v].w * y[v].w;
#pragma unroll
        for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        const float f = 1.f / sqrtf(sum / (2 * HD) + p.eps);
#pragma unroll
        for (int v = 0; v < V4; ++v) {
            const float *g = p.gain + v * 128 + lane * 4;  // (a vector of any alignment)
            y[v] = make_float4(y[v].x * f * __ldg(g), y[v].y * f * __ldg(g + 1), y[v].z * f * __ldg(g + 2), y[v].w * f * __ldg(g + 3));
        }
    }
    uint2 *dst = reinterpret_cast<uint2 *>(p.out + out_row * 2 * HD);
#pragma unroll
    for (int v = 0; v < V4; ++v) dst[v * 32 + lane] = make_uint2(pack_bf16(y[v].x, y[v].y), pack_bf16(y[v].z, y[v].w));
}

}  // namespace pe
