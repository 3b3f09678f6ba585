// What the attention kernels on e4m3 codes share (pe_q8_attn.cu, pe_q8_rows.cu): chunks of key tiles, and their merge.
#pragma once

#include "q8_mma.cuh"

namespace pe {

namespace {

constexpr int kQ8Keys = 128;  // of a tile

// A chunk: tiles [t0, t1) of an item (sequence si, kv-head, row block).  The item's full chunks have ids first + k
// stride, k < nfull, and its shorter remainder, if any, id rem.
struct Q8Chunk {
    int32_t si, kvh, blk, t0, t1;
};

__device__ __forceinline__ int q8_tiles(const Q8Seq &sq) { return (sq.n_keys + kQ8Keys - 1) / kQ8Keys; }

// a / d with inv = ceil(2^32 / d), for a below 2^26: the product is at most one too high (no call of the compiler's
// division: the kernel's code has to stay in the instruction cache)
__device__ __forceinline__ int div_by(int a, int d, uint32_t inv)
{
    const int q = d == 1 ? a : static_cast<int>(__umulhi(static_cast<uint32_t>(a), inv));
    return q * d > a ? q - 1 : q;
}

// seqs, rem: shared-memory copies; rem[j]: (first id, sequence) of the j-th sequence with remainder chunks
__device__ __forceinline__ Q8Chunk q8_chunk(const Q8AttnParams &p, const Q8Seq *seqs, const int2 *rem, int c)
{
    Q8Chunk ci;
    int lo = 0;
    if (c < p.full_chunks) {
        int hi = p.n_seqs;
        while (hi - lo > 1) {  // the last sequence whose first full chunk is at most c
            const int mid = (lo + hi) >> 1;
            if (seqs[mid].full0 <= c) lo = mid; else hi = mid;
        }
        const Q8Seq &sq = seqs[lo];
        const int off = c - sq.full0, u = div_by(off, sq.n_blocks, sq.blocks_inv);
        ci.si = lo;
        ci.blk = off - u * sq.n_blocks;
        ci.kvh = div_by(u, sq.n_full, sq.full_inv);
        ci.t0 = (u - ci.kvh * sq.n_full) * sq.ct;
        ci.t1 = ci.t0 + sq.ct;
    } else {
        int hi = p.n_rem;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (rem[mid].x <= c) lo = mid; else hi = mid;
        }
        ci.si = rem[lo].y;
        const Q8Seq &sq = seqs[ci.si];
        const int off = c - rem[lo].x;
        ci.kvh = div_by(off, sq.n_blocks, sq.blocks_inv);
        ci.blk = off - ci.kvh * sq.n_blocks;
        ci.t0 = sq.n_full * sq.ct;
        ci.t1 = q8_tiles(sq);
    }
    return ci;
}

// Merge of the items held in several chunks: M = max_k m_k, O = sum_k 2^(m_k - M) O_k / sum_k 2^(m_k - M) l_k, in
// the item's chunk order.  A block per item and row; its groups of HD / 4 threads take every kGroups-th chunk, eight of
// them a round trip to L2.  Items of many chunks take the form with 512 threads: 94 chunks (8 rows on 120k keys) in one
// round trip, not three.  ROWS, for blocks of many rows held in few chunks: a group has a row to itself, and a block
// several (8 sequences of 4000 keys, 64 rows, with the attention: 39.2 -> 33.1 us; of 32k, 128 rows: 221 -> 217; but one
// of 32k, 19 chunks, 36.8 -> 39.1).
template <int HD, int RB, int THREADS, bool ROWS>
__global__ void __launch_bounds__(THREADS) attn_q8_combine_kernel(const __grid_constant__ Q8AttnParams p)
{
    constexpr int kLanes = HD / 4;
    constexpr int kGroups = THREADS / kLanes;
    constexpr int kOB = 8;
    __shared__ float4 s_acc[kGroups][kLanes];
    __shared__ float s_m[kGroups], s_l[kGroups];
    const int item = static_cast<int>(blockIdx.x), r0 = static_cast<int>(blockIdx.y) * (ROWS ? kGroups : 1);
    int lo = 0, hi = p.n_seqs;
    while (hi - lo > 1) {  // the last sequence whose first item is at most this one
        const int mid = (lo + hi) >> 1;
        if (p.seqs[mid].item0 <= item) lo = mid; else hi = mid;
    }
    const Q8Seq &sq = p.seqs[lo];
    const int blk = (item - sq.item0) % sq.n_blocks, kvh = (item - sq.item0) / sq.n_blocks;
    const int nfull = sq.n_full, cpi = nfull + (sq.rem0 >= 0 ? 1 : 0);
    const int first = sq.full0 + kvh * nfull * sq.n_blocks + blk;
    const int rem = sq.rem0 + kvh * sq.n_blocks + blk;
    const int grp = static_cast<int>(threadIdx.x) / kLanes;
    const int r = ROWS ? r0 + grp : r0, row = blk * RB + r;
    const int t = static_cast<int>(threadIdx.x) % kLanes;
    const float *pm = p.part + static_cast<int64_t>(p.total_chunks) * RB * HD;
    const float *pl = pm + static_cast<int64_t>(p.total_chunks) * RB;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    if (cpi <= 1 || row >= sq.n_q * p.group) return;
    float mx = -INFINITY, den = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kStep = ROWS ? 1 : kGroups;  // from one of the group's chunks to the next
    for (int k0 = ROWS ? 0 : grp; k0 < cpi; k0 += kStep * kOB) {
        float mv[kOB], lv[kOB];
        float4 ov[kOB];
#pragma unroll
        for (int u = 0; u < kOB; ++u) {
            const int k = k0 + u * kStep;
            const bool in = k < cpi;
            const int64_t c = k < nfull ? first + static_cast<int64_t>(k) * sq.n_blocks : (in ? rem : (nfull ? first : rem));
            mv[u] = in ? __ldcg(pm + c * RB + r) : -INFINITY;
            lv[u] = in ? __ldcg(pl + c * RB + r) : 0.f;
            ov[u] = in && p.out ? __ldcg(reinterpret_cast<const float4 *>(p.part + (c * RB + r) * HD) + t)
                                : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float bmx = mx;
#pragma unroll
        for (int u = 0; u < kOB; ++u) bmx = fmaxf(bmx, mv[u]);
        if (bmx == -INFINITY) {  // no visible key so far, or NaN keys only
#pragma unroll
            for (int u = 0; u < kOB; ++u) den += lv[u];
            continue;
        }
        const float f = mx == -INFINITY ? 0.f : ex2(mx - bmx);
        den *= f;
        acc.x *= f;
        acc.y *= f;
        acc.z *= f;
        acc.w *= f;
        mx = bmx;
#pragma unroll
        for (int u = 0; u < kOB; ++u) {
            if (mv[u] == -INFINITY && lv[u] == 0.f) continue;  // O_k and l_k hold nothing
            const float w = ex2(mv[u] - bmx);
            den += w * lv[u];
            acc.x += w * ov[u].x;
            acc.y += w * ov[u].y;
            acc.z += w * ov[u].z;
            acc.w += w * ov[u].w;
        }
    }
    float M = mx, l = den;
    float4 o = acc;
    if constexpr (!ROWS) {
        s_acc[grp][t] = acc;
        if (t == 0) {
            s_m[grp] = mx;
            s_l[grp] = den;
        }
        __syncthreads();
        if (grp != 0) return;
#pragma unroll
        for (int q = 0; q < kGroups; ++q) M = fmaxf(M, s_m[q]);
        o = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
    }
#pragma unroll
    for (int q = 0; q < (ROWS ? 0 : kGroups); ++q) {
        if (s_m[q] == -INFINITY) {
            l += s_l[q];  // 0 or NaN
            continue;
        }
        const float w = ex2(s_m[q] - M);
        const float4 x = s_acc[q][t];
        l += w * s_l[q];
        o.x += w * x.x;
        o.y += w * x.y;
        o.z += w * x.z;
        o.w += w * x.w;
    }
    const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : NAN);
    const int64_t at = static_cast<int64_t>(sq.q_row0 + row / p.group) * p.hq + kvh * p.group + row % p.group;
    if (p.out) reinterpret_cast<uint2 *>(p.out + at * HD)[t] = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (p.lse && t == 0) p.lse[at] = M + __log2f(l);
}

template <int HD, int RB>
cudaError_t launch_q8_merge(const Q8AttnParams &p, cudaStream_t st)
{
    const bool many = p.max_chunks > 8 * 128 / (HD / 4);
    constexpr int kRows = 128 / (HD / 4);
    const bool rows = RB >= 32 && (p.max_chunks <= 8 || p.total_items * RB >= 2048);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.total_items), rows ? RB / kRows : RB);
    cfg.blockDim = dim3(many && !rows ? 512 : 128);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if constexpr (RB >= 32)
        if (rows) return cudaLaunchKernelEx(&cfg, attn_q8_combine_kernel<HD, RB, 128, true>, p);
    return cudaLaunchKernelEx(&cfg, many ? attn_q8_combine_kernel<HD, RB, 512, false> : attn_q8_combine_kernel<HD, RB, 128, false>, p);
}

}  // namespace

}  // namespace pe
