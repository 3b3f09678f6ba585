// Device helpers of differential attention's kernels (pe_diff.cu, pe_diff_many.cu).
#pragma once

#include "dev_common.cuh"

namespace pe {

constexpr float kDiffSumLimit = 1.8446744e19f;  // 2^64: larger tile sums move a row's reference (pe_attn.cu)

// A pair of weights as two bf16 parts each: their upper ones, and in `lo` what those leave over, so that a weight is off by
// 2^-16 of itself.  One part is not enough here: what the maps share cancels, and the errors of both maps' weights stay while the
// difference shrinks (maps 2 % apart, lambda 0.95: up to 3.6e-2 off in the 2-norm with one part, 1.7e-3 with two, which is the
// output's own rounding).
__device__ __forceinline__ uint32_t two_parts(float2 e, uint32_t &lo)
{
    const uint32_t hi = pack_bf16(e.x, e.y);
    const float2 h = unpack_bf16(hi);
    lo = pack_bf16(e.x - h.x, e.y - h.y);
    return hi;
}

// A taker's pieces, one after another: every role walks them alike.
template <typename Shape>
struct DiffWalk {
    const DiffParams &p;
    int u, t, u1, t1;  // next piece, end of the stretch
    int taker;
    int rank, ranks;   // of the CTAs that share a piece, and their number
    int si, pair, map, block, t0, n, slot;
    __device__ __forceinline__ DiffWalk(const DiffParams &p_, int cta, int rank_ = 0, int ranks_ = 1)
        : p(p_), taker(cta), rank(rank_), ranks(ranks_), map(0)
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
            if (ranks > 1) {
                const int all = n;
                t0 += all * rank / ranks;
                n = all * (rank + 1) / ranks - all * rank / ranks;
            }
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

// And the one that holds its last.
__device__ __forceinline__ int diff_last_taker(const DiffParams &p, int u)
{
    int lo = 0, hi = p.n_takers - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.start[mid].u <= u) lo = mid; else hi = mid - 1;
    }
    return lo;
}

}  // namespace pe
