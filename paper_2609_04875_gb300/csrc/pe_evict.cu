// Eviction from a cache by accumulated attention weight: select the positions
// a sequence keeps, copy their K and V into fresh pages (8-bit pages quantised
// again from their values), then replace the page table and compact the weights.
//
// Select: of T positions the first `sinks` and the last `recent` stay, and of
// the others the `want` with the largest weight, ties to the lowest index, NaN
// below every number.  Weights are mapped to unsigned keys in the same order;
// a radix select (8 bits a pass) finds the key of the last one kept and how
// many of its equals are kept, then one scan in position order writes the
// kept positions.
#include <algorithm>

#include "pe_internal.h"
#include "ptx.cuh"
#include "q8.cuh"

namespace pe {

namespace {

constexpr int kSelThreads = 1024;

__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0u;                         // NaN: evicted first
    const uint32_t b = __float_as_uint(w + 0.f);   // -0 and 0 are equal
    return b >> 31 ? ~b : b | 0x80000000u;         // -inf is 0x007fffff
}

// exclusive prefix sum of a flag over the block (in thread order); total: the block's sum
__device__ __forceinline__ int block_rank(bool flag, int *s_warp, int &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t b = __ballot_sync(0xffffffffu, flag);
    __syncthreads();
    if (lane == 0) s_warp[warp] = __popc(b);
    __syncthreads();
    int before = __popc(b & ((1u << lane) - 1)), all = 0;
    for (int w = 0; w < kSelThreads / 32; ++w) {
        const int n = s_warp[w];
        before += w < warp ? n : 0;
        all += n;
    }
    total = all;
    return before;
}

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const __grid_constant__ EvictParams p)
{
    __shared__ int s_hist[256];
    __shared__ int s_warp[kSelThreads / 32];
    __shared__ uint32_t s_key;
    __shared__ int s_left;
    const EvictSeg &sg = p.segs[blockIdx.x];
    const float *w = p.weights + static_cast<int64_t>(sg.row) * p.weights_stride;
    int32_t *kept = p.kept + static_cast<int64_t>(sg.row) * p.kept_stride;
    for (int j = sg.keep + static_cast<int>(threadIdx.x); j < p.kept_cols; j += kSelThreads) kept[j] = -1;
    if (sg.keep >= sg.len) {
        for (int j = threadIdx.x; j < sg.len; j += kSelThreads) kept[j] = j;
        return;
    }
    const int lo = sg.sinks, hi = sg.len - sg.recent;  // the candidates
    const int want = sg.keep - sg.sinks - sg.recent;
    // key: the candidates' want-th largest key; left: how many equal to it are kept
    uint32_t key = 0xffffffffu;
    int left = 0;
    if (want > 0) {
        key = 0;
        left = want;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) s_hist[threadIdx.x] = 0;
            __syncthreads();
            const uint32_t done = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int j = lo + static_cast<int>(threadIdx.x); j < hi; j += kSelThreads) {
                const uint32_t k = weight_key(w[j]);
                if ((k & done) == key) atomicAdd(&s_hist[k >> shift & 255u], 1);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int b = 255;
                while (b > 0 && s_hist[b] < left) left -= s_hist[b--];
                s_key = key | static_cast<uint32_t>(b) << shift;
                s_left = left;
            }
            __syncthreads();
            key = s_key;
            left = s_left;
        }
    }
    int n = 0, ties = 0;  // kept and equal ones met so far
    for (int j0 = 0; j0 < sg.len; j0 += kSelThreads) {
        const int j = j0 + static_cast<int>(threadIdx.x);
        const bool mid = j >= lo && j < hi;
        const uint32_t k = mid && want > 0 ? weight_key(w[j]) : 0u;
        const bool tie = mid && want > 0 && k == key;
        int all = 0;
        const int tie_rank = ties + block_rank(tie, s_warp, all);
        ties += all;
        const bool take = j < sg.len && (!mid || (want > 0 && (k > key || (tie && tie_rank < left))));
        const int at = n + block_rank(take, s_warp, all);
        if (take) kept[at] = j;
        n += all;
    }
}

// One unit is a new page of one kv-head and layer: row r of it is the position kept[page * ps + r], read through
// the table that still holds the old pages.
template <bool Q8, int CPR, int NC>
__global__ void __launch_bounds__(kQ8Block) evict_copy_kernel(const __grid_constant__ EvictParams p, int threads)
{
    __shared__ uint32_t s_max[kQ8Block / 32];
    constexpr int HD = CPR * 8;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kQ8Block / threads) + threadIdx.x / threads;
    const bool on = unit < static_cast<int64_t>(p.L) * p.n_new * p.hkv;
    const int64_t u = on ? unit : 0;
    const int h = static_cast<int>(u % p.hkv);
    const int pg = static_cast<int>(u / p.hkv % p.n_new);
    const int64_t l = u / p.hkv / p.n_new;
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {  // last segment with new0 <= pg
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].new0 <= pg) lo = mid; else hi = mid - 1;
    }
    const EvictSeg &sg = p.segs[lo];
    const int lp = sg.first_lp + (pg - sg.new0);
    const int32_t *kept = p.kept + static_cast<int64_t>(sg.row) * p.kept_stride + lp * p.ps;
    const int32_t *table = p.page_table + sg.table_row;
    const int rows = min(p.ps, sg.keep - lp * p.ps);
    const int64_t head = (l * p.num_pages + p.new_pages[pg]) * p.hkv + h;
    constexpr int kBytes = Q8 ? HD : 2 * HD;  // of a row
    uint8_t *kd = static_cast<uint8_t *>(p.k_pool) + head * p.ps * kBytes;
    uint8_t *vd = static_cast<uint8_t *>(p.v_pool) + head * p.ps * kBytes;
    auto load = [&](int row, int col8, uint4 &k, uint4 &v) {
        const int pos = kept[row];
        const int64_t from = (l * p.num_pages + table[pos / p.ps]) * p.hkv + h;
        const int64_t at = (from * p.ps + pos % p.ps) * CPR + col8;
        if constexpr (Q8) {
            k = q8_to_bf16(static_cast<const uint2 *>(p.k_pool)[at], pow2i(p.exps[2 * from]));
            v = q8_to_bf16(static_cast<const uint2 *>(p.v_pool)[at], pow2i(p.exps[2 * from + 1]));
        } else {
            k = static_cast<const uint4 *>(p.k_pool)[at];
            v = static_cast<const uint4 *>(p.v_pool)[at];
        }
    };
    if constexpr (Q8) {
        q8_write_page<CPR, NC>(on, threadIdx.x % threads, threads, rows, kd, vd, p.exps + 2 * head, s_max, load);
    } else {
        if (!on) return;
        for (int c = threadIdx.x % threads; c < rows * CPR; c += threads) {
            uint4 k, v;
            load(c / CPR, c % CPR, k, v);
            reinterpret_cast<uint4 *>(kd)[c] = k;
            reinterpret_cast<uint4 *>(vd)[c] = v;
        }
    }
}

// The table entries of this launch's new pages.
__global__ void __launch_bounds__(256) evict_table_kernel(const __grid_constant__ EvictParams p)
{
    for (int s = 0; s < p.n; ++s) {
        const EvictSeg &sg = p.segs[s];
        for (int i = threadIdx.x; i < sg.n_new; i += 256)
            p.page_table[sg.table_row + sg.first_lp + i] = p.new_pages[sg.new0 + i];
    }
}

// One block per sequence, last of all: the table past the kept pages, the length, and the weights: kept[j] >= j, so
// taken a block's width at a time in ascending order they move down in place.
__global__ void __launch_bounds__(kSelThreads) evict_finish_kernel(const __grid_constant__ EvictParams p)
{
    const EvictSeg &sg = p.segs[blockIdx.x];
    if (sg.keep >= sg.len) return;
    float *w = p.weights + static_cast<int64_t>(sg.row) * p.weights_stride;
    const int32_t *kept = p.kept + static_cast<int64_t>(sg.row) * p.kept_stride;
    for (int j0 = 0; j0 < sg.keep; j0 += kSelThreads) {
        const int j = j0 + static_cast<int>(threadIdx.x);
        const float x = j < sg.keep ? w[kept[j]] : 0.f;
        __syncthreads();
        if (j < sg.keep) w[j] = x;
    }
    __syncthreads();
    for (int j = sg.keep + static_cast<int>(threadIdx.x); j < sg.len; j += kSelThreads) w[j] = 0.f;
    const int now = (sg.keep + p.ps - 1) / p.ps;
    for (int e = now + static_cast<int>(threadIdx.x); e < sg.old_n; e += kSelThreads) p.page_table[sg.table_row + e] = -1;
    if (threadIdx.x == 0) p.seq_len[sg.seq] = sg.keep;
}

}  // namespace

cudaError_t launch_evict_select(const EvictParams &p, cudaStream_t st)
{
    evict_select_kernel<<<p.n, kSelThreads, 0, st>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_evict_copy(bool q8, int head_dim, const EvictParams &p, cudaStream_t st)
{
    const int elems = p.ps * head_dim, threads = q8_unit_threads(elems), nc = q8_unit_chunks(elems);
    const int64_t blocks = (static_cast<int64_t>(p.L) * p.n_new * p.hkv * threads + kQ8Block - 1) / kQ8Block;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    const unsigned n = static_cast<unsigned>(blocks);
    if (n > 0) {
        if (!q8) {
            if (head_dim == 128) evict_copy_kernel<false, 16, 1><<<n, kQ8Block, 0, st>>>(p, threads);
            else evict_copy_kernel<false, 8, 1><<<n, kQ8Block, 0, st>>>(p, threads);
        } else if (head_dim == 128) {
            if (nc == 8) evict_copy_kernel<true, 16, 8><<<n, kQ8Block, 0, st>>>(p, threads);
            else evict_copy_kernel<true, 16, 4><<<n, kQ8Block, 0, st>>>(p, threads);
        } else {
            if (nc == 8) evict_copy_kernel<true, 8, 8><<<n, kQ8Block, 0, st>>>(p, threads);
            else if (nc == 4) evict_copy_kernel<true, 8, 4><<<n, kQ8Block, 0, st>>>(p, threads);
            else evict_copy_kernel<true, 8, 2><<<n, kQ8Block, 0, st>>>(p, threads);
        }
    }
    return cudaGetLastError();
}

cudaError_t launch_evict_table(const EvictParams &p, cudaStream_t st)
{
    evict_table_kernel<<<1, 256, 0, st>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_evict_finish(const EvictParams &p, cudaStream_t st)
{
    evict_finish_kernel<<<p.n, kSelThreads, 0, st>>>(p);
    return cudaGetLastError();
}

}  // namespace pe
