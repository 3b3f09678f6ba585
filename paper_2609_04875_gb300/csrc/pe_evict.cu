// Eviction from a cache by accumulated attention weight: select the positions
// a sequence keeps, copy their K and V into fresh pages (8-bit pages quantised
// again from their values), then replace the page table and compact the weights.
//
// Select: of T positions the first `sinks` and the last `recent` stay, and of
// the others the `want` with the largest weight, ties to the lowest index, NaN
// below every number.  Weights are mapped to unsigned keys in the same order;
// a radix select (11, 11 and 10 bits) finds the key of the last one kept and how
// many of its equals are kept; then every warp takes a stretch of positions,
// counts what it keeps, and writes it behind the warps before it.
//
// One block a sequence, the keys in shared memory where they fit: a pass over
// 32k keys is then 32 reads a thread.  With 8-bit digits (of which the first, sign
// and exponent, has few values: atomics on the same bins), every pass over global
// memory and a scan by 1024 positions at a time, 8 sequences of 20k to 33k took
// 103 us.
#include <algorithm>
#include <cstddef>
#include <cstring>

#include "pe_internal.h"
#include "ptx.cuh"
#include "q8.cuh"

namespace pe {

namespace {

constexpr int kSelThreads = 1024, kSelWarps = kSelThreads / 32;
constexpr int kSelBins = 2048;
constexpr int kSelSmemKeys = 48 * 1024;   // keys held in shared memory (192 KB)

__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0u;                         // NaN: evicted first
    const uint32_t b = __float_as_uint(w + 0.f);   // -0 and 0 are equal
    return b >> 31 ? ~b : b | 0x80000000u;         // -inf is 0x007fffff
}

template <typename Params>
__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const __grid_constant__ Params p, int smem_keys)
{
    extern __shared__ uint32_t s_keys[];           // [smem_keys]: the candidates' keys, when they fit
    __shared__ int s_hist[kSelBins];
    __shared__ int s_gt[kSelWarps], s_tie[kSelWarps];
    __shared__ int s_bin, s_left;
    ptx::griddep_wait();  // launched with programmatic serialization
    ptx::griddep_launch_dependents();
    const EvictSeg &sg = p.segs[blockIdx.x];
    const float *w = p.weights + static_cast<int64_t>(sg.row) * p.weights_stride;
    int32_t *kept = p.kept + static_cast<int64_t>(sg.row) * p.kept_stride;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (p.done && threadIdx.x == 0) p.done[sg.row] = EvictDone{sg.seq, sg.len, sg.keep, 0};
    for (int j = sg.keep + static_cast<int>(threadIdx.x); j < p.kept_cols; j += kSelThreads) kept[j] = -1;
    if (sg.keep >= sg.len) {
        for (int j = threadIdx.x; j < sg.len; j += kSelThreads) kept[j] = j;
        return;
    }
    const int lo = sg.sinks, n = sg.len - sg.recent - lo;  // the candidates: positions lo + [0, n)
    const int want = sg.keep - sg.sinks - sg.recent;
    const bool held = n <= smem_keys;
    auto key_at = [&](int j) -> uint32_t { return held ? s_keys[j] : weight_key(w[lo + j]); };
    if (held)
        for (int j = threadIdx.x; j < n; j += kSelThreads) s_keys[j] = weight_key(w[lo + j]);
    // key: the candidates' want-th largest key; left: how many equal to it are kept
    uint32_t key = 0xffffffffu;
    int left = 0;
    if (want > 0) {
        key = 0;
        left = want;
        uint32_t done = 0;  // mask of the digits found
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            const uint32_t digit = pass == 2 ? 1023u : 2047u;
            for (int b = threadIdx.x; b < kSelBins; b += kSelThreads) s_hist[b] = 0;
            __syncthreads();
            for (int j = threadIdx.x; j < n; j += kSelThreads) {
                const uint32_t k = key_at(j);
                if ((k & done) == key) atomicAdd(&s_hist[k >> shift & digit], 1);
            }
            __syncthreads();
            // the bin, from the top, that holds the left-th: warp w counts the w-th 64 bins from the top, then the warp
            // that holds it looks among its own, two a lane
            const int top = kSelBins - 1 - warp * 64 - lane * 2;
            const int a = s_hist[top], b = s_hist[top - 1];
            int before = a + b;  // inclusive prefix over the warp
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, before, off);
                if (lane >= off) before += o;
            }
            if (lane == 31) s_gt[warp] = before;
            __syncthreads();
            for (int x = 0; x < warp; ++x) before += s_gt[x];
            before -= a + b;
            if (before < left && left <= before + a + b) {
                const bool second = before + a < left;
                s_bin = second ? top - 1 : top;
                s_left = left - before - (second ? a : 0);
            }
            __syncthreads();
            key |= static_cast<uint32_t>(s_bin) << shift;
            left = s_left;
            done |= digit << shift;
        }
    } else {
        __syncthreads();
    }
    // warp `warp` takes candidates [j0, j1): how many are above the key, and equal to it
    const int per = ((n + kSelWarps - 1) / kSelWarps + 31) & ~31;
    const int j0 = min(n, warp * per), j1 = min(n, j0 + per);
    int gt = 0, tie = 0;
    for (int j = j0 + lane; j < j1; j += 32) {
        const uint32_t k = key_at(j);
        gt += k > key;
        tie += k == key;
    }
    gt = __reduce_add_sync(0xffffffffu, gt);
    tie = __reduce_add_sync(0xffffffffu, tie);
    if (lane == 0) {
        s_gt[warp] = gt;
        s_tie[warp] = tie;
    }
    __syncthreads();
    int at = lo, ties = 0;  // kept before this warp's stretch (the sinks first), and equal ones
    for (int x = 0; x < warp; ++x) {
        at += s_gt[x] + min(s_tie[x], max(0, left - ties));
        ties += s_tie[x];
    }
    for (int b = j0; b < j1; b += 32) {
        const int j = b + lane;
        const uint32_t k = j < j1 ? key_at(j) : 0u;
        const bool is_tie = j < j1 && want > 0 && k == key;
        const uint32_t before = (1u << lane) - 1, t = __ballot_sync(0xffffffffu, is_tie);
        const bool take = j < j1 && want > 0 && (k > key || (is_tie && ties + __popc(t & before) < left));
        const uint32_t m = __ballot_sync(0xffffffffu, take);
        if (take) kept[at + __popc(m & before)] = lo + j;
        at += __popc(m);
        ties += __popc(t);
    }
    for (int j = threadIdx.x; j < lo; j += kSelThreads) kept[j] = j;
    for (int j = threadIdx.x; j < sg.recent; j += kSelThreads) kept[sg.keep - sg.recent + j] = sg.len - sg.recent + j;
}

// One unit is a new page of one kv-head and layer: row r of it is the position kept[page * ps + r], read through
// the table that still holds the old pages.  Thread t of the unit's `threads` holds chunks c = i * threads + t of 16
// bytes, 16 or 8 values.
//
// 8 bits: codes stay codes.  The page's largest magnitude is the largest of its rows' largest codes, each with its old
// page's scale; a row whose scale stays moves as it is, another's codes are scaled by the difference.  (Through
// bf16 values in registers, eight codes a load, 8 sequences x 8 layers down to 4k tokens took 545 us; with divisions and
// rows in 64 bits, 94 registers a thread, 272.)  Bound by the rows' scattered reads, 128 bytes each at d = 128, at the end
// of a chain of three loads: 214 us, 5.0 TB/s of reads and writes.
template <typename Params, bool Q8, int CPR, int NC>
__global__ void __launch_bounds__(kQ8Block) evict_copy_kernel(const __grid_constant__ Params p, int threads)
{
    __shared__ uint2 s_max[kQ8Block / 32];
    ptx::griddep_wait();  // launched with programmatic serialization
    ptx::griddep_launch_dependents();
    const int log_threads = 31 - __clz(threads);
    const uint32_t unit = (blockIdx.x << (kLogQ8Block - log_threads)) + (threadIdx.x >> log_threads);  // (below 2^31: the pools' pages)
    const bool on = unit < static_cast<uint32_t>(p.L * p.n_new * p.hkv);
    const uint32_t u = on ? unit : 0, page = u / p.hkv;
    const int h = static_cast<int>(u - page * p.hkv);
    const int pg = static_cast<int>(page % p.n_new);
    const int l = static_cast<int>(page / p.n_new);
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {  // last segment with new0 <= pg
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].new0 <= pg) lo = mid; else hi = mid - 1;
    }
    const EvictSeg &sg = p.segs[lo];
    const int lp = sg.first_lp + (pg - sg.new0), lps = p.log_ps, t = threadIdx.x % threads;
    const int32_t *kept = p.kept + static_cast<int64_t>(sg.row) * p.kept_stride + (lp << lps);
    const int32_t *table = p.page_table + sg.table_row;
    const int rows = on ? min(p.ps, sg.keep - (lp << lps)) : 0;
    const int head = (l * p.num_pages + p.new_pages[pg]) * p.hkv + h;
    const uint4 *kp = static_cast<const uint4 *>(p.k_pool), *vp = static_cast<const uint4 *>(p.v_pool);
    int from[NC];  // the source row, of all layers' rows (a cache's rows are below 2^31)
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int row = (i * threads + t) / CPR;
        from[i] = -1;
        if (row < rows) {
            const int pos = kept[row];
            from[i] = (((l * p.num_pages + table[pos >> lps]) * p.hkv + h) << lps) + (pos & (p.ps - 1));
        }
    }
    uint4 k[NC], v[NC];
    int ke[NC], ve[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
        ke[i] = ve[i] = -126;
        if (from[i] < 0) continue;
        const int64_t c = static_cast<int64_t>(from[i]) * CPR + (i * threads + t) % CPR;
        k[i] = kp[c];
        v[i] = vp[c];
        if constexpr (Q8) {
            const char2 e = reinterpret_cast<const char2 *>(p.exps)[from[i] >> lps];
            ke[i] = static_cast<int8_t>(e.x);
            ve[i] = static_cast<int8_t>(e.y);
        }
    }
    if constexpr (Q8) {
        // the largest magnitudes as float bits; a row held as NaN (its K codes) counts for nothing and stays
        uint32_t km = 0, vm = 0;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            if (k[i].x == kQ8NanWord) continue;
            km = max(km, __float_as_uint(e4m3x2_to_float2(codes_absmax(k[i])).x * pow2i(ke[i])));
            vm = max(vm, __float_as_uint(e4m3x2_to_float2(codes_absmax(v[i])).x * pow2i(ve[i])));
        }
        km = __reduce_max_sync(0xffffffffu, km);
        vm = __reduce_max_sync(0xffffffffu, vm);
        if (threads > 32) {  // uniform over the block
            if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = make_uint2(km, vm);
            __syncthreads();
            const int w0 = (threadIdx.x / threads) * (threads >> 5);
            for (int w = w0; w < w0 + (threads >> 5); ++w) {
                km = max(km, s_max[w].x);
                vm = max(vm, s_max[w].y);
            }
        }
        const int kn = q8_exponent(km >> 16), vn = q8_exponent(vm >> 16);  // (four significant bits: exact in bf16)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            if (from[i] < 0) continue;
            if (ke[i] != kn && k[i].x != kQ8NanWord) k[i] = rescale_codes(k[i], ke[i] - kn);
            if (ve[i] != vn) v[i] = rescale_codes(v[i], ve[i] - vn);
        }
        if (on && t == 0) reinterpret_cast<char2 *>(p.exps)[head] = make_char2(static_cast<char>(kn), static_cast<char>(vn));
    }
    const int64_t to = (static_cast<int64_t>(head) << lps) * CPR;
    uint4 *kd = static_cast<uint4 *>(p.k_pool) + to, *vd = static_cast<uint4 *>(p.v_pool) + to;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if (from[i] < 0) continue;
        kd[i * threads + t] = k[i];
        vd[i * threads + t] = v[i];
    }
}

// The table entries of a group of new pages, where there are several (their copies read the table, so they wait).
__global__ void __launch_bounds__(256) evict_table_kernel(const __grid_constant__ EvictParams p)
{
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const EvictSeg &sg = p.segs[blockIdx.x];
    for (int i = threadIdx.x; i < sg.n_new; i += 256) p.page_table[sg.table_row + sg.first_lp + i] = p.new_pages[sg.new0 + i];
}

// A sequence's weights, the end of its table row and its length, last of all.  kept[j] >= j, so taken some positions at
// a time in ascending order the weights move down in place.  (One block; all of its threads.)
__device__ __forceinline__ void finish_sequence(float *w, const int32_t *kept, int32_t *table, int64_t *len_out, int len, int keep, int ps,
                                                int log_ps)
{
    constexpr int kAt = 4;  // positions of a thread in flight
    for (int j0 = 0; j0 < keep; j0 += kAt * kSelThreads) {
        float x[kAt];
#pragma unroll
        for (int u = 0; u < kAt; ++u) {
            const int j = j0 + u * kSelThreads + static_cast<int>(threadIdx.x);
            x[u] = j < keep ? w[kept[j]] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kAt; ++u) {
            const int j = j0 + u * kSelThreads + static_cast<int>(threadIdx.x);
            if (j < keep) w[j] = x[u];
        }
    }
    __syncthreads();
    for (int j = keep + static_cast<int>(threadIdx.x); j < len; j += kSelThreads) w[j] = 0.f;
    const int now = (keep + ps - 1) >> log_ps, before = (len + ps - 1) >> log_ps;
    for (int e = now + static_cast<int>(threadIdx.x); e < before; e += kSelThreads) table[e] = -1;
    if (threadIdx.x == 0) *len_out = keep;
}

// One block per sequence of the only group, whose new pages it enters.
template <typename Params>
__global__ void __launch_bounds__(kSelThreads) evict_finish_kernel(const __grid_constant__ Params p)
{
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const EvictSeg &sg = p.segs[blockIdx.x];
    if (sg.keep >= sg.len) return;
    for (int i = threadIdx.x; i < sg.n_new; i += kSelThreads) p.page_table[sg.table_row + sg.first_lp + i] = p.new_pages[sg.new0 + i];
    finish_sequence(p.weights + static_cast<int64_t>(sg.row) * p.weights_stride, p.kept + static_cast<int64_t>(sg.row) * p.kept_stride,
                    p.page_table + sg.table_row, p.seq_len + sg.seq, sg.len, sg.keep, p.ps, p.log_ps);
}

// One block per sequence of the call, from the records that the selections left: a single launch, however many groups
// there were, so that no sequence's weights move unless all do.
__global__ void __launch_bounds__(kSelThreads) evict_finish_all_kernel(const __grid_constant__ EvictFinishParams p)
{
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int row = static_cast<int>(blockIdx.x);
    const EvictDone s = p.done[row];
    if (s.keep >= s.len) return;
    finish_sequence(p.weights + static_cast<int64_t>(row) * p.weights_stride, p.kept + static_cast<int64_t>(row) * p.kept_stride,
                    p.page_table + static_cast<int64_t>(s.seq) * p.max_pages, p.seq_len + s.seq, s.len, s.keep, p.ps, p.log_ps);
}

cudaLaunchConfig_t serial_config(unsigned blocks, unsigned threads, size_t smem, cudaStream_t st, cudaLaunchAttribute *attr)
{
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

// A launch's parameter block is copied by the host, by CUDA and by the GPU's front end (append_kv_kernel): few sequences
// and pages take the small one.
using Small = EvictParamsT<16, 128>;
bool fits_small(const EvictParams &p, bool pages) { return p.n <= 16 && (!pages || p.n_new <= 128); }
Small small_of(const EvictParams &p, bool pages)
{
    Small q;
    static_assert(offsetof(Small, segs) == offsetof(EvictParams, segs), "the same header");
    std::memcpy(static_cast<void *>(&q), static_cast<const void *>(&p), offsetof(Small, segs));
    std::copy(p.segs, p.segs + p.n, q.segs);
    if (pages) std::copy(p.new_pages, p.new_pages + p.n_new, q.new_pages);
    return q;
}

template <typename Params>
cudaError_t launch_copy_t(const cudaLaunchConfig_t &cfg, bool q8, int head_dim, int nc, const Params &p, int threads)
{
    if (q8 && head_dim == 128) {
        if (nc == 4) return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, true, 8, 4>, p, threads);
        return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, true, 8, 2>, p, threads);
    }
    if (q8) {
        if (nc == 4) return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, true, 4, 4>, p, threads);
        if (nc == 2) return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, true, 4, 2>, p, threads);
        return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, true, 4, 1>, p, threads);
    }
    if (head_dim == 128) {
        if (nc == 8) return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, false, 16, 8>, p, threads);
        return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, false, 16, 4>, p, threads);
    }
    if (nc == 8) return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, false, 8, 8>, p, threads);
    if (nc == 4) return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, false, 8, 4>, p, threads);
    return cudaLaunchKernelEx(&cfg, evict_copy_kernel<Params, false, 8, 2>, p, threads);
}

template <typename Params>
cudaError_t launch_select_t(const Params &p, int max_len, cudaStream_t st)
{
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = set_dyn_smem_once(evict_select_kernel<Params>, kSelSmemKeys * 4, configured);
    if (e != cudaSuccess) return e;
    const int keys = max_len <= kSelSmemKeys ? max_len : 0;  // (longer candidates are read from global memory)
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(p.n), kSelThreads, static_cast<size_t>(keys) * 4, st, &attr);
    return cudaLaunchKernelEx(&cfg, evict_select_kernel<Params>, p, keys);
}

}  // namespace

cudaError_t launch_evict_select(const EvictParams &p, int max_len, cudaStream_t st)
{
    return fits_small(p, false) ? launch_select_t(small_of(p, false), max_len, st) : launch_select_t(p, max_len, st);
}

cudaError_t launch_evict_copy(bool q8, int head_dim, const EvictParams &p, cudaStream_t st)
{
    // a thread holds at most 4 chunks of 16 bytes of K, and of V (bf16: 8)
    const int chunks = p.ps * head_dim / (q8 ? 16 : 8), threads = std::min(kQ8Block, std::max(32, chunks / 4)), nc = chunks / threads;
    const int64_t blocks = (static_cast<int64_t>(p.L) * p.n_new * p.hkv * threads + kQ8Block - 1) / kQ8Block;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    if (blocks == 0) return cudaSuccess;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(blocks), kQ8Block, 0, st, &attr);
    if (fits_small(p, true)) return launch_copy_t(cfg, q8, head_dim, nc, small_of(p, true), threads);
    return launch_copy_t(cfg, q8, head_dim, nc, p, threads);
}

cudaError_t launch_evict_table(const EvictParams &p, cudaStream_t st)
{
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(p.n), 256, 0, st, &attr);
    return cudaLaunchKernelEx(&cfg, evict_table_kernel, p);
}

cudaError_t launch_evict_finish(const EvictParams &p, cudaStream_t st)
{
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(p.n), kSelThreads, 0, st, &attr);
    if (fits_small(p, true)) return cudaLaunchKernelEx(&cfg, evict_finish_kernel<Small>, small_of(p, true));
    return cudaLaunchKernelEx(&cfg, evict_finish_kernel<EvictParams>, p);
}

cudaError_t launch_evict_finish_all(const EvictFinishParams &p, cudaStream_t st)
{
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(p.n), kSelThreads, 0, st, &attr);
    return cudaLaunchKernelEx(&cfg, evict_finish_all_kernel, p);
}

}  // namespace pe
