// The 8-bit cache's writes and reads (formats: q8.cuh): append (quantised page
// by page on the way into the pool), the bf16 copy of one layer that the bf16
// attention kernels read, and the read-back of a range of tokens.  All are
// bound by memory: each reads its input once and writes its output once.
#include <algorithm>
#include <cstddef>
#include <cstring>

#include "pe_internal.h"
#include "ptx.cuh"
#include "q8.cuh"

namespace pe {

namespace {

constexpr int kSmallSegs8 = 16, kSmallPages8 = 128;  // the small parameter block (as in pe_kv.cu)

// One unit is a touched page of one kv-head and layer (kv-heads fastest, so neighbouring units read neighbouring
// rows of K and V).  A partly filled page is quantised again as a whole: its kept rows' values and the new rows.
// p.segs[].cum0 counts pages here, p.seg_tokens the launch's pages.
template <typename Params, int CPR, int NC>
__global__ void __launch_bounds__(kQ8Block) append_q8_kernel(const __grid_constant__ Params p, int threads)
{
    __shared__ uint32_t s_max[kQ8Block / 32];
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();  // launched with programmatic serialization: only the launch overlaps the kernel before
    if (blockIdx.x == 0) {
        for (int s = 0; s < p.n_segs; ++s) {
            const AppendSeg &sg = p.segs[s];
            for (int i = threadIdx.x; i < sg.n_new; i += kQ8Block)
                p.page_table[sg.table_row + sg.first_new_lp + i] = p.new_pages[sg.new0 + i];
            if (threadIdx.x == 0) p.seq_len[sg.seq] = static_cast<int64_t>(sg.len0) + sg.n_tokens;
        }
    }
    constexpr int HD = CPR * 8;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kQ8Block / threads) + threadIdx.x / threads;
    const bool on = unit < static_cast<int64_t>(p.L) * p.seg_tokens * p.hkv;
    const int64_t u = on ? unit : 0;
    const int h = static_cast<int>(u % p.hkv);
    const int64_t r = u / p.hkv;
    const int pg = static_cast<int>(r % p.seg_tokens);
    const int64_t l = r / p.seg_tokens;
    int lo = 0, hi = p.n_segs - 1;
    while (lo < hi) {  // last segment with cum0 <= pg
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].cum0 <= pg) lo = mid; else hi = mid - 1;
    }
    const AppendSeg &sg = p.segs[lo];
    const int lp = sg.len0 / p.ps + (pg - sg.cum0);
    const int page = lp < sg.first_new_lp ? sg.last_page : p.new_pages[sg.new0 + (lp - sg.first_new_lp)];
    const int pos0 = lp * p.ps;
    const int old = max(0, sg.len0 - pos0);                          // rows the page keeps
    const int rows = min(p.ps, sg.len0 + sg.n_tokens - pos0);        // rows it holds afterwards
    const int64_t head = (l * p.num_pages + page) * p.hkv + h;
    uint8_t *kp = reinterpret_cast<uint8_t *>(p.k_pool) + head * p.ps * HD;
    uint8_t *vp = reinterpret_cast<uint8_t *>(p.v_pool) + head * p.ps * HD;
    int8_t *ex = p.exps + head * 2;
    int ke0 = 0, ve0 = 0;
    if (on && old > 0) {
        ke0 = ex[0];
        ve0 = ex[1];
    }
    const float kes = pow2i(ke0), ves = pow2i(ve0);
    const int64_t src0 = ((l * p.n_total + sg.tok0 + (pos0 - sg.len0)) * p.hkv + h) * CPR;  // of the page's row 0
    if (threads <= 32) __syncwarp();
    else __syncthreads();  // the old exponents are read before they are written
    q8_write_page<CPR, NC>(on, threadIdx.x % threads, threads, rows, old, ke0, ve0, kp, vp, ex, s_max,
                           [&](int row, int col8, uint4 &k, uint4 &v) {
                               if (row < old) {
                                   k = q8_to_bf16(*reinterpret_cast<const uint2 *>(kp + row * HD + col8 * 8), kes);
                                   v = q8_to_bf16(*reinterpret_cast<const uint2 *>(vp + row * HD + col8 * 8), ves);
                               } else {
                                   const int64_t s = src0 + static_cast<int64_t>(row) * p.hkv * CPR + col8;
                                   k = __ldcs(p.K + s);
                                   v = __ldcs(p.V + s);
                               }
                           });
}

template <typename Params>
cudaError_t launch_append_t(const cudaLaunchConfig_t &cfg, int head_dim, int nc, const Params &p, int threads)
{
    if (head_dim == 128) {
        if (nc == 8) return cudaLaunchKernelEx(&cfg, append_q8_kernel<Params, 16, 8>, p, threads);
        return cudaLaunchKernelEx(&cfg, append_q8_kernel<Params, 16, 4>, p, threads);
    }
    if (nc == 8) return cudaLaunchKernelEx(&cfg, append_q8_kernel<Params, 8, 8>, p, threads);
    if (nc == 4) return cudaLaunchKernelEx(&cfg, append_q8_kernel<Params, 8, 4>, p, threads);
    return cudaLaunchKernelEx(&cfg, append_q8_kernel<Params, 8, 2>, p, threads);
}

// A page of one layer is Hkv x ps x d contiguous codes: a block takes 1024 chunks of eight of K and of V of one page
// (blockIdx.y), a thread four of each, so that a warp's loads and stores are contiguous.
constexpr int kUnpackChunks = 4;
__global__ void __launch_bounds__(256) unpack_q8_kernel(const __grid_constant__ UnpackParams p)
{
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    int lo = 0, hi = p.n - 1;
    const int b = static_cast<int>(blockIdx.x);
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].page0 <= b) lo = mid; else hi = mid - 1;
    }
    const int page = p.page_table[p.segs[lo].table_row + (b - p.segs[lo].page0)];
    if (page < 0 || page >= p.num_pages) return;
    const int per_head = p.ps * p.d / 8, n = p.hkv * per_head;
    const int c0 = static_cast<int>(blockIdx.y) * 256 * kUnpackChunks + static_cast<int>(threadIdx.x);
    const int64_t src = (static_cast<int64_t>(p.layer) * p.num_pages + page) * p.hkv;
    const uint2 *k8 = reinterpret_cast<const uint2 *>(p.k8) + src * per_head, *v8 = reinterpret_cast<const uint2 *>(p.v8) + src * per_head;
    const char2 *ex = reinterpret_cast<const char2 *>(p.exps) + src;
    uint4 *k = p.k + static_cast<int64_t>(page) * n, *v = p.v + static_cast<int64_t>(page) * n;
    uint2 a[kUnpackChunks], w[kUnpackChunks];
    char2 e[kUnpackChunks];
#pragma unroll
    for (int u = 0; u < kUnpackChunks; ++u) {
        const int c = c0 + u * 256;
        if (c >= n) continue;
        a[u] = k8[c];
        w[u] = v8[c];
        e[u] = ex[c / per_head];
    }
#pragma unroll
    for (int u = 0; u < kUnpackChunks; ++u) {
        const int c = c0 + u * 256;
        if (c >= n) continue;
        k[c] = q8_to_bf16(a[u], pow2i(static_cast<int8_t>(e[u].x)));
        v[c] = q8_to_bf16(w[u], pow2i(static_cast<int8_t>(e[u].y)));
    }
}

// A block per page and layer.  Bound by memory: 32 pages of 32 layers and 8 kv-heads of 16 x 128, 34 MB read and written, add
// 8 us to a call of rounds.
__global__ void __launch_bounds__(256) save_pages_kernel(const __grid_constant__ SaveParams p)
{
    ptx::griddep_wait();  // launched with programmatic serialization
    ptx::griddep_launch_dependents();
    const int l = static_cast<int>(blockIdx.y), n = p.hkv * p.ps * p.d / 16;
    const int64_t head = (static_cast<int64_t>(l) * p.num_pages + p.pages[blockIdx.x]) * p.hkv;
    uint4 *k = p.k8 + head * (p.ps * p.d / 16), *v = p.v8 + head * (p.ps * p.d / 16);
    char2 *e = reinterpret_cast<char2 *>(p.exps) + head;
    uint8_t *slot = p.slots + static_cast<int64_t>(blockIdx.x) * p.slot_bytes;
    uint4 *sk = reinterpret_cast<uint4 *>(slot) + static_cast<int64_t>(l) * n, *sv = sk + static_cast<int64_t>(p.L) * n;
    char2 *se = reinterpret_cast<char2 *>(slot + static_cast<int64_t>(p.L) * n * 32) + static_cast<int64_t>(l) * p.hkv;
    for (int i = threadIdx.x; i < n; i += 256) {
        if (p.back) {
            k[i] = sk[i];
            v[i] = sv[i];
        } else {
            sk[i] = k[i];
            sv[i] = v[i];
        }
    }
    for (int h = threadIdx.x; h < p.hkv; h += 256) {
        if (p.back) e[h] = se[h];
        else se[h] = e[h];
    }
}

// One block per touched page and layer: its tokens' rows, kv-heads and chunks fastest, so that a warp writes contiguous
// memory and reads whole rows.  (Eight codes a load, and so contiguous 16-byte stores, took 12 % more.)
template <bool Q8>
__global__ void __launch_bounds__(256) read_kv_kernel(const __grid_constant__ ReadParams p)
{
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int pg = static_cast<int>(blockIdx.x % static_cast<unsigned>(p.pages));
    const int64_t l = blockIdx.x / static_cast<unsigned>(p.pages);
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].page0 <= pg) lo = mid; else hi = mid - 1;
    }
    const ReadSeg &sg = p.segs[lo];
    const int lp = (sg.begin >> p.log_ps) + (pg - sg.page0);
    const int first = max(sg.begin, lp << p.log_ps), rows = min(sg.end, (lp + 1) << p.log_ps) - first;
    const int page = p.page_table[sg.table_row + lp];
    if (page < 0 || page >= p.num_pages) return;  // (no valid token lies there)
    const int log_cpr = 31 - __clz(p.d / (Q8 ? 16 : 8)), cpr = 1 << log_cpr;  // 16-byte chunks of a stored row
    const int64_t head0 = (l * p.num_pages + page) * p.hkv;
    const int64_t out0 = (l * p.n_total + sg.tok0 + (first - sg.begin)) * p.hkv;
    const uint4 *kp = static_cast<const uint4 *>(p.k_pool), *vp = static_cast<const uint4 *>(p.v_pool);
#pragma unroll 4
    for (int i = threadIdx.x; i < rows * p.hkv * cpr; i += 256) {
        const int col = i & (cpr - 1), r = i >> log_cpr;
        const int row = static_cast<int>(static_cast<unsigned>(r) / static_cast<unsigned>(p.hkv)), h = r - row * p.hkv;
        const int64_t src = (((head0 + h) << p.log_ps) + (first & (p.ps - 1)) + row) * cpr + col;
        const int64_t dst = (out0 + r) * cpr + col;
        const uint4 k = kp[src], v = vp[src];
        if constexpr (Q8) {
            const char2 e = reinterpret_cast<const char2 *>(p.exps)[head0 + h];
            const float ks = pow2i(static_cast<int8_t>(e.x)), vs = pow2i(static_cast<int8_t>(e.y));
            const uint4 k0 = q8_to_bf16(make_uint2(k.x, k.y), ks), k1 = q8_to_bf16(make_uint2(k.z, k.w), ks);
            const bool nan = k.x == kQ8NanWord;  // a token held as NaN
            __stcs(p.K + 2 * dst, k0);
            __stcs(p.K + 2 * dst + 1, k1);
            __stcs(p.V + 2 * dst, nan ? k0 : q8_to_bf16(make_uint2(v.x, v.y), vs));
            __stcs(p.V + 2 * dst + 1, nan ? k1 : q8_to_bf16(make_uint2(v.z, v.w), vs));
        } else {
            __stcs(p.K + dst, k);
            __stcs(p.V + dst, v);
        }
    }
}

cudaLaunchConfig_t serial_config(unsigned blocks, unsigned threads, cudaStream_t st, cudaLaunchAttribute *attr)
{
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

}  // namespace

cudaError_t launch_append_q8(int head_dim, const AppendParams &p, cudaStream_t st)
{
    const int elems = p.ps * head_dim, threads = q8_unit_threads(elems), nc = q8_unit_chunks(elems);
    const int64_t units = static_cast<int64_t>(p.L) * p.seg_tokens * p.hkv;
    const int64_t blocks = (units * threads + kQ8Block - 1) / kQ8Block;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(std::max<int64_t>(1, blocks)), kQ8Block, st, &attr);
    if (p.n_segs <= kSmallSegs8 && p.n_new <= kSmallPages8) {
        using Small = AppendParamsT<kSmallSegs8, kSmallPages8>;
        Small q;
        static_assert(offsetof(Small, segs) == offsetof(AppendParams, segs), "the same header");
        std::memcpy(static_cast<void *>(&q), static_cast<const void *>(&p), offsetof(Small, segs));
        std::copy(p.segs, p.segs + p.n_segs, q.segs);
        std::copy(p.new_pages, p.new_pages + p.n_new, q.new_pages);
        return launch_append_t(cfg, head_dim, nc, q, threads);
    }
    return launch_append_t(cfg, head_dim, nc, p, threads);
}

cudaError_t launch_unpack_q8(const UnpackParams &p, int pages, cudaStream_t st)
{
    if (pages <= 0) return cudaSuccess;
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(pages), 256, st, &attr);
    cfg.gridDim.y = static_cast<unsigned>((p.hkv * p.ps * p.d / 8 + 256 * kUnpackChunks - 1) / (256 * kUnpackChunks));
    return cudaLaunchKernelEx(&cfg, unpack_q8_kernel, p);
}

cudaError_t launch_save_pages(const SaveParams &p, cudaStream_t st)
{
    if (p.n <= 0) return cudaSuccess;
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(p.n), 256, st, &attr);
    cfg.gridDim.y = static_cast<unsigned>(p.L);
    return cudaLaunchKernelEx(&cfg, save_pages_kernel, p);
}

cudaError_t launch_read_kv(bool q8, const ReadParams &p, cudaStream_t st)
{
    const int64_t blocks = static_cast<int64_t>(p.L) * p.pages;
    if (blocks <= 0) return cudaSuccess;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(blocks), 256, st, &attr);
    return q8 ? cudaLaunchKernelEx(&cfg, read_kv_kernel<true>, p) : cudaLaunchKernelEx(&cfg, read_kv_kernel<false>, p);
}

}  // namespace pe
