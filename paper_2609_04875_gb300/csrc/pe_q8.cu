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
    float kes = 0.f, ves = 0.f;
    if (on && old > 0) {
        kes = pow2i(ex[0]);
        ves = pow2i(ex[1]);
    }
    const int64_t src0 = ((l * p.n_total + sg.tok0 + (pos0 - sg.len0)) * p.hkv + h) * CPR;  // of the page's row 0
    if (threads <= 32) __syncwarp();
    else __syncthreads();  // the old exponents are read before they are written
    q8_write_page<CPR, NC>(on, threadIdx.x % threads, threads, rows, kp, vp, ex, s_max,
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

// One block per (sequence, page): the page of one layer is Hkv x ps x d contiguous codes.
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
    const int per_head = p.ps * p.d / 16;  // 16-code chunks
    const int64_t src = static_cast<int64_t>(p.layer) * p.num_pages + page;
    const uint4 *k8 = p.k8 + src * p.hkv * per_head, *v8 = p.v8 + src * p.hkv * per_head;
    uint4 *k = p.k + static_cast<int64_t>(page) * p.hkv * per_head * 2;
    uint4 *v = p.v + static_cast<int64_t>(page) * p.hkv * per_head * 2;
    const int8_t *ex = p.exps + src * p.hkv * 2;
    for (int c = threadIdx.x; c < p.hkv * per_head; c += 256) {
        const int h = c / per_head;
        const float ks = pow2i(ex[2 * h]), vs = pow2i(ex[2 * h + 1]);
        const uint4 a = k8[c], w = v8[c];
        k[2 * c] = q8_to_bf16(make_uint2(a.x, a.y), ks);
        k[2 * c + 1] = q8_to_bf16(make_uint2(a.z, a.w), ks);
        v[2 * c] = q8_to_bf16(make_uint2(w.x, w.y), vs);
        v[2 * c + 1] = q8_to_bf16(make_uint2(w.z, w.w), vs);
    }
}

// A thread moves eight values of K and of V.  Tokens [begin_i, begin_i + n_i) of each sequence, every layer.
template <bool Q8>
__global__ void __launch_bounds__(256) read_kv_kernel(const __grid_constant__ ReadParams p, int64_t chunks)
{
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int cpr = p.d / 8;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t c = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; c < chunks; c += stride) {
        const int col8 = static_cast<int>(c % cpr);
        int64_t r = c / cpr;
        const int h = static_cast<int>(r % p.hkv);
        r /= p.hkv;
        const int t = static_cast<int>(r % p.seg_tokens);
        const int64_t l = r / p.seg_tokens;
        int lo = 0, hi = p.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.segs[mid].cum0 <= t) lo = mid; else hi = mid - 1;
        }
        const ReadSeg &sg = p.segs[lo];
        const int pos = sg.begin + (t - sg.cum0);
        const int page = p.page_table[sg.table_row + pos / p.ps];
        const int64_t head = (l * p.num_pages + page) * p.hkv + h;
        const int64_t src = (head * p.ps + pos % p.ps) * cpr + col8;
        uint4 k, v;
        if (page < 0 || page >= p.num_pages) {
            k = v = make_uint4(kBf16NanPair, kBf16NanPair, kBf16NanPair, kBf16NanPair);
        } else if constexpr (Q8) {
            const uint2 kc = static_cast<const uint2 *>(p.k_pool)[src], vc = static_cast<const uint2 *>(p.v_pool)[src];
            k = q8_to_bf16(kc, pow2i(p.exps[2 * head]));
            v = q8_to_bf16(vc, pow2i(p.exps[2 * head + 1]));
            if (kc.x == kQ8NanWord) v = k;  // a token held as NaN
        } else {
            k = static_cast<const uint4 *>(p.k_pool)[src];
            v = static_cast<const uint4 *>(p.v_pool)[src];
        }
        const int64_t dst = ((l * p.n_total + sg.tok0 + (t - sg.cum0)) * p.hkv + h) * cpr + col8;
        __stcs(p.K + dst, k);
        __stcs(p.V + dst, v);
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
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(pages), 256, st, &attr);
    return cudaLaunchKernelEx(&cfg, unpack_q8_kernel, p);
}

cudaError_t launch_read_kv(bool q8, const ReadParams &p, int num_sms, cudaStream_t st)
{
    const int64_t chunks = static_cast<int64_t>(p.L) * p.seg_tokens * p.hkv * (p.d / 8);
    if (chunks <= 0) return cudaSuccess;
    const int64_t blocks = std::min<int64_t>((chunks + 255) / 256, static_cast<int64_t>(num_sms) * 16);
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(static_cast<unsigned>(blocks), 256, st, &attr);
    return q8 ? cudaLaunchKernelEx(&cfg, read_kv_kernel<true>, p, chunks) : cudaLaunchKernelEx(&cfg, read_kv_kernel<false>, p, chunks);
}

}  // namespace pe
