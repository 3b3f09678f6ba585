// Position rotation: of keys on their way into the cache and of the queries beside them (append), and of one tensor alone.
//
// Pair i of a head's columns -- (i, i + n_pairs), or neighbours (2i, 2i + 1) -- turns by the angle that frequency i has at
// the token's position on i's axis:
//     a' = scale (a cos - b sin),  b' = scale (b cos + a sin)
// in 32 bits, rounded once.  Columns past the pairs are copied.
#include <algorithm>
#include <cstddef>
#include <cstring>

#include "pe_internal.h"
#include "dev_common.cuh"
#include "q8.cuh"

namespace pe {

namespace {

// (cos, sin) times the scale of pair i for token tok (of the whole tensor), whose position in its sequence is pos.
__device__ __forceinline__ float2 rope_turn(const RopeParams &r, int i, int64_t tok, int pos)
{
    const int at = r.positions ? r.positions[r.axis[i] * r.positions_stride + tok] : pos;
    const uint64_t phase = static_cast<uint64_t>(static_cast<int64_t>(at)) * r.turn[i];
    float s, c;
    sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 4.656612873077393e-10f, &s, &c);  // 2^-31 half turns
    return make_float2(c * r.scale, s * r.scale);
}

__device__ __forceinline__ float bf16_at(const uint4 *row, int col)
{
    return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(row)[col]);
}

// Columns 8 chunk .. + 7 of a row, rotated.
__device__ __forceinline__ void rope_chunk(const RopeParams &r, const uint4 *row, int chunk, int64_t tok, int pos, float (&y)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int col = chunk * 8 + k;
        const float x = bf16_at(row, col);
        y[k] = x;
        if (col >= 2 * r.n_pairs) continue;
        const bool second = r.interleaved ? col & 1 : col >= r.n_pairs;
        const int i = r.interleaved ? col >> 1 : (second ? col - r.n_pairs : col);
        const int other = r.interleaved ? col ^ 1 : (second ? i : col + r.n_pairs);
        const float2 t = rope_turn(r, i, tok, pos);
        const float z = bf16_at(row, other);
        y[k] = second ? x * t.x + z * t.y : x * t.x - z * t.y;
    }
}

__device__ __forceinline__ uint4 pack8(const float (&y)[8])
{
    return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

template <typename Segs>
__device__ __forceinline__ int find_seg(const Segs &segs, int n, int t)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (segs[mid].cum0 <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// A thread per 16-byte chunk, whole rows within a warp: reads come before writes there, so out may be X.
template <int CPR>
__global__ void __launch_bounds__(256) rotate_kernel(const __grid_constant__ RotateParams p, int64_t chunks)
{
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const bool on = c < chunks;
    const int64_t r = on ? c / CPR : 0;
    const int h = static_cast<int>(r % p.heads);
    const int64_t t = r / p.heads;
    const int tok = p.tok0 + static_cast<int>(t % p.n_tokens);
    const int64_t row = ((t / p.n_tokens) * p.n_total + tok) * p.heads + h;
    int lo = 0, hi = p.n_segs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].tok0 <= tok) lo = mid; else hi = mid - 1;
    }
    const int pos = p.segs[lo].pos0 + tok - p.segs[lo].tok0;
    float y[8];
    if (on) rope_chunk(p.r, p.X + row * CPR, static_cast<int>(c % CPR), tok, pos, y);
    __syncwarp();
    if (on) p.out[row * CPR + c % CPR] = pack8(y);
}

// K's rows rotated and V's copied into their slots, and Q's rows rotated: `rows` of each token, Hkv and then Hq.
template <typename Params, int CPR>
__global__ void __launch_bounds__(256) append_rope_kernel(const __grid_constant__ Params p, int64_t chunks)
{
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const auto &a = p.a;
    if (blockIdx.x == 0) {
        for (int s = 0; s < a.n_segs; ++s) {
            const AppendSeg &sg = a.segs[s];
            for (int i = threadIdx.x; i < sg.n_new; i += 256)
                a.page_table[sg.table_row + sg.first_new_lp + i] = a.new_pages[sg.new0 + i];
            if (threadIdx.x == 0) a.seq_len[sg.seq] = static_cast<int64_t>(sg.len0) + sg.n_tokens;
        }
    }
    const int heads = a.hkv + (p.c.Q ? p.c.hq : 0);
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const bool on = c < chunks;
    const int64_t r = on ? c / CPR : 0;
    const int chunk = static_cast<int>(c % CPR);
    const int h = static_cast<int>(r % heads);
    const int64_t lt = r / heads;
    const int t = static_cast<int>(lt % a.seg_tokens);
    const int64_t l = lt / a.seg_tokens;
    const AppendSeg &sg = a.segs[find_seg(a.segs, a.n_segs, t)];
    const int local = t - sg.cum0, pos = sg.len0 + local;
    const int64_t tok = sg.tok0 + local;
    const bool is_q = h >= a.hkv;
    const int64_t src = is_q ? ((l * a.n_total + tok) * p.c.hq + (h - a.hkv)) * CPR : ((l * a.n_total + tok) * a.hkv + h) * CPR;
    float y[8];
    if (on) rope_chunk(p.c.r, (is_q ? p.c.Q : a.K) + src, chunk, tok, pos, y);
    __syncwarp();
    if (!on) return;
    if (is_q) {
        p.c.Q_out[src + chunk] = pack8(y);
        return;
    }
    const int lp = pos / a.ps;
    const int page = lp < sg.first_new_lp ? sg.last_page : a.new_pages[sg.new0 + (lp - sg.first_new_lp)];
    const int64_t dst = (((l * a.num_pages + page) * a.hkv + h) * a.ps + (pos - lp * a.ps)) * CPR + chunk;
    a.k_pool[dst] = pack8(y);
    a.v_pool[dst] = a.V[src + chunk];
}

cudaLaunchConfig_t serial_config(int64_t blocks, unsigned threads, cudaStream_t st, cudaLaunchAttribute *attr)
{
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::max<int64_t>(1, blocks)));
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

// Page by page (append_q8_kernel): the new rows of K rotated in 32 bits, so that a value is rounded once, to its code.
template <typename Params, int CPR, int NC>
__global__ void __launch_bounds__(kQ8Block) append_rope_q8_kernel(const __grid_constant__ Params p, int threads, int page_blocks)
{
    __shared__ uint32_t s_max[kQ8Block / 32];
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const auto &a = p.a;
    constexpr int HD = CPR * 8;
    if (static_cast<int>(blockIdx.x) >= page_blocks) {  // Q's rows
        const int64_t c = static_cast<int64_t>(blockIdx.x - page_blocks) * kQ8Block + threadIdx.x;
        int n_tok = 0;
        for (int s = 0; s < a.n_segs; ++s) n_tok += a.segs[s].n_tokens;
        const bool on = c < static_cast<int64_t>(a.L) * n_tok * p.c.hq * CPR;
        const int64_t r = on ? c / CPR : 0;
        const int h = static_cast<int>(r % p.c.hq);
        const int64_t lt = r / p.c.hq;
        int t = static_cast<int>(lt % n_tok), s = 0;
        for (; t >= a.segs[s].n_tokens; ++s) t -= a.segs[s].n_tokens;
        const int64_t tok = a.segs[s].tok0 + t;
        const int64_t src = (((lt / n_tok) * a.n_total + tok) * p.c.hq + h) * CPR;
        float y[8];
        if (on) rope_chunk(p.c.r, p.c.Q + src, static_cast<int>(c % CPR), tok, a.segs[s].len0 + t, y);
        __syncwarp();
        if (on) p.c.Q_out[src + c % CPR] = pack8(y);
        return;
    }
    if (blockIdx.x == 0) {
        for (int s = 0; s < a.n_segs; ++s) {
            const AppendSeg &sg = a.segs[s];
            for (int i = threadIdx.x; i < sg.n_new; i += kQ8Block)
                a.page_table[sg.table_row + sg.first_new_lp + i] = a.new_pages[sg.new0 + i];
            if (threadIdx.x == 0) a.seq_len[sg.seq] = static_cast<int64_t>(sg.len0) + sg.n_tokens;
        }
    }
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kQ8Block / threads) + threadIdx.x / threads;
    const bool on = unit < static_cast<int64_t>(a.L) * a.seg_tokens * a.hkv;
    const int64_t u = on ? unit : 0;
    const int h = static_cast<int>(u % a.hkv);
    const int64_t r = u / a.hkv;
    const int pg = static_cast<int>(r % a.seg_tokens);
    const int64_t l = r / a.seg_tokens;
    const AppendSeg &sg = a.segs[find_seg(a.segs, a.n_segs, pg)];
    const int lp = sg.len0 / a.ps + (pg - sg.cum0);
    const int page = lp < sg.first_new_lp ? sg.last_page : a.new_pages[sg.new0 + (lp - sg.first_new_lp)];
    const int pos0 = lp * a.ps;
    const int old = max(0, sg.len0 - pos0);
    const int rows = min(a.ps, sg.len0 + sg.n_tokens - pos0);
    const int64_t head = (l * a.num_pages + page) * a.hkv + h;
    uint8_t *kp = reinterpret_cast<uint8_t *>(a.k_pool) + head * a.ps * HD;
    uint8_t *vp = reinterpret_cast<uint8_t *>(a.v_pool) + head * a.ps * HD;
    int8_t *ex = a.exps + head * 2;
    int ke0 = 0, ve0 = 0;
    if (on && old > 0) {
        ke0 = ex[0];
        ve0 = ex[1];
    }
    const float kes = pow2i(ke0), ves = pow2i(ve0);
    const int64_t tok0 = sg.tok0 + (pos0 - sg.len0);  // of the page's row 0
    if (threads <= 32) __syncwarp();
    else __syncthreads();  // the old exponents are read before they are written
    q8_write_page_f32<CPR, NC>(on, threadIdx.x % threads, threads, rows, old, ke0, ve0, kp, vp, ex, s_max,
                               [&](int row, int col8, float (&k)[8], uint4 &v) {
                                   if (row < old) {
                                       q8_to_float(*reinterpret_cast<const uint2 *>(kp + row * HD + col8 * 8), kes, k);
                                       v = q8_to_bf16(*reinterpret_cast<const uint2 *>(vp + row * HD + col8 * 8), ves);
                                   } else {
                                       const int64_t tok = tok0 + row;
                                       const int64_t s = ((l * a.n_total + tok) * a.hkv + h) * CPR;
                                       rope_chunk(p.c.r, a.K + s, col8, tok, pos0 + row, k);
                                       v = a.V[s + col8];
                                   }
                               });
}

constexpr int kSmallSegs = 16, kSmallPages = 128;  // the small parameter block (as in pe_kv.cu)

template <typename Params>
cudaError_t launch_append_rope_t(bool q8, int head_dim, const Params &p, cudaStream_t st)
{
    cudaLaunchAttribute attr;
    if (!q8) {
        const int64_t chunks = static_cast<int64_t>(p.a.L) * p.a.seg_tokens * (p.a.hkv + (p.c.Q ? p.c.hq : 0)) * (head_dim / 8);
        const cudaLaunchConfig_t cfg = serial_config((chunks + 255) / 256, 256, st, &attr);
        return head_dim == 128 ? cudaLaunchKernelEx(&cfg, append_rope_kernel<Params, 16>, p, chunks)
                               : cudaLaunchKernelEx(&cfg, append_rope_kernel<Params, 8>, p, chunks);
    }
    const int elems = p.a.ps * head_dim, threads = q8_unit_threads(elems), nc = q8_unit_chunks(elems);
    const int64_t units = static_cast<int64_t>(p.a.L) * p.a.seg_tokens * p.a.hkv;
    const int64_t page_blocks = (units * threads + kQ8Block - 1) / kQ8Block;
    int64_t tokens = 0;
    for (int i = 0; i < p.a.n_segs; ++i) tokens += p.a.segs[i].n_tokens;
    const int64_t q_blocks = p.c.Q ? (p.a.L * tokens * p.c.hq * (head_dim / 8) + kQ8Block - 1) / kQ8Block : 0;
    if (page_blocks + q_blocks > INT32_MAX) return cudaErrorInvalidValue;
    const cudaLaunchConfig_t cfg = serial_config(page_blocks + q_blocks, kQ8Block, st, &attr);
    const int pb = static_cast<int>(page_blocks);
    if (head_dim == 128) {
        if (nc == 8) return cudaLaunchKernelEx(&cfg, append_rope_q8_kernel<Params, 16, 8>, p, threads, pb);
        return cudaLaunchKernelEx(&cfg, append_rope_q8_kernel<Params, 16, 4>, p, threads, pb);
    }
    if (nc == 8) return cudaLaunchKernelEx(&cfg, append_rope_q8_kernel<Params, 8, 8>, p, threads, pb);
    if (nc == 4) return cudaLaunchKernelEx(&cfg, append_rope_q8_kernel<Params, 8, 4>, p, threads, pb);
    return cudaLaunchKernelEx(&cfg, append_rope_q8_kernel<Params, 8, 2>, p, threads, pb);
}

template <int SEGS, int PAGES>
cudaError_t launch_sized(bool q8, int head_dim, const AppendParams &a, const RopeCall &rope, cudaStream_t st)
{
    AppendRopeParamsT<SEGS, PAGES> p;
    using Block = AppendParamsT<SEGS, PAGES>;
    static_assert(offsetof(Block, segs) == offsetof(AppendParams, segs), "the same header");
    p.c = rope;
    std::memcpy(static_cast<void *>(&p.a), static_cast<const void *>(&a), offsetof(AppendParams, segs));
    std::copy(a.segs, a.segs + a.n_segs, p.a.segs);
    std::copy(a.new_pages, a.new_pages + a.n_new, p.a.new_pages);
    return launch_append_rope_t(q8, head_dim, p, st);
}

}  // namespace

cudaError_t launch_append_rope(bool q8, int head_dim, const AppendParams &a, const RopeCall &rope, cudaStream_t st)
{
    if (a.n_segs <= kSmallSegs && a.n_new <= kSmallPages) return launch_sized<kSmallSegs, kSmallPages>(q8, head_dim, a, rope, st);
    return launch_sized<kMaxSegs, kAppendMaxPages>(q8, head_dim, a, rope, st);
}

cudaError_t launch_rotate(int head_dim, const RotateParams &p, cudaStream_t st)
{
    const int64_t chunks = static_cast<int64_t>(p.layers) * p.n_tokens * p.heads * (head_dim / 8);
    if (chunks <= 0) return cudaSuccess;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config((chunks + 255) / 256, 256, st, &attr);
    return head_dim == 128 ? cudaLaunchKernelEx(&cfg, rotate_kernel<16>, p, chunks) : cudaLaunchKernelEx(&cfg, rotate_kernel<8>, p, chunks);
}

}  // namespace pe
