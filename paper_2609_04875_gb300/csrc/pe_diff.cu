// Differential attention over the paged cache.  Heads 2i and 2i + 1 of Q are the two maps of head i, which reads kv-heads
// 2j and 2j + 1 (j = i / group): their keys, one head a map, and side by side their values, of width 2d.
//     A_m = softmax(scale q_m K_{2j+m}^T),  O = (A_0 - lambda_i A_1) [V_2j | V_2j+1],
//     out = gain O / sqrt(mean(O^2) + eps)   (or O, without a gain)
#include "dev_common.cuh"

namespace pe {

namespace {

// A block per query row and head: each warp takes every eighth key, with sums of its own; the block's first warp joins them.
template <int HD>
__global__ void __launch_bounds__(256) diff_attn_kernel(const __grid_constant__ DiffParams p)
{
    constexpr int E = HD / 32, W = 2 * HD / 32;  // columns of q and of O that a lane holds
    __shared__ float s_m[2][8], s_l[2][8], s_o[2][8][2 * HD];
    ptx::griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int i = static_cast<int>(blockIdx.y), j = i / p.group;
    int row = static_cast<int>(blockIdx.x), si = 0;
    while (row >= p.seqs[si].n_q) row -= p.seqs[si++].n_q;
    const DiffSeq &sq = p.seqs[si];
    const int keys = sq.n_keys - sq.n_q + row + 1;
    const int64_t q_row = sq.q_row0 + row;
    float q[2][E], o[2][W], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    for (int x = 0; x < 2; ++x) {
        for (int e = 0; e < E; ++e) q[x][e] = __bfloat162float(p.q[(q_row * p.hq + 2 * i + x) * HD + e * 32 + lane]);
        for (int w = 0; w < W; ++w) o[x][w] = 0.f;
    }
    for (int k = warp; k < keys; k += 8) {
        const int page = p.page_table[sq.table_row + k / p.ps];
        if (page < 0 || page >= p.num_pages) continue;
        const int64_t at = (((static_cast<int64_t>(p.layer) * p.num_pages + page) * p.hkv + 2 * j) * p.ps + k % p.ps) * HD;
        const int64_t next = static_cast<int64_t>(p.ps) * HD;  // the same token of kv-head 2j + 1
        float v[W];
        for (int w = 0; w < W; ++w) v[w] = __bfloat162float(p.v_pool[at + (w * 32 / HD) * next + (w * 32 % HD) + lane]);
        for (int x = 0; x < 2; ++x) {
            float s = 0.f;
            for (int e = 0; e < E; ++e) s += q[x][e] * __bfloat162float(p.k_pool[at + x * next + e * 32 + lane]);
            for (int w = 16; w; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
            s *= p.scale_log2;
            const float m_new = fmaxf(m[x], s);
            if (m_new == -INFINITY && s == -INFINITY) continue;  // (a NaN goes on)
            const float f = m[x] == -INFINITY ? 0.f : ex2(m[x] - m_new), pw = ex2(s - m_new);
            l[x] = l[x] * f + pw;
            for (int w = 0; w < W; ++w) o[x][w] = o[x][w] * f + pw * v[w];
            m[x] = m_new;
        }
    }
    for (int x = 0; x < 2; ++x) {
        if (lane == 0) {
            s_m[x][warp] = m[x];
            s_l[x][warp] = l[x];
        }
        for (int w = 0; w < W; ++w) s_o[x][warp][w * 32 + lane] = o[x][w];
    }
    __syncthreads();
    if (warp > 0) return;
    float r[W], sum = 0.f;
    for (int w = 0; w < W; ++w) r[w] = 0.f;
    for (int x = 0; x < 2; ++x) {
        float mx = -INFINITY, den = 0.f, acc[W];
        for (int u = 0; u < 8; ++u) mx = fmaxf(mx, s_m[x][u]);
        for (int w = 0; w < W; ++w) acc[w] = 0.f;
        for (int u = 0; u < 8; ++u) {
            const float f = s_m[x][u] == -INFINITY ? (s_l[x][u] == 0.f ? 0.f : s_l[x][u]) : ex2(s_m[x][u] - mx);
            den += f * s_l[x][u];
            if (f != 0.f)
                for (int w = 0; w < W; ++w) acc[w] += f * s_o[x][u][w * 32 + lane];
        }
        const float inv = den == 0.f ? 0.f : 1.f / den, part = x ? -p.lambda[i] : 1.f;
        for (int w = 0; w < W; ++w) r[w] += part * acc[w] * inv;
    }
    if (p.gain) {
        for (int w = 0; w < W; ++w) sum += r[w] * r[w];
        for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        const float f = 1.f / sqrtf(sum / (2 * HD) + p.eps);
        for (int w = 0; w < W; ++w) r[w] *= f * p.gain[w * 32 + lane];
    }
    for (int w = 0; w < W; ++w) p.out[(q_row * (p.hq / 2) + i) * 2 * HD + w * 32 + lane] = __float2bfloat16(r[w]);
}

}  // namespace

cudaError_t launch_diff_attn(int head_dim, const DiffParams &p, int64_t rows, cudaStream_t st)
{
    if (rows <= 0) return cudaSuccess;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows), static_cast<unsigned>(p.hq / 2));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return head_dim == 128 ? cudaLaunchKernelEx(&cfg, diff_attn_kernel<128>, p) : cudaLaunchKernelEx(&cfg, diff_attn_kernel<64>, p);
}

}  // namespace pe
