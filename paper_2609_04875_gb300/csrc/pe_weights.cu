// The keys' accumulated softmax weights: acc[j] += sum over q-heads h and
// queries i of w_ij^h, w = softmax(scale q_i^h K^T)_j, for the queries of one
// attention call.  Two passes over K (bf16): the log-sum-exp of every query row,
// then, one thread per key, the sum of its weights over the rows in a fixed
// order (nothing is added atomically).
#include "dev_common.cuh"

namespace pe {

namespace {

constexpr int kLseThreads = 128;
constexpr int kWtKeys = 128;
constexpr int kWtRows = 16;

// scores of bf16 q (fp32 in shared memory) against one bf16 key row
template <int HD>
__device__ __forceinline__ float dot_row(const float *q, const uint4 *k)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) {
        const uint4 w = k[i];
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s = fmaf(__uint_as_float(u[j] << 16), q[8 * i + 2 * j], s);
            s = fmaf(__uint_as_float(u[j] & 0xffff0000u), q[8 * i + 2 * j + 1], s);
        }
    }
    return s;
}

__device__ __forceinline__ int64_t key_row(const WeightParams &p, const WeightSeg &sg, int h, int key)
{
    const int page = p.page_table[sg.table_row + key / p.ps];
    return (static_cast<int64_t>(page) * p.hkv + h) * p.ps + key % p.ps;
}

// One block per query row: its log2-sum-exp over the keys it sees.
template <int HD>
__global__ void __launch_bounds__(kLseThreads) weights_lse_kernel(const __grid_constant__ WeightParams p)
{
    __shared__ float s_q[HD], s_m[kLseThreads / 32], s_l[kLseThreads / 32];
    const int64_t row = blockIdx.x;  // q row x Hq
    const int qr = static_cast<int>(row / p.hq), hq = static_cast<int>(row % p.hq);
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].q_row0 - p.segs[0].q_row0 <= qr) lo = mid; else hi = mid - 1;
    }
    const WeightSeg &sg = p.segs[lo];
    const int i = qr - (sg.q_row0 - p.segs[0].q_row0);
    const int n_keys = sg.n_keys - sg.n_q + i + 1;
    for (int c = threadIdx.x; c < HD; c += kLseThreads)
        s_q[c] = __bfloat162float(p.q[(static_cast<int64_t>(sg.q_row0 + i) * p.hq + hq) * HD + c]);
    __syncthreads();
    float m = -INFINITY, l = 0.f;
    for (int key = threadIdx.x; key < n_keys; key += kLseThreads) {
        const float x = p.scale_log2 * dot_row<HD>(s_q, reinterpret_cast<const uint4 *>(p.k + key_row(p, sg, hq / p.group, key) * HD));
        const float mn = x > m || x != x ? x : m;
        l = l * (m == -INFINITY ? 0.f : exp2f(m - mn)) + exp2f(x - mn);
        m = mn;
    }
    // the warp's, then the block's
    for (int off = 16; off >= 1; off >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, off), ol = __shfl_xor_sync(0xffffffffu, l, off);
        const float mn = om > m || om != om ? om : m;
        l = (m == -INFINITY ? 0.f : l * exp2f(m - mn)) + (om == -INFINITY ? 0.f : ol * exp2f(om - mn));
        m = mn;
    }
    if ((threadIdx.x & 31) == 0) {
        s_m[threadIdx.x >> 5] = m;
        s_l[threadIdx.x >> 5] = l;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    m = -INFINITY;
    for (float x : s_m) m = x > m || x != x ? x : m;
    l = 0.f;
    for (int w = 0; w < kLseThreads / 32; ++w) l += s_m[w] == -INFINITY ? 0.f : s_l[w] * exp2f(s_m[w] - m);
    p.lse[static_cast<int64_t>(sg.q_row0 + i) * p.hq + hq] = m + log2f(l);
}

// One block per 128 keys of a sequence.
template <int HD>
__global__ void __launch_bounds__(kWtKeys) weights_sum_kernel(const __grid_constant__ WeightParams p)
{
    __shared__ float s_q[kWtRows][HD], s_lse[kWtRows];
    const WeightSeg &sg = p.segs[blockIdx.y];
    const int key = static_cast<int>(blockIdx.x) * kWtKeys + static_cast<int>(threadIdx.x);
    if (static_cast<int>(blockIdx.x) * kWtKeys >= sg.n_keys) return;
    const bool on = key < sg.n_keys;
    const int pos0 = sg.n_keys - sg.n_q;
    const int rows = sg.n_q * p.group;
    float sum = 0.f;
    for (int h = 0; h < p.hkv; ++h) {
        uint4 k[HD / 8];
        if (on) {
            const uint4 *src = reinterpret_cast<const uint4 *>(p.k + key_row(p, sg, h, key) * HD);
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) k[c] = src[c];
        }
        for (int r0 = 0; r0 < rows; r0 += kWtRows) {
            const int nr = min(kWtRows, rows - r0);
            __syncthreads();
            for (int c = threadIdx.x; c < nr * HD; c += kWtKeys) {
                const int r = r0 + c / HD;
                s_q[c / HD][c % HD] = __bfloat162float(
                    p.q[(static_cast<int64_t>(sg.q_row0 + r / p.group) * p.hq + h * p.group + r % p.group) * HD + c % HD]);
            }
            if (static_cast<int>(threadIdx.x) < nr) {
                const int r = r0 + static_cast<int>(threadIdx.x);
                s_lse[threadIdx.x] = p.lse[static_cast<int64_t>(sg.q_row0 + r / p.group) * p.hq + h * p.group + r % p.group];
            }
            __syncthreads();
            if (!on) continue;
            for (int r = 0; r < nr; ++r)
                if (key <= pos0 + (r0 + r) / p.group)
                    sum += exp2f(p.scale_log2 * dot_row<HD>(s_q[r], k) - s_lse[r]);
        }
    }
    if (on) {
        float *a = p.weights + static_cast<int64_t>(sg.row) * p.weights_stride + key;
        *a += sum;
    }
}

// The same sum from kept scores.  A block per 32 keys: warp w takes the rows w, w + 8, .. of every kv-head (a key per
// lane, eight rows in flight), and the warps' sums are added in order.  Bound by the scores' latency and bytes (L2).
constexpr int kKeptWarps = 8, kKeptRows = 8;
__global__ void __launch_bounds__(32 * kKeptWarps) weights_kept_kernel(const __grid_constant__ WeightParams p)
{
    __shared__ float s_sum[kKeptWarps][32];
    const WeightSeg &sg = p.segs[blockIdx.y];
    const int key0 = static_cast<int>(blockIdx.x) * 32;
    if (key0 >= sg.n_keys) return;
    ptx::griddep_wait();  // launched with programmatic serialization
    ptx::griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_head = sg.n_q * p.group, rows = per_head * p.hkv;  // row R: kv-head R / per_head
    const float *s = p.scores + sg.score0 + key0 + lane;
    float sum = 0.f;
    for (int r0 = warp; r0 < rows; r0 += kKeptWarps * kKeptRows) {
        float x[kKeptRows], l[kKeptRows];
#pragma unroll
        for (int u = 0; u < kKeptRows; ++u) {
            const int R = r0 + u * kKeptWarps;
            const int h = R / per_head, r = R - h * per_head;
            x[u] = R < rows ? s[static_cast<int64_t>(R) * sg.score_stride] : -INFINITY;
            l[u] = R < rows ? p.lse[static_cast<int64_t>(sg.q_row0 + r / p.group) * p.hq + h * p.group + r % p.group] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kKeptRows; ++u) sum += ex2(x[u] - l[u]);
    }
    s_sum[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || key0 + lane >= sg.n_keys) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kKeptWarps; ++w) sum += s_sum[w][lane];
    p.weights[static_cast<int64_t>(sg.row) * p.weights_stride + key0 + lane] += sum;
}

}  // namespace

cudaError_t launch_weights_kept(const WeightParams &p, int max_keys, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((max_keys + 31) / 32), static_cast<unsigned>(p.n));
    cfg.blockDim = dim3(32 * kKeptWarps);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, weights_kept_kernel, p);
}

cudaError_t launch_weights(int head_dim, const WeightParams &p, int64_t q_rows, int max_keys, cudaStream_t st)
{
    const unsigned rows = static_cast<unsigned>(q_rows * p.hq);
    const dim3 tiles(static_cast<unsigned>((max_keys + kWtKeys - 1) / kWtKeys), static_cast<unsigned>(p.n));
    if (head_dim == 128) {
        weights_lse_kernel<128><<<rows, kLseThreads, 0, st>>>(p);
        weights_sum_kernel<128><<<tiles, kWtKeys, 0, st>>>(p);
    } else {
        weights_lse_kernel<64><<<rows, kLseThreads, 0, st>>>(p);
        weights_sum_kernel<64><<<tiles, kWtKeys, 0, st>>>(p);
    }
    return cudaGetLastError();
}

}  // namespace pe
