// The keys' accumulated softmax weights: acc[j] += sum over q-heads h and
// queries i of w_ij^h, w = softmax(scale q_i^h K^T)_j, for the queries of one
// attention call.  Two passes over K (bf16): the log-sum-exp of every query row,
// then, one thread per key, the sum of its weights over the rows in a fixed
// order (nothing is added atomically).  That is the form for bf16 caches, and on
// an 8-bit cache for what does not fit its workspace or is kept off the codes by
// an option.  Otherwise 8-bit caches take one of two others:
//   - few rows: the attention keeps its scores, which are summed here;
//   - more rows: the scores are computed again on the tensor cores
//     (weights_q8_kernel), from the codes and the attention's log-sum-exp.
#include "q8_mma.cuh"

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
        if (x == -INFINITY) continue;  // adds nothing (and -inf - -inf, before a thread's first other key, would be NaN)
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

// The same sum from kept scores.  A block per 128 keys: warp w takes the rows w, w + 8, .. of every kv-head (four keys a
// lane, four rows in flight), and the warps' sums are added in order.  Bound by the latency of its reads (from L2).
constexpr int kKeptWarps = 8, kKeptRows = 4, kKeptKeys = 128;
__global__ void __launch_bounds__(32 * kKeptWarps) weights_kept_kernel(const __grid_constant__ WeightParams p)
{
    __shared__ float4 s_sum[kKeptWarps][32];
    const WeightSeg &sg = p.segs[blockIdx.y];
    const int key0 = static_cast<int>(blockIdx.x) * kKeptKeys;
    ptx::griddep_wait();  // launched with programmatic serialization
    ptx::griddep_launch_dependents();
    if (key0 >= sg.n_keys) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_head = sg.n_q * p.group, rows = per_head * p.hkv;  // row R: kv-head R / per_head
    const float *s = p.scores + sg.score0 + key0 + 4 * lane;  // (a row's last tile is whole: -inf past the keys)
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r0 = warp; r0 < rows; r0 += kKeptWarps * kKeptRows) {
        float4 x[kKeptRows];
        float l[kKeptRows];
#pragma unroll
        for (int u = 0; u < kKeptRows; ++u) {
            const int R = r0 + u * kKeptWarps;
            const int h = R / per_head, r = R - h * per_head;
            x[u] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            l[u] = 0.f;
            if (R < rows) {
                x[u] = *reinterpret_cast<const float4 *>(s + static_cast<int64_t>(R) * sg.score_stride);
                l[u] = p.lse[static_cast<int64_t>(sg.q_row0 + r / p.group) * p.hq + h * p.group + r % p.group];
            }
        }
#pragma unroll
        for (int u = 0; u < kKeptRows; ++u) {
            sum.x += ex2(x[u].x - l[u]);
            sum.y += ex2(x[u].y - l[u]);
            sum.z += ex2(x[u].z - l[u]);
            sum.w += ex2(x[u].w - l[u]);
        }
    }
    s_sum[warp][lane] = sum;
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= kKeptKeys || key0 + t >= sg.n_keys) return;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kKeptWarps; ++w) total += reinterpret_cast<const float *>(s_sum[w])[t];
    p.weights[static_cast<int64_t>(sg.row) * p.weights_stride + key0 + t] += total;
}

// ---- many rows of an 8-bit cache: S^T again, keys on the M side
//     S^T [128 keys x 128 rows] = K8 [128 x d] . Q8^T, q in two e4m3 parts added up in the same columns (q8_mma.cuh),
//     acc[key] += sum over rows of 2^(S 2^(ek + eq) scale_log2 - lse)
// A CTA takes 128 keys of a sequence and goes through all kv-heads and groups of 128 rows (a unit each), so that a key
// has one writer; a thread owns a key and adds up its rows in order.  Where the tiles of keys are fewer than the SMs, a
// cluster of up to 8 CTAs shares a tile's units (1.6 us each, one after another) and its first CTA adds up the others'
// sums in order: 128 queries of 32 q-heads on 1000 keys 55 -> 12 us.  Bound by the exponentials: rows x keys
// of them.
// q's parts, 2^eq scale_log2 and -lse of each group are laid out once (weights_rows_kernel) as the kernel's shared
// memory holds them, so a group is one bulk copy.  For 2 x 32 queries of 32 q-heads on 9k and 16k keys the scores kept by
// the attention, 8 bytes a row and key, took 99 us to add up; this takes 28, its layout of q included.
//
// Roles (320 threads): warps 0-3 and 4-7 the sums of every other unit, warp 8 copies, warp 9 MMAs.
constexpr int kWqThreads = 320, kWqStages = 2, kWqRows = 128;
template <int HD>
struct WqCfg {
    static constexpr int kPart = kWqRows * HD;                 // q's high parts, then its low parts
    static constexpr int kGroup = q8_row_group_bytes(HD);      // .. then 2^eq scale_log2 [128], -lse [128]
    static constexpr int kTile = 128 * HD;                     // K codes
    static constexpr int kOffK = kWqStages * kGroup;
    static constexpr int kOffBar = kOffK + kWqStages * kTile;  // k_full, k_empty, q_full, q_empty, s_full, s_empty [2], drain
    static constexpr int kOffMisc = kOffBar + 13 * 8;          // tmem slot, abort
    static constexpr int kOffSum = kOffMisc + 8;               // float [128]
    static constexpr int kDynSmem = kOffSum + 512 + 1024;
    static constexpr uint32_t kTmemCols = 2 * kWqRows;
    static_assert(kGroup % 1024 == 0 && kGroup == 2 * kPart + 1024, "operand alignment");
};

template <int HD>
__global__ void __launch_bounds__(256) weights_rows_kernel(const __grid_constant__ WeightQ8Params p)
{
    using C = WqCfg<HD>;
    ptx::griddep_wait();  // launched with programmatic serialization: the attention's log-sum-exp
    ptx::griddep_launch_dependents();
    const int grp = static_cast<int>(blockIdx.x);
    int lo = 0, hi = p.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.segs[mid].group0 <= grp) lo = mid; else hi = mid;
    }
    const WeightQ8Seg &sg = p.segs[lo];
    const int kvh = (grp - sg.group0) / sg.n_groups, row0 = (grp - sg.group0) % sg.n_groups * kWqRows;
    const int rows = sg.n_q << p.log_group;
    uint8_t *dst = p.groups + static_cast<int64_t>(grp) * C::kGroup;
    float *coef = reinterpret_cast<float *>(dst + 2 * C::kPart);
    constexpr int kPieces = HD / 8;
    // a piece of eight columns a thread (rows do not straddle warps)
    const int e = static_cast<int>(blockIdx.y) * 256 + static_cast<int>(threadIdx.x);
    const int r = e / kPieces, pc = e % kPieces, row = row0 + r;
    const int64_t at = static_cast<int64_t>(sg.q_row0 + (row >> p.log_group)) * p.hq + (kvh << p.log_group) + (row & ((1 << p.log_group) - 1));
    const uint4 v = row < rows ? *reinterpret_cast<const uint4 *>(p.q + at * HD + pc * 8) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t a = bf16x8_absmax(v);
#pragma unroll
    for (int off = kPieces / 2; off >= 1; off >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, off));
    const bool bad = a >= 0x7f80u;
    const int eq = bad ? 0 : q8_exponent(a);
    uint2 vh, vl;
    q8_split(v, pow2i(-eq), 1.f, vh, vl);
    if (bad) vh = make_uint2(kQ8NanWord, kQ8NanWord);
    *reinterpret_cast<uint2 *>(dst + row_chunk<HD>(r, pc >> 1) + (pc & 1) * 8) = vh;
    *reinterpret_cast<uint2 *>(dst + C::kPart + row_chunk<HD>(r, pc >> 1) + (pc & 1) * 8) = vl;
    if (pc == 0) {  // a row past the last adds 2^-inf
        coef[r] = row < rows ? pow2i(eq) * p.scale_log2 : 0.f;
        coef[kWqRows + r] = row < rows ? -p.lse[at] : -INFINITY;
    }
}

template <int HD>
__global__ void __launch_bounds__(kWqThreads, 2)
    weights_q8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ WeightQ8Params p, int split)
{
    using C = WqCfg<HD>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t sbase = ptx::smem_addr(smem), bar0 = sbase + C::kOffBar;
    auto bar = [&](int kind, int i) { return bar0 + 8u * (2 * kind + (i & 1)); };
    enum { kKFull, kKEmpty, kQFull, kQEmpty, kSFull, kSEmpty, kDrain };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::kOffMisc + 4);
    float *s_sum = reinterpret_cast<float *>(smem + C::kOffSum);
    const WaitCtx wctx{abort_flag, p.status};
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(bar(kKFull, i), 1);
            ptx::mbar_init(bar(kKEmpty, i), 1);
            ptx::mbar_init(bar(kQFull, i), 1);
            ptx::mbar_init(bar(kQEmpty, i), 128);
            ptx::mbar_init(bar(kSFull, i), 1);
            ptx::mbar_init(bar(kSEmpty, i), 128);
        }
        ptx::mbar_init(bar(kDrain, 0), 1);
        *abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&tm_k);
    }
    if (warp == 9) {
        ptx::tmem_alloc(ptx::smem_addr(tmem_slot), C::kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    ptx::griddep_wait();  // launched with programmatic serialization: the row groups
    ptx::griddep_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    const int b = static_cast<int>(blockIdx.x) / split, rank = static_cast<int>(blockIdx.x) % split;
    int lo = 0, hi = p.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.segs[mid].tile0 <= b) lo = mid; else hi = mid;
    }
    const WeightQ8Seg &sg = p.segs[lo];
    const int key0 = (b - sg.tile0) * 128, all_units = p.hkv * sg.n_groups;
    // the CTA's units (kv-head u / n_groups, group u % n_groups): unit0 + [0, units), of kv-heads head0 + ..
    const int unit0 = static_cast<int>(static_cast<int64_t>(all_units) * rank / split);
    const int units = static_cast<int>(static_cast<int64_t>(all_units) * (rank + 1) / split) - unit0;
    const int head0 = unit0 / sg.n_groups, group0 = unit0 - head0 * sg.n_groups;
    int issued = 0;  // copies: stages filled (K in the low half, groups in the high)

    if (warp == 8) {
        // ============================================================ copies
        const int slot_key = key0 + (lane << p.log_ps);
        int row0 = p.oob_row, step = 0;  // the lane's box: a page of kv-head 0, and the way to the next head
        if (lane < (128 >> p.log_ps) && slot_key < sg.n_keys) {
            const int page = p.page_table[sg.table_row + (slot_key >> p.log_ps)];
            if (page >= 0 && page < p.num_pages) {
                row0 = (p.layer * p.num_pages + page) * p.hkv << p.log_ps;
                step = p.ps;
            } else {
                atomicCAS(p.status, 0, kStatusBadPage);
            }
        }
        bool ok = true;
        for (int u = 0, h = 0, g = group0; u < units && ok; ++u) {
            if (u == 0 || g == 0) {
                if (h >= kWqStages && !(ok = wait_spin(bar(kKEmpty, h), ((h / kWqStages) - 1) & 1, wctx))) break;
                if (lane == 0) ptx::mbar_arrive_expect_tx(bar(kKFull, h), C::kTile);
                __syncwarp();
                if (lane < (128 >> p.log_ps))
                    ptx::tma_load_2d(sbase + C::kOffK + (h & 1) * C::kTile + (lane << p.log_ps) * HD, &tm_k, 0, row0 + (head0 + h) * step, bar(kKFull, h));
                __syncwarp();
                issued += 1;
            }
            if (u >= kWqStages && !(ok = wait_spin(bar(kQEmpty, u), ((u / kWqStages) - 1) & 1, wctx))) break;
            if (lane == 0) {
                ptx::mbar_arrive_expect_tx(bar(kQFull, u), C::kGroup);
                ptx::bulk_load(sbase + (u & 1) * C::kGroup, p.groups + static_cast<int64_t>(sg.group0 + unit0 + u) * C::kGroup, C::kGroup, bar(kQFull, u));
            }
            __syncwarp();
            issued += 1 << 16;
            if (++g == sg.n_groups) {
                g = 0;
                ++h;
            }
        }
        // after an abort, copies may still be in flight: bounded wait for the last ones issued
        if (lane == 0 && *abort_flag) {
            const uint64_t start = ptx::globaltimer();
            for (int ring = 0; ring < 2; ++ring) {
                const int n = ring ? issued >> 16 : issued & 0xffff;
                for (int i = max(0, n - kWqStages); i < n; ++i)
                    while (!ptx::mbar_try_wait(bar(ring ? kQFull : kKFull, i), (i / kWqStages) & 1) && ptx::globaltimer() - start < 4000000ull) {
                    }
            }
        }
    } else if (warp == 9) {
        // ============================================================ MMAs
        constexpr uint32_t kId = idesc_e4m3_f32(128, kWqRows, false);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint64_t k_desc = row_desc<HD>(sbase + C::kOffK, 16), q_desc = row_desc<HD>(sbase, 16);
        bool ok = true;
        for (int u = 0, h = 0, g = group0; u < units; ++u) {
            if ((u == 0 || g == 0) && !(ok = wait_spin(bar(kKFull, h), (h / kWqStages) & 1, wctx))) break;
            if (!(ok = wait_spin(bar(kQFull, u), (u / kWqStages) & 1, wctx))) break;
            if (u >= 2 && !(ok = wait_spin(bar(kSEmpty, u), ((u / 2) - 1) & 1, wctx))) break;
            ptx::tc_fence_after();
            const uint64_t kd = k_desc + (h & 1) * (C::kTile >> 4), qd = q_desc + (u & 1) * (C::kGroup >> 4);
#pragma unroll
            for (int kk = 0; kk < 2 * (HD / 32); ++kk) {
                const int col = kk % (HD / 32) * 32, part = kk / (HD / 32);
                mma_e4m3_warp(tm + kWqRows * (u & 1), kd + (col >> 4), qd + ((part * C::kPart + col) >> 4), kId, kk > 0 ? 1u : 0u);
            }
            mma_commit_warp(bar(kSFull, u));
            if (++g == sg.n_groups) {
                mma_commit_warp(bar(kKEmpty, h));
                g = 0;
                ++h;
            }
        }
        mma_commit_warp(bar(kDrain, 0));
        if (lane == 0) {
            const uint64_t start = ptx::globaltimer();
            while (!ptx::mbar_try_wait(bar(kDrain, 0), 0) && ptx::globaltimer() - start < 4000000ull) {
            }
        }
        __syncwarp();
    } else {
        // ============================================================ sums (thread = key)
        const int side = warp >> 2, t = threadIdx.x & 127, key = key0 + t;
        const uint32_t taddr = tmem + kWqRows * side + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const int qpos0 = sg.n_keys - sg.n_q;
        int head = -1;  // exponents' index of kv-head 0
        if (key < sg.n_keys) {
            const int page = p.page_table[sg.table_row + (key >> p.log_ps)];
            if (page >= 0 && page < p.num_pages) head = (p.layer * p.num_pages + page) * p.hkv;
        }
        float sum = 0.f;
        bool ok = true;
        for (int u = side; u < units && ok; u += 2) {
            const int h = (unit0 + u) / sg.n_groups, row0 = (unit0 + u - h * sg.n_groups) * kWqRows;
            const float ks = head >= 0 ? pow2i(p.exps[2 * (head + h)]) : 0.f;
            const float2 ks2 = make_float2(ks, ks);
            const float *coef = reinterpret_cast<const float *>(smem + side * C::kGroup + 2 * C::kPart);
            // does the group's first row see all 128 keys?
            const bool all = key0 + 127 <= qpos0 + (row0 >> p.log_group);
            if (!(ok = wait_spin(bar(kSFull, u), (u / 2) & 1, wctx))) break;
            ptx::tc_fence_after();
            float2 acc = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int c0 = 0; c0 < kWqRows; c0 += 16) {
                float s[16];
                ptx::tmem_ld_n<16>(taddr + c0, s);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float4 a = *reinterpret_cast<const float4 *>(coef + c0 + r), l = *reinterpret_cast<const float4 *>(coef + kWqRows + c0 + r);
                    const float2 x = fma2(make_float2(s[r], s[r + 1]), mul2(ks2, make_float2(a.x, a.y)), make_float2(l.x, l.y));
                    const float2 y = fma2(make_float2(s[r + 2], s[r + 3]), mul2(ks2, make_float2(a.z, a.w)), make_float2(l.z, l.w));
                    s[r] = ex2(x.x);
                    s[r + 1] = ex2(x.y);
                    s[r + 2] = ex2(y.x);
                    s[r + 3] = ex2(y.y);
                }
                if (!all) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (key > qpos0 + ((row0 + c0 + r) >> p.log_group) || row0 + c0 + r >= sg.n_q << p.log_group) s[r] = 0.f;
                }
#pragma unroll
                for (int r = 0; r < 16; r += 2) acc = add2(acc, make_float2(s[r], s[r + 1]));
            }
            sum += acc.x + acc.y;
            ptx::tc_fence_before();
            ptx::mbar_arrive(bar(kSEmpty, u));
            ptx::mbar_arrive(bar(kQEmpty, u));
        }
        if (side == 1) s_sum[t] = sum;
        ptx::bar_sync(1, 256);
        if (side == 0) s_sum[t] += sum;
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (split > 1) ptx::cluster_sync();  // every CTA's sums are in its shared memory
    if (rank == 0 && threadIdx.x < 128) {
        const int t = static_cast<int>(threadIdx.x);
        float sum = s_sum[t];
        for (int r = 1; r < split; ++r) sum += ptx::ld_cluster_f32(ptx::smem_addr(s_sum + t), r);
        if (key0 + t < sg.n_keys) p.weights[static_cast<int64_t>(sg.row) * p.weights_stride + key0 + t] += sum;
    }
    if (split > 1) ptx::cluster_sync();  // .. and has been read
    if (warp == 9) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, C::kTmemCols);
    }
}

template <int HD>
cudaError_t launch_weights_q8_t(const CUtensorMap &tm_k, const WeightQ8Params &p, int groups, int tiles, int split, cudaStream_t st)
{
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = set_dyn_smem_once(weights_q8_kernel<HD>, WqCfg<HD>::kDynSmem, configured);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(groups), kWqRows * (HD / 8) / 256);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if ((e = cudaLaunchKernelEx(&cfg, weights_rows_kernel<HD>, p)) != cudaSuccess) return e;
    cudaLaunchAttribute both[2] = {attr[0], {}};
    both[1].id = cudaLaunchAttributeClusterDimension;
    both[1].val.clusterDim.x = static_cast<unsigned>(split);
    both[1].val.clusterDim.y = both[1].val.clusterDim.z = 1;
    cfg.attrs = both;
    cfg.numAttrs = split > 1 ? 2 : 1;
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * split));
    cfg.blockDim = dim3(kWqThreads);
    cfg.dynamicSmemBytes = WqCfg<HD>::kDynSmem;
    return cudaLaunchKernelEx(&cfg, weights_q8_kernel<HD>, tm_k, p, split);
}

}  // namespace

cudaError_t launch_weights_q8(int head_dim, const CUtensorMap &tm_k, const WeightQ8Params &p, int groups, int tiles, int split, cudaStream_t st)
{
    return head_dim == 128 ? launch_weights_q8_t<128>(tm_k, p, groups, tiles, split, st) : launch_weights_q8_t<64>(tm_k, p, groups, tiles, split, st);
}

cudaError_t launch_weights_kept(const WeightParams &p, int max_keys, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((max_keys + kKeptKeys - 1) / kKeptKeys), static_cast<unsigned>(p.n));
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
