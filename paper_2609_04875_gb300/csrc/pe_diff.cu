// Differential attention over the paged cache.  Heads 2i and 2i + 1 of Q are the two maps of head i, which reads kv-heads
// 2j and 2j + 1 (j = i / group): their keys, one head a map, and side by side their values, of width 2d.
//     A_m = softmax(scale q_m K_{2j+m}^T),  O = (A_0 - lambda_i A_1) [V_2j | V_2j+1],
//     out = gain O / sqrt(mean(O^2) + eps)   (or O, without a gain)
//
// One pass over keys and values for both maps: the M side of the products holds 64 rows of each map, the maps of the same
// queries.  Per tile of 64 keys
//     S [128 x 128]  = Q [128 x d] . [K_2j ; K_2j+1]^T        (a row uses the 64 columns of its own map)
//     O [128 x 2d]  += P [128 x 64] . [V_2j | V_2j+1]         (A = P from TMEM, in two parts: two_parts)
// so half of S is not used, and where there are few rows most of M is not; both cost less than the keys' way from memory
// (64 keys, d = 128: 64 KB, 2800 cycles of an SM's share of HBM; its MMAs 1536).
//
// Work is cut into equal stretches of tiles, a CTA each (pe_internal.h); every piece writes O / l and its log-sum-exp, and
// the merge joins a row's pieces of both maps, subtracts and norms.  Where keys are few a cluster takes a whole unit and joins
// its parts through shared memory (plan_diff, pe_host.cu).
//
// Bound by HBM, and by what does not shrink with the bytes.  16 agents of 2k to 8k keys, 32 / 8 heads, d = 128: 60 us (5.6
// TB/s); 64 query heads on 120k keys 82 us (6.0); 8 agents of 32k keys and 16 queries (64 rows) 180 us (6.0).  Of the 82: first
// scores 3.6 us after the launch before ends; the SMs finish over 16 us, for some groups of eight take their bytes 13 % slower
// than others; 1 us to the merge and 4 in it.  (Equal shares of bytes; shares taken as the SMs come free would need pieces
// short enough that the merge, or the pieces' own starts, cost what they save.)
#include <algorithm>

#include "dev_common.cuh"
#include "diff.cuh"
#include "q8.cuh"

namespace pe {

namespace {

constexpr int kDiffThreads = 288;               // warps 0-3 softmax, 4-7 producers, 8 MMA

template <int HD>
struct DiffCfg {
    static constexpr int kRegions = HD / 64;                  // 128-byte swizzle atoms along d
    static constexpr int kStages = HD == 128 ? 3 : 6;
    static constexpr int kQBytes = 128 * HD * 2;
    static constexpr int kKBytes = 2 * DiffFew::kKeys * HD * 2;    // both maps' keys of a tile
    static constexpr int kKRegion = 2 * DiffFew::kKeys * 128;
    static constexpr int kVBytes = DiffFew::kKeys * 2 * HD * 2;
    static constexpr int kVRegion = DiffFew::kKeys * 128;
    static constexpr int kOffK = kQBytes;
    static constexpr int kOffV = kOffK + kStages * kKBytes;
    static constexpr int kOffBar = kOffV + kStages * kVBytes;
    // k_full, k_empty, v_full, v_empty [stages]; q_full, edge; s_full, p_full, o_done [2]
    static constexpr int kNumBars = 4 * kStages + 2 + 6;
    static constexpr int kOffMisc = kOffBar + kNumBars * 8;   // tmem slot, abort flag, keys not finite [2][2]
    static constexpr int kOffLse = kOffMisc + 24;             // float [128]: whole units
    static constexpr int kRowFloats = 2 * HD + 4;             // of a row's O there, in the stages' memory: 16 bytes past a multiple of 128
    static constexpr int kDynSmem = kOffLse + 128 * 4 + 1024;
    static constexpr int kTmemO = 256;                        // S at 0 and 128, P over S
    static constexpr uint32_t kTmemCols = 512;
    static_assert(kDynSmem <= 232448, "shared memory budget");
    static_assert(128 * kRowFloats * 4 <= kOffBar - kOffK, "rows of a whole unit");
};

// One row of a head, joined from its pieces by a warp: lane t has the columns 4t .. + 3 of every 128.
template <int HD>
struct DiffRow {
    static constexpr int V4 = 2 * HD / 128;  // float4 a lane
    float m[2], l[2];
    float4 o[2][V4];
    __device__ __forceinline__ DiffRow()
    {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            m[x] = -INFINITY;
            l[x] = 0.f;
#pragma unroll
            for (int v = 0; v < V4; ++v) o[x][v] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    // A piece of map x: O / l and log-sum-exp.
    __device__ __forceinline__ void add(int x, float lse, const float4 (&z)[V4])
    {
        if (lse == -INFINITY) return;  // (no key seen: its row may hold anything)
        const float mn = fmaxf(m[x], lse);
        const float f = m[x] == -INFINITY ? 0.f : ex2(m[x] - mn), g = ex2(lse - mn);  // (NaN where lse is)
        m[x] = mn;
        l[x] = l[x] * f + g;
#pragma unroll
        for (int v = 0; v < V4; ++v)
            o[x][v] = make_float4(o[x][v].x * f + z[v].x * g, o[x][v].y * f + z[v].y * g, o[x][v].z * f + z[v].z * g, o[x][v].w * f + z[v].w * g);
    }
    // The difference of the maps, the norm, and the output row.
    __device__ __forceinline__ void finish(const DiffParams &p, int64_t q_row, int head, int lane)
    {
        const float g0 = l[0] == 0.f ? 0.f : 1.f / l[0], g1 = l[1] == 0.f ? 0.f : -__ldg(p.lambda + head) / l[1];
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < V4; ++v) {
            const float4 a = o[0][v], b = o[1][v];
            o[0][v] = make_float4(g0 * a.x + g1 * b.x, g0 * a.y + g1 * b.y, g0 * a.z + g1 * b.z, g0 * a.w + g1 * b.w);
            sum += o[0][v].x * o[0][v].x + o[0][v].y * o[0][v].y + o[0][v].z * o[0][v].z + o[0][v].w * o[0][v].w;
        }
        if (p.gain) {
#pragma unroll
            for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
            const float f = 1.f / sqrtf(sum / (2 * HD) + p.eps);
#pragma unroll
            for (int v = 0; v < V4; ++v) {
                const float *g = p.gain + v * 128 + lane * 4;  // (a vector of any alignment)
                o[0][v] = make_float4(o[0][v].x * f * __ldg(g), o[0][v].y * f * __ldg(g + 1), o[0][v].z * f * __ldg(g + 2), o[0][v].w * f * __ldg(g + 3));
            }
        }
        uint2 *dst = reinterpret_cast<uint2 *>(p.out + (q_row * (p.hq / 2) + head) * 2 * HD);
#pragma unroll
        for (int v = 0; v < V4; ++v) dst[v * 32 + lane] = make_uint2(pack_bf16(o[0][v].x, o[0][v].y), pack_bf16(o[0][v].z, o[0][v].w));
    }
};

// ld_cluster_f32 (ptx.cuh), four
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr, uint32_t rank)
{
    float4 v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr), "r"(rank)
                 : "memory");
    return v;
}

template <int HD>
__global__ void __launch_bounds__(kDiffThreads, 1)
    diff_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const __grid_constant__ DiffParams p)
{
    using C = DiffCfg<HD>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_addr(smem_raw);
    const uint32_t sbase = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (sbase - raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ranks = max(1, p.whole), rank = static_cast<int>(blockIdx.x) % ranks, taker = static_cast<int>(blockIdx.x) / ranks;

    const uint32_t b_k_full = sbase + C::kOffBar;
    const uint32_t b_k_empty = b_k_full + 8 * C::kStages;
    const uint32_t b_v_full = b_k_empty + 8 * C::kStages;
    const uint32_t b_v_empty = b_v_full + 8 * C::kStages;
    const uint32_t b_q_full = b_v_empty + 8 * C::kStages;
    const uint32_t b_edge = b_q_full + 8;      // the softmax threads among themselves
    const uint32_t b_s_full = b_edge + 8;      // [2]
    const uint32_t b_p_full = b_s_full + 16;   // [2]
    const uint32_t b_o_done = b_p_full + 16;   // [2]
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::kOffMisc + 4);
    uint32_t *odd_keys = reinterpret_cast<uint32_t *>(smem + C::kOffMisc + 8);  // [2][2]
    float *s_rows = reinterpret_cast<float *>(smem + C::kOffK), *s_lse = reinterpret_cast<float *>(smem + C::kOffLse);
    const WaitCtx wctx{abort_flag, p.status};

    if (threadIdx.x < 128) s_lse[threadIdx.x] = -INFINITY;  // (a CTA may have no tile of its cluster's unit)
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            ptx::mbar_init(b_k_full + 8 * s, 2);
            ptx::mbar_init(b_k_empty + 8 * s, 1);
            ptx::mbar_init(b_v_full + 8 * s, 2);
            ptx::mbar_init(b_v_empty + 8 * s, 1);
        }
        ptx::mbar_init(b_q_full, 128);
        ptx::mbar_init(b_edge, 128);
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(b_s_full + 8 * s, 1);
            ptx::mbar_init(b_p_full + 8 * s, 128);
            ptx::mbar_init(b_o_done + 8 * s, 1);
        }
        *abort_flag = 0;
        for (int k = 0; k < 4; ++k) odd_keys[k] = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
        ptx::prefetch_tensormap(&tm_k);
        ptx::prefetch_tensormap(&tm_v);
    }
    if (warp == 8) {
        ptx::tmem_alloc(ptx::smem_addr(tmem_slot), C::kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // everything before this overlapped the kernel before; the merge's blocks may come in from here on
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();

    DiffWalk<DiffFew> w(p, taker, rank, ranks);
    int i = 0;  // tiles of the pieces before
    if (warp >= 4 && warp < 8) {
        // =================================================== producers: K of a map, or V of a kv-head
        const bool is_v = warp >= 6;
        const int head = warp & 1;
        const CUtensorMap *map = is_v ? &tm_v : &tm_k;
        const uint32_t b_full = is_v ? b_v_full : b_k_full, b_empty = is_v ? b_v_empty : b_k_empty;
        const int rows = min(p.ps, DiffFew::kKeys);                 // of a box
        const int n_ops = DiffFew::kKeys / rows * C::kRegions;      // <= 16
        const int op_page = lane / C::kRegions, op_reg = lane % C::kRegions;
        const bool on = lane < n_ops;
        const uint32_t base = sbase + (is_v ? C::kOffV + (head * C::kRegions + op_reg) * C::kVRegion
                                            : C::kOffK + op_reg * C::kKRegion + head * DiffFew::kKeys * 128) + op_page * rows * 128;
        bool ok = true;
        while (ok && w.next()) {
            const DiffSeq &sq = p.seqs[w.si];
            const int kvh = 2 * w.pair + head;
            auto row_of = [&](int k) -> int {  // of the pool, of this lane's box of tile k
                const int key = (w.t0 + k) * DiffFew::kKeys + op_page * rows, lp = key >> p.log_ps;
                const int page = on && lp < sq.n_pages ? p.page_table[sq.table_row + lp] : -1;
                return page >= 0 && page < p.num_pages ? (((p.layer * p.num_pages + page) * p.hkv + kvh) << p.log_ps) + (key & (p.ps - 1))
                                                       : p.oob_row;
            };
            int y = row_of(0);
            for (int k = 0; k < w.n; ++k, ++i) {
                const int next = k + 1 < w.n ? row_of(k + 1) : 0, s = i % C::kStages;
                if (i >= C::kStages && !wait_bar_warp(b_empty + 8 * s, ((i / C::kStages) - 1) & 1, wctx)) { ok = false; break; }
                if (lane == 0) ptx::mbar_arrive_expect_tx(b_full + 8 * s, DiffFew::kKeys * HD * 2);
                __syncwarp();
                if (on) ptx::tma_load_2d(base + s * (is_v ? C::kVBytes : C::kKBytes), map, op_reg * 64, y, b_full + 8 * s);
                y = next;
            }
        }
        __syncwarp();
        if (*abort_flag && lane == 0) {  // a bounded chance for copies in flight to land
            const uint64_t g0 = ptx::globaltimer();
            for (int k = max(0, i - C::kStages); k < i; ++k)
                while (!ptx::mbar_try_wait(b_full + 8 * (k % C::kStages), (k / C::kStages) & 1) && ptx::globaltimer() - g0 < 4000000ull) {}
        }
    } else if (warp == 8) {
        // =================================================== MMA (the converged warp; one elected lane issues)
        constexpr uint32_t kIdescS = ptx::idesc_bf16_f32(128, 2 * DiffFew::kKeys, false);
        constexpr uint32_t kIdescO = ptx::idesc_bf16_f32(128, 2 * HD, true);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint64_t q_desc = ptx::smem_desc_sw128(sbase, 16, 1024);
        const uint64_t k_desc = ptx::smem_desc_sw128(sbase + C::kOffK, 16, 1024);
        const uint64_t v_desc = ptx::smem_desc_sw128(sbase + C::kOffV, C::kVRegion, 1024);
        auto full = [&](uint32_t bar, int j) { return wait_bar_warp(bar + 8 * (j % C::kStages), (j / C::kStages) & 1, wctx); };
        auto issue_s = [&](int j) {
            if (!full(b_k_full, j)) return false;
            ptx::tc_fence_after();
            const uint64_t kd = k_desc + (j % C::kStages) * (C::kKBytes >> 4);
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk)
                mma_bf16_warp(tm + 128 * (j & 1), q_desc + (((kk >> 2) * (128 * 128) + (kk & 3) * 32) >> 4),
                              kd + (((kk >> 2) * C::kKRegion + (kk & 3) * 32) >> 4), kIdescS, kk > 0 ? 1u : 0u);
            mma_commit_warp(b_s_full + 8 * (j & 1));
            mma_commit_warp(b_k_empty + 8 * (j % C::kStages));
            return true;
        };
        bool ok = true;
        for (int piece = 0; ok && w.next(); ++piece) {
            const int n = __shfl_sync(0xffffffffu, w.n, 0);
            if (!wait_bar_warp(b_q_full, piece & 1, wctx)) break;
            ok = issue_s(i) && (n < 2 || issue_s(i + 1));
            for (int k = 0; ok && k < n; ++k, ++i) {
                if (!full(b_v_full, i) || !wait_bar_warp(b_p_full + 8 * (i & 1), (i >> 1) & 1, wctx)) { ok = false; break; }
                ptx::tc_fence_after();
                const uint64_t vd = v_desc + (i % C::kStages) * (C::kVBytes >> 4);
#pragma unroll
                for (int kk = 0; kk < 2 * DiffFew::kKeys / 16; ++kk)  // the weights' upper parts, then their lower ones
                    mma_bf16_ts_warp(tm + C::kTmemO, tm + 128 * (i & 1) + kk * 8, vd + ((kk & 3) * 16 * 128 >> 4), kIdescO,
                                     (k > 0 || kk > 0) ? 1u : 0u);
                mma_commit_warp(b_o_done + 8 * (i & 1));
                mma_commit_warp(b_v_empty + 8 * (i % C::kStages));
                if (k + 2 < n) ok = issue_s(i + 2);  // (P(i), over S(i), is read by then)
            }
        }
    } else {
        // =================================================== softmax: thread r owns row r (TMEM lane r)
        const int row = threadIdx.x, m = row / DiffFew::kRows;
        const uint32_t lane_off = static_cast<uint32_t>(warp * 32) << 16;
        const float2 sl2 = make_float2(p.scale_log2, p.scale_log2);
        bool ok = true;
        int met = 0;
        auto meet = [&]() {  // of all softmax threads; bounded, as every wait
            ptx::mbar_arrive(b_edge);
            return wait_bar_warp(b_edge, met++ & 1, wctx);
        };
        while (ok && w.next()) {
            const DiffSeq &sq = p.seqs[w.si];
            const int r = w.block * DiffFew::kRows + (row & (DiffFew::kRows - 1));  // packed row of its map
            const int qi = r / p.group, head = 2 * (w.pair * p.group + r - qi * p.group) + m;
            const bool valid = qi < sq.n_q, any = __any_sync(0xffffffffu, valid);
            const int pos = sq.n_keys - sq.n_q + qi;
            const int pos_first = sq.n_keys - sq.n_q + w.block * DiffFew::kRows / p.group;
            // Q's row into shared memory (the S products of the piece before are done), 16-byte chunks swizzled by row & 7
            if (valid) {
                const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (static_cast<int64_t>(sq.q_row0 + qi) * p.hq + head) * HD);
#pragma unroll
                for (int c = 0; c < HD / 8; ++c) {
                    const uint4 v = __ldg(src + c);
                    *reinterpret_cast<uint4 *>(smem + (c >> 3) * (128 * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = v;
                }
            }
            ptx::fence_proxy_async_smem();
            ptx::mbar_arrive(b_q_full);
            float m_ref = -INFINITY, l = 0.f;
            for (int k = 0; k < w.n; ++k, ++i) {
                const int kbase = (w.t0 + k) * DiffFew::kKeys;
                const uint32_t tS = tmem + 128 * (i & 1) + lane_off;
                const bool edge = kbase + DiffFew::kKeys - 1 > pos_first;  // a row of the block does not see some key of the tile
                if (edge) {
                    // V of keys that some row does not see: 0 times an infinity or NaN would reach that row.  Such keys' V
                    // become 0, and rows that see them NaN.
                    if (!wait_bar_warp(b_v_full + 8 * (i % C::kStages), (i / C::kStages) & 1, wctx)) { ok = false; break; }
                    const int key = row & 63;
                    uint8_t *v = smem + C::kOffV + (i % C::kStages) * C::kVBytes + (row >> 6) * C::kRegions * C::kVRegion + key * 128;
                    uint32_t odd = 0;
#pragma unroll
                    for (int c = 0; c < HD / 8; ++c)
                        odd = max(odd, bf16x8_absmax(*reinterpret_cast<const uint4 *>(v + (c >> 3) * C::kVRegion + (((c & 7) ^ (key & 7)) << 4))));
                    const bool is_odd = odd >= 0x7f80u;
                    // Two sets of words in turn (a tile has one meeting or three, so their parity tells it from the next):
                    // a thread that is ahead may mark the next tile's keys before all have read this one's, but not those
                    // of the tile after, which is past the next one's meeting.
                    volatile uint32_t *odd_set = odd_keys + 2 * (met & 1);
                    if (is_odd) atomicOr(const_cast<uint32_t *>(odd_set) + (key >> 5), 1u << (key & 31));
                    if (!meet()) { ok = false; break; }
                    const uint64_t odd_mask = odd_set[0] | static_cast<uint64_t>(odd_set[1]) << 32;
                    if (odd_mask) {
                        if (is_odd)
                            for (int c = 0; c < HD / 8; ++c)
                                *reinterpret_cast<uint4 *>(v + (c >> 3) * C::kVRegion + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        ptx::fence_proxy_async_smem();
                        const int sees = pos - kbase + 1;  // keys of the tile
                        if (sees > 0 && (odd_mask & (sees >= 64 ? ~0ull : (1ull << sees) - 1))) l = NAN;
                        if (!meet()) { ok = false; break; }  // the mask is read
                        if (row < 2) odd_set[row] = 0;
                        if (!meet()) { ok = false; break; }  // and cleared
                    }
                }
                if (!wait_bar_warp(b_s_full + 8 * (i & 1), (i >> 1) & 1, wctx)) { ok = false; break; }
                ptx::tc_fence_after();
                if (any) {
                    float s[DiffFew::kKeys];
                    {
                        float (&s0)[32] = *reinterpret_cast<float (*)[32]>(&s[0]);
                        float (&s1)[32] = *reinterpret_cast<float (*)[32]>(&s[32]);
                        ptx::tmem_ld32(tS + 64 * m, s0);
                        ptx::tmem_ld32(tS + 64 * m + 32, s1);
                        ptx::tmem_wait_ld();
                    }
                    if (edge) {
#pragma unroll
                        for (int c = 0; c < DiffFew::kKeys; ++c)
                            if (kbase + c > pos) s[c] = -INFINITY;
                    }
                    // weights against the row's reference, which moves only when a tile's sum passes 2^64 (pe_attn.cu)
                    auto exp_tile = [&](float ref) -> float {
                        const float2 nref = make_float2(-ref, -ref);
                        float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                        for (int ch = 0; ch < DiffFew::kKeys / 32; ++ch) {
                            uint32_t pk[16], lo[16];
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const int c = ch * 32 + 2 * x;
                                const float2 y = fma2(make_float2(s[c], s[c + 1]), sl2, nref);
                                const float2 e = make_float2(ex2(y.x), ex2(y.y));
                                pk[x] = two_parts(e, lo[x]);
                                acc[x & 3] = add2(acc[x & 3], e);
                            }
                            tmem_st16(tS + ch * 16, pk);
                            tmem_st16(tS + DiffFew::kKeys / 2 + ch * 16, lo);
                        }
                        const float2 a = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
                        return a.x + a.y;
                    };
                    float rs = 0.f;
                    bool need = valid && m_ref == -INFINITY;
                    if (!__all_sync(0xffffffffu, need)) {
                        rs = exp_tile(m_ref == -INFINITY ? 0.f : m_ref);
                        need = need || (valid && !(rs <= kDiffSumLimit));
                    }
                    if (__any_sync(0xffffffffu, need)) {
                        float mx[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) mx[x] = max3(s[x], s[4 + x], s[8 + x]);
#pragma unroll
                        for (int c = 12; c < 60; c += 8)
#pragma unroll
                            for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], s[c + x], s[c + 4 + x]);
                        const float mt = fmaxf(max3(mx[0], mx[1], mx[2]), max3(mx[3], fmaxf(s[60], s[61]), fmaxf(s[62], s[63])));
                        const float m_new = fmaxf(m_ref, mt * sl2.x);
                        if (k > 0 && __any_sync(0xffffffffu, need && m_ref != -INFINITY)) {
                            // O holds P V of the tiles before once the last of them is done
                            if (!wait_bar_warp(b_o_done + 8 * ((i - 1) & 1), ((i - 1) >> 1) & 1, wctx)) { ok = false; break; }
                            ptx::tc_fence_after();
                            const float alpha = need && m_ref != -INFINITY ? ex2(m_ref - m_new) : 1.f;
#pragma unroll 1
                            for (int ch = 0; ch < 2 * HD / 16; ++ch) {
                                uint32_t o[16];
                                tmem_ld16(tmem + C::kTmemO + lane_off + ch * 16, o);
                                ptx::tmem_wait_ld();
#pragma unroll
                                for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                                tmem_st16(tmem + C::kTmemO + lane_off + ch * 16, o);
                            }
                            if (need) l *= alpha;
                        }
                        if (need) m_ref = m_new;
                        ptx::tmem_wait_st();
                        rs = exp_tile(m_ref == -INFINITY ? 0.f : m_ref);
                    }
                    l += rs;
                    ptx::tmem_wait_st();
                }
                ptx::tc_fence_before();
                ptx::mbar_arrive(b_p_full + 8 * (i & 1));
            }
            if (!ok || !wait_bar_warp(b_o_done + 8 * ((i - 1) & 1), ((i - 1) >> 1) & 1, wctx)) break;
            ptx::tc_fence_after();
            if (any) {
                const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one)
                const int64_t at = static_cast<int64_t>(w.slot) * 128 + row;
                float4 *dst = reinterpret_cast<float4 *>(p.whole ? s_rows + row * C::kRowFloats : p.part + at * 2 * HD);
#pragma unroll 1
                for (int ch = 0; ch < 2 * HD / 32; ++ch) {
                    float o[32];
                    ptx::tmem_ld32(tmem + C::kTmemO + lane_off + ch * 32, o);
                    ptx::tmem_wait_ld();
                    if (valid && l != 0.f)
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            dst[ch * 8 + x] = make_float4(o[4 * x] * inv, o[4 * x + 1] * inv, o[4 * x + 2] * inv, o[4 * x + 3] * inv);
                }
                if (valid) (p.whole ? s_lse[row] : p.part_lse[at]) = l == 0.f ? -INFINITY : m_ref + __log2f(l);
            }
            ptx::tc_fence_before();
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, C::kTmemCols);
    }
    if (p.whole) {  // the cluster's parts of its unit, a warp a row
        __syncwarp();
        ptx::cluster_sync();
        DiffWalk<DiffFew> unit(p, taker);
        if (unit.next()) {
            const DiffSeq &sq = p.seqs[unit.si];
            const int r0 = unit.block * DiffFew::kRows, rows = min(DiffFew::kRows, sq.n_q * p.group - r0);
            for (int x = rank + warp * ranks; x < rows; x += ranks * (kDiffThreads / 32)) {
                const int q = (r0 + x) / p.group, head = unit.pair * p.group + r0 + x - q * p.group;
                DiffRow<HD> a;
#pragma unroll 2
                for (int c = 0; c < ranks; ++c) {
                    float lse[2];
                    float4 z[2][2 * HD / 128];
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        lse[m] = ptx::ld_cluster_f32(ptx::smem_addr(s_lse + m * DiffFew::kRows + x), c);
#pragma unroll
                        for (int v = 0; v < 2 * HD / 128; ++v)
                            z[m][v] = ld_cluster_f32x4(ptx::smem_addr(s_rows + (m * DiffFew::kRows + x) * C::kRowFloats + v * 128 + lane * 4), c);
                    }
#pragma unroll
                    for (int m = 0; m < 2; ++m) a.add(m, lse[m], z[m]);
                }
                a.finish(p, sq.q_row0 + q, head, lane);
            }
        }
        __syncwarp();
        ptx::cluster_sync();  // the others have read this CTA's rows
    }
}

constexpr int kMergeWarps = 8, kMergeBatch = 4;  // warps of a row's columns; pieces that a group of lanes has in flight

// A block per output row and head, a warp per eighth of its columns (SETS of eight warps), in each warp groups of lanes with
// every fourth (d = 64: eighth) of the set's pieces.  A round of loads takes about a microsecond, so that pieces are taken
// 16 (d = 64: 32) a set at a time: 39 of 32 rows and heads, 9 us with one set.
// With one set it has registers and shared memory enough to be resident, waiting, while the attention still runs.
template <int HD, int SETS>
__global__ void __launch_bounds__(32 * kMergeWarps * SETS, SETS == 1 ? 4 : 1) diff_combine_kernel(const __grid_constant__ DiffParams p)
{
    constexpr int kLanes = 2 * HD / kMergeWarps / 4;  // of a group: a float4 each
    constexpr int kGroups = 32 / kLanes;
    __shared__ float s_sum[kMergeWarps];
    __shared__ float s_m[SETS][2], s_l[SETS][2];
    __shared__ float4 s_o[SETS > 1 ? SETS : 1][SETS > 1 ? 2 * HD / 2 : 1];  // [set][map, column]
    const int set = threadIdx.x / (32 * kMergeWarps), warp = (threadIdx.x >> 5) % kMergeWarps, lane = threadIdx.x & 31;
    const int col = warp * kLanes + lane % kLanes;    // in float4
    int lo = 0, hi = p.n_seqs - 1;
    const int id = static_cast<int>(blockIdx.x);
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.seqs[mid].out0 <= id) lo = mid; else hi = mid - 1;
    }
    const DiffSeq &sq = p.seqs[lo];
    const int heads = p.hq / 2, local = id - sq.out0, qi = local / heads, head = local - qi * heads;
    const int pair = head / p.group, r = qi * p.group + head - pair * p.group;
    const int u = sq.unit0 + pair * sq.n_blocks + r / DiffFew::kRows, row = r % DiffFew::kRows;
    const int c0 = diff_first_taker(p, u), c1 = diff_last_taker(p, u);
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float4 o[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int cb = c0 + set * kMergeBatch * kGroups + lane / kLanes; cb <= c1; cb += SETS * kMergeBatch * kGroups) {
        float lse[kMergeBatch][2];
        float4 y[kMergeBatch][2];
#pragma unroll
        for (int b = 0; b < kMergeBatch; ++b) {
            const int c = min(cb + b * kGroups, c1);
            const int64_t at = static_cast<int64_t>(u + c) * DiffFew::kSlotRows + row;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                lse[b][x] = __ldcg(p.part_lse + at + x * DiffFew::kRows);
                y[b][x] = __ldcg(reinterpret_cast<const float4 *>(p.part + (at + x * DiffFew::kRows) * 2 * HD) + col);
            }
        }
#pragma unroll
        for (int b = 0; b < kMergeBatch; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (cb + b * kGroups > c1 || lse[b][x] == -INFINITY) continue;  // (no key seen: its row may hold anything)
                const float mn = fmaxf(m[x], lse[b][x]);
                const float f = m[x] == -INFINITY ? 0.f : ex2(m[x] - mn), g = ex2(lse[b][x] - mn);  // (NaN where lse is)
                const float4 z = y[b][x];
                m[x] = mn;
                l[x] = l[x] * f + g;
                o[x] = make_float4(o[x].x * f + z.x * g, o[x].y * f + z.y * g, o[x].z * f + z.z * g, o[x].w * f + z.w * g);
            }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        float mx = m[x];
#pragma unroll
        for (int k = kLanes; k < 32; k <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, k));
        const float f = l[x] == 0.f ? 0.f : ex2(m[x] - mx);
        m[x] = mx;
        l[x] *= f;
        o[x] = make_float4(o[x].x * f, o[x].y * f, o[x].z * f, o[x].w * f);
#pragma unroll
        for (int k = kLanes; k < 32; k <<= 1) {
            l[x] += __shfl_xor_sync(0xffffffffu, l[x], k);
            o[x].x += __shfl_xor_sync(0xffffffffu, o[x].x, k);
            o[x].y += __shfl_xor_sync(0xffffffffu, o[x].y, k);
            o[x].z += __shfl_xor_sync(0xffffffffu, o[x].z, k);
            o[x].w += __shfl_xor_sync(0xffffffffu, o[x].w, k);
        }
    }
    if constexpr (SETS > 1) {  // the sets' sums, joined by the first
        if (lane < kLanes) {
#pragma unroll
            for (int x = 0; x < 2; ++x) s_o[set][x * (2 * HD / 4) + col] = o[x];
        }
        if (warp == 0 && lane == 0) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                s_m[set][x] = m[x];
                s_l[set][x] = l[x];
            }
        }
        __syncthreads();
        if (set > 0) return;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float mx = -INFINITY;
#pragma unroll
            for (int k = 0; k < SETS; ++k) mx = fmaxf(mx, s_m[k][x]);
            l[x] = 0.f;
            o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < SETS; ++k) {
                const float f = s_l[k][x] == 0.f ? 0.f : ex2(s_m[k][x] - mx);
                const float4 z = s_o[k][x * (2 * HD / 4) + col];
                l[x] += s_l[k][x] * f;
                o[x] = make_float4(o[x].x + z.x * f, o[x].y + z.y * f, o[x].z + z.z * f, o[x].w + z.w * f);
            }
        }
    }
    const float g0 = l[0] == 0.f ? 0.f : 1.f / l[0], g1 = l[1] == 0.f ? 0.f : -__ldg(p.lambda + head) / l[1];
    float4 y = make_float4(g0 * o[0].x + g1 * o[1].x, g0 * o[0].y + g1 * o[1].y, g0 * o[0].z + g1 * o[1].z, g0 * o[0].w + g1 * o[1].w);
    if (p.gain) {
        float sum = y.x * y.x + y.y * y.y + y.z * y.z + y.w * y.w;
#pragma unroll
        for (int k = 1; k < kLanes; k <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        if (lane == 0) s_sum[warp] = sum;
        ptx::bar_sync(1, 32 * kMergeWarps);  // (the first set's)
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < kMergeWarps; ++k) sum += s_sum[k];
        const float f = 1.f / sqrtf(sum / (2 * HD) + p.eps);
        const float *g = p.gain + col * 4;  // (a vector of any alignment)
        y = make_float4(y.x * f * __ldg(g), y.y * f * __ldg(g + 1), y.z * f * __ldg(g + 2), y.w * f * __ldg(g + 3));
    }
    if (lane < kLanes)
        reinterpret_cast<uint2 *>(p.out + (static_cast<int64_t>(sq.q_row0 + qi) * heads + head) * 2 * HD)[col] =
            make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
}

constexpr int kRowMergeWarps = 4;

// A warp per output row and head, two pieces of both maps in flight.
template <int HD>
__global__ void __launch_bounds__(32 * kRowMergeWarps) diff_row_combine_kernel(const __grid_constant__ DiffParams p)
{
    const int lane = threadIdx.x & 31, id = static_cast<int>(blockIdx.x) * kRowMergeWarps + (threadIdx.x >> 5);
    ptx::griddep_launch_dependents();
    if (id >= p.n_out) return;
    int lo = 0, hi = p.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.seqs[mid].out0 <= id) lo = mid; else hi = mid - 1;
    }
    const DiffSeq &sq = p.seqs[lo];
    const int heads = p.hq / 2, local = id - sq.out0, qi = local / heads, head = local - qi * heads;
    const int pair = head / p.group, r = qi * p.group + head - pair * p.group;
    const int u = sq.unit0 + pair * sq.n_blocks + r / DiffFew::kRows, row = r % DiffFew::kRows;
    const int c0 = diff_first_taker(p, u), c1 = diff_last_taker(p, u);
    ptx::griddep_wait();
    DiffRow<HD> a;
    for (int c = c0; c <= c1; c += 2) {
        float lse[2][2];
        float4 z[2][2][DiffRow<HD>::V4];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                lse[b][x] = -INFINITY;
                if (c + b > c1) continue;
                const int64_t at = static_cast<int64_t>(u + c + b) * DiffFew::kSlotRows + x * DiffFew::kRows + row;
                lse[b][x] = __ldcg(p.part_lse + at);
#pragma unroll
                for (int v = 0; v < DiffRow<HD>::V4; ++v) z[b][x][v] = __ldcg(reinterpret_cast<const float4 *>(p.part + at * 2 * HD) + v * 32 + lane);
            }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) a.add(x, lse[b][x], z[b][x]);
    }
    a.finish(p, sq.q_row0 + qi, head, lane);
}

// A block per 32 consecutive rows of a pair of kv-heads, lane t on row t, the columns over WARPS warps (the partials' layout:
// part_chunk), BATCH pieces in flight.
template <int HD, int WARPS, int BATCH>
__global__ void __launch_bounds__(32 * WARPS) diff_many_combine_kernel(const __grid_constant__ DiffParams p)
{
    constexpr int N = 2 * HD / 4 / WARPS;  // 16-byte chunks of a warp
    __shared__ float s_sum[WARPS][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int lo = 0, hi = p.n_seqs - 1;
    const int id = static_cast<int>(blockIdx.x);
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.seqs[mid].out0 <= id) lo = mid; else hi = mid - 1;
    }
    const DiffSeq &sq = p.seqs[lo];
    const int groups = (sq.n_q * p.group + 31) / 32, pair = (id - sq.out0) / groups, r0 = ((id - sq.out0) - pair * groups) * 32;
    const int r = r0 + lane, qi = r / p.group, head = pair * p.group + r - qi * p.group;
    int u[2], c0[2], c1[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        u[x] = sq.unit0 + (2 * pair + x) * sq.n_blocks + r0 / DiffMany::kRows;
        c0[x] = diff_first_taker(p, u[x]);
        c1[x] = diff_last_taker(p, u[x]);
    }
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const bool valid = qi < sq.n_q;
    float4 y[N];
#pragma unroll
    for (int k = 0; k < N; ++k) y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        float m = -INFINITY, l = 0.f;
        float4 o[N];
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int cb = c0[x]; cb <= c1[x]; cb += BATCH) {
            float lse[BATCH];
            float4 z[BATCH][N];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int64_t at = static_cast<int64_t>(u[x] + cb + b) * DiffMany::kSlotRows + r % DiffMany::kRows;
                const bool in = valid && cb + b <= c1[x];
                lse[b] = in ? __ldcg(p.part_lse + at) : -INFINITY;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    z[b][k] = in ? __ldcg(part_chunk<2 * HD>(p.part, at, warp * N + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (lse[b] == -INFINITY) continue;  // (no key seen, or no row; what it holds is anything)
                const float mn = fmaxf(m, lse[b]), f = m == -INFINITY ? 0.f : ex2(m - mn), g = ex2(lse[b] - mn);  // (NaN where lse is)
                m = mn;
                l = l * f + g;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    o[k] = make_float4(o[k].x * f + z[b][k].x * g, o[k].y * f + z[b][k].y * g, o[k].z * f + z[b][k].z * g,
                                       o[k].w * f + z[b][k].w * g);
            }
        }
        if (l == 0.f) continue;
        const float g = (x ? -__ldg(p.lambda + head) : 1.f) / l;
#pragma unroll
        for (int k = 0; k < N; ++k) y[k] = make_float4(y[k].x + g * o[k].x, y[k].y + g * o[k].y, y[k].z + g * o[k].z, y[k].w + g * o[k].w);
    }
    if (p.gain) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) sum += y[k].x * y[k].x + y[k].y * y[k].y + y[k].z * y[k].z + y[k].w * y[k].w;
        s_sum[warp][lane] = sum;
        __syncthreads();
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) sum += s_sum[k][lane];
        const float f = 1.f / sqrtf(sum / (2 * HD) + p.eps);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float *g = p.gain + (warp * N + k) * 4;
            y[k] = make_float4(y[k].x * f * __ldg(g), y[k].y * f * __ldg(g + 1), y[k].z * f * __ldg(g + 2), y[k].w * f * __ldg(g + 3));
        }
    }
    if (!valid) return;
    uint4 *dst = reinterpret_cast<uint4 *>(p.out + (static_cast<int64_t>(sq.q_row0 + qi) * (p.hq / 2) + head) * 2 * HD + warp * N * 4);
#pragma unroll
    for (int k = 0; k < N; k += 2)
        dst[k / 2] = make_uint4(pack_bf16(y[k].x, y[k].y), pack_bf16(y[k].z, y[k].w), pack_bf16(y[k + 1].x, y[k + 1].y),
                                pack_bf16(y[k + 1].z, y[k + 1].w));
}

cudaLaunchConfig_t diff_config(int blocks, int threads, int smem, cudaStream_t st, cudaLaunchAttribute *attr)
{
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(smem);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

// n clusters of `ranks` CTAs.
template <int HD>
cudaError_t diff_attn_config(int n, int ranks, cudaStream_t st, cudaLaunchAttribute (&attr)[2], cudaLaunchConfig_t &cfg)
{
    static std::atomic<uint64_t> configured{0};
    cfg = diff_config(n * ranks, kDiffThreads, DiffCfg<HD>::kDynSmem, st, attr);
    if (ranks > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = static_cast<unsigned>(ranks);
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    return set_dyn_smem_once(diff_attn_kernel<HD>, DiffCfg<HD>::kDynSmem, configured);
}

template <int HD>
cudaError_t launch_diff_t(const CUtensorMap &k, const CUtensorMap &v, const DiffParams &p, cudaStream_t st)
{
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg;
    if (cudaError_t e = diff_attn_config<HD>(p.n_takers, std::max(1, p.whole), st, attr, cfg); e != cudaSuccess) return e;
    return cudaLaunchKernelEx(&cfg, diff_attn_kernel<HD>, k, v, p);
}

template <int HD>
cudaError_t diff_clusters_t(int ranks, int *n)
{
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg;
    if (cudaError_t e = diff_attn_config<HD>(1, ranks, nullptr, attr, cfg); e != cudaSuccess) return e;
    return cudaOccupancyMaxActiveClusters(n, diff_attn_kernel<HD>, &cfg);
}

}  // namespace

cudaError_t launch_diff_attn(int head_dim, const CUtensorMap &tm_k, const CUtensorMap &tm_v, const DiffParams &p, cudaStream_t st)
{
    if (p.n_takers <= 0) return cudaSuccess;
    return head_dim == 128 ? launch_diff_t<128>(tm_k, tm_v, p, st) : launch_diff_t<64>(tm_k, tm_v, p, st);
}

cudaError_t diff_resident_clusters(int head_dim, int ranks, int *n)
{
    return head_dim == 128 ? diff_clusters_t<128>(ranks, n) : diff_clusters_t<64>(ranks, n);
}

cudaError_t launch_diff_combine(int head_dim, bool many, const DiffParams &p, cudaStream_t st)
{
    if (p.n_out <= 0) return cudaSuccess;
    cudaLaunchAttribute attr;
    if (many) {
        const DiffSeq &last = p.seqs[p.n_seqs - 1];
        const bool pieces = p.n_takers > 2 * (last.unit0 + last.n_blocks * p.hkv);  // more than two or three of a unit
        const int warps = pieces ? head_dim / 4 : head_dim / 8;
        const cudaLaunchConfig_t cfg = diff_config(p.n_out, 32 * warps, 0, st, &attr);
        if (head_dim == 128)
            return pieces ? cudaLaunchKernelEx(&cfg, diff_many_combine_kernel<128, 32, 3>, p)
                          : cudaLaunchKernelEx(&cfg, diff_many_combine_kernel<128, 16, 1>, p);
        return pieces ? cudaLaunchKernelEx(&cfg, diff_many_combine_kernel<64, 16, 4>, p)
                      : cudaLaunchKernelEx(&cfg, diff_many_combine_kernel<64, 8, 1>, p);
    }
    // Few pieces of many rows go a warp a row: 8 agents of 32k keys and 16 queries, normed (6 pieces of 4096 rows and heads) 189
    // us, by blocks 197.  Very many pieces of few rows take three sets of warps: one agent of 120k keys (39 pieces of 32) 82.6 us,
    // with one set 89.5.
    const DiffSeq &last = p.seqs[p.n_seqs - 1];
    if (p.n_takers <= 8 * (last.unit0 + last.n_blocks * (p.hkv / 2)) && p.n_out >= 1024) {
        const cudaLaunchConfig_t cfg = diff_config((p.n_out + kRowMergeWarps - 1) / kRowMergeWarps, 32 * kRowMergeWarps, 0, st, &attr);
        return head_dim == 128 ? cudaLaunchKernelEx(&cfg, diff_row_combine_kernel<128>, p)
                               : cudaLaunchKernelEx(&cfg, diff_row_combine_kernel<64>, p);
    }
    const bool sets = p.n_takers > 16 * (last.unit0 + last.n_blocks * (p.hkv / 2)) && p.n_out <= 512;
    const cudaLaunchConfig_t cfg = diff_config(p.n_out, 32 * kMergeWarps * (sets ? 3 : 1), 0, st, &attr);
    if (head_dim == 128) return sets ? cudaLaunchKernelEx(&cfg, diff_combine_kernel<128, 3>, p) : cudaLaunchKernelEx(&cfg, diff_combine_kernel<128, 1>, p);
    return sets ? cudaLaunchKernelEx(&cfg, diff_combine_kernel<64, 3>, p) : cudaLaunchKernelEx(&cfg, diff_combine_kernel<64, 1>, p);
}

}  // namespace pe
