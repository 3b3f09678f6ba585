// Differential attention of many rows (mathematics, units and partials: pe_diff.cu, pe_internal.h).
//
// A unit is one map of 256 query rows: O [256 x 2d] takes all of TMEM that two S buffers leave at d = 128, so the maps are
// units of their own.  Per tile of 128 keys, by tcgen05 over a pair of CTAs (128 rows each)
//     S [256 x 128] = Q [256 x d] . K_2j+m^T            (each CTA's shared memory holds 64 of the keys)
//     O [256 x 2d] += P [256 x 128] . [V_2j | V_2j+1]   (A = P from TMEM; each CTA's shared memory holds one kv-head's V)
// P goes to the second product as two bf16 parts (two_parts, diff.cuh), which take the columns of S that they come from.
// So a CTA loads half of a tile: 48 KB (d = 128) for 2560 cycles of MMAs.
//
// Bound by the tensor cores.  S(j + 1) is computed before P(j) is waited for, so a tile's softmax has the time of a tile's
// MMAs; it is spread over two warpgroups, each with half of the tile's keys (64 exponentials a thread).  The halves of a row
// share its reference: it moves only when a tile's sum passes 2^64 (pe_attn.cu), so per tile they exchange one vote, and the
// maxima only then and at a piece's first tile.
//
// Measured: 1638 queries on 16k keys, 32 / 8 heads, d = 128: 542 to 578 us (1.8 to 1.9 PFLOP/s of products, P's two parts counted;
// tensor cores 90 % busy, the card's power limit), 400 queries 150 us; d = 64, whose softmax has half the MMAs' time to hide in,
// 360 to 374 us.  Weights in one part took 378 and 309 and were not accurate enough (two_parts).  Not kept, all measured with one
// part (309, 395, 24.4 and 71 us): P in columns of its own at d = 64, so that S(j + 2) need
// not wait for P V(j), 362 us; four warpgroups with a quarter of the keys each 341 (d = 128 406); both maps of a block in a
// cluster of four that finishes its rows itself: 500 queries on 1000 keys 26.6 us against 24.4, 2000 on 2000 97 against 71.
//
// Roles (352 threads): warps 0-3 and 4-7 softmax, 8 producer of Q and K, 9 of V, 10 MMA (the pair's first CTA issues).  A piece's Q
// is loaded as soon as the S products of the piece before are done, so that it is there when that one's outputs are written.
#include <algorithm>

#include "diff.cuh"
#include "q8.cuh"

namespace pe {

namespace {

constexpr int kManyThreads = 352;
constexpr int kSoftWarps = 8;

template <int HD>
struct ManyCfg {
    static constexpr int kRegions = HD / 64;
    static constexpr int kStages = HD == 128 ? 4 : 7;
    static constexpr int kQBytes = 128 * HD * 2;
    static constexpr int kKRegion = 64 * 128;                 // 64 keys x 64 columns
    static constexpr int kKBytes = kRegions * kKRegion;
    static constexpr int kVRegion = 128 * 128;                // 128 keys x 64 columns
    static constexpr int kVBytes = kRegions * kVRegion;
    static constexpr int kOffK = kQBytes;
    static constexpr int kOffV = kOffK + kStages * kKBytes;
    static constexpr int kOffMax = kOffV + kStages * kVBytes; // float [2][128]: the halves' maxima, or sums
    static constexpr int kOffNeed = kOffMax + 2 * 128 * 4;    // bool [2][128]: whose reference has to move
    static constexpr int kOffBar = kOffNeed + 2 * 128;
    // k_full, k_empty, v_full, v_empty, v_peer [stages]; q_full, q_empty, meet, edge; s_full, p_full, o_done [2]
    static constexpr int kNumBars = 5 * kStages + 4 + 6;
    static constexpr int kOffMisc = kOffBar + kNumBars * 8;   // tmem slot, abort, votes [2], keys not finite [2][4]
    static constexpr int kDynSmem = kOffMisc + 48 + 1024;
    static constexpr int kTmemO = 256;                        // S at 0 and 128
    static constexpr uint32_t kTmemCols = 512;
    static_assert(kDynSmem <= 232448, "shared memory budget");
    static_assert(kOffV % 1024 == 0, "operand alignment");
};

// ---- a pair of CTAs
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}

__device__ __forceinline__ void arrive_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// The same where no generic memory is handed over: what was written is tensor memory (tcgen05.wait::st, tcgen05.fence) or this
// CTA's shared memory for its own tensor core (fence.proxy.async).  The release of all memory at cluster scope makes a warp wait
// for its stores: at every tile it took 1.8 of 3.4 thousand cycles.
__device__ __forceinline__ void arrive_peer(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

__device__ __forceinline__ void or_cluster(uint32_t cluster_addr, uint32_t bits)
{
    asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(cluster_addr), "r"(bits) : "memory");
}

__device__ __forceinline__ bool try_wait_cluster(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// wait_bar_warp (dev_common.cuh) on a barrier at which threads of both CTAs arrive
__device__ __forceinline__ bool wait_cluster_warp(uint32_t bar, uint32_t parity, const WaitCtx &w)
{
    bool ok = try_wait_cluster(bar, parity);
    if (!ok) {
        const uint64_t t0 = ptx::globaltimer();
        for (;;) {
            if ((ok = try_wait_cluster(bar, parity))) break;
            if (*w.abort) break;
            if (ptx::globaltimer() - t0 > kWaitNs) {
                *w.abort = 1;
                atomicCAS(w.status, 0, kStatusWaitTimeout);
                break;
            }
        }
    }
    return __all_sync(0xffffffffu, ok);
}

// A box into this CTA's shared memory, its bytes counted on a barrier of either CTA of the pair.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t cluster_bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(cluster_bar)
        : "memory");
}

__device__ __forceinline__ void tma_load_pair_4d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, int32_t w,
                                                 uint32_t cluster_bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(cluster_bar)
        : "memory");
}

__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void mma_pair_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Arrive once on `bar` of both CTAs when every MMA that the elected lane issued so far completes.
__device__ __forceinline__ void commit_pair(uint32_t bar)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(bar),
        "h"(static_cast<uint16_t>(3))
        : "memory");
}

template <int HD>
__global__ void __launch_bounds__(kManyThreads, 1)
    diff_many_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                     const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ DiffParams p)
{
    using C = ManyCfg<HD>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_addr(smem_raw);
    const uint32_t sbase = (raw + 1023u) & ~1023u;  // (the same in both CTAs)
    uint8_t *smem = smem_raw + (sbase - raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1;

    const uint32_t b_k_full = sbase + C::kOffBar;          // (the first CTA's count the loads of both)
    const uint32_t b_k_empty = b_k_full + 8 * C::kStages;
    const uint32_t b_v_full = b_k_empty + 8 * C::kStages;
    const uint32_t b_v_empty = b_v_full + 8 * C::kStages;
    const uint32_t b_v_peer = b_v_empty + 8 * C::kStages;  // (the first CTA's: the other's V is there)
    const uint32_t b_q_full = b_v_peer + 8 * C::kStages;   // (the first CTA's counts the loads of both)
    const uint32_t b_q_empty = b_q_full + 8;
    const uint32_t b_meet = b_q_empty + 8;                 // this CTA's softmax warps among themselves
    const uint32_t b_edge = b_meet + 8;                    // the softmax warps of both
    const uint32_t b_s_full = b_edge + 8;                  // [2]
    const uint32_t b_p_full = b_s_full + 16;               // [2] (the first CTA's: the softmax warps of both)
    const uint32_t b_o_done = b_p_full + 16;               // [2]
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::kOffMisc + 4);
    volatile uint32_t *votes = reinterpret_cast<volatile uint32_t *>(smem + C::kOffMisc + 8);      // [2]
    volatile uint32_t *odd_keys = reinterpret_cast<volatile uint32_t *>(smem + C::kOffMisc + 16);  // [2][4]
    const WaitCtx wctx{abort_flag, p.status};

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            ptx::mbar_init(b_k_full + 8 * s, 1);
            ptx::mbar_init(b_k_empty + 8 * s, 1);
            ptx::mbar_init(b_v_full + 8 * s, 1);
            ptx::mbar_init(b_v_empty + 8 * s, 1);
            ptx::mbar_init(b_v_peer + 8 * s, 1);
        }
        ptx::mbar_init(b_q_full, 1);
        ptx::mbar_init(b_q_empty, 1);
        ptx::mbar_init(b_meet, kSoftWarps);
        ptx::mbar_init(b_edge, 2 * kSoftWarps);
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(b_s_full + 8 * s, 1);
            ptx::mbar_init(b_p_full + 8 * s, 2 * kSoftWarps);
            ptx::mbar_init(b_o_done + 8 * s, 1);
        }
        *abort_flag = 0;
        votes[0] = votes[1] = 0;
        for (int k = 0; k < 8; ++k) odd_keys[k] = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
        ptx::prefetch_tensormap(&tm_q);
        ptx::prefetch_tensormap(&tm_k);
        ptx::prefetch_tensormap(&tm_v);
    }
    if (warp == 10) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::smem_addr(tmem_slot)), "r"(C::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    ptx::tc_fence_before();
    __syncthreads();
    __syncwarp();
    ptx::cluster_sync();  // the pair's barriers are there
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();

    DiffWalk<DiffMany> w(p, static_cast<int>(blockIdx.x >> 1));
    int i = 0;  // tiles of the pieces before
    if (warp == 8 || warp == 9) {
        // =================================================== producers: Q's 128 rows and 64 keys of K, or one kv-head's V of 128
        const bool is_v = warp == 9;
        const CUtensorMap *map = is_v ? &tm_v : &tm_k;
        const uint32_t b_full = is_v ? b_v_full : b_k_full, b_empty = is_v ? b_v_empty : b_k_empty;
        const bool both = !is_v;  // K's loads of both CTAs are counted in the first; V's each in its own, whose softmax waits too
        const uint32_t b_count = peer_addr(b_full, both ? 0 : rank);
        const int rows = min(p.ps, 64), keys = is_v ? 128 : 64;
        const int n_ops = keys / rows * C::kRegions;  // <= 32
        const int op_page = lane / C::kRegions, op_reg = lane % C::kRegions;
        const bool on = lane < n_ops;
        const uint32_t bytes = is_v ? C::kVBytes : C::kKBytes;
        const uint32_t base = sbase + (is_v ? C::kOffV + op_reg * C::kVRegion : C::kOffK + op_reg * C::kKRegion) + op_page * rows * 128;
        const uint32_t q_count = peer_addr(b_q_full, 0);
        bool ok = true;
        int pieces = 0;
        for (; ok && w.next(); ++pieces) {
            const DiffSeq &sq = p.seqs[w.si];
            if (!is_v) {
                if (pieces > 0 && !wait_bar_warp(b_q_empty, (pieces - 1) & 1, wctx)) { ok = false; break; }
                if (lane == 0) {
                    if (rank == 0) ptx::mbar_arrive_expect_tx(b_q_full, 2 * C::kQBytes);
                    // (rows past the sequence's last are others', or zeros)
                    const int q0 = sq.q_row0 + (w.block * DiffMany::kRows + static_cast<int>(rank) * 128) / p.group;
                    for (int r = 0; r < C::kRegions; ++r)
                        tma_load_pair_4d(sbase + r * (128 * 128), &tm_q, r * 64, w.map, w.pair * p.group, q0, q_count);
                }
                __syncwarp();
            }
            const int kvh = 2 * w.pair + (is_v ? static_cast<int>(rank) : w.map);
            auto row_of = [&](int k) -> int {  // of the pool, of this lane's box of tile k
                const int key = (w.t0 + k) * 128 + (is_v ? 0 : 64 * static_cast<int>(rank)) + op_page * rows, lp = key >> p.log_ps;
                const int page = on && lp < sq.n_pages ? p.page_table[sq.table_row + lp] : -1;
                return page >= 0 && page < p.num_pages ? (((p.layer * p.num_pages + page) * p.hkv + kvh) << p.log_ps) + (key & (p.ps - 1))
                                                       : p.oob_row;
            };
            int y = row_of(0);
            for (int k = 0; k < w.n; ++k, ++i) {
                const int next = k + 1 < w.n ? row_of(k + 1) : 0, s = i % C::kStages;
                if (i >= C::kStages && !wait_bar_warp(b_empty + 8 * s, ((i / C::kStages) - 1) & 1, wctx)) { ok = false; break; }
                if (lane == 0 && (!both || rank == 0)) ptx::mbar_arrive_expect_tx(b_full + 8 * s, both ? 2 * bytes : bytes);
                __syncwarp();
                if (on) tma_load_pair(base + s * bytes, map, op_reg * 64, y, b_count + 8 * s);
                y = next;
            }
        }
        // what the pair's first CTA still sends to this CTA's barriers is waited for: they have to be there
        if (ok && !is_v && pieces > 0) ok = wait_bar_warp(b_q_empty, (pieces - 1) & 1, wctx);
        for (int k = max(0, i - C::kStages); ok && k < i; ++k)
            ok = wait_bar_warp(b_empty + 8 * (k % C::kStages), (k / C::kStages) & 1, wctx);
        __syncwarp();
        if (*abort_flag && lane == 0 && (!both || rank == 0)) {  // a bounded chance for copies in flight to land
            const uint64_t g0 = ptx::globaltimer();
            if (!is_v && pieces > 0)
                while (!ptx::mbar_try_wait(b_q_full, (pieces - 1) & 1) && ptx::globaltimer() - g0 < 4000000ull) {}
            for (int k = max(0, i - C::kStages); k < i; ++k)
                while (!ptx::mbar_try_wait(b_full + 8 * (k % C::kStages), (k / C::kStages) & 1) && ptx::globaltimer() - g0 < 4000000ull) {}
        }
    } else if (warp == 10) {
        // =================================================== MMA (the converged warp of the first CTA)
        constexpr uint32_t kIdescS = ptx::idesc_bf16_f32(256, 128, false);
        constexpr uint32_t kIdescO = ptx::idesc_bf16_f32(256, 2 * HD, true);
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
                mma_pair(tm + 128 * (j & 1), q_desc + (((kk >> 2) * (128 * 128) + (kk & 3) * 32) >> 4),
                         kd + (((kk >> 2) * C::kKRegion + (kk & 3) * 32) >> 4), kIdescS, kk > 0 ? 1u : 0u);
            commit_pair(b_s_full + 8 * (j & 1));
            commit_pair(b_k_empty + 8 * (j % C::kStages));
            return true;
        };
        if (rank == 1) {  // tells the first CTA that this one's V is there
            const uint32_t peer = peer_addr(b_v_peer, 0);
            for (bool ok = true; ok && w.next();)
                for (int k = 0; ok && k < w.n; ++k, ++i)
                    if ((ok = full(b_v_full, i)) && lane == 0) arrive_peer(peer + 8 * (i % C::kStages));
        }
        bool ok = rank == 0;
        for (int piece = 0; ok && w.next(); ++piece) {
            const int n = __shfl_sync(0xffffffffu, w.n, 0);
            if (!wait_bar_warp(b_q_full, piece & 1, wctx)) break;
            ok = issue_s(i) && (n < 2 || issue_s(i + 1));
            if (n <= 2) commit_pair(b_q_empty);
            for (int k = 0; ok && k < n; ++k, ++i) {
                if (!full(b_v_full, i) || !full(b_v_peer, i) || !wait_bar_warp(b_p_full + 8 * (i & 1), (i >> 1) & 1, wctx)) { ok = false; break; }
                ptx::tc_fence_after();
                const uint64_t vd = v_desc + (i % C::kStages) * (C::kVBytes >> 4);
#pragma unroll
                for (int kk = 0; kk < 16; ++kk)  // P's halves over S's: of each the weights' upper parts, then their lower ones
                    mma_pair_ts(tm + C::kTmemO, tm + 128 * (i & 1) + kk * 8, vd + (((kk >> 3) * 4 + (kk & 3)) * 16 * 128 >> 4), kIdescO,
                                (k > 0 || kk > 0) ? 1u : 0u);
                commit_pair(b_o_done + 8 * (i & 1));
                commit_pair(b_v_empty + 8 * (i % C::kStages));
                if (k + 2 < n) {
                    ok = issue_s(i + 2);  // (P(i), over S(i), is read by then)
                    if (k + 3 == n) commit_pair(b_q_empty);
                }
            }
        }
    } else if (warp < kSoftWarps) {
        // =================================================== softmax: thread (half, row) owns 64 of a tile's keys
        const int row = threadIdx.x & 127, half = warp >> 2;
        const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t p_full = peer_addr(b_p_full, 0);
        const uint32_t edge0 = peer_addr(b_edge, 0), edge1 = peer_addr(b_edge, 1);
        const uint32_t odd0 = peer_addr(sbase + C::kOffMisc + 16, 0), odd1 = peer_addr(sbase + C::kOffMisc + 16, 1);
        float *s_max = reinterpret_cast<float *>(smem + C::kOffMax);
        bool *s_need = reinterpret_cast<bool *>(smem + C::kOffNeed);
        const float2 sl2 = make_float2(p.scale_log2, p.scale_log2);
        bool ok = true;
        int met = 0, edges = 0;
        auto meet = [&]() {  // of this CTA's softmax warps
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(b_meet);
            return wait_bar_warp(b_meet, met++ & 1, wctx);
        };
        auto meet_pair = [&](bool tells) {  // tells: this warp wrote to the other CTA
            __syncwarp();
            if (lane == 0) {
                if (tells) {
                    arrive_cluster(edge0);
                    arrive_cluster(edge1);
                } else {
                    arrive_peer(edge0);
                    arrive_peer(edge1);
                }
            }
            return wait_cluster_warp(b_edge, edges++ & 1, wctx);
        };
        int pos, pos_first;
        bool valid, any;
        auto begin = [&]() {  // the next piece's row
            if (!w.next()) return false;
            const DiffSeq &sq = p.seqs[w.si];
            const int qi = (w.block * DiffMany::kRows + static_cast<int>(rank) * 128 + row) / p.group;
            valid = qi < sq.n_q;
            any = __any_sync(0xffffffffu, valid);
            pos = sq.n_keys - sq.n_q + qi;
            pos_first = sq.n_keys - sq.n_q + w.block * DiffMany::kRows / p.group;  // of the pair's rows
            return true;
        };
        for (bool more = begin(); ok && more;) {
            float m_ref = -INFINITY, l = 0.f;
            const int n = w.n, t0 = w.t0;
            for (int k = 0; k < n; ++k, ++i) {
                const int kbase = (t0 + k) * 128;
                const uint32_t tS = tmem + 128 * (i & 1) + 64 * half + lane_off;
                const bool edge = kbase + 127 > pos_first;  // a row of the pair does not see some key of the tile
                if (edge) {
                    // V of such keys (pe_diff.cu): each CTA looks through the kv-head that it holds, for both
                    if (!wait_bar_warp(b_v_full + 8 * (i % C::kStages), (i / C::kStages) & 1, wctx)) { ok = false; break; }
                    const int key = threadIdx.x & 127, c0 = half * (HD / 16);
                    uint8_t *v = smem + C::kOffV + (i % C::kStages) * C::kVBytes + key * 128;
                    uint32_t odd = 0;
#pragma unroll
                    for (int c = 0; c < HD / 16; ++c)
                        odd = max(odd, bf16x8_absmax(*reinterpret_cast<const uint4 *>(v + ((c0 + c) >> 3) * C::kVRegion + (((c0 + c) & 7) << 4))));
                    const bool is_odd = odd >= 0x7f80u;
                    // two sets of words in turn, by the meetings' parity (pe_diff.cu): the other CTA may be a tile ahead
                    const int odd_set = 4 * (edges & 1);
                    if (is_odd) {
                        or_cluster(odd0 + 4 * (odd_set + (key >> 5)), 1u << (key & 31));
                        or_cluster(odd1 + 4 * (odd_set + (key >> 5)), 1u << (key & 31));
                    }
                    if (!meet_pair(__any_sync(0xffffffffu, is_odd))) { ok = false; break; }
                    uint32_t mask[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) mask[x] = odd_keys[odd_set + x];
                    if (mask[0] | mask[1] | mask[2] | mask[3]) {
                        if (odd_keys[odd_set + (key >> 5)] >> (key & 31) & 1u)
                            for (int c = 0; c < HD / 16; ++c)
                                *reinterpret_cast<uint4 *>(v + ((c0 + c) >> 3) * C::kVRegion + (((c0 + c) & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                        ptx::fence_proxy_async_smem();
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int sees = pos - kbase - 32 * x + 1;  // of this word's keys
                            if (sees > 0 && (mask[x] & (sees >= 32 ? ~0u : (1u << sees) - 1))) l = NAN;
                        }
                        if (!meet_pair(false)) { ok = false; break; }  // the mask is read
                        if (threadIdx.x < 4) odd_keys[odd_set + threadIdx.x] = 0;
                        if (!meet_pair(true)) { ok = false; break; }   // and cleared
                    }
                }
                if (!wait_bar_warp(b_s_full + 8 * (i & 1), (i >> 1) & 1, wctx)) { ok = false; break; }
                ptx::tc_fence_after();
                float s[64];
                if (any) {
                    float (&s0)[32] = *reinterpret_cast<float (*)[32]>(&s[0]);
                    float (&s1)[32] = *reinterpret_cast<float (*)[32]>(&s[32]);
                    ptx::tmem_ld32(tS, s0);
                    ptx::tmem_ld32(tS + 32, s1);
                    ptx::tmem_wait_ld();
                    if (edge) {
#pragma unroll
                        for (int c = 0; c < 64; ++c)
                            if (kbase + 64 * half + c > pos) s[c] = -INFINITY;
                    }
                }
                auto exp_tile = [&](float ref) -> float {
                    const float2 nref = make_float2(-ref, -ref);
                    float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int ch = 0; ch < 2; ++ch) {
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
                        tmem_st16(tS + 32 + ch * 16, lo);
                    }
                    const float2 a = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
                    return a.x + a.y;
                };
                float rs = 0.f;
                bool move = k == 0, need = true;  // move: uniform over the CTA's softmax threads
                if (k > 0) {
                    if (any) rs = exp_tile(m_ref == -INFINITY ? 0.f : m_ref);
                    need = valid && (m_ref == -INFINITY || !(rs <= kDiffSumLimit));
                    const bool vote = __any_sync(0xffffffffu, need);
                    if (vote && lane == 0) votes[i & 1] = 1;
                    if (!meet()) { ok = false; break; }
                    move = votes[i & 1] != 0;
                }
                if (move) {
                    float mt = -INFINITY;
                    if (any) {
                        float mx[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) mx[x] = max3(s[x], s[4 + x], s[8 + x]);
#pragma unroll
                        for (int c = 12; c < 60; c += 8)
#pragma unroll
                            for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], s[c + x], s[c + 4 + x]);
                        mt = fmaxf(max3(mx[0], mx[1], mx[2]), max3(mx[3], fmaxf(s[60], s[61]), fmaxf(s[62], s[63])));
                    }
                    s_max[half * 128 + row] = mt;
                    s_need[half * 128 + row] = need;
                    if (!meet()) { ok = false; break; }
                    if (threadIdx.x == 0) votes[i & 1] = 0;  // (read by all; of use again in two tiles)
                    // (rows that need not keep theirs, and so their bits, whatever the other rows hold)
                    const float m_new = need || s_need[(half ^ 1) * 128 + row] ? fmaxf(m_ref, fmaxf(mt, s_max[(half ^ 1) * 128 + row]) * sl2.x) : m_ref;
                    if (k > 0) {
                        // O holds P V of the tiles before once the last of them is done
                        if (!wait_bar_warp(b_o_done + 8 * ((i - 1) & 1), ((i - 1) >> 1) & 1, wctx)) { ok = false; break; }
                        ptx::tc_fence_after();
                        const float alpha = m_ref == -INFINITY ? 1.f : ex2(m_ref - m_new);  // (no score so far: O and l are 0)
                        if (any && __any_sync(0xffffffffu, valid && m_new != m_ref)) {
                            const uint32_t tO = tmem + C::kTmemO + half * HD + lane_off;
#pragma unroll 1
                            for (int ch = 0; ch < HD / 16; ++ch) {
                                uint32_t o[16];
                                tmem_ld16(tO + ch * 16, o);
                                ptx::tmem_wait_ld();
#pragma unroll
                                for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                                tmem_st16(tO + ch * 16, o);
                            }
                            l *= alpha;
                        }
                    }
                    m_ref = m_new;
                    ptx::tmem_wait_st();
                    if (any) rs = exp_tile(m_ref == -INFINITY ? 0.f : m_ref);
                }
                l += rs;
                ptx::tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_peer(p_full + 8 * (i & 1));
            }
            if (!ok) break;
            const bool had = valid, had_any = any;
            const int64_t at = static_cast<int64_t>(w.slot) * DiffMany::kSlotRows + rank * 128 + row;
            more = begin();
            if (!wait_bar_warp(b_o_done + 8 * ((i - 1) & 1), ((i - 1) >> 1) & 1, wctx)) break;
            ptx::tc_fence_after();
            s_max[half * 128 + row] = l;  // (P V waited for every warp: no maxima of the last tile are read any more)
            if (!meet()) break;
            l += s_max[(half ^ 1) * 128 + row];
            if (!meet()) break;           // (of use again in the next piece's first tile)
            if (had_any) {
                const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one)
#pragma unroll 1
                for (int ch = 0; ch < HD / 32; ++ch) {
                    float o[32];
                    ptx::tmem_ld32(tmem + C::kTmemO + half * HD + lane_off + ch * 32, o);
                    ptx::tmem_wait_ld();
                    if (had && l != 0.f)
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            *part_chunk<2 * HD>(p.part, at, half * (HD / 4) + ch * 8 + x) =
                                make_float4(o[4 * x] * inv, o[4 * x + 1] * inv, o[4 * x + 2] * inv, o[4 * x + 3] * inv);
                }
                if (had && half == 0) p.part_lse[at] = l == 0.f ? -INFINITY : m_ref + __log2f(l);
            }
            ptx::tc_fence_before();
        }
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync();  // both CTAs are done with each other's barriers and memory
    if (warp == 10) {
        ptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
    }
}

template <int HD>
cudaError_t launch_many_t(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const DiffParams &p, cudaStream_t st)
{
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = set_dyn_smem_once(diff_many_kernel<HD>, ManyCfg<HD>::kDynSmem, configured);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(2 * p.n_takers));
    cfg.blockDim = dim3(kManyThreads);
    cfg.dynamicSmemBytes = ManyCfg<HD>::kDynSmem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, diff_many_kernel<HD>, q, k, v, p);
}

}  // namespace

cudaError_t launch_diff_attn_many(int head_dim, const CUtensorMap &tm_q, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                                  const DiffParams &p, cudaStream_t st)
{
    if (p.n_takers <= 0) return cudaSuccess;
    return head_dim == 128 ? launch_many_t<128>(tm_q, tm_k, tm_v, p, st) : launch_many_t<64>(tm_q, tm_k, tm_v, p, st);
}

}  // namespace pe
