// Attention of few query rows over the 8-bit cache, on its codes: tcgen05
// kind::f8f6f4 with keys on the M side, so that K and V go from HBM to the
// tensor cores as they are stored.
//
//     S^T [128 keys x 16] = K8 [128 x d] . Q8^T     (A = K codes, K-major)
//     O^T [d x NP]       += V8^T [d x 128] . P8^T   (A = V codes, MN-major; B too)
//
// Both factors must be e4m3, so q and the softmax weights are split into parts
// of four significant bits:
//   q   = 2^eq (q_hi + 2^-4 q_lo): bf16 has eight bits, so two parts are exact
//         for elements down to 2^-14 of the row's largest; S = S_hi + 2^-4 S_lo
//         in columns of their own.  With 16 rows q_lo is not scaled and both add
//         up in the same columns, or TMEM would hold chunks of half the length:
//         exact down to 2^-10 (smaller elements err by at most 2^-18 of the
//         largest).
//   p   = 2^-8 (p_hi + 2^-4 p_mid + 2^-8 p_lo): the eleven bits of the weight in
//         fp16, in which the parts are taken two at a time, and an absolute floor
//         of 2^-26 of the largest.
// The products are exact and accumulate in fp32 (measured: within 2^-22 of the
// sum of magnitudes), so what is rounded is the output alone, to bf16.
//
// A key's V scale goes into its weight: with ev its page's exponent and evm the
// largest of the chunk, y = x + ev - evm (x the score in log2 units) gets the
// weight pv = 2^(y - m), the sum of weights adds pv 2^(evm - ev) = 2^(x - m),
// and O = 2^evm sum pv code.  The reference m is the largest y of the chunk's
// row, so that pages of any scale use the codes' range.  (ev - evm is held at
// -100 or more.)
//
// The scores of a whole chunk stay in TMEM: one group of warps takes their
// maximum as the tiles arrive, another, a chunk behind, reads them again for the
// weights.  So nothing is ever rescaled and no tile waits at a barrier of the
// group.  With a running maximum, moved when a tile passed it and O^T rescaled
// then, the chain from a tile's scores to its weights took 1200 cycles with 4
// rows and 4500 with 16 (a tile's share of HBM is 1390).
//
// Up to 16 query rows R = query * g + head-in-group of a kv-head, in one block of
// RB; more rows go on the M side (pe_q8_rows.cu).
//
// Bound by HBM: 2 d bytes a key and kv-head.  One CTA a SM takes chunks of up to
// kQ8MaxChunk tiles from a counter, longest first; partials (O, m, l) of items
// held in several chunks are merged by a second launch.
//
// Roles (544 threads): warps 0-3 maxima (thread = key of the tile), 4-7 and 8-11
// weights of every other tile (thread = key) and, a chunk behind, the epilogue of
// every other chunk (thread = d-column), 12 K producer, 13 S^T MMAs, 14 V producer, 15 scheduler
// (takes chunk ids, reads page ids and scales, splits the q rows), 16 O^T MMAs.
// A commit takes its warp 80 cycles and an MMA 45, a probe of a barrier as long:
// one warp for both products spent 1500 cycles a tile, more than a tile's share
// of HBM, so each product has its warp, and each MMA group one commit.
#include <algorithm>

#include "q8_chunks.cuh"
#include "q8_mma.cuh"

namespace pe {

namespace {

constexpr int kQ8Stages = 5;                 // K ring, and V ring
constexpr int kQ8Threads = 544;
constexpr int kQ8Ring = 4;                   // chunks between the scheduler and the weights
constexpr int kQ8Desc = 3;                   // chunk descriptors of the producers (V is one behind K)
constexpr int kQ8DescInts = 8 + 16 * kQ8MaxChunk;
constexpr int kQ8BarMax = 1, kQ8BarWeights = 2;  // named barriers of the two groups
constexpr float kQ8Unpart = 1.f / 16.f;
constexpr int kNQ = 16;                      // columns of a tile's scores

__device__ __forceinline__ uint32_t half2_to_e4m3(__half2 w)
{
    return __nv_cvt_halfraw2_to_fp8x2(static_cast<__half2_raw>(w), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ __half2 e4m3_to_half2(uint32_t codes)
{
    return __half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes), __NV_E4M3));
}

// P^T as the B operand, MN-major without swizzle: 16 columns of a key are 16 bytes, keys 16 bytes apart, groups of 16
// columns 2 KB apart.  So a thread, which holds one key, stores a key's parts 16 bytes at a time; K-major, a byte for
// each row and part (48 for 16 rows), a tile's weights took twice as long.
__device__ __forceinline__ uint64_t weights_desc(uint32_t addr)
{
    return ptx::smem_desc_sw128(addr, 8 * 16, 2048) & ~(7ull << 61);
}

template <int HD, int RB>
struct Q8Cfg {
    static constexpr int kTile = kQ8Keys * HD;                   // a K or V stage
    static constexpr int kOffV = kQ8Stages * kTile;
    static constexpr int kOffZero = 2 * kQ8Stages * kTile;       // d = 64: O^T rows 64..127 read zeros here
    static constexpr int kZero = HD == 64 ? kTile : 0;
    static constexpr int kParts = 3;                             // of a weight, RB columns of O^T each
    static constexpr int kNP = (kParts * RB + 15) / 16 * 16;
    static constexpr int kOffQ = kOffZero + kZero;
    static constexpr bool kQSum = RB > 8;                        // both parts of q in the same columns
    static constexpr int kQPart = kNQ * HD;                      // .. from two operands; else rows 0.. and 8.. of one
    static constexpr int kQBytes = (kQSum ? 2 : 1) * kQPart;     // per ring entry
    static constexpr int kOffP = kOffQ + kQ8Ring * kQBytes;
    static constexpr int kPBytes = kNP * 128;
    static constexpr int kCT = q8_max_chunk(RB);                 // tiles of a chunk whose scores TMEM holds, twice
    static constexpr int kOffRed = kOffP + 2 * kPBytes;          // float [12 warps][16], then the maxima [2][16], 8 - them
    static constexpr int kOffBar = kOffRed + (12 + 4) * 16 * 4;
    // k_full, v_full, v_empty [stages]; s_full [2][kCT]; s_free, m_full, p_full, drain [2];
    // ch_full, ch_empty [ring]; o_item, o_free, stats [2]; desc_full, desc_empty [kQ8Desc]
    static constexpr int kNumBars = 3 * kQ8Stages + 2 * kCT + 8 + 2 * kQ8Ring + 6 + 2 * kQ8Desc;
    static constexpr int kOffMisc = kOffBar + kNumBars * 8;      // tmem slot, abort, K / V tiles issued
    static constexpr int kStatsFloats = 8 + 2 * RB;              // id, 2^(evm - 8), Q8Chunk, -, m[RB], l[RB]
    static constexpr int kOffStats = kOffMisc + 16;
    // per ring entry: id, evm, Q8Chunk, -, 2^eq [16], then (ek, ev) of page slot j of tile k as int8 pairs [k][16]
    static constexpr int kEntryEq = 32, kEntryEx = 96;
    static constexpr int kEntryBytes = kEntryEx + kQ8MaxChunk * 32;
    static constexpr int kOffEntry = (kOffStats + 2 * kStatsFloats * 4 + 15) / 16 * 16;
    static constexpr int kOffDesc = kOffEntry + kQ8Ring * kEntryBytes;
    static constexpr int kOffSeqs = kOffDesc + kQ8Desc * kQ8DescInts * 4;
    static constexpr int kSmem = kOffSeqs + kMaxSegs * static_cast<int>(sizeof(Q8Seq) + 8);
    static constexpr int kDynSmem = kSmem + 1024;
    static constexpr int kTmemO = 2 * kCT * kNQ;                 // two O^T buffers after the scores of two chunks
    static constexpr uint32_t kTmemCols = 512;
    static_assert(kTmemO + 2 * kNP <= static_cast<int>(kTmemCols), "tensor memory");
    static_assert(kCT <= kQ8MaxChunk, "chunk length");
    static_assert(kOffP % 1024 == 0 && kPBytes % 1024 == 0 && kQBytes % 1024 == 0, "operand alignment");
    static_assert(kDynSmem <= 232448, "shared memory budget");
    static_assert(sizeof(Q8Seq) % 4 == 0, "copied by words");
};

// Reduces v[r] over the warp's lanes for every r < N (4, 8 or 16), always in the same order: each step halves the rows
// that a lane still holds.  The lane keeps v[0], of row reduced_row<N>().
template <int N, typename Op>
__device__ __forceinline__ void reduce_rows(float (&v)[N], const Op &op)
{
    const int lane = threadIdx.x & 31;
    int m = 16;
#pragma unroll
    for (int c = N / 2; c >= 1; c >>= 1, m >>= 1) {
        const bool up = lane & m;
#pragma unroll
        for (int i = 0; i < c; ++i) {
            const float got = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + c], m);
            v[i] = op(up ? v[i + c] : v[i], got);
        }
    }
    for (; m >= 1; m >>= 1) v[0] = op(v[0], __shfl_xor_sync(0xffffffffu, v[0], m));
}
template <int N>
__device__ __forceinline__ int reduced_row()
{
    constexpr int kBits = N == 16 ? 4 : (N == 8 ? 3 : 2);
    return (threadIdx.x & 31) >> (5 - kBits);  // lane bit 4 chose the upper half of the rows, bit 3 of those, ..
}

template <int HD, int RB>
__global__ void __launch_bounds__(kQ8Threads, 1)
    attn_q8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const __grid_constant__ Q8AttnParams p)
{
    using C = Q8Cfg<HD, RB>;
    constexpr int R = kQ8Ring;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    const uint32_t sbase = ptx::smem_addr(smem);
    float *s_red = reinterpret_cast<float *>(smem + C::kOffRed);
    const uint32_t bar0 = sbase + C::kOffBar;
    auto k_full = [&](int s) { return bar0 + 8u * s; };
    auto v_full = [&](int s) { return bar0 + 8u * (kQ8Stages + s); };
    auto v_empty = [&](int s) { return bar0 + 8u * (2 * kQ8Stages + s); };  // P V done: also frees the tile's P^T
    // [2][kCT] a tile's scores, by chunk parity; also frees its K stage
    const uint32_t b_s_full = bar0 + 8u * 3 * kQ8Stages;
    const uint32_t b_s_free = b_s_full + 8 * 2 * C::kCT;      // [2] a chunk's scores have been read
    const uint32_t b_m_full = b_s_free + 16;                  // [2] a chunk's maxima are in s_max
    const uint32_t b_p_full = b_m_full + 16;                  // [2]
    const uint32_t b_drain = b_p_full + 16;                   // [2] S^T, O^T
    const uint32_t b_ch_full = b_drain + 16;                  // [R] a chunk's id, scales and q parts are in its entry
    const uint32_t b_ch_empty = b_ch_full + 8 * R;            // [R] the weights are done with the chunk
    const uint32_t b_o_item = b_ch_empty + 8 * R;             // [2] a chunk's O^T is complete
    const uint32_t b_o_free = b_o_item + 16;                  // [2] the epilogue has read that O^T buffer
    const uint32_t b_stats = b_o_free + 16;                   // [2] a chunk's statistics are in s_stats
    const uint32_t b_desc_full = b_stats + 16;                // [kQ8Desc] a chunk's TMA rows are in s_desc
    const uint32_t b_desc_empty = b_desc_full + 8 * kQ8Desc;  // [kQ8Desc] both producers have issued that chunk
    float *s_stats = reinterpret_cast<float *>(smem + C::kOffStats);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::kOffMisc + 4);
    volatile int *s_issued = reinterpret_cast<volatile int *>(smem + C::kOffMisc + 8);  // [2]: K, V
    Q8Seq *s_seqs = reinterpret_cast<Q8Seq *>(smem + C::kOffSeqs);
    int2 *s_rem = reinterpret_cast<int2 *>(smem + C::kOffSeqs + kMaxSegs * sizeof(Q8Seq));
    int *s_desc = reinterpret_cast<int *>(smem + C::kOffDesc);
    auto entry = [&](int n) { return smem + C::kOffEntry + (n % R) * C::kEntryBytes; };
    const WaitCtx wctx{abort_flag, p.status};

    if (threadIdx.x == 384) {
        for (int s = 0; s < kQ8Stages; ++s) {
            ptx::mbar_init(k_full(s), 1);
            ptx::mbar_init(v_full(s), 1);
            ptx::mbar_init(v_empty(s), 1);
        }
        for (int b = 0; b < 2 * C::kCT; ++b) ptx::mbar_init(b_s_full + 8 * b, 1);
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(b_s_free + 8 * b, 256);
            ptx::mbar_init(b_m_full + 8 * b, 1);
            ptx::mbar_init(b_p_full + 8 * b, 128);
            ptx::mbar_init(b_drain + 8 * b, 1);
            ptx::mbar_init(b_o_item + 8 * b, 1);
            ptx::mbar_init(b_o_free + 8 * b, 128);
            ptx::mbar_init(b_stats + 8 * b, 1);
        }
        for (int r = 0; r < R; ++r) {
            ptx::mbar_init(b_ch_full + 8 * r, 1);
            ptx::mbar_init(b_ch_empty + 8 * r, 2 + 256);  // MMA warps, weight threads
        }
        for (int d = 0; d < kQ8Desc; ++d) {
            ptx::mbar_init(b_desc_full + 8 * d, 1);
            ptx::mbar_init(b_desc_empty + 8 * d, 2);      // K and V producers
        }
        *abort_flag = 0;
        s_issued[0] = 0;
        s_issued[1] = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&tm_k);
        ptx::prefetch_tensormap(&tm_v);
    }
    if (warp == 13) {
        ptx::tmem_alloc(ptx::smem_addr(tmem_slot), C::kTmemCols);
        ptx::tmem_relinquish();
    }
    if (warp < 4) {
        // columns that hold no part of a weight or of q stay zero
        for (int e = threadIdx.x; e < (R * C::kQBytes + 2 * C::kPBytes) / 16; e += 128)
            reinterpret_cast<uint4 *>(smem + C::kOffQ)[e] = make_uint4(0u, 0u, 0u, 0u);
        for (int e = threadIdx.x; e < C::kZero / 16; e += 128)
            reinterpret_cast<uint4 *>(smem + C::kOffZero)[e] = make_uint4(0u, 0u, 0u, 0u);
        ptx::fence_proxy_async_smem();
    } else if (warp >= 4 && warp < 12) {
        const int n_words = p.n_seqs * static_cast<int>(sizeof(Q8Seq) / 4);
        const int32_t *src = reinterpret_cast<const int32_t *>(p.seqs);
        for (int e = threadIdx.x - 128; e < n_words; e += 256) reinterpret_cast<int32_t *>(s_seqs)[e] = src[e];
        for (int e = threadIdx.x - 128; e < p.n_rem; e += 256)
            s_rem[e] = make_int2(p.seqs[p.rem_seq[e]].rem0, p.rem_seq[e]);
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    // Launched with programmatic serialization: nothing written by earlier kernels is read before this point.
    ptx::griddep_wait();
    const uint32_t tmem = *tmem_slot;

    if (warp == 12 || warp == 14) {
        // ============================================================ producers (warp 12: K, warp 14: V)
        const bool is_v = warp == 14;
        const CUtensorMap *map = is_v ? &tm_v : &tm_k;
        const int n_boxes = kQ8Keys / p.ps;  // a page a box
        int i = 0;                           // tile ordinal in this CTA
        uint32_t used[kQ8Stages] = {};       // K: the score barrier (and its parity << 8) of the last tiles, newest first
        for (int n = 0;; ++n) {
            const int d = n % kQ8Desc;
            if (!wait_spin(b_desc_full + 8 * d, (n / kQ8Desc) & 1, wctx)) break;
            const int *desc = s_desc + d * kQ8DescInts;
            if (desc[0] < 0) break;  // no more chunks
            const int nt = desc[1];
            bool ok = true;
            for (int k = 0; k < nt; ++k) {
                const int s = i % kQ8Stages;
                const uint32_t b_full = is_v ? v_full(s) : k_full(s);
                if (i >= kQ8Stages) {
                    const uint32_t u = used[kQ8Stages - 1];
                    if (!(is_v ? wait_spin(v_empty(s), ((i / kQ8Stages) - 1) & 1, wctx) : wait_spin(b_s_full + 8 * (u & 255u), u >> 8, wctx))) {
                        ok = false;
                        break;
                    }
                }
#pragma unroll
                for (int x = kQ8Stages - 1; x > 0; --x) used[x] = used[x - 1];
                used[0] = (n & 1) * C::kCT + k + (((n >> 1) & 1) << 8);
                if (lane == 0) ptx::mbar_arrive_expect_tx(b_full, C::kTile);
                __syncwarp();
                if (lane < n_boxes)
                    ptx::tma_load_2d(sbase + (is_v ? C::kOffV : 0) + s * C::kTile + lane * p.ps * HD, map, 0,
                                     desc[8 + 16 * k + lane], b_full);
                __syncwarp();
                ++i;
                if (lane == 0) s_issued[is_v ? 1 : 0] = i;
            }
            if (!ok) break;
            if (lane == 0) ptx::mbar_arrive(b_desc_empty + 8 * d);
        }
    } else if (warp == 15) {
        // ============================================================ scheduler
        const int lg = p.log_group, lps = p.log_ps;
        const int n_slots = kQ8Keys >> lps;  // <= 16
        constexpr int kPer = kQ8MaxChunk / 2;
        constexpr int kPieces = HD / 8;       // of a q row, eight columns each; lane e: row e / kPieces, piece e % kPieces
        constexpr int kRowsAt = 32 / kPieces;
        constexpr int kPasses = RB / kRowsAt, kAt = kPasses < 4 ? kPasses : 4;  // passes over the rows, at a time
        const int pc = lane % kPieces;
        auto load_q = [&](const Q8Chunk &ci, int j0, uint4 (&qv)[kAt]) {
            const Q8Seq &sq = s_seqs[ci.si];
#pragma unroll
            for (int j = 0; j < kAt; ++j) {
                qv[j] = make_uint4(0u, 0u, 0u, 0u);
                const int row = ci.blk * RB + (j0 + j) * kRowsAt + lane / kPieces;
                if (row < sq.n_q << lg)
                    qv[j] = *reinterpret_cast<const uint4 *>(
                        p.q + (static_cast<int64_t>(sq.q_row0 + (row >> lg)) * p.hq + (ci.kvh << lg) + (row & ((1 << lg) - 1))) * HD + pc * 8);
            }
        };
        auto claim = [&](int n) -> int {  // lane 0's is the id of chunk ordinal n (-1: no more)
            int c = -1;
            if (lane == 0) {
                c = n < 2 ? n * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x)
                          : 2 * static_cast<int>(gridDim.x) + atomicAdd(p.sched, 1);
                if (c >= p.total_chunks) c = -1;
            }
            return c;
        };
        // page ids of a chunk: entry e = 32 u + lane is tile e / 16, page slot e % 16
        auto load_pages = [&](const Q8Chunk &ci, int (&pg)[kPer]) {
            const Q8Seq &sq = s_seqs[ci.si];
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int e = 32 * u + lane;
                const int key0 = (ci.t0 + (e >> 4)) * kQ8Keys + ((e & 15) << lps);
                const bool in = ci.t0 + (e >> 4) < ci.t1 && (e & 15) < n_slots && key0 < sq.n_keys;
                pg[u] = in ? p.page_table[sq.table_row + (key0 >> lps)] : INT32_MIN;
            }
        };
        // Loads under load take 2000 cycles, so the next chunk's are in flight while this one's are used.
        int c = 0;  // (round -1 only takes the first)
        Q8Chunk ci{};
        int pg[kPer];
        for (int n = -1;; ++n) {
            const int d = n % kQ8Desc;
            const int claimed = c >= 0 ? claim(n + 1) : -1;
            if (n >= kQ8Desc && !wait_spin(b_desc_empty + 8 * d, ((n / kQ8Desc) - 1) & 1, wctx)) c = -1;
            int *desc = s_desc + d * kQ8DescInts;
            int ex[kPer];  // (ek, ev)
            uint4 qv[kAt];
            if (n < 0) {
            } else if (c >= 0) {
#pragma unroll
                for (int u = 0; u < kPer; ++u) {
                    const bool ok_page = pg[u] >= 0 && pg[u] < p.num_pages;
                    if (!ok_page && pg[u] != INT32_MIN) atomicCAS(p.status, 0, kStatusBadPage);
                    pg[u] = ok_page ? (p.layer * p.num_pages + pg[u]) * p.hkv + ci.kvh : -1;
                    desc[8 + 32 * u + lane] = pg[u] >= 0 ? pg[u] << lps : p.oob_row;  // past the sequence (or a bad id): zeros
                }
                if (lane == 0) {
                    desc[0] = c;
                    desc[1] = ci.t1 - ci.t0;
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(b_desc_full + 8 * d);  // release: the producers read the rows
#pragma unroll
                for (int u = 0; u < kPer; ++u)
                    ex[u] = pg[u] >= 0 ? reinterpret_cast<const uint16_t *>(p.exps)[pg[u]] : 0x8282;  // -126, -126
                load_q(ci, 0, qv);
            } else if (lane == 0) {
                desc[0] = -1;
                ptx::mbar_arrive(b_desc_full + 8 * d);
            }
            const int c_next = __shfl_sync(0xffffffffu, claimed, 0);
            Q8Chunk ci_next{};
            if (c_next >= 0) {
                ci_next = q8_chunk(p, s_seqs, s_rem, c_next);
                load_pages(ci_next, pg);
            }
            if (n < 0) {
                c = c_next;
                ci = ci_next;
                continue;
            }
            if (n >= R && !wait_spin(b_ch_empty + 8 * (n % R), ((n / R) - 1) & 1, wctx)) break;
            uint8_t *en = entry(n);
            if (c >= 0) {
                int evm = -126;
#pragma unroll
                for (int u = 0; u < kPer; ++u) {
                    evm = max(evm, static_cast<int>(static_cast<int8_t>(ex[u] >> 8)));
                    reinterpret_cast<uint16_t *>(en + C::kEntryEx)[32 * u + lane] = static_cast<uint16_t>(ex[u]);
                }
                evm = __reduce_max_sync(0xffffffffu, evm);
                if (lane == 0) {
                    reinterpret_cast<int *>(en)[1] = evm;
                    *reinterpret_cast<Q8Chunk *>(en + 8) = ci;
                }
                uint8_t *qb = smem + C::kOffQ + (n % R) * C::kQBytes;
#pragma unroll 1
                for (int j0 = 0;;) {
                    uint32_t amax[kAt];
#pragma unroll
                    for (int j = 0; j < kAt; ++j) amax[j] = bf16x8_absmax(qv[j]);
#pragma unroll
                    for (int off = kPieces / 2; off >= 1; off >>= 1)
#pragma unroll
                        for (int j = 0; j < kAt; ++j) amax[j] = max(amax[j], __shfl_xor_sync(0xffffffffu, amax[j], off));
#pragma unroll
                    for (int j = 0; j < kAt; ++j) {
                        const int r = (j0 + j) * kRowsAt + lane / kPieces;
                        const bool bad = amax[j] >= 0x7f80u;  // an infinity or NaN in the row: the row becomes NaN
                        const int eq = bad ? 0 : q8_exponent(amax[j]);
                        uint2 vh, vl;
                        q8_split(qv[j], pow2i(-eq), C::kQSum ? 1.f : 16.f, vh, vl);
                        if (bad) vh = make_uint2(kQ8NanWord, kQ8NanWord);
                        *reinterpret_cast<uint2 *>(qb + row_chunk<HD>(r, pc >> 1) + (pc & 1) * 8) = vh;
                        *reinterpret_cast<uint2 *>(qb + (C::kQSum ? C::kQPart + row_chunk<HD>(r, pc >> 1) : row_chunk<HD>(kNQ / 2 + r, pc >> 1)) +
                                                   (pc & 1) * 8) = vl;
                        if (pc == 0) reinterpret_cast<float *>(en + C::kEntryEq)[r] = pow2i(eq);
                    }
                    if ((j0 += kAt) >= kPasses) break;
                    load_q(ci, j0, qv);
                }
                ptx::fence_proxy_async_smem();
            }
            if (lane == 0) reinterpret_cast<int *>(en)[0] = c;
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(b_ch_full + 8 * (n % R));  // release: the other roles read the entry
            if (c < 0) break;
            c = c_next;
            ci = ci_next;
        }
        ptx::griddep_launch_dependents();  // the merge's blocks come as CTAs end
        // the last scheduler to stop resets the counter for the next launch
        if (lane == 0) {
            __threadfence();
            if (atomicAdd(p.sched + 1, 1) == static_cast<int>(gridDim.x) - 1) {
                p.sched[0] = 0;
                p.sched[1] = 0;
                __threadfence();
            }
        }
    } else if (warp == 13 || warp == 16) {
        // ============================================================ MMA issuers (converged warps; one lane issues)
        const bool is_s = warp == 13;
        constexpr uint32_t kIdS = idesc_e4m3_f32(128, kNQ, false);
        constexpr uint32_t kIdPV = idesc_e4m3_f32(128, C::kNP, true);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint64_t k_desc = row_desc<HD>(sbase, 16);
        const uint64_t q_desc = row_desc<HD>(sbase + C::kOffQ, 16);
        const uint64_t p_desc = weights_desc(sbase + C::kOffP);
        int i = 0;  // tile ordinal in this CTA
        bool ok = true;
        for (int n = 0; ok; ++n) {
            if (!wait_spin(b_ch_full + 8 * (n % R), (n / R) & 1, wctx)) break;
            const int c = reinterpret_cast<volatile int *>(entry(n))[0];
            if (c < 0) break;
            const Q8Chunk *ci = reinterpret_cast<const Q8Chunk *>(entry(n) + 8);
            const int nt = __shfl_sync(0xffffffffu, ci->t1 - ci->t0, 0);
            if (lane == 0) ptx::mbar_arrive(b_ch_empty + 8 * (n % R));
            // the scores, or the O^T, of the chunk before the last have been read
            if (n >= 2 && !wait_spin((is_s ? b_s_free : b_o_free) + 8 * (n & 1), ((n - 2) >> 1) & 1, wctx)) break;
            for (int j = 0; j < nt; ++j, ++i) {
                const int s = i % kQ8Stages;
                if (is_s) {
                    if (!(ok = wait_spin(k_full(s), (i / kQ8Stages) & 1, wctx))) break;
                    ptx::tc_fence_after();
                    const int at = (n & 1) * C::kCT + j;
                    const uint64_t kd = k_desc + s * (C::kTile >> 4);
                    const uint64_t qd = q_desc + (n % R) * (C::kQBytes >> 4);
#pragma unroll
                    for (int part = 0; part < (C::kQSum ? 2 : 1); ++part)
#pragma unroll
                        for (int col = 0; col < HD; col += 32)
                            mma_e4m3_warp(tm + kNQ * at, kd + (col >> 4), qd + ((part * C::kQPart + col) >> 4), kIdS, part + col > 0 ? 1u : 0u);
                    mma_commit_warp(b_s_full + 8 * at);
                } else {
                    // (the weights are written once the scores are complete, so P^T(i) stands for S^T(i) too)
                    if (!(ok = wait_spin(v_full(s), (i / kQ8Stages) & 1, wctx) && wait_spin(b_p_full + 8 * (i & 1), (i >> 1) & 1, wctx))) break;
                    ptx::tc_fence_after();
                    const uint32_t va = sbase + C::kOffV + s * C::kTile;
                    const uint64_t vd = row_desc<HD>(va, HD == 64 ? sbase + C::kOffZero - va : 16);
                    const uint64_t pd = p_desc + (i & 1) * (C::kPBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)  // 32 keys each
                        mma_e4m3_warp(tm + C::kTmemO + C::kNP * (n & 1), vd + (kk * 32 * HD >> 4), pd + (kk * 32 * 16 >> 4), kIdPV,
                                      (j > 0 || kk > 0) ? 1u : 0u);
                    mma_commit_warp(v_empty(s));
                    if (j == nt - 1) mma_commit_warp(b_o_item + 8 * (n & 1));
                }
            }
        }
        // every tcgen05 op of this warp completes before TMEM is released
        const uint32_t b_mine = b_drain + (is_s ? 0 : 8);
        mma_commit_warp(b_mine);
        if (lane == 0) {
            const uint64_t start = ptx::globaltimer();
            while (!ptx::mbar_try_wait(b_mine, 0) && ptx::globaltimer() - start < 4000000ull) {
            }
        }
        __syncwarp();
    } else {
        // ============================================================ maxima (warps 0-3), weights and epilogue (4-11)
        const bool is_max = warp < 4;
        const int t = threadIdx.x & 127;      // key of the tile, or d-column
        const int grp = (warp >> 2) - 1;      // weights: the tiles of ordinal grp mod 2
        const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;  // the TMEM lanes this warp may access
        const int slot = t >> p.log_ps;
        float *s_max = s_red + 12 * 16;       // [2][16], then 8 - them: the largest weight is 2^8
        const int lg = p.log_group;
        // the output, or the partial, of chunk ordinal n, four rows at a time
        auto epilogue = [&](int n) -> bool {
            if (!wait_spin(b_stats + 8 * (n & 1), (n >> 1) & 1, wctx)) return false;
            const float *st = s_stats + (n & 1) * C::kStatsFloats;
            const int c = __float_as_int(st[0]);
            const float scale = st[1];
            const Q8Chunk ci = *reinterpret_cast<const Q8Chunk *>(st + 2);
            if (!wait_spin(b_o_item + 8 * (n & 1), (n >> 1) & 1, wctx)) return false;
            ptx::tc_fence_after();
            const Q8Seq &sq = s_seqs[ci.si];
            const int row0 = ci.blk * RB;
            const int n_rows = min(RB, (sq.n_q << lg) - row0);
            const bool whole = sq.n_full + (sq.rem0 >= 0 ? 1 : 0) == 1;
            float *po = p.part + static_cast<int64_t>(c) * RB * HD + t;
#pragma unroll 1
            for (int r0 = 0; r0 < RB; r0 += 4) {
                const uint32_t to = tmem + C::kTmemO + C::kNP * (n & 1) + r0 + lane_off;
                float o[C::kParts][4];
#pragma unroll
                for (int k = 0; k < C::kParts; ++k) ptx::tmem_ld_n<4>(to + k * RB, o[k]);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int r = r0 + x;
                    float v = o[C::kParts - 1][x];
#pragma unroll
                    for (int k = C::kParts - 2; k >= 0; --k) v = fmaf(v, kQ8Unpart, o[k][x]);
                    v *= scale;
                    if (!whole) {
                        if (t < HD) po[r * HD] = v;
                    } else if (r < n_rows) {
                        const int row = row0 + r;
                        const int64_t at = static_cast<int64_t>(sq.q_row0 + (row >> lg)) * p.hq + (ci.kvh << lg) + (row & ((1 << lg) - 1));
                        const float l = st[8 + RB + r];  // (NaN: the row sees a NaN)
                        if (t < HD && p.out) p.out[at * HD + t] = __float2bfloat16_rn(v * (l > 0.f ? __fdividef(1.0f, l) : l));
                        if (p.lse && t == r) p.lse[at] = st[8 + r] + __log2f(l);
                    }
                }
            }
            if (!whole && t < RB) {
                float *pm = p.part + static_cast<int64_t>(p.total_chunks) * RB * HD + static_cast<int64_t>(c) * RB + t;
                pm[0] = st[8 + t];
                pm[static_cast<int64_t>(p.total_chunks) * RB] = st[8 + RB + t];
            }
            ptx::tc_fence_before();
            ptx::mbar_arrive(b_o_free + 8 * (n & 1));  // O^T buffer and stats slot may be reused
            return true;
        };
        int n = 0;   // chunk ordinal
        int i = 0;   // tile ordinal in this CTA
        bool stopped = false;
        for (;; ++n) {
            // (a wait that gave up is voted on, here and after a chunk's tiles, so that a group leaves together)
            if (!wait_spin(b_ch_full + 8 * (n % R), (n / R) & 1, wctx)) stopped = true;
            if (ptx::bar_sync_or(is_max ? kQ8BarMax : kQ8BarWeights, is_max ? 128 : 256, stopped)) break;
            const uint8_t *en = entry(n);
            const int c = reinterpret_cast<const volatile int *>(en)[0];
            if (c < 0 && is_max) break;
            const int evm = reinterpret_cast<const volatile int *>(en)[1];
            const Q8Chunk ci = c >= 0 ? *reinterpret_cast<const Q8Chunk *>(en + 8) : Q8Chunk{};
            const Q8Seq &sq = s_seqs[ci.si];
            const int row0 = ci.blk * RB;
            const int qpos0 = sq.n_keys - sq.n_q;
            // tiles from this one on hold keys that the block's first row does not see
            const int masked_from = (qpos0 + (row0 >> lg) + 1) / kQ8Keys;
            const float4 *qs = reinterpret_cast<const float4 *>(en + C::kEntryEq);  // four rows' 2^eq
            // s = scores without their scales, of tile j of the chunk; ks, dv: the key's K scale times scale_log2, and
            // its V scale against the chunk's largest
            float s[RB], ks;
            int dv;
            auto load_scores = [&](int j) -> bool {
                const char2 ex = reinterpret_cast<const char2 *>(en + C::kEntryEx)[16 * j + slot];
                ks = pow2i(static_cast<int8_t>(ex.x)) * p.scale_log2;
                dv = max(static_cast<int8_t>(ex.y) - evm, -100);
                const int at = (n & 1) * C::kCT + j;
                if (is_max) {  // (the weights come after the maxima of the whole chunk)
                    if (!wait_spin(b_s_full + 8 * at, (n >> 1) & 1, wctx)) return false;
                    ptx::tc_fence_after();
                }
                ptx::tmem_ld_n<RB>(tmem + kNQ * at + lane_off, s);
                if constexpr (!C::kQSum) {
                    float low[RB];
                    ptx::tmem_ld_n<RB>(tmem + kNQ * at + kNQ / 2 + lane_off, low);
                    ptx::tmem_wait_ld();
#pragma unroll
                    for (int r = 0; r < RB; ++r) s[r] = fmaf(low[r], kQ8Unpart, s[r]);
                } else {
                    ptx::tmem_wait_ld();
                }
                return true;
            };
            auto sees = [&](int key, int r) { return key <= qpos0 + ((row0 + r) >> lg); };
            if (is_max) {
                const int n_rows = min(RB, (sq.n_q << lg) - row0);
                float *sc = p.scores ? p.scores + sq.score0 + (static_cast<int64_t>(ci.kvh) * (sq.n_q << lg) + row0) * sq.score_stride : nullptr;
                float m[RB];
#pragma unroll
                for (int r = 0; r < RB; ++r) m[r] = -INFINITY;
                for (int lt = ci.t0; lt < ci.t1; ++lt) {
                    if (!load_scores(lt - ci.t0)) {
                        stopped = true;
                        break;
                    }
                    const int key = lt * kQ8Keys + t;
                    const float2 fdv = make_float2(static_cast<float>(dv), static_cast<float>(dv)), ks2 = make_float2(ks, ks);
#pragma unroll
                    for (int r = 0; r < RB; r += 4) {
                        const float4 q = qs[r / 4];
                        const float2 x = mul2(make_float2(s[r], s[r + 1]), mul2(ks2, make_float2(q.x, q.y)));
                        const float2 y = mul2(make_float2(s[r + 2], s[r + 3]), mul2(ks2, make_float2(q.z, q.w)));
                        s[r] = x.x;
                        s[r + 1] = x.y;
                        s[r + 2] = y.x;
                        s[r + 3] = y.y;
                    }
                    if (lt >= masked_from) {
#pragma unroll
                        for (int r = 0; r < RB; ++r) s[r] = sees(key, r) && key < sq.n_keys ? s[r] : -INFINITY;
                    }
                    if (sc) {
#pragma unroll
                        for (int r = 0; r < RB; ++r)
                            if (r < n_rows) sc[r * sq.score_stride + key] = s[r];
                    }
#pragma unroll
                    for (int r = 0; r < RB; r += 2) {
                        const float2 y = add2(make_float2(s[r], s[r + 1]), fdv);
                        m[r] = fmaxf(m[r], y.x);  // (a NaN is not taken)
                        m[r + 1] = fmaxf(m[r + 1], y.y);
                    }
                }
                ptx::tc_fence_before();
                if (ptx::bar_sync_or(kQ8BarMax, 128, stopped)) break;
                reduce_rows<RB>(m, [](float x, float y) { return fmaxf(x, y); });
                if (lane % (32 / RB) == 0) s_red[warp * 16 + reduced_row<RB>()] = m[0];
                ptx::bar_sync(kQ8BarMax, 128);
                // (the slot's chunk n - 2 has been read: its scores were freed before this chunk's were computed)
                if (t < RB) {
                    const float x = fmaxf(fmaxf(s_red[t], s_red[16 + t]), fmaxf(s_red[32 + t], s_red[48 + t]));
                    s_max[(n & 1) * 16 + t] = x;
                    s_max[(2 + (n & 1)) * 16 + t] = x == -INFINITY ? 0.f : 8.f - x;
                }
                if (warp == 0) {
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(b_m_full + 8 * (n & 1));  // release: the weights read them
                }
                continue;
            }
            // ------------------------------------------------ weights
            if (c >= 0) {
                stopped = !wait_spin(b_m_full + 8 * (n & 1), (n >> 1) & 1, wctx);
                ptx::tc_fence_after();
                const float my_max = s_max[(n & 1) * 16 + lane % RB];
                const float4 *m8 = reinterpret_cast<const float4 *>(s_max + (2 + (n & 1)) * 16);
                float2 lpart[RB / 2];
#pragma unroll
                for (int r = 0; r < RB / 2; ++r) lpart[r] = make_float2(0.f, 0.f);
                for (int lt = ci.t0; lt < ci.t1 && !stopped; ++lt, ++i) {
                    if ((i & 1) != grp) continue;
                    (void)load_scores(lt - ci.t0);
                    const int key = lt * kQ8Keys + t;
                    const float2 fdv = make_float2(static_cast<float>(dv), static_cast<float>(dv)), ks2 = make_float2(ks, ks);
                    const float2 unv = make_float2(pow2i(-dv), pow2i(-dv));
#pragma unroll
                    for (int r = 0; r < RB; r += 4) {
                        const float4 q = qs[r / 4], m = m8[r / 4];
                        const float2 x = fma2(make_float2(s[r], s[r + 1]), mul2(ks2, make_float2(q.x, q.y)), add2(make_float2(m.x, m.y), fdv));
                        const float2 y = fma2(make_float2(s[r + 2], s[r + 3]), mul2(ks2, make_float2(q.z, q.w)), add2(make_float2(m.z, m.w), fdv));
                        s[r] = ex2(x.x);
                        s[r + 1] = ex2(x.y);
                        s[r + 2] = ex2(y.x);
                        s[r + 3] = ex2(y.y);
                    }
                    if (lt >= masked_from) {
#pragma unroll
                        for (int r = 0; r < RB; ++r)
                            if (!(sees(key, r) && key < sq.n_keys)) s[r] = 0.f;
                    }
#pragma unroll
                    for (int r = 0; r < RB; r += 2) lpart[r / 2] = fma2(make_float2(s[r], s[r + 1]), unv, lpart[r / 2]);
                    // P^T(i) into buffer i & 1 once O^T += V^T P^T(i - 2) has read it
                    if (i >= 2 && !wait_spin(v_empty((i - 2) % kQ8Stages), ((i - 2) / kQ8Stages) & 1, wctx)) {
                        stopped = true;
                        break;
                    }
                    uint32_t pw[C::kNP / 4];  // column part * RB + r of O^T, a byte each
#pragma unroll
                    for (int x = C::kParts * RB / 4; x < C::kNP / 4; ++x) pw[x] = 0u;
#pragma unroll
                    for (int r = 0; r < RB; r += 4) {
                        __half2 w0 = __floats2half2_rn(s[r], s[r + 1]), w1 = __floats2half2_rn(s[r + 2], s[r + 3]);
#pragma unroll
                        for (int part = 0; part < C::kParts; ++part) {
                            const uint32_t q0 = half2_to_e4m3(w0), q1 = half2_to_e4m3(w1);
                            pw[(part * RB + r) / 4] = q0 | q1 << 16;
                            if (part + 1 < C::kParts) {  // 16 (w - part), exact
                                const __half2 up = __float2half2_rn(16.f), down = __float2half2_rn(-16.f);
                                w0 = __hfma2(e4m3_to_half2(q0), down, __hmul2(w0, up));
                                w1 = __hfma2(e4m3_to_half2(q1), down, __hmul2(w1, up));
                            }
                        }
                    }
                    uint4 *pt = reinterpret_cast<uint4 *>(smem + C::kOffP + grp * C::kPBytes) + t;
#pragma unroll
                    for (int x = 0; x < C::kNP / 16; ++x) pt[x * 128] = make_uint4(pw[4 * x], pw[4 * x + 1], pw[4 * x + 2], pw[4 * x + 3]);
                    ptx::fence_proxy_async_smem();
                    ptx::tc_fence_before();
                    ptx::mbar_arrive(b_p_full + 8 * grp);
                }
                // ---------------------------------------------------- row statistics for the epilogue
                float lsum[RB];
#pragma unroll
                for (int r = 0; r < RB; r += 2) {
                    lsum[r] = lpart[r / 2].x;
                    lsum[r + 1] = lpart[r / 2].y;
                }
                reduce_rows<RB>(lsum, [](float x, float y) { return x + y; });
                if (lane % (32 / RB) == 0) s_red[warp * 16 + reduced_row<RB>()] = lsum[0];
                if (ptx::bar_sync_or(kQ8BarWeights, 256, stopped)) break;
                ptx::mbar_arrive(b_s_free + 8 * (n & 1));
                if (warp == 4) {
                    // the stats slot of chunk n - 2 must have been read
                    if (n >= 2) (void)wait_spin(b_o_free + 8 * (n & 1), ((n - 2) >> 1) & 1, wctx);
                    float *st = s_stats + (n & 1) * C::kStatsFloats;
                    if (lane == 31) {
                        st[0] = __int_as_float(c);
                        // 2^(evm - 8), subnormal where the chunk's V is
                        st[1] = evm - 8 >= -126 ? pow2i(evm - 8) : pow2i(evm + 56) * 0x1p-64f;
                        *reinterpret_cast<Q8Chunk *>(st + 2) = ci;
                    }
                    if (lane < RB) {
                        float l = 0.f;
#pragma unroll
                        for (int w = 4; w < 12; ++w) l += s_red[w * 16 + lane];
                        st[8 + lane] = my_max;
                        st[8 + RB + lane] = l * (1.f / 256.f);
                    }
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(b_stats + 8 * (n & 1));  // release: the epilogue reads the slot
                }
                ptx::mbar_arrive(b_ch_empty + 8 * (n % R));  // (warp 4 last: s_red is read)
            }
            // the chunk before, whose O^T is complete by now (or, after the last chunk, will be soon), by the two groups in turn
            if (n >= 1 && ((n - 1) & 1) == grp) stopped = !epilogue(n - 1);
            if (c < 0) break;
        }
    }

    ptx::tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) {
        // after an abort, copies may still be in flight: bounded wait for the last ones issued
        const uint64_t start = ptx::globaltimer();
        for (int ring = 0; ring < 2; ++ring) {
            const int issued = s_issued[ring];
            for (int i = max(0, issued - kQ8Stages); i < issued; ++i) {
                const uint32_t b = ring ? v_full(i % kQ8Stages) : k_full(i % kQ8Stages);
                while (!ptx::mbar_try_wait(b, (i / kQ8Stages) & 1) && ptx::globaltimer() - start < 4000000ull) {
                }
            }
        }
    }
    if (warp == 13) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, C::kTmemCols);
    }
}

template <int HD, int RB>
cudaError_t launch_q8_t(const CUtensorMap &tm_k, const CUtensorMap &tm_v, const Q8AttnParams &p, cudaStream_t st)
{
    using C = Q8Cfg<HD, RB>;
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = set_dyn_smem_once(attn_q8_kernel<HD, RB>, C::kDynSmem, configured);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.total_ctas));
    cfg.blockDim = dim3(kQ8Threads);
    cfg.dynamicSmemBytes = C::kDynSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, attn_q8_kernel<HD, RB>, tm_k, tm_v, p);
    return e != cudaSuccess || !p.any_split ? e : launch_q8_merge<HD, RB>(p, st);
}

}  // namespace

cudaError_t launch_attn_q8(int head_dim, int rows_cap, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                           const Q8AttnParams &p, cudaStream_t st)
{
    if (p.total_ctas <= 0) return cudaSuccess;
    if (head_dim == 128) {
        if (rows_cap == 4) return launch_q8_t<128, 4>(tm_k, tm_v, p, st);
        if (rows_cap == 8) return launch_q8_t<128, 8>(tm_k, tm_v, p, st);
        if (rows_cap == 16) return launch_q8_t<128, 16>(tm_k, tm_v, p, st);
    } else if (head_dim == 64) {
        if (rows_cap == 4) return launch_q8_t<64, 4>(tm_k, tm_v, p, st);
        if (rows_cap == 8) return launch_q8_t<64, 8>(tm_k, tm_v, p, st);
        if (rows_cap == 16) return launch_q8_t<64, 16>(tm_k, tm_v, p, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace pe
