// Attention of up to some hundred query rows a kv-head over the 8-bit cache, on its codes: tcgen05 kind::f8f6f4 with the
// rows on the M side.
//
//     S [128 x 128 keys] = Q8 [128 x d] . K8^T       (A = q from shared memory, B = K codes, K-major)
//     O [128 x d]       += P8 [128 x 128] . V8       (A = weights from TMEM, B = V codes, MN-major)
//
// Blocks of RB = 32, 64 or 128 rows.  The M side holds 128 / RB copies of the block, and copy a's weights are those of
// the a-th part of a tile's keys, zero elsewhere; the copies' outputs add up in the epilogue.  So a row's exponentials
// are spread over all four quarters of the SM whatever RB is.  Two threads hold a lane (of S, P and O), one for each half
// of its keys.
//
// Both factors of a product have eight bits, so q and the weights are split into parts:
//   q   = 2^eq (q_hi + q_lo), e4m3, which add up in the same S: bf16 has eight significant bits, a code four, so this is
//         exact for elements down to 2^-10 of the row's largest (smaller ones err by at most 2^-18 of the largest);
//   p   = p_hi + p_mid + p_low, e5m2, which add up in the same O: the weight as fp16, whose upper byte is an e5m2 number;
//         what it leaves over is fp16 again.  Three significant bits a part, the last one rounded: nine of the weight, and
//         an absolute floor of 2^-17 where the largest weight is 2^kRowsTop.
// The products are exact and accumulate in fp32.
//
// A key's V scale goes into its weight: with ev its page's exponent and evm the largest of the chunk, y = x + ev - evm (x
// the score in log2 units), weight 2^(y - m), sum of weights 2^(evm - ev) times that, O = 2^evm sum weight code.
//
// m, the exponent of the weight 2^kRowsTop, is put kRowsSlack above the largest y of the chunk's first tile, and again of
// every later tile that passes it; then O and the sum so far are scaled, which waits for the tile before's P V.  So the
// floor is 2^-24 of the largest weight.
//
// One pass over the keys for up to 128 rows, where the swap-AB kernel (pe_q8_attn.cu), whose blocks hold at most 16, goes
// through them once for every 16 and for each reads 58 KB of shared memory a tile besides what its warps exchange.  HBM's
// share of a tile is 1390 cycles, its 20 MMAs of 64 cycles are 1280; what bounds is the chain of a tile's steps (scores
// read, maxima exchanged, weights, parts, O scaled): 2200 cycles with 64 rows, of which leaving out any one of the
// loads, MMAs, exponentials, parts and scaling saves 2 to 8 %.  8 sequences of 32k keys and 8 kv-heads, d = 128, with the
// merge: 32 rows 123 us, 64 rows 144 (the swap-AB kernel 286), 128 rows 214; HBM's time for the codes is 79.  Not kept, 64 rows:
// four threads a lane 161; groups that take every other tile and pass the references on 148; the next tile's scores read
// before the parts are stored 153 (128 rows spill, 357); q as an operand in TMEM and six stages 147 (128 rows 211); chunks of
// 28 tiles 149; weights as three e4m3 parts, which need two accumulators, 166.
//
// Roles (512 threads): warps 0-3 and 4-7 weights (lane = thread % 128, the first and second half of its keys), 8-11 q's
// parts and the epilogue, 12 producer, 13 S, 14 P V, 15 scheduler.
#include <algorithm>

#include "q8_chunks.cuh"

namespace pe {

namespace {

constexpr int kRowsThreads = 512;
constexpr int kRowsRing = 3;                 // chunk entries
constexpr int kRowsDesc = 3;                 // chunk descriptors of the producer
constexpr int kRowsDescInts = 8 + 16 * kQ8MaxChunk;
constexpr int kRowsBarVote = 1, kRowsBarEpi = 2, kRowsBarMax = 3;  // named barriers (3 to 6)
constexpr float kRowsTop = 15.f, kRowsSlack = 8.f;

// D[tmem] (+)= A[tmem] * B[smem], A packed four per column
__device__ __forceinline__ void mma_f8_ts_warp(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                                 uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ uint32_t half2_bits(__half2 w) { return *reinterpret_cast<uint32_t *>(&w); }
__device__ __forceinline__ __half2 bits_half2(uint32_t b) { return *reinterpret_cast<__half2 *>(&b); }

template <int HD, int RB>
struct RowsCfg {
    static constexpr int kCopies = 128 / RB;
    static constexpr int kEPT = RB / 2;                          // keys of a tile that a thread holds
    static constexpr int kStages = HD == 128 ? 4 : 6;
    static constexpr int kTile = kQ8Keys * HD;                   // K, then V, of a stage
    static constexpr int kOffQ = 2 * kStages * kTile;
    static constexpr int kQPart = 128 * HD;
    static constexpr int kOffStage = kOffQ + 4 * kQPart;         // two chunks' q, high and low
    static constexpr int kStageRow = 36;                         // floats: 32 columns of a lane's O
    static constexpr int kOffBar = kOffStage + 128 * kStageRow * 4;
    // k_full, v_full, kv_empty [stages]; s_full, s_free, o_item, o_free; p_full, q_full, stats, drain [2];
    // ch_full, ch_empty [ring]; desc_full, desc_empty [kRowsDesc]
    static constexpr int kNumBars = 3 * kStages + 4 + 8 + 2 * kRowsRing + 2 * kRowsDesc;
    static constexpr int kOffMisc = kOffBar + kNumBars * 8;      // tmem slot, abort, tiles issued
    static constexpr int kOffMax = (kOffMisc + 16 + 15) / 16 * 16;  // float [2][256]: the threads' maxima
    static constexpr int kOffEq = kOffMax + 2 * 256 * 4;         // float [2][RB]: 2^eq scale_log2
    static constexpr int kOffL = kOffEq + 2 * RB * 4;            // float [2][256]: the threads' sums of weights
    static constexpr int kOffM = kOffL + 2 * 256 * 4;            // float [2][RB]: the rows' references
    static constexpr int kOffInv = kOffM + 2 * RB * 4;           // float [RB]
    // per ring entry: id, evm, Q8Chunk, -, then (ek, ev) of page slot j of tile k as int8 pairs [k][16]
    static constexpr int kEntryEx = 32;
    static constexpr int kEntryBytes = kEntryEx + kQ8MaxChunk * 32;
    static constexpr int kOffEntry = kOffInv + RB * 4;
    static constexpr int kOffDesc = kOffEntry + kRowsRing * kEntryBytes;
    static constexpr int kOffSeqs = kOffDesc + kRowsDesc * kRowsDescInts * 4;
    static constexpr int kSmem = kOffSeqs + kMaxSegs * static_cast<int>(sizeof(Q8Seq) + 8);
    static constexpr int kDynSmem = kSmem + 1024;
    static constexpr int kTmemP = 128;                           // S at 0; two tiles' three parts of 32 columns
    static constexpr int kTmemO = kTmemP + 2 * 96;
    static constexpr uint32_t kTmemCols = 512;
    static_assert(kTmemO + HD <= static_cast<int>(kTmemCols), "tensor memory");
    static_assert(kOffQ % 1024 == 0 && kQPart % 1024 == 0 && kOffEntry % 16 == 0, "operand alignment");
    static_assert(kDynSmem <= 232448, "shared memory budget");
};

template <int HD, int RB>
__global__ void __launch_bounds__(kRowsThreads, 1)
    attn_q8_rows_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                        const __grid_constant__ Q8AttnParams p)
{
    using C = RowsCfg<HD, RB>;
    constexpr int R = kRowsRing, kS = C::kStages;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    const uint32_t sbase = ptx::smem_addr(smem);
    const uint32_t bar0 = sbase + C::kOffBar;
    auto k_full = [&](int s) { return bar0 + 8u * s; };
    auto v_full = [&](int s) { return bar0 + 8u * (kS + s); };
    auto kv_empty = [&](int s) { return bar0 + 8u * (2 * kS + s); };  // the tile's P V is done: also frees P
    const uint32_t b_s_full = bar0 + 8u * 3 * kS;
    const uint32_t b_s_free = b_s_full + 8;                   // the scores have been read
    const uint32_t b_p_full = b_s_free + 8;                   // [2]
    const uint32_t b_o_item = b_p_full + 16;                  // a chunk's O is complete
    const uint32_t b_o_free = b_o_item + 8;                   // the epilogue has read it
    const uint32_t b_q_full = b_o_free + 8;                   // [2] a chunk's q parts and 2^eq
    const uint32_t b_stats = b_q_full + 16;                   // [2] a chunk's references and sums
    const uint32_t b_drain = b_stats + 16;                    // [2] S, P V
    const uint32_t b_ch_full = b_drain + 16;                  // [R] a chunk's id and scales are in its entry
    const uint32_t b_ch_empty = b_ch_full + 8 * R;            // [R]
    const uint32_t b_desc_full = b_ch_empty + 8 * R;          // [kRowsDesc] a chunk's TMA rows
    const uint32_t b_desc_empty = b_desc_full + 8 * kRowsDesc;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + C::kOffMisc + 4);
    volatile int *s_issued = reinterpret_cast<volatile int *>(smem + C::kOffMisc + 8);
    float *s_max = reinterpret_cast<float *>(smem + C::kOffMax);
    float *s_eq = reinterpret_cast<float *>(smem + C::kOffEq);
    float *s_l = reinterpret_cast<float *>(smem + C::kOffL);
    float *s_m = reinterpret_cast<float *>(smem + C::kOffM);
    Q8Seq *s_seqs = reinterpret_cast<Q8Seq *>(smem + C::kOffSeqs);
    int2 *s_rem = reinterpret_cast<int2 *>(smem + C::kOffSeqs + kMaxSegs * sizeof(Q8Seq));
    int *s_desc = reinterpret_cast<int *>(smem + C::kOffDesc);
    auto entry = [&](int n) { return smem + C::kOffEntry + (n % R) * C::kEntryBytes; };
    const WaitCtx wctx{abort_flag, p.status};

    if (threadIdx.x == 384) {
        for (int s = 0; s < kS; ++s) {
            ptx::mbar_init(k_full(s), 1);
            ptx::mbar_init(v_full(s), 1);
            ptx::mbar_init(kv_empty(s), 1);
        }
        ptx::mbar_init(b_s_full, 1);
        ptx::mbar_init(b_s_free, 8);
        ptx::mbar_init(b_o_item, 1);
        ptx::mbar_init(b_o_free, 4);
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(b_p_full + 8 * b, 8);
            ptx::mbar_init(b_q_full + 8 * b, 4);
            ptx::mbar_init(b_stats + 8 * b, 8);
            ptx::mbar_init(b_drain + 8 * b, 1);
        }
        for (int r = 0; r < R; ++r) {
            ptx::mbar_init(b_ch_full + 8 * r, 1);
            ptx::mbar_init(b_ch_empty + 8 * r, 2 + 8 + 4);  // MMA warps, weights, epilogue
        }
        for (int d = 0; d < kRowsDesc; ++d) {
            ptx::mbar_init(b_desc_full + 8 * d, 1);
            ptx::mbar_init(b_desc_empty + 8 * d, 1);
        }
        *abort_flag = 0;
        *s_issued = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&tm_k);
        ptx::prefetch_tensormap(&tm_v);
    }
    if (warp == 13) {
        ptx::tmem_alloc(ptx::smem_addr(tmem_slot), C::kTmemCols);
        ptx::tmem_relinquish();
    }
    if (warp < 8) {
        const int n_words = p.n_seqs * static_cast<int>(sizeof(Q8Seq) / 4);
        const int32_t *src = reinterpret_cast<const int32_t *>(p.seqs);
        for (int e = threadIdx.x; e < n_words; e += 256) reinterpret_cast<int32_t *>(s_seqs)[e] = src[e];
        for (int e = threadIdx.x; e < p.n_rem; e += 256) s_rem[e] = make_int2(p.seqs[p.rem_seq[e]].rem0, p.rem_seq[e]);
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (warp < 4) {  // the weights of keys that are not a copy's stay zero
        const float zero[32] = {};
        for (int k = 0; k < 6; ++k) ptx::tmem_st32(tmem + C::kTmemP + 32 * k + (static_cast<uint32_t>(warp * 32) << 16), zero);
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
    }
    __syncthreads();
    ptx::tc_fence_after();
    // Launched with programmatic serialization: nothing written by earlier kernels is read before this point.
    ptx::griddep_wait();

    if (warp == 12) {
        // ============================================================ producer
        const int n_boxes = kQ8Keys / p.ps;  // a page a box
        const bool is_v = lane >= 16;
        const CUtensorMap *map = is_v ? &tm_v : &tm_k;
        const int box = lane & 15;
        int i = 0;                           // tile ordinal in this CTA
        for (int n = 0;; ++n) {
            const int d = n % kRowsDesc;
            if (!wait_spin(b_desc_full + 8 * d, (n / kRowsDesc) & 1, wctx)) break;
            const int *desc = s_desc + d * kRowsDescInts;
            if (desc[0] < 0) break;  // no more chunks
            const int nt = desc[1];
            bool ok = true;
            for (int k = 0; k < nt; ++k, ++i) {
                const int s = i % kS;
                if (i >= kS && !(ok = wait_spin(kv_empty(s), ((i / kS) - 1) & 1, wctx))) break;
                if (box == 0) ptx::mbar_arrive_expect_tx(is_v ? v_full(s) : k_full(s), C::kTile);
                __syncwarp();
                if (box < n_boxes)
                    ptx::tma_load_2d(sbase + (2 * s + (is_v ? 1 : 0)) * C::kTile + box * p.ps * HD, map, 0, desc[8 + 16 * k + box],
                                     is_v ? v_full(s) : k_full(s));
                __syncwarp();
                if (lane == 0) *s_issued = i + 1;
            }
            if (!ok) break;
            if (lane == 0) ptx::mbar_arrive(b_desc_empty + 8 * d);
        }
    } else if (warp == 15) {
        // ============================================================ scheduler
        const int lps = p.log_ps;
        const int n_slots = kQ8Keys >> lps;  // <= 16
        constexpr int kPer = kQ8MaxChunk / 2;
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
        // the next chunk's loads are in flight while this one's are used
        int c = 0;  // (round -1 only takes the first)
        Q8Chunk ci{};
        int pg[kPer];
        for (int n = -1;; ++n) {
            const int d = n % kRowsDesc;
            const int claimed = c >= 0 ? claim(n + 1) : -1;
            if (n >= kRowsDesc && !wait_spin(b_desc_empty + 8 * d, ((n / kRowsDesc) - 1) & 1, wctx)) c = -1;
            int *desc = s_desc + d * kRowsDescInts;
            int ex[kPer];  // (ek, ev)
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
                if (lane == 0) ptx::mbar_arrive(b_desc_full + 8 * d);  // release: the producer reads the rows
#pragma unroll
                for (int u = 0; u < kPer; ++u)
                    ex[u] = pg[u] >= 0 ? reinterpret_cast<const uint16_t *>(p.exps)[pg[u]] : 0x8282;  // -126, -126
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
    } else if (warp == 13 || warp == 14) {
        // ============================================================ MMA issuers (converged warps; one lane issues)
        const bool is_s = warp == 13;
        constexpr uint32_t kIdS = idesc_e4m3_f32(128, kQ8Keys, false);
        constexpr uint32_t kIdPV = idesc_e4m3_f32(128, HD, false) | (1u << 7) | (1u << 16);  // A e5m2, B MN-major
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        int i = 0;  // tile ordinal in this CTA
        bool ok = true;
        for (int n = 0; ok; ++n) {
            if (!wait_spin(b_ch_full + 8 * (n % R), (n / R) & 1, wctx)) break;
            const int c = reinterpret_cast<volatile int *>(entry(n))[0];
            if (c < 0) break;
            const Q8Chunk *ci = reinterpret_cast<const Q8Chunk *>(entry(n) + 8);
            const int nt = __shfl_sync(0xffffffffu, ci->t1 - ci->t0, 0);
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(b_ch_empty + 8 * (n % R));
            // the chunk's q; or the O of the chunk before has been read
            if (is_s ? !wait_spin(b_q_full + 8 * (n & 1), (n >> 1) & 1, wctx) : n >= 1 && !wait_spin(b_o_free, (n - 1) & 1, wctx)) break;
            const uint64_t qd = row_desc<HD>(sbase + C::kOffQ + (n & 1) * 2 * C::kQPart, 16);
            for (int j = 0; j < nt; ++j, ++i) {
                const int s = i % kS;
                if (is_s) {
                    if (!(ok = wait_spin(k_full(s), (i / kS) & 1, wctx) && (i < 1 || wait_spin(b_s_free, (i - 1) & 1, wctx)))) break;
                    ptx::tc_fence_after();
                    const uint64_t kd = row_desc<HD>(sbase + 2 * s * C::kTile, 16);
#pragma unroll
                    for (int part = 0; part < 2; ++part)
#pragma unroll
                        for (int col = 0; col < HD; col += 32)
                            mma_e4m3_warp(tm, qd + ((part * C::kQPart + col) >> 4), kd + (col >> 4), kIdS, part + col > 0 ? 1u : 0u);
                    mma_commit_warp(b_s_full);
                } else {
                    if (!(ok = wait_spin(v_full(s), (i / kS) & 1, wctx) && wait_spin(b_p_full + 8 * (i & 1), (i >> 1) & 1, wctx))) break;
                    ptx::tc_fence_after();
                    const uint64_t vd = row_desc<HD>(sbase + (2 * s + 1) * C::kTile, 16);
#pragma unroll
                    for (int part = 0; part < 3; ++part)
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)  // 32 keys each
                            mma_f8_ts_warp(tm + C::kTmemO, tm + C::kTmemP + 96 * (i & 1) + 32 * part + 8 * kk, vd + (kk * 32 * HD >> 4), kIdPV,
                                           (j > 0 || kk > 0 || part > 0) ? 1u : 0u);
                    mma_commit_warp(kv_empty(s));
                    if (j == nt - 1) mma_commit_warp(b_o_item);
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
    } else if (warp >= 8) {
        // ============================================================ q's parts, epilogue (thread = lane of O)
        const int t = threadIdx.x & 127;
        const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const int lg = p.log_group;
        float *stage = reinterpret_cast<float *>(smem + C::kOffStage);
        float *s_inv = reinterpret_cast<float *>(smem + C::kOffInv);
        bool stopped = false, ended = false;
        // q of chunk ordinal n in parts, for every copy; its buffer is free: the O of chunk n - 2 is complete
        auto prepare = [&](int n) {
            if (ended) return;
            if (!wait_spin(b_ch_full + 8 * (n % R), (n / R) & 1, wctx)) stopped = true;
            stopped = ptx::bar_sync_or(kRowsBarEpi, 128, stopped);
            const uint8_t *en = entry(n);
            if (stopped || reinterpret_cast<const volatile int *>(en)[0] < 0) {
                ended = true;
                return;
            }
            const Q8Chunk ci = *reinterpret_cast<const Q8Chunk *>(en + 8);
            const Q8Seq &sq = s_seqs[ci.si];
            constexpr int kPieces = HD / 8;            // of a row, eight columns each
            constexpr int kRowsAt = 128 / kPieces, kAt = 4;
            const int pc = t % kPieces;
            uint8_t *qb = smem + C::kOffQ + (n & 1) * 2 * C::kQPart;
#pragma unroll 1
            for (int j0 = 0; j0 < RB / kRowsAt; j0 += kAt) {
                uint4 qv[kAt];
#pragma unroll
                for (int j = 0; j < kAt; ++j) {
                    const int r = (j0 + j) * kRowsAt + t / kPieces, row = ci.blk * RB + r;
                    qv[j] = make_uint4(0u, 0u, 0u, 0u);
                    if (r < RB && row < sq.n_q << lg)
                        qv[j] = *reinterpret_cast<const uint4 *>(
                            p.q + (static_cast<int64_t>(sq.q_row0 + (row >> lg)) * p.hq + (ci.kvh << lg) + (row & ((1 << lg) - 1))) * HD + pc * 8);
                }
#pragma unroll
                for (int j = 0; j < kAt; ++j) {
                    const int r = (j0 + j) * kRowsAt + t / kPieces;
                    uint32_t amax = bf16x8_absmax(qv[j]);
#pragma unroll
                    for (int off = kPieces / 2; off >= 1; off >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, off));
                    const bool bad = amax >= 0x7f80u;  // an infinity or NaN in the row: the row becomes NaN
                    const int eq = bad ? 0 : q8_exponent(amax);
                    uint2 vh, vl;
                    q8_split(qv[j], pow2i(-eq), 1.f, vh, vl);
                    if (bad) vh = make_uint2(kQ8NanWord, kQ8NanWord);
                    if (r < RB) {
#pragma unroll
                        for (int a = 0; a < C::kCopies; ++a) {
                            uint8_t *at = qb + row_chunk<HD>(a * RB + r, pc >> 1) + (pc & 1) * 8;
                            *reinterpret_cast<uint2 *>(at) = vh;
                            *reinterpret_cast<uint2 *>(at + C::kQPart) = vl;
                        }
                        if (pc == 0) s_eq[(n & 1) * RB + r] = pow2i(eq) * p.scale_log2;
                    }
                }
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(b_q_full + 8 * (n & 1));
        };
        int last = -1;  // the last chunk prepared
        for (int n = 0;; ++n) {
            while (!ended && last < n + 1) {
                prepare(last + 1);
                if (!ended) ++last;
            }
            if (n > last) break;
            const uint8_t *en = entry(n);
            const int c = reinterpret_cast<const int *>(en)[0], evm = reinterpret_cast<const int *>(en)[1];
            const Q8Chunk ci = *reinterpret_cast<const Q8Chunk *>(en + 8);
            const Q8Seq &sq = s_seqs[ci.si];
            const int row0 = ci.blk * RB;
            const int n_rows = min(RB, (sq.n_q << lg) - row0);
            const int out_rows = p.out ? n_rows : 0;  // (no output: the log-sum-exp alone is asked for)
            const bool whole = sq.n_full + (sq.rem0 >= 0 ? 1 : 0) == 1;
            auto out_row = [&](int r) {  // of row r of the block
                const int row = row0 + r;
                return static_cast<int64_t>(sq.q_row0 + (row >> lg)) * p.hq + (ci.kvh << lg) + (row & ((1 << lg) - 1));
            };
            // 2^(evm - kRowsTop), subnormal where the chunk's V is
            constexpr int kTop = static_cast<int>(kRowsTop);
            const float scale = evm - kTop >= -126 ? pow2i(evm - kTop) : pow2i(evm - kTop + 64) * 0x1p-64f;
            if (!wait_spin(b_stats + 8 * (n & 1), (n >> 1) & 1, wctx)) stopped = true;
            if (!wait_spin(b_o_item, n & 1, wctx)) stopped = true;
            if (ptx::bar_sync_or(kRowsBarEpi, 128, stopped)) break;
            ptx::tc_fence_after();
            if (t < RB) {
                float l = 0.f;
#pragma unroll
                for (int a = 0; a < 2 * C::kCopies; ++a) l += s_l[(n & 1) * 256 + a * RB + t];
                l *= 1.f / (1 << static_cast<int>(kRowsTop));
                const float m = s_m[(n & 1) * RB + t];
                s_inv[t] = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);  // (NaN: the row sees a NaN)
                if (!whole) {
                    float *pm = p.part + static_cast<int64_t>(p.total_chunks) * RB * HD + static_cast<int64_t>(c) * RB + t;
                    pm[0] = m;
                    pm[static_cast<int64_t>(p.total_chunks) * RB] = l;
                } else if (p.lse && t < n_rows) {
                    p.lse[out_row(t)] = m + __log2f(l);
                }
            }
#pragma unroll 1
            for (int x = 0; x < HD; x += 32) {
                float o[32];
                ptx::tmem_ld32(tmem + C::kTmemO + x + lane_off, o);
                ptx::tmem_wait_ld();
                if (x == HD - 32) {
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(b_o_free);
                }
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                    *reinterpret_cast<float4 *>(stage + t * C::kStageRow + k) =
                        make_float4(o[k] * scale, o[k + 1] * scale, o[k + 2] * scale, o[k + 3] * scale);
                ptx::bar_sync(kRowsBarEpi, 128);
#pragma unroll 4
                for (int r = t / 8; r < out_rows; r += 16) {
                    const int col = t % 8 * 4;
                    float4 v = *reinterpret_cast<const float4 *>(stage + r * C::kStageRow + col);
#pragma unroll
                    for (int a = 1; a < C::kCopies; ++a) {
                        const float4 w = *reinterpret_cast<const float4 *>(stage + (a * RB + r) * C::kStageRow + col);
                        v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
                    }
                    if (!whole) {
                        *reinterpret_cast<float4 *>(p.part + (static_cast<int64_t>(c) * RB + r) * HD + x + col) = v;
                    } else {
                        const float inv = s_inv[r];
                        *reinterpret_cast<uint2 *>(p.out + out_row(r) * HD + x + col) =
                            make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
                    }
                }
                ptx::bar_sync(kRowsBarEpi, 128);
            }
            if (lane == 0) ptx::mbar_arrive(b_ch_empty + 8 * (n % R));
        }
    } else {
        // ============================================================ weights
        const int t = threadIdx.x;            // 0..255
        const int L = t & 127, r = L % RB;    // lane, row of the block
        const int key0 = L / RB * RB + (t >> 7) * C::kEPT;  // first key of a tile that the thread holds (copy's part: RB keys)
        const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const int lg = p.log_group;
        constexpr int kSub = C::kEPT < 32 ? C::kEPT : 32;   // keys at a time
        constexpr int kShare = RB / 32;       // warps of a row: those of its lanes in every copy, 8 / kShare
        int i = 0;                            // tile ordinal
        bool stopped = false;
        for (int n = 0;; ++n) {
            // (a wait that gave up is voted on, so that all leave together)
            if (!wait_spin(b_ch_full + 8 * (n % R), (n / R) & 1, wctx)) stopped = true;
            if (ptx::bar_sync_or(kRowsBarVote, 256, stopped)) break;
            const uint8_t *en = entry(n);
            if (reinterpret_cast<const volatile int *>(en)[0] < 0) break;
            const int evm = reinterpret_cast<const volatile int *>(en)[1];
            const Q8Chunk ci = *reinterpret_cast<const Q8Chunk *>(en + 8);
            const Q8Seq &sq = s_seqs[ci.si];
            const int row0 = ci.blk * RB;
            const int seen0 = sq.n_keys - sq.n_q + 1;  // keys that query 0 sees
            const int seen = row0 + r < sq.n_q << lg ? seen0 + ((row0 + r) >> lg) : 0;
            const int masked_from = (seen0 + (row0 >> lg)) / kQ8Keys;
            if (!wait_spin(b_q_full + 8 * (n & 1), (n >> 1) & 1, wctx)) stopped = true;
            const float qs = s_eq[(n & 1) * RB + r];
            float m = -INFINITY, l = 0.f;  // (-inf: the row has seen no key)
            for (int lt = ci.t0; lt < ci.t1; ++lt, ++i) {
                const uint16_t *ex = reinterpret_cast<const uint16_t *>(en + C::kEntryEx) + 16 * (lt - ci.t0);
                const int left = lt >= masked_from ? seen - lt * kQ8Keys - key0 : 1 << 30;  // of the thread's keys, those the row sees
                if (!wait_spin(b_s_full, i & 1, wctx)) stopped = true;
                ptx::tc_fence_after();
                float y[C::kEPT];
#pragma unroll
                for (int at = 0; at < C::kEPT; at += kSub) {
                    float v[kSub];
                    if constexpr (kSub == 32) ptx::tmem_ld32(tmem + lane_off + key0 + at, v);
                    else ptx::tmem_ld_n<16>(tmem + lane_off + key0 + at, v);
#pragma unroll
                    for (int x = 0; x < kSub; ++x) y[at + x] = v[x];
                }
                ptx::tmem_wait_ld();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(b_s_free);
                // of eight keys from `at`: the factor of their scores, and their V exponent against the chunk's largest
                auto exps = [&](int at) { return static_cast<uint32_t>(ex[(key0 + at) >> p.log_ps]); };
                auto v_exp = [&](uint32_t e) { return max(static_cast<int8_t>(e >> 8) - evm, -100); };
                float mx = -INFINITY;
#pragma unroll
                for (int at = 0; at < C::kEPT; at += 8) {
                    const uint32_t e = exps(at);
                    const float f = pow2i(static_cast<int8_t>(e & 255u)) * qs, dv = static_cast<float>(v_exp(e));
#pragma unroll
                    for (int x = at; x < at + 8; x += 2) {
                        const float2 z = fma2(make_float2(y[x], y[x + 1]), make_float2(f, f), make_float2(dv, dv));
                        y[x] = z.x;
                        y[x + 1] = z.y;
                    }
                }
                if (left < C::kEPT) {
#pragma unroll
                    for (int x = 0; x < C::kEPT; ++x) y[x] = x < left ? y[x] : -INFINITY;
                }
#pragma unroll
                for (int x = 0; x < C::kEPT; x += 2) mx = max3(mx, y[x], y[x + 1]);  // (a NaN is not taken)
                // the rows' references, if this tile passes them
                float *mine = s_max + (i & 1) * 256;
                mine[t] = mx;
                ptx::bar_sync(kRowsBarMax + (warp & 3) % kShare, 256 / kShare);
#pragma unroll
                for (int a = 0; a < 2 * C::kCopies; ++a) mx = fmaxf(mx, mine[a * RB + r]);
                float f = 1.f;
                if (mx > m) {
                    if (lt + 1 < ci.t1) mx += kRowsSlack;
                    f = m == -INFINITY ? 0.f : ex2(m - mx);
                    m = mx;
                    l *= f;
                }
                __half2 w[C::kEPT / 2];
                const float ref = m == -INFINITY ? 0.f : kRowsTop - m;
                const float2 off = make_float2(ref, ref);
#pragma unroll
                for (int at = 0; at < C::kEPT; at += 8) {
                    float2 acc = make_float2(0.f, 0.f);
#pragma unroll
                    for (int x = at; x < at + 8; x += 2) {
                        float2 z = add2(make_float2(y[x], y[x + 1]), off);
                        z = make_float2(ex2(z.x), ex2(z.y));
                        acc = add2(acc, z);
                        w[x / 2] = __floats2half2_rn(z.x, z.y);
                    }
                    l = fmaf(acc.x + acc.y, pow2i(-v_exp(exps(at))), l);
                }
                float word[3][C::kEPT / 4];
#pragma unroll
                for (int x = 0; x < C::kEPT / 4; ++x) {
                    __half2 a = w[2 * x], b = w[2 * x + 1];
#pragma unroll
                    for (int part = 0; part < 3; ++part) {
                        const uint32_t half_ulp = part == 2 ? 0x00800080u : 0u;
                        word[part][x] = __uint_as_float(__byte_perm(half2_bits(a) + half_ulp, half2_bits(b) + half_ulp, 0x7531));
                        a = __hsub2(a, bits_half2(half2_bits(a) & 0xff00ff00u));  // exact
                        b = __hsub2(b, bits_half2(half2_bits(b) & 0xff00ff00u));
                    }
                }
                // O holds the tile before; or P V of the tile before that has read its weights
                const bool scaled = lt > ci.t0 && __any_sync(0xffffffffu, f != 1.f);
                const int done = i - (scaled ? 1 : 2);
                if (done >= 0 && !wait_spin(kv_empty(done % kS), (done / kS) & 1, wctx)) stopped = true;
                ptx::tc_fence_after();
#pragma unroll
                for (int part = 0; part < 3; ++part)
                    ptx::tmem_st_n<C::kEPT / 4>(tmem + C::kTmemP + 96 * (i & 1) + 32 * part + key0 / 4 + lane_off, word[part]);
                if (scaled) {
                    constexpr int kN = HD / 64;  // half of O each of the lane's two threads
                    const uint32_t at = tmem + C::kTmemO + (t >> 7) * (HD / 2) + lane_off;
                    float o[kN][32];
#pragma unroll
                    for (int x = 0; x < kN; ++x) ptx::tmem_ld32(at + 32 * x, o[x]);
                    ptx::tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < kN; ++x) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[x][k] *= f;
                        ptx::tmem_st32(at + 32 * x, o[x]);
                    }
                }
                ptx::tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(b_p_full + 8 * (i & 1));
            }
            s_l[(n & 1) * 256 + t] = l;
            if (t < RB) s_m[(n & 1) * RB + t] = m;
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive(b_stats + 8 * (n & 1));
                ptx::mbar_arrive(b_ch_empty + 8 * (n % R));
            }
        }
    }

    ptx::tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) {
        // after an abort, copies may still be in flight: bounded wait for the last ones issued
        const uint64_t start = ptx::globaltimer();
        const int issued = *s_issued;
        for (int i = max(0, issued - kS); i < issued; ++i)
            for (int v = 0; v < 2; ++v) {
                const uint32_t b = v ? v_full(i % kS) : k_full(i % kS);
                while (!ptx::mbar_try_wait(b, (i / kS) & 1) && ptx::globaltimer() - start < 4000000ull) {
                }
            }
    }
    if (warp == 13) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, C::kTmemCols);
    }
}

template <int HD, int RB>
cudaError_t launch_rows_t(const CUtensorMap &tm_k, const CUtensorMap &tm_v, const Q8AttnParams &p, cudaStream_t st)
{
    using C = RowsCfg<HD, RB>;
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = set_dyn_smem_once(attn_q8_rows_kernel<HD, RB>, C::kDynSmem, configured);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.total_ctas));
    cfg.blockDim = dim3(kRowsThreads);
    cfg.dynamicSmemBytes = C::kDynSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, attn_q8_rows_kernel<HD, RB>, tm_k, tm_v, p);
    return e != cudaSuccess || !p.any_split ? e : launch_q8_merge<HD, RB>(p, st);
}

}  // namespace

cudaError_t launch_attn_q8_rows(int head_dim, int rows_cap, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                                const Q8AttnParams &p, cudaStream_t st)
{
    if (p.total_ctas <= 0) return cudaSuccess;
    if (head_dim == 128) {
        if (rows_cap == 32) return launch_rows_t<128, 32>(tm_k, tm_v, p, st);
        if (rows_cap == 64) return launch_rows_t<128, 64>(tm_k, tm_v, p, st);
        if (rows_cap == 128) return launch_rows_t<128, 128>(tm_k, tm_v, p, st);
    } else if (head_dim == 64) {
        if (rows_cap == 32) return launch_rows_t<64, 32>(tm_k, tm_v, p, st);
        if (rows_cap == 64) return launch_rows_t<64, 64>(tm_k, tm_v, p, st);
        if (rows_cap == 128) return launch_rows_t<64, 128>(tm_k, tm_v, p, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace pe
