// Private to the pe library: kernel parameter blocks shared by the host code
// (pe_host.cu) and the kernels (pe_kv.cu, pe_attn.cu).
#pragma once

#include <atomic>
#include <cstdint>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

namespace pe {

constexpr int kBM = 128;               // query rows (GQA-packed) per attention tile
constexpr int kBN = 128;               // keys per attention tile
constexpr int kMaxSegs = 64;           // sequences per append / attention launch
constexpr int kMaxCropSegs = 256;      // sequences per crop launch
constexpr int kAppendMaxPages = 3072;  // new page ids carried by one append launch

// Device status word codes (pe_device_status).
constexpr int kStatusWaitTimeout = 1;
constexpr int kStatusBadPage = 2;      // page id outside the pool
constexpr int kStatusBadPlan = 3;      // the persistent kernel met a partial slot outside its workspace (skipped)

// ---------------------------------------------------------------- append
struct AppendSeg {
    int32_t tok0;          // first token of this segment inside the packed K/V
    int32_t cum0;          // prefix of segment tokens inside this launch
    int32_t n_tokens;
    int32_t len0;          // sequence length before this segment
    int32_t first_new_lp;  // logical index of the first page popped for this segment
    int32_t last_page;     // physical page holding logical page first_new_lp-1 (-1 if none)
    int32_t new0;          // offset of this segment's new page ids in new_pages
    int32_t n_new;
    int32_t table_row;     // seq * max_pages_per_seq
    int32_t seq;
};

template <int SEGS, int PAGES>
struct AppendParamsT {
    const uint4 *K;        // packed [L][n_total][Hkv][d] bf16, viewed as 16-byte chunks
    const uint4 *V;
    uint4 *k_pool;         // [L][num_pages][Hkv][ps][d]
    uint4 *v_pool;
    int32_t *page_table;   // device mirror [max_seqs][max_pages_per_seq]
    int64_t *seq_len;      // device mirror [max_seqs]
    int32_t L, hkv, dvec, ps, num_pages, n_total, n_segs, seg_tokens;
    int32_t n_new;         // page ids carried
    int32_t beside;        // 1: runs beside the decode merge launched just before (append_kv_kernel)
    int8_t *exps;          // 8-bit cache: scale exponents [L][num_pages][Hkv][2] (K, V); the pools hold codes
    AppendSeg segs[SEGS];
    int32_t new_pages[PAGES];
};
using AppendParams = AppendParamsT<kMaxSegs, kAppendMaxPages>;

// ---------------------------------------------------------------- copy-on-write
struct CowCopy {
    int32_t src, dst;      // pages
    int32_t slots;         // valid slots of the shared page
    int32_t entry;         // index of the device table entry to point at dst
};

struct CowParams {
    uint4 *k_pool;
    uint4 *v_pool;
    int8_t *exps;          // 8-bit cache: scale exponents, copied too (else null)
    int32_t *page_table;
    int32_t n, L, hkv, ps, dvec, num_pages;
    CowCopy copies[kMaxSegs];
};

// ---------------------------------------------------------------- 8-bit cache
struct UnpackSeg {
    int32_t table_row;     // seq * max_pages_per_seq
    int32_t page0;         // prefix of pages inside this launch
};

// One layer's codes of the listed sequences' pages as bf16, at the same page ids.
struct UnpackParams {
    const int32_t *page_table;
    const uint4 *k8, *v8;  // codes [L][num_pages][Hkv][ps][d]
    const int8_t *exps;    // [L][num_pages][Hkv][2]
    uint4 *k, *v;          // bf16 [num_pages][Hkv][ps][d]
    int32_t n, layer, hkv, ps, d, num_pages;
    UnpackSeg segs[kMaxSegs];
};

struct ReadSeg {
    int32_t table_row;
    int32_t begin, end;    // tokens read
    int32_t page0;         // prefix of touched pages inside this launch
    int32_t tok0;          // first row of K / V
};

struct ReadParams {
    const int32_t *page_table;
    const void *k_pool, *v_pool;
    const int8_t *exps;    // 8-bit cache only
    uint4 *K, *V;          // bf16 [L][n_total][Hkv][d]
    int32_t n, L, hkv, ps, log_ps, d, num_pages, n_total, pages;
    ReadSeg segs[kMaxSegs];
};

// Stored pages, codes and scales of all layers, copied out or back: a slot a page.
constexpr int kMaxSavedPages = 512;    // of one launch
struct SaveParams {
    uint4 *k8, *v8;
    int8_t *exps;
    uint8_t *slots;        // page i: K codes [L][Hkv][ps][d], V codes, exponents [L][Hkv][2], from i * slot_bytes on
    int64_t slot_bytes;
    int32_t n, L, hkv, ps, d, num_pages;
    int32_t back;          // 1: from the slots into the pages
    int32_t pages[kMaxSavedPages];
};

// Attention of few rows on the codes (pe_q8_attn.cu, pe_q8_rows.cu): items are (sequence, kv-head, block of query rows).
constexpr int kQ8MaxChunk = 14;        // key tiles (128 keys) of a chunk, and with blocks of rb rows:
__host__ __device__ constexpr int q8_max_chunk(int rb) { return rb == 16 ? 12 : 14; }

struct Q8Seq {
    int32_t table_row;     // seq * max_pages_per_seq
    int32_t q_row0, n_q;   // rows of Q / out
    int32_t n_keys;        // the last query sees all of them
    int32_t n_blocks;      // of n_q x group rows
    int32_t ct;            // tiles per full chunk
    int32_t n_full;        // full chunks
    uint32_t blocks_inv, full_inv;  // ceil(2^32 / n_blocks), ceil(2^32 / n_full) (for more than one)
    int32_t full0;         // first full chunk id: full0 + (kv-head * nfull + k) * n_blocks + block
    int32_t rem0;          // first remainder chunk id (rem0 + kv-head * n_blocks + block), -1: none
    int32_t item0;         // first item (merge): item0 + kv-head * n_blocks + block
    int32_t score_stride;  // scores: of a row, a multiple of 128
    int32_t pad_;
    int64_t score0;        // scores: first row (kv-head * n_q x group + row)
};

struct Q8AttnParams {
    const int32_t *page_table;
    const __nv_bfloat16 *q;  // bf16 [rows][Hq][d]
    __nv_bfloat16 *out;      // the same, or null
    const int8_t *exps;      // [L][num_pages][Hkv][2]
    float *part;             // partials: O [chunks][RB][d], then m [chunks][RB], then l [chunks][RB]
    float *lse;              // null, or log2-sum-exp [rows][Hq]
    float *scores;           // null, or every row's scores in log2 units (-inf: not seen)
    int32_t *sched;          // [0] next chunk, [1] CTAs that stopped taking; zero between launches
    int32_t *status;
    int32_t n_seqs, hq, hkv, group, log_group, layer, num_pages, ps, log_ps;
    int32_t oob_row;         // a pool row past the end: boxes there read zeros
    int32_t full_chunks, total_chunks, total_items, total_ctas, any_split, n_rem;
    int32_t max_chunks;      // of an item
    float scale_log2;        // softmax_scale * log2(e)
    Q8Seq seqs[kMaxSegs];
    int32_t rem_seq[kMaxSegs];  // sequences with remainder chunks, longest remainder first
};

// ---------------------------------------------------------------- eviction
struct EvictSeg {
    int32_t row;           // of weights and kept
    int32_t seq, table_row;
    int32_t len, keep;     // tokens before and after
    int32_t sinks, recent;
    int32_t first_lp;      // logical index of the first new page in this launch
    int32_t new0, n_new;   // this launch's new pages of the sequence, in new_pages
};

// What the finish of an eviction of several groups needs of a sequence: device memory, one a row of weights and kept.
struct EvictDone {
    int32_t seq, len, keep, pad_;
};

template <int SEGS, int PAGES>
struct EvictParamsT {
    int32_t *page_table;
    int64_t *seq_len;
    void *k_pool, *v_pool;
    int8_t *exps;          // 8-bit cache only
    float *weights;        // [rows][weights_stride]
    int32_t *kept;         // [rows][kept_stride]
    EvictDone *done;       // null, or the rows' records (the selection writes them)
    int64_t weights_stride, kept_stride;
    int32_t n, L, hkv, ps, log_ps, num_pages, n_new, kept_cols;
    EvictSeg segs[SEGS];
    int32_t new_pages[PAGES];
};
using EvictParams = EvictParamsT<kMaxSegs, kAppendMaxPages>;

struct EvictFinishParams {
    int32_t *page_table;
    int64_t *seq_len;
    float *weights;
    const int32_t *kept;
    const EvictDone *done;
    int64_t weights_stride, kept_stride;
    int32_t n, ps, log_ps, max_pages;
};

// ---------------------------------------------------------------- accumulated weights
struct WeightSeg {
    int32_t row;           // of weights
    int32_t table_row;
    int32_t q_row0, n_q, n_keys;
    int32_t score_stride;  // scores kept by the attention (Q8Seq)
    int64_t score0;
};

struct WeightParams {
    const int32_t *page_table;
    const __nv_bfloat16 *q;  // bf16 [rows][Hq][d]
    const __nv_bfloat16 *k;  // bf16 [num_pages][Hkv][ps][d], one layer
    float *lse;            // workspace [rows][Hq], log2 units
    const float *scores;   // kept by the attention, or null
    float *weights;        // [rows][weights_stride]
    int64_t weights_stride;
    int32_t n, hq, hkv, group, ps;
    float scale_log2;
    WeightSeg segs[kMaxSegs];
};

// ---------------------------------------------------------------- crop
constexpr int kMaxCropFreed = 2048;  // freed page ids carried by one crop launch (debug poison)

struct CropSeg {
    int32_t table_row;
    int32_t keep;          // pages kept
    int32_t old_n;         // pages before the crop
    int32_t seq;
    int64_t new_len;
    int32_t freed0;        // debug poison: this sequence's pages whose last reference went,
    int32_t n_freed;       //   as a range of CropParams::freed
    int32_t tail_page;     // debug poison: last kept page when this sequence is its only holder, else -1
    int32_t pad_;
};

template <int SEGS, int FREED>
struct CropParamsT {
    int32_t *page_table;
    int64_t *seq_len;
    uint4 *k_pool;
    uint4 *v_pool;
    int32_t n, poison, L, hkv, ps, dvec, num_pages;
    uint32_t poison_word;  // debug poison: what a word of a freed slot becomes
    CropSeg segs[SEGS];
    int32_t freed[FREED];
};
using CropParams = CropParamsT<kMaxCropSegs, kMaxCropFreed>;

// ---------------------------------------------------------------- attention
struct AttnSeq {
    int32_t table_row;     // seq * max_pages_per_seq
    int32_t n_pages;       // ceil(len / ps)
    int32_t q_row0;        // first row of this sequence in packed Q / out
    int32_t n_q;
    int32_t n_keys;        // len
    int32_t item0;         // first CTA work item of this sequence
    int32_t n_qtiles;      // ceil(n_q * group / kBM)
    int32_t n_splits;      // key splits per q-tile (1 without split-KV)
    int64_t part_row0;     // first partial row in the workspace (split-KV)
    int32_t comb0;         // first combine row item (split-KV)
    int32_t pair_top;      // the launch covers q-tile pairs [pair_top - items / (Hkv x splits), pair_top),
                           // heaviest first (pair_top = all pairs, unless a tail launch takes the lightest)
};

struct AttnParams {
    const int32_t *page_table;
    void *out;             // bf16 [rows][Hq][d]
    float *part_o;         // split-KV partial outputs, rows of d fp32 in blocks of 32 rows (part_chunk)
    float *part_lse;       // split-KV partial log2-sum-exp [rows]
    int32_t *status;
    int32_t n_seqs, hq, hkv, group, layer, num_pages, ps, oob_row;
    int32_t split_tiles;   // key tiles per split
    int32_t total_items;
    int32_t total_comb;
    int32_t pairs_fastest;  // one-item kernel: number a sequence's items pairs fastest (else kv-heads fastest)
    int32_t next_stride;   // one-item kernel: CTA b prefetches item b + next_stride's Q tiles into L2 (0: off)
    int32_t rounded_sums;  // rows divided by the sum of their weights as rounded to bf16 (else: before it)
    float scale_log2;      // softmax_scale * log2(e)
    AttnSeq seqs[kMaxSegs];
};

// ---------------------------------------------------------------- persistent (stream-K) attention
// A launch group's work units are (sequence, kv-head, q-tile pair), numbered
// sequence by sequence from AttnSeq::item0 (kv-head fastest, pairs heaviest
// first); a unit loads the key tiles [0, n) of its pair.  The persistent
// kernel runs one CTA per SM: whole units in lockstep rounds, then CTA c's
// contiguous stretch of the remaining (unit, key tile) work; the pieces of
// units cut by a stretch boundary write fp32 partials (O / l and log2-sum-exp)
// into slot `slot`, part `part`, and the warp that writes a slot's last part
// (counted on its ticket) merges the slot's parts.
constexpr int kMaxSkCtas = 160;        // >= SMs of the GPU
constexpr int kSkTicketsPerSlot = 8;   // one per (q-tile, warp of 32 rows)

struct SkCta {
    int32_t u0, t0;        // first unit and its first key tile
    int32_t u1, t1;        // last unit and the key tile it stops before (t1 = 0: u1 is not taken)
    int32_t slot0, part0;  // partial slot and part of u0's piece (slot -1: the whole unit, written directly)
    int32_t slot1, part1;  // the same for u1's piece when u1 > u0
};

struct SkSlot {
    int32_t unit;          // the unit cut into parts
    int32_t n_parts;
};

struct SkParams {
    AttnParams a;          // sequences, shapes, output; part_o / part_lse hold the partials
    int32_t n_ctas, n_slots, max_parts;
    int32_t rounds;        // whole units first: in round r < rounds CTA k takes unit r n_ctas + k (odd r:
                           // r n_ctas + n_ctas - 1 - k); then its tail stretch (cta[k], u0 > u1: none)
    int32_t *tickets;      // [n_slots][2][4] parts written per (slot, q-tile, warp); zero between launches
    SkCta cta[kMaxSkCtas];
    SkSlot slots[kMaxSkCtas];
};

// ---------------------------------------------------------------- decode attention
// Sequences whose queries pack into at most kDecMaxRows rows per kv-head
// (n_q x group) take the decode kernel (pe_decode.cu): CUDA cores, 64-key
// tiles streamed by bulk copies, split-KV merged in-kernel by the last split.
constexpr int kDecMaxRows = 16;
constexpr int kDecKeys = 64;           // keys per decode tile

struct DecodeSeq {
    int32_t table_row;     // seq * max_pages_per_seq
    int32_t n_pages;
    int32_t q_row0;        // first row of this sequence in Q / out
    int32_t n_q;
    int32_t n_keys;        // len
    int32_t cta0;          // CUDA-core kernel: first CTA of this sequence (hkv x n_splits CTAs, kv-head major);
                           // tensor-core kernel: tiles per chunk of this sequence's items
    int32_t n_splits;
    int32_t tile0;         // tensor-core kernel: the first full chunk id of this sequence's items (full
                           // chunks numbered sequence-major, kv-head next)
    int32_t rem0;          // tensor-core kernel: the id of kv-head 0's remainder chunk (kv-head h: rem0 + h),
                           // -1 when the tile count is a multiple of the chunk size
};

struct DecodeParams {
    const int32_t *page_table;
    const void *q;         // bf16 [rows][Hq][d]
    void *out;             // bf16 [rows][Hq][d]
    const void *k_pool;    // bf16 [L][num_pages][Hkv][ps][d]
    const void *v_pool;
    float *part;           // split partials: O [ctas][RB][d], then m [ctas][RB], then l [ctas][RB]
    int32_t *tickets;      // one counter per (sequence, kv-head) of the launch; zero between launches
    int32_t *sched;        // tensor-core kernel: [0] next chunk, [1] CTAs that stopped taking; zero between launches
    int32_t *status;
    int32_t n_seqs, hq, hkv, group, layer, num_pages, ps;
    int32_t oob_row;       // a pool row past the end: boxes there read zeros
    int32_t split_tiles;   // decode tiles per split (CUDA-core kernel) / per chunk (tensor-core kernel, <= 8)
    int32_t total_ctas;
    int32_t total_tiles;   // tensor-core kernel: chunks of all (sequence, kv-head) items
    int32_t full_chunks;   // tensor-core kernel: ids below this are full chunks, the rest remainder chunks
    int32_t any_split;     // tensor-core kernel: some item has several chunks (a combine launch follows)
    int32_t two_parts;     // tensor-core kernel: the form whose weights have two bf16 parts (TcCfg::kPRows)
    float scale_log2;      // softmax_scale * log2(e)
    DecodeSeq seqs[kMaxSegs];
    int32_t rem_seq[kMaxSegs];  // tensor-core kernel: the sequence of remainder block j (ids
                                // full_chunks + j hkv .., one per kv-head), blocks longest first
};

// Weights of many rows from the codes: rows R = query * group + head-in-group of a kv-head in groups of 128.
__host__ __device__ constexpr int q8_row_group_bytes(int head_dim) { return 2 * 128 * head_dim + 1024; }

struct WeightQ8Seg {
    int32_t row;           // of weights
    int32_t table_row;
    int32_t q_row0, n_q, n_keys;
    int32_t tile0;         // first tile of 128 keys (a block each)
    int32_t n_groups;      // groups of 128 rows of a kv-head
    int32_t group0;        // first group: group0 + kv-head * n_groups + i
};

struct WeightQ8Params {
    const int32_t *page_table;
    const __nv_bfloat16 *q;
    const int8_t *exps;
    const float *lse;      // [rows][Hq], log2 units
    uint8_t *groups;       // workspace, q8_row_group_bytes each
    float *weights;
    int64_t weights_stride;
    int32_t *status;
    int32_t n, hq, hkv, log_group, layer, num_pages, ps, log_ps, oob_row;
    float scale_log2;
    WeightQ8Seg segs[kMaxSegs];
};

// Records `msg` as this thread's last error (pe_last_error) and returns code.
int32_t report_error(int32_t code, const char *msg);

// Launchers (defined in the .cu files).
cudaError_t launch_append(const AppendParams &p, int64_t chunks, cudaStream_t st);
cudaError_t launch_crop(const CropParams &p, cudaStream_t st);
// Fork: copies n device page-table entries from row src_row to dst_row and sets
// the new sequence's device length.
cudaError_t launch_table_copy(int32_t *page_table, int32_t src_row, int32_t dst_row, int32_t n, int64_t *seq_len,
                              int32_t dst_seq, int64_t len, cudaStream_t st);
// Copy-on-write: copies slots [0, slots) of each copy's page src to its page dst
// (every layer and kv-head, K and V) and points its device table entry at dst.
cudaError_t launch_cow_copy(const CowParams &p, cudaStream_t st);
// tm_o: the output as a map of the same shape as tm_q (full q-tiles are stored by TMA); unused when split
cudaError_t launch_replay_attn(int head_dim, bool split, const CUtensorMap &tm_q, const CUtensorMap &tm_k,
                               const CUtensorMap &tm_v, const CUtensorMap &tm_o, const AttnParams &p, cudaStream_t st);
cudaError_t launch_splitkv_combine(int head_dim, const AttnParams &p, int num_sms, cudaStream_t st);
// Persistent stream-K attention (p.n_ctas CTAs), cut units merged in the kernel.
cudaError_t launch_replay_attn_sk(int head_dim, const CUtensorMap &tm_q, const CUtensorMap &tm_k,
                                  const CUtensorMap &tm_v, const SkParams &p, cudaStream_t st);
// rows_cap: 4, 8 or 16 (every sequence's n_q x group fits).
// tm_k / tm_v: the pools as 2-D maps {d, L*num_pages*Hkv*ps} with 64 x min(ps, 64) boxes, 128-byte swizzle.
// tensor_core (d = 128 only): keys on the MMA's M side, 128-key tiles (split_tiles
// counts 128-key tiles); otherwise CUDA cores, 64-key tiles.
cudaError_t launch_decode_attn(int head_dim, int rows_cap, bool tensor_core, const CUtensorMap &tm_k,
                               const CUtensorMap &tm_v, const DecodeParams &p, cudaStream_t st);
// 8-bit cache: p's pools hold codes, p.exps their scales, p.segs[].cum0 and p.seg_tokens count touched pages.
cudaError_t launch_append_q8(int head_dim, const AppendParams &p, cudaStream_t st);
cudaError_t launch_unpack_q8(const UnpackParams &p, int pages, cudaStream_t st);
cudaError_t launch_save_pages(const SaveParams &p, cudaStream_t st);
cudaError_t launch_read_kv(bool q8, const ReadParams &p, cudaStream_t st);
// Eviction, in this order on one stream: select for each group of sequences, then copy for each group of new pages.  One
// group: finish, which enters its pages; else a table after each copy and finish_all over all sequences, the only step
// that changes their weights.
cudaError_t launch_evict_select(const EvictParams &p, int max_len, cudaStream_t st);
cudaError_t launch_evict_copy(bool q8, int head_dim, const EvictParams &p, cudaStream_t st);
cudaError_t launch_evict_table(const EvictParams &p, cudaStream_t st);
cudaError_t launch_evict_finish(const EvictParams &p, cudaStream_t st);
cudaError_t launch_evict_finish_all(const EvictFinishParams &p, cudaStream_t st);
// q_rows: query rows of the launch's sequences (consecutive from segs[0].q_row0).
cudaError_t launch_weights(int head_dim, const WeightParams &p, int64_t q_rows, int max_keys, cudaStream_t st);
// The same from scores and lse that launch_attn_q8 left.
cudaError_t launch_weights_kept(const WeightParams &p, int max_keys, cudaStream_t st);
cudaError_t launch_weights_q8(int head_dim, const CUtensorMap &tm_k, const WeightQ8Params &p, int groups, int tiles, int split,
                              cudaStream_t st);
// rows_cap: 4, 8 or 16 rows a block.  tm_k / tm_v: the codes as 2-D maps {d, L*num_pages*Hkv*ps} with d x ps boxes,
// swizzled over d bytes.
cudaError_t launch_attn_q8(int head_dim, int rows_cap, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                           const Q8AttnParams &p, cudaStream_t st);
cudaError_t launch_attn_q8_rows(int head_dim, int rows_cap, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                                const Q8AttnParams &p, cudaStream_t st);
cudaError_t launch_bounded_wait_selftest(int32_t *status, uint64_t limit_ns, cudaStream_t st);

// Raises `kernel`'s dynamic shared-memory limit to `bytes` on the current
// device, once per device: the attribute is set on the device that is current
// at the call, so a process that runs caches on several GPUs sets it on each.
// `done` holds one bit per device (devices past 63 set it on every call).
template <typename Kernel>
inline cudaError_t set_dyn_smem_once(Kernel kernel, int bytes, std::atomic<uint64_t> &done)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = (dev >= 0 && dev < 64) ? (1ull << dev) : 0;
    if (bit && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && bit) done.fetch_or(bit, std::memory_order_acq_rel);
    return e;
}

// Fixed split-KV scratch compiled into the library (pe_attn.cu), used only by
// pe_replay_attn_static_scratch.  static_scratch() returns its device address
// on the current device; the address is looked up once per device.
constexpr int64_t kStaticScratchBytes = 16ll << 20;
cudaError_t static_scratch(float **ptr);

}  // namespace pe
