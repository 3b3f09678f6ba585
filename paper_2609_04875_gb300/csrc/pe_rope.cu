// Position rotation: of keys on their way into the cache and of the queries beside them (append), and of one tensor alone.
//
// Pair i of a head's columns -- (i, i + n_pairs), or neighbours (2i, 2i + 1) -- turns by the angle that frequency i has at
// the token's position on i's axis:
//     a' = scale (a cos - b sin),  b' = scale (b cos + a sin)
// in 32 bits, rounded once.  Columns past the pairs are copied.
//
// Bound by memory: every row is read once and written once, and an angle, a token's for all its rows, costs a sine and
// a cosine for each pair.  A thread keeps the angles of the same eight pairs (16 registers) and goes through the rows of a token,
// layer by layer and head by head, four of 32 bytes in flight; a warp reads and writes whole rows.  1638 tokens of 32 layers, 32 query heads and 8 kv-heads of
// 128: 189 us, 6.8 TB/s (a thread per chunk that computes its own angles: 713); the queries of 4 x 1500 tokens of 8 layers 117
// us, 6.7 TB/s (696).  Small calls are bound by their launch: 16 tokens of one layer 2.9 us on the GPU.
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
    const int at = r.positions ? __ldg(r.positions + r.axis[i] * r.positions_stride + tok) : pos;
    const uint64_t phase = static_cast<uint64_t>(static_cast<int64_t>(at)) * r.turn[i];
    float s, c;
    sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 4.656612873077393e-10f, &s, &c);  // 2^-31 half turns
    return make_float2(c * r.scale, s * r.scale);
}

__device__ __forceinline__ void unpack8(uint4 v, float (&y)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = unpack_bf16(w[k]);
        y[2 * k] = f.x;
        y[2 * k + 1] = f.y;
    }
}

__device__ __forceinline__ uint4 pack8(const float (&y)[8])
{
    return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

// Columns 8 chunk .. + 7 of a row, rotated, one by one: for any number of pairs.
__device__ __forceinline__ void rope_chunk(const RopeParams &r, const uint4 *row, int chunk, int64_t tok, int pos, float (&y)[8])
{
    const __nv_bfloat16 *x = reinterpret_cast<const __nv_bfloat16 *>(row);
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
        const int col = chunk * 8 + k;
        float v = __bfloat162float(x[col]);
        if (col < 2 * r.n_pairs) {
            const bool second = r.interleaved ? col & 1 : col >= r.n_pairs;
            const int i = r.interleaved ? col >> 1 : (second ? col - r.n_pairs : col);
            const float2 t = rope_turn(r, i, tok, pos);
            const float z = __bfloat162float(x[r.interleaved ? col ^ 1 : (second ? i : col + r.n_pairs)]);
            v = second ? v * t.x + z * t.y : v * t.x - z * t.y;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (u == k) y[u] = v;
    }
}

// A thread's share of every row of a token: two chunks of eight columns, a and b, which are either copied or eight whole
// pairs, whose angles it keeps.  In halves those are chunks c and c + n_pairs / 8, of neighbours 2c and 2c + 1.
struct PairOfChunks {
    int a, b;
    bool turns, interleaved;
    float2 t[8];
    __device__ __forceinline__ PairOfChunks(const RopeParams &r, int c, int64_t tok, int pos)
    {
        const int whole = r.n_pairs / 8;
        turns = c < whole;
        interleaved = r.interleaved;
        a = turns && !interleaved ? c : 2 * c;
        b = turns && !interleaved ? c + whole : 2 * c + 1;
        if (turns)
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = rope_turn(r, 8 * c + k, tok, pos);
    }
    __device__ __forceinline__ void turn(uint4 &va, uint4 &vb) const
    {
        if (!turns) return;
        float x[8], y[8];
        unpack8(va, x);
        unpack8(vb, y);
        if (interleaved) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p = x[2 * k], q = x[2 * k + 1], u = y[2 * k], w = y[2 * k + 1];
                x[2 * k] = p * t[k].x - q * t[k].y;
                x[2 * k + 1] = q * t[k].x + p * t[k].y;
                y[2 * k] = u * t[4 + k].x - w * t[4 + k].y;
                y[2 * k + 1] = w * t[4 + k].x + u * t[4 + k].y;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float p = x[k], q = y[k];
                x[k] = p * t[k].x - q * t[k].y;
                y[k] = q * t[k].x + p * t[k].y;
            }
        }
        va = pack8(x);
        vb = pack8(y);
    }
};

// (reads and writes of a row are one thread's, or come one after the other within a warp: out may be the input)
__device__ __forceinline__ uint4 ld_once(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

// Rows [r0, r1) of one token, a warp, numbered layer by layer and head by head: at(l, h) is a row's offset in chunks, of src and
// of dst; with V it is copied alike (v_src, v_dst).
template <int CPR, bool WHOLE, bool V, typename From, typename To>
__device__ __forceinline__ void rotate_rows(const RopeParams &r, const uint4 *src, uint4 *dst, const uint4 *v_src, uint4 *v_dst, int heads,
                                            int r0, int r1, int64_t tok, int pos, const From &from, const To &to)
{
    constexpr int CP = CPR / 2, RPW = 32 / CP, U = V ? 2 : 4;
    const int lane = threadIdx.x & 31, c = lane % CP;
    if constexpr (WHOLE) {
        const PairOfChunks pc(r, c, tok, pos);
        for (int x0 = r0 + lane / CP; x0 < r1; x0 += U * RPW) {
            uint4 a[U], b[U], va[U], vb[U];
            int64_t at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = x0 + u * RPW, l = x / heads, h = x - l * heads;
                if (x >= r1) continue;
                const int64_t f = from(l, h);
                at[u] = to(l, h);
                a[u] = ld_once(src + f + pc.a);
                b[u] = ld_once(src + f + pc.b);
                if constexpr (V) {
                    va[u] = ld_once(v_src + f + pc.a);
                    vb[u] = ld_once(v_src + f + pc.b);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (x0 + u * RPW >= r1) continue;
                pc.turn(a[u], b[u]);
                dst[at[u] + pc.a] = a[u];
                dst[at[u] + pc.b] = b[u];
                if constexpr (V) {
                    v_dst[at[u] + pc.a] = va[u];
                    v_dst[at[u] + pc.b] = vb[u];
                }
            }
        }
    } else {
        for (int x0 = r0; x0 < r1; x0 += RPW) {
            const int x = x0 + lane / CP, l = x / heads, h = x - l * heads;
            float y[8], z[8];
            int64_t f = 0;
            if (x < r1) {
                f = from(l, h);
                rope_chunk(r, src + f, 2 * c, tok, pos, y);
                rope_chunk(r, src + f, 2 * c + 1, tok, pos, z);
            }
            __syncwarp();
            if (x < r1) {
                const int64_t t = to(l, h);
                dst[t + 2 * c] = pack8(y);
                dst[t + 2 * c + 1] = pack8(z);
                if constexpr (V) {
                    v_dst[t + 2 * c] = v_src[f + 2 * c];
                    v_dst[t + 2 * c + 1] = v_src[f + 2 * c + 1];
                }
            }
        }
    }
}

// The queries of token tok: a part of part_rows rows.
template <int CPR, bool WHOLE>
__device__ __forceinline__ void rotate_part(const RopeParams &r, const uint4 *X, uint4 *out, int layers, int64_t n_total, int heads, int part,
                                            int part_rows, int64_t tok, int pos)
{
    const auto at = [&](int l, int h) { return ((l * n_total + tok) * heads + h) * CPR; };
    rotate_rows<CPR, WHOLE, false>(r, X, out, nullptr, nullptr, heads, part * part_rows, min((part + 1) * part_rows, layers * heads), tok, pos, at, at);
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

constexpr int kRowThreads = 128;  // of a block of rows: 4 tasks, a warp each

// A warp per token and part of its rows (tokens fastest: neighbouring warps read neighbouring rows).
template <int CPR, bool WHOLE>
__global__ void __launch_bounds__(kRowThreads) rotate_kernel(const __grid_constant__ RotateParams p, int parts, int part_rows)
{
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int64_t id = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5);
    const int part = static_cast<int>(id / p.n_tokens), tok = p.tok0 + static_cast<int>(id - static_cast<int64_t>(part) * p.n_tokens);
    if (part >= parts) return;
    int lo = 0, hi = p.n_segs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.segs[mid].tok0 <= tok) lo = mid; else hi = mid - 1;
    }
    rotate_part<CPR, WHOLE>(p.r, p.X, p.out, p.layers, p.n_total, p.heads, part, part_rows, tok, p.segs[lo].pos0 + tok - p.segs[lo].tok0);
}

template <typename Block>
__device__ __forceinline__ void enter_pages(const Block &a)
{
    for (int s = 0; s < a.n_segs; ++s) {
        const AppendSeg &sg = a.segs[s];
        for (int i = threadIdx.x; i < sg.n_new; i += blockDim.x)
            a.page_table[sg.table_row + sg.first_new_lp + i] = a.new_pages[sg.new0 + i];
        if (threadIdx.x == 0) a.seq_len[sg.seq] = static_cast<int64_t>(sg.len0) + sg.n_tokens;
    }
}

// A warp per token and part: of K's rows and V's, into their slots, or of Q's.
template <typename Params, int CPR, bool WHOLE>
__global__ void __launch_bounds__(kRowThreads) append_rope_kernel(const __grid_constant__ Params p, int kv_parts, int kv_rows, int q_parts, int q_rows)
{
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const auto &a = p.a;
    if (blockIdx.x == 0) enter_pages(a);
    const int64_t id = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5);
    const int part = static_cast<int>(id / a.seg_tokens), t = static_cast<int>(id - static_cast<int64_t>(part) * a.seg_tokens);
    if (part >= kv_parts + q_parts) return;
    const AppendSeg &sg = a.segs[find_seg(a.segs, a.n_segs, t)];
    const int local = t - sg.cum0, pos = sg.len0 + local;
    const int64_t tok = sg.tok0 + local;
    if (part >= kv_parts) {
        rotate_part<CPR, WHOLE>(p.c.r, p.c.Q, p.c.Q_out, a.L, a.n_total, p.c.hq, part - kv_parts, q_rows, tok, pos);
        return;
    }
    const int lp = pos / a.ps, slot = pos - lp * a.ps;
    const int64_t page = lp < sg.first_new_lp ? sg.last_page : a.new_pages[sg.new0 + (lp - sg.first_new_lp)];
    rotate_rows<CPR, WHOLE, true>(
        p.c.r, a.K, a.k_pool, a.V, a.v_pool, a.hkv, part * kv_rows, min((part + 1) * kv_rows, a.L * a.hkv), tok, pos,
        [&](int l, int h) { return ((l * static_cast<int64_t>(a.n_total) + tok) * a.hkv + h) * CPR; },
        [&](int l, int h) { return (((static_cast<int64_t>(l) * a.num_pages + page) * a.hkv + h) * a.ps + slot) * CPR; });
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

// (cos, sin) of a page's new rows, in shared memory.  Where n_pairs is a multiple of 8, pair 8c + k of a row stands at k *
// (n_pairs / 8) + c, so that lanes on neighbouring chunks read neighbouring entries.
template <bool WHOLE>
__device__ __forceinline__ int turn_at(int n_pairs, int i)
{
    return WHOLE ? (i & 7) * (n_pairs >> 3) + (i >> 3) : i;
}

template <bool WHOLE>
__device__ __forceinline__ void rope_chunk_table(const RopeParams &r, const float2 *turns, const uint4 *row, int chunk, float (&y)[8])
{
    const int n = r.n_pairs;
    unpack8(__ldg(row + chunk), y);
    if (chunk * 8 >= 2 * n) return;
    if (r.interleaved) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!WHOLE && 4 * chunk + k >= n) break;
            const float2 t = turns[turn_at<WHOLE>(n, 4 * chunk + k)];
            const float a = y[2 * k], b = y[2 * k + 1];
            y[2 * k] = a * t.x - b * t.y;
            y[2 * k + 1] = b * t.x + a * t.y;
        }
    } else if (WHOLE) {
        const int whole = n >> 3, c = chunk < whole ? chunk : chunk - whole;
        const float sign = chunk < whole ? -1.f : 1.f;
        float z[8];
        unpack8(__ldg(row + (chunk < whole ? chunk + whole : c)), z);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 t = turns[k * whole + c];
            y[k] = y[k] * t.x + z[k] * (sign * t.y);
        }
    } else {
        const __nv_bfloat16 *x = reinterpret_cast<const __nv_bfloat16 *>(row);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int col = chunk * 8 + k;
            if (col >= 2 * n) break;
            const bool second = col >= n;
            const float2 t = turns[second ? col - n : col];
            const float z = __bfloat162float(x[second ? col - n : col + n]);
            y[k] = y[k] * t.x + (second ? z : -z) * t.y;
        }
    }
}

// A block per page and layer (append_q8_kernel works head by head), heads [h0, h1) of it one group after another: the angles
// of the page's new rows are computed once.  K's new rows turn in 32 bits, so that a value is rounded once, to its code.
// Bound by the latency of its steps (page, exponents, angles, rows, maximum, codes): 16 agents x 32 layers, one token, 17 us
// (with the angles computed where a chunk is read, 8 times unrolled: 27), 8 agents' 333 tokens of 2 layers 12 us (20).
template <typename Params, int CPR, int NC, bool WHOLE>
__global__ void __launch_bounds__(kQ8Block, NC == 8 ? 1 : 3) append_rope_q8_kernel(const __grid_constant__ Params p, int threads, int page_blocks, int parts,
                                                                  int tokens, int q_parts, int q_rows)
{
    extern __shared__ float2 turns[];
    __shared__ uint32_t s_max[kQ8Block / 32];
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const auto &a = p.a;
    constexpr int HD = CPR * 8;
    if (static_cast<int>(blockIdx.x) >= page_blocks) {  // Q's rows, a warp per token and part
        const int64_t id = static_cast<int64_t>(blockIdx.x - page_blocks) * (kQ8Block / 32) + (threadIdx.x >> 5);
        const int q_part = static_cast<int>(id / tokens);
        if (q_part >= q_parts) return;
        int t = static_cast<int>(id - static_cast<int64_t>(q_part) * tokens), s = 0;
        for (; t >= a.segs[s].n_tokens; ++s) t -= a.segs[s].n_tokens;
        rotate_part<CPR, WHOLE>(p.c.r, p.c.Q, p.c.Q_out, a.L, a.n_total, p.c.hq, q_part, q_rows, a.segs[s].tok0 + t, a.segs[s].len0 + t);
        return;
    }
    if (blockIdx.x == 0) enter_pages(a);
    int r = static_cast<int>(blockIdx.x);
    const int part = r % parts;
    r /= parts;
    const int pg = r % a.seg_tokens;
    const int64_t l = r / a.seg_tokens;
    const AppendSeg &sg = a.segs[find_seg(a.segs, a.n_segs, pg)];
    const int lp = sg.len0 / a.ps + (pg - sg.cum0);
    const int page = lp < sg.first_new_lp ? sg.last_page : a.new_pages[sg.new0 + (lp - sg.first_new_lp)];
    const int pos0 = lp * a.ps;
    const int old = max(0, sg.len0 - pos0);
    const int rows = min(a.ps, sg.len0 + sg.n_tokens - pos0);
    const int64_t tok0 = sg.tok0 + (pos0 - sg.len0);  // of the page's row 0
    const int n = p.c.r.n_pairs;
    for (int x = threadIdx.x; x < (rows - old) * n; x += kQ8Block) {
        const int row = x / n, i = x - row * n;
        turns[row * n + turn_at<WHOLE>(n, i)] = rope_turn(p.c.r, i, tok0 + old + row, pos0 + old + row);
    }
    __syncthreads();
    const int groups = kQ8Block / threads, share = (a.hkv + parts - 1) / parts, h1 = min(a.hkv, (part + 1) * share);
    for (int hb = part * share; hb < h1; hb += groups) {
        const int h = hb + threadIdx.x / threads;
        const bool on = h < h1;
        const int64_t head = (l * a.num_pages + page) * a.hkv + (on ? h : 0);
        uint8_t *kp = reinterpret_cast<uint8_t *>(a.k_pool) + head * a.ps * HD;
        uint8_t *vp = reinterpret_cast<uint8_t *>(a.v_pool) + head * a.ps * HD;
        int8_t *ex = a.exps + head * 2;
        int ke0 = 0, ve0 = 0;
        if (on && old > 0) {
            ke0 = ex[0];
            ve0 = ex[1];
        }
        const float kes = pow2i(ke0), ves = pow2i(ve0);
        if (threads <= 32) __syncwarp();
        else __syncthreads();  // the old exponents are read before they are written
        q8_write_page_f32<CPR, NC>(on, threadIdx.x % threads, threads, rows, old, ke0, ve0, kp, vp, ex, s_max,
                                   [&](int row, int col8, float (&k)[8], uint4 &v) {
                                       if (row < old) {
                                           q8_to_float(*reinterpret_cast<const uint2 *>(kp + row * HD + col8 * 8), kes, k);
                                           v = q8_to_bf16(*reinterpret_cast<const uint2 *>(vp + row * HD + col8 * 8), ves);
                                       } else {
                                           const int64_t s = ((l * a.n_total + tok0 + row) * a.hkv + h) * CPR;
                                           v = __ldg(a.V + s + col8);
                                           rope_chunk_table<WHOLE>(p.c.r, turns + (row - old) * n, a.K + s, col8, k);
                                       }
                                   });
    }
}

constexpr int kSmallSegs = 16, kSmallPages = 128;  // the small parameter block (as in pe_kv.cu)

// Rows of a part: eight steps of a warp's rows, or fewer (a whole number of steps) until the warps are 16 an SM.  A part's rows
// share their angles, whose eight sines and cosines take a thread longer than a step does.  A warp per token and layer / parts, 3890
// tokens of 10 layers, 16 heads of Q and 2 of K of 128: 98 / 65 us; 3509 tokens of 21 layers, 8 and 8 of 64: 137 / 74.
int part_of_rows(int64_t tokens, int rows, int cpr)
{
    const int step = 64 / cpr;  // rows of a warp
    int n = 8;
    while (n > 1 && (tokens * ((rows + n * step - 1) / (n * step)) < 152 * 16 || (n / 2) * step >= rows)) n /= 2;
    return n * step;
}

template <typename Params, int CPR, bool WHOLE>
cudaError_t launch_append_rope_t(bool q8, const Params &p, cudaStream_t st)
{
    cudaLaunchAttribute attr;
    int64_t tokens = 0;
    for (int i = 0; i < p.a.n_segs; ++i) tokens += p.a.segs[i].n_tokens;
    const int q_all = p.c.Q ? p.a.L * p.c.hq : 0, q_rows = part_of_rows(tokens, std::max(1, q_all), CPR), q_parts = (q_all + q_rows - 1) / q_rows;
    if (!q8) {
        const int kv_all = p.a.L * p.a.hkv, kv_rows = part_of_rows(tokens, kv_all, CPR), kv_parts = (kv_all + kv_rows - 1) / kv_rows;
        const int64_t blocks = (tokens * (kv_parts + q_parts) + kRowThreads / 32 - 1) / (kRowThreads / 32);
        if (blocks > INT32_MAX) return cudaErrorInvalidValue;
        const cudaLaunchConfig_t cfg = serial_config(blocks, kRowThreads, st, &attr);
        return cudaLaunchKernelEx(&cfg, append_rope_kernel<Params, CPR, WHOLE>, p, kv_parts, kv_rows, q_parts, q_rows);
    }
    // threads that share a page of one kv-head: half as many chunks each as append_q8_kernel's, for K takes twice the registers
    const int elems = p.a.ps * CPR * 8, threads = std::max(32, std::min(kQ8Block, elems / 32)), nc = elems / 8 / threads;
    // a page's heads over as many blocks as there are groups of them, while the blocks are few
    const int64_t pages = static_cast<int64_t>(p.a.L) * p.a.seg_tokens;
    const int groups = kQ8Block / threads, most = (p.a.hkv + groups - 1) / groups;
    int parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, 8 * 152 / std::max<int64_t>(1, pages))));
    parts = (most + (most + parts - 1) / parts - 1) / ((most + parts - 1) / parts);  // (none without a group)
    int64_t longest = 0;
    for (int i = 0; i < p.a.n_segs; ++i) longest = std::max<int64_t>(longest, p.a.segs[i].n_tokens);
    const int64_t page_blocks = pages * parts, blocks = page_blocks + (tokens * q_parts + kQ8Block / 32 - 1) / (kQ8Block / 32);
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = serial_config(blocks, kQ8Block, st, &attr);
    cfg.dynamicSmemBytes = static_cast<size_t>(std::min<int64_t>(p.a.ps, longest)) * p.c.r.n_pairs * sizeof(float2);
    const int pb = static_cast<int>(page_blocks), n = static_cast<int>(tokens);
    auto launch = [&](auto kernel, std::atomic<uint64_t> &configured) {
        if (cudaError_t e = set_dyn_smem_once(kernel, 128 * kRopeMaxPairs * static_cast<int>(sizeof(float2)), configured); e != cudaSuccess)
            return e;
        return cudaLaunchKernelEx(&cfg, kernel, p, threads, pb, parts, n, q_parts, q_rows);
    };
    static std::atomic<uint64_t> done[3];
    if (nc == 8) return launch(append_rope_q8_kernel<Params, CPR, 8, WHOLE>, done[0]);
    if (CPR == 16 || nc == 4) return launch(append_rope_q8_kernel<Params, CPR, 4, WHOLE>, done[1]);
    return launch(append_rope_q8_kernel<Params, CPR, 2, WHOLE>, done[2]);
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
    const bool whole = rope.r.n_pairs % 8 == 0;
    using P = AppendRopeParamsT<SEGS, PAGES>;
    if (head_dim == 128) return whole ? launch_append_rope_t<P, 16, true>(q8, p, st) : launch_append_rope_t<P, 16, false>(q8, p, st);
    return whole ? launch_append_rope_t<P, 8, true>(q8, p, st) : launch_append_rope_t<P, 8, false>(q8, p, st);
}

}  // namespace

cudaError_t launch_append_rope(bool q8, int head_dim, const AppendParams &a, const RopeCall &rope, cudaStream_t st)
{
    if (a.n_segs <= kSmallSegs && a.n_new <= kSmallPages) return launch_sized<kSmallSegs, kSmallPages>(q8, head_dim, a, rope, st);
    return launch_sized<kMaxSegs, kAppendMaxPages>(q8, head_dim, a, rope, st);
}

template <int CPR>
static cudaError_t launch_rotate_t(const RotateParams &p, cudaStream_t st)
{
    const int rows = p.layers * p.heads;
    if (p.n_tokens <= 0 || rows <= 0) return cudaSuccess;
    const int part_rows = part_of_rows(p.n_tokens, rows, CPR), parts = (rows + part_rows - 1) / part_rows;
    const int64_t blocks = (static_cast<int64_t>(p.n_tokens) * parts + kRowThreads / 32 - 1) / (kRowThreads / 32);
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = serial_config(blocks, kRowThreads, st, &attr);
    return p.r.n_pairs % 8 == 0 ? cudaLaunchKernelEx(&cfg, rotate_kernel<CPR, true>, p, parts, part_rows)
                                : cudaLaunchKernelEx(&cfg, rotate_kernel<CPR, false>, p, parts, part_rows);
}

cudaError_t launch_rotate(int head_dim, const RotateParams &p, cudaStream_t st)
{
    return head_dim == 128 ? launch_rotate_t<16>(p, st) : launch_rotate_t<8>(p, st);
}

}  // namespace pe
