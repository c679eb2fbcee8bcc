// Attention over packed sequences for sm_100a: what its kernels share. Parameters, the work of a block, tiles.
//
//   S = scale Q K^T (a query sees the keys of its sequence, if causal up to its own row)   P = softmax(S)   O = P V
//
// Rows are tokens, T of them; head h of a tensor is D columns from column h D on, rows are ld elements apart. Sequence i is
// the rows [cu[i], cu[i+1]) (or T / n rows each), queries' heads h = 0..heads-1 read the keys of head h / (heads / kv_heads).
// Tiles are rows of a sequence by 64 or 128 columns (D rounded up: what lies beyond D reads as zero): 128 rows of an item's own, 64 or 128 of those that it
// walks over. TMA fetches them in boxes of so many rows x 64 columns of one head with the 128-byte swizzle. A sequence's last tile ends inside a box: the
// rows after it are another sequence's or nobody's, and where they would enter a sum as 0 x value they are overwritten with zeros
// in shared memory (they may hold infinities or NaN), or, of queries that keys walk over, with the sequence's last query.
#pragma once
#include "attention.h"
#include "gemm_sm100.cuh"

namespace nb {

constexpr uint32_t kAttnBox = 128 * 128;  // bytes of a box
constexpr float kLog2e = 1.4426950408889634f;

struct AttnSpan {
    int start, len;  // rows of the sequence
    int block;       // block of `rows` rows of it, or -1: nothing to do
};

__host__ __device__ __forceinline__ bool attn_wide(const void *p, long long ld, int D)
{
    return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * 2) | static_cast<uintptr_t>(D * 2)) & 31u) == 0;
}

// The order of the items, of blocks of 128 rows, told by one warp. With a causal mask a block has work in proportion to its place in its sequence (dQ and the
// forward pass: more towards the end; dK, dV: more towards the start), so items come in falling order of that over all sequences: the l-th
// level is block l (or l-th from the end) of every sequence that has so many, highest level first. A lane holds up to kOwn sequences, and the level
// of the k-th item is found by sums over the warp. (In order of the sequences 16 of 1024 rows left a fifth of the SMs' time unused at the end.) For more
// sequences than that, sequence i has the slots from cu[i] / 128 + i on, at least as many as it has blocks, so that no sums over the sequences before
// it are needed. Bounds outside [0, T] or falling ones are cut to an empty or shorter sequence (and reported by attn_report_bounds).
class AttnOrder {
    static constexpr int kOwn = 4;
    int start_[kOwn], len_[kOwn];
    int top_;  // levels

    __device__ __forceinline__ static int blocks(int len) { return (len + 127) / 128; }
    __device__ __forceinline__ int above(int level) const  // items of this level and higher ones
    {
        int n = 0;
#pragma unroll
        for (int c = 0; c < kOwn; ++c) n += max(blocks(len_[c]) - level, 0);
        return __reduce_add_sync(0xffffffffu, n);
    }

public:
    __device__ __forceinline__ void load(const AttnParams &p)
    {
        const int lane = static_cast<int>(threadIdx.x & 31);
        int most = 0;
#pragma unroll
        for (int c = 0; c < kOwn; ++c) {
            const int i = c * 32 + lane;
            start_[c] = len_[c] = 0;
            if (i < p.n && p.n <= 32 * kOwn) {
                if (p.cu) {
                    start_[c] = min(max(__ldcg(p.cu + i), 0), p.T);
                    len_[c] = min(max(__ldcg(p.cu + i + 1), start_[c]), p.T) - start_[c];
                } else {
                    len_[c] = p.T / p.n;
                    start_[c] = i * len_[c];
                }
            }
            most = max(most, blocks(len_[c]));
        }
        top_ = __reduce_max_sync(0xffffffffu, most);
    }
    // the k-th item of a head; from_end: blocks at the start of a sequence have the most work
    __device__ __forceinline__ AttnSpan item(const AttnParams &p, int k, bool from_end) const
    {
        const int lane = static_cast<int>(threadIdx.x & 31);
        AttnSpan s{0, 0, -1};
        if (p.n > 32 * kOwn) {
            int first;
            if (p.cu == nullptr) {
                s.len = p.T / p.n;
                first = blocks(s.len);
                s.start = k / first * s.len;
                if (k / first >= p.n) s.len = 0;
                first = k / first * first;
            } else {
                int lo = 0, hi = p.n;  // the last i with cu[i] / 128 + i <= k lies in [lo, hi)
                while (hi - lo > 1) {
                    const int step = (hi - lo + 31) / 32;
                    const int i = lo + lane * step;
                    const unsigned before = __ballot_sync(0xffffffffu, i < hi && max(__ldcg(p.cu + i), 0) / 128 + i <= k);
                    const int last = before ? 31 - __clz(before) : 0;
                    lo += last * step;
                    hi = min(hi, lo + step);
                }
                first = max(__ldcg(p.cu + lo), 0) / 128 + lo;
                s.start = min(max(__ldcg(p.cu + lo), 0), p.T);
                s.len = min(max(__ldcg(p.cu + lo + 1), s.start), p.T) - s.start;
            }
            const int local = k - first, n = blocks(s.len);
            if (local >= 0 && local < n) s.block = from_end ? local : n - 1 - local;
            return s;
        }
        if (above(0) <= k) return s;
        int lo = 0, hi = top_;  // the level is the last with more than k items from it on up
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (above(mid) > k) lo = mid;
            else hi = mid;
        }
        int rank = k - above(lo + 1);  // among the sequences that have the level
#pragma unroll
        for (int c = 0; c < kOwn; ++c) {
            const bool has = blocks(len_[c]) > lo;
            const unsigned all = __ballot_sync(0xffffffffu, has);
            const unsigned here = __ballot_sync(0xffffffffu, has && __popc(all & ((1u << lane) - 1u)) == rank);
            if (here) {
                s.start = __shfl_sync(0xffffffffu, start_[c], __ffs(here) - 1);
                s.len = __shfl_sync(0xffffffffu, len_[c], __ffs(here) - 1);
                s.block = from_end ? blocks(s.len) - 1 - lo : lo;
            }
            rank -= __popc(all);  // below zero from there on: no sequence of the lanes to come
        }
        return s;
    }
};

// Reports bounds that fall or leave [0, T]; by one warp of a launch.
__device__ __forceinline__ void attn_report_bounds(const int *cu, int n, int T, int *status)
{
    for (int i = static_cast<int>(threadIdx.x & 31); i <= n; i += 32)
        if (__ldcg(cu + i) < (i ? __ldcg(cu + i - 1) : 0) || __ldcg(cu + i) > T)
            if (atomicCAS(status, 0, kStatusBadSequences) == 0) status[1] = i;
}

__device__ __forceinline__ bool warp_wait(const WaitCtx &w, uint32_t bar, uint32_t parity, int where)
{
    return __all_sync(0xffffffffu, wait_barrier(w, bar, parity, where));
}

// ---------------------------------------------------------------- the items of a block
// A block begins with the item of its own place in the grid. When its loading warp has the tiles of an item on their way it asks for the next
// one, which the hardware takes off the blocks that have not started; items pass from the loading warp to the others by two slots in shared memory.
struct AttnItem {
    int start, len, block, head;  // block < 0: no more
};
struct AttnItems {
    static constexpr int kBars = 5;  // barriers: an item is there (two), it has been read by all (two), the next one has come
    uint32_t bars, memory;           // kBars of 8 bytes; 48 bytes, 16-byte aligned
    __device__ __forceinline__ uint32_t there(int k) const { return bars + 8u * (k & 1); }
    __device__ __forceinline__ uint32_t read(int k) const { return bars + 16u + 8u * (k & 1); }
    // by lane `lane` of the warp that initialises barriers
    __device__ __forceinline__ void init(int lane, int readers) const
    {
        if (lane < kBars) ptx::mbar_init(bars + 8u * lane, lane == 2 || lane == 3 ? readers : 1);
    }
    // the loading warp asks for the next item: its place in the grid, or -1. (Asked for earlier, an item may wait for a block that has much to do.)
    __device__ __forceinline__ bool next(const WaitCtx &w, uint32_t &asked, int &at) const
    {
        if (ptx::elect_one()) {
            ptx::mbar_expect_tx(bars + 32u, 16);
            ptx::launch_cancel(memory, bars + 32u);
        }
        __syncwarp();
        if (!warp_wait(w, bars + 32u, asked++ & 1u, 520)) return false;
        at = ptx::launch_cancelled(memory);
        ptx::fence_proxy_async_smem();  // the next answer is written where this one was read
        __syncwarp();
        return true;
    }
    // the loading warp puts the k-th item down
    __device__ __forceinline__ bool put(const WaitCtx &w, int k, const AttnItem &m) const
    {
        if (!warp_wait(w, read(k), (static_cast<uint32_t>(k >> 1) & 1u) ^ 1u, 510)) return false;
        if ((threadIdx.x & 31) == 0) {
            ptx::st_shared_v4(memory + 16u + 16u * (k & 1), static_cast<uint32_t>(m.start), static_cast<uint32_t>(m.len), static_cast<uint32_t>(m.block),
                              static_cast<uint32_t>(m.head));
            ptx::mbar_arrive(there(k));
        }
        __syncwarp();
        return true;
    }
    // the k-th item, for one thread that stands for its warp, or for all of a warp; false: there is none, or a wait ran out
    template <bool WARP>
    __device__ __forceinline__ bool take(const WaitCtx &w, int k, AttnItem &m) const
    {
        const uint32_t par = static_cast<uint32_t>(k >> 1) & 1u;
        if (!(WARP ? warp_wait(w, there(k), par, 500) : wait_barrier(w, there(k), par, 500))) return false;
        uint32_t v[4];
        ptx::ld_shared_v4(memory + 16u + 16u * (k & 1), v[0], v[1], v[2], v[3]);
        m = {static_cast<int>(v[0]), static_cast<int>(v[1]), static_cast<int>(v[2]), static_cast<int>(v[3])};
        if (WARP) __syncwarp();
        if (!WARP || (threadIdx.x & 31) == 0) ptx::mbar_arrive(read(k));
        return m.block >= 0;
    }
};

// ---------------------------------------------------------------- items that a cluster of blocks shares
// The tiles that a block walks over for an item: n from the first-th on. Of a cluster's blocks as many take part as have LEAST of them each.
struct AttnPart {
    int first, n;
};
template <int LEAST>
__device__ __forceinline__ int attn_sharers(int parts, int tiles)
{
    return max(1, min(parts, tiles / LEAST));
}
template <bool SPLIT, int LEAST>
__device__ __forceinline__ AttnPart attn_part(int parts, int tiles)
{
    if (!SPLIT) return {0, tiles};
    const int sharers = attn_sharers<LEAST>(parts, tiles), i = static_cast<int>(ptx::cluster_ctarank());
    if (i >= sharers) return {0, 0};
    const int first = static_cast<int>(static_cast<long long>(tiles) * i / sharers);
    return {first, static_cast<int>(static_cast<long long>(tiles) * (i + 1) / sharers) - first};
}
// The sums of an item's blocks are joined by all blocks of the cluster (a power of two of them): a block owns 128 / parts of the item's rows and takes its cluster's sums of these,
// written by the others into its shared memory as `parts` groups of that many rows, [128][D] fp32. Pieces of 16 bytes change places so that eight rows meet no bank twice.
constexpr int kAttnParts = 8;  // blocks of a cluster, at most
struct AttnShare {
    int parts, rank, rows;  // of the cluster; this block; that a block owns
    __device__ __forceinline__ explicit AttnShare(int n) : parts(n), rank(static_cast<int>(ptx::cluster_ctarank())), rows(128 / n) {}
    __device__ __forceinline__ uint32_t owner(int row) const { return static_cast<uint32_t>(row / rows); }
    __device__ __forceinline__ int slot(int part, int row) const { return part * rows + row % rows; }
    // whether a wait has run out in a block of the cluster, by a whole warp, when all their waits are over
    __device__ __forceinline__ bool failed(uint32_t abort_addr) const
    {
        const int lane = static_cast<int>(threadIdx.x & 31);
        return __any_sync(0xffffffffu, lane < parts && ptx::ld_cluster_u32_volatile(ptx::mapa(abort_addr, static_cast<uint32_t>(min(lane, parts - 1)))) != 0);
    }
};
// W columns of a row per lane, from column col on, from the fp32 accumulator at `acc` to the row's owner
template <int W, int D>
__device__ __forceinline__ void attn_give_row(const AttnShare &c, uint32_t acc, uint32_t sums, int row, int col)
{
    const int slot = c.slot(c.rank, row);
    const uint32_t to = ptx::mapa(sums + slot * (D * 4), c.owner(row));
#pragma unroll
    for (int k = 0; k < W; k += 32) {
        uint32_t o[32];
        __syncwarp();
        ptx::tmem_ld_32x32_wait(acc + k, o);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            ptx::st_cluster_v4(to + ((((col + k) / 4 + i) ^ (slot & 7)) << 4), o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    }
    __syncwarp();
}
// The block's own rows (of `rows` of the item): the sums of the cluster's first `sharers` blocks, weighed, added in their order and written as bf16 by THREADS threads.
// weight(part, row): of a part's sums
template <int D, int THREADS, class Weight>
__device__ __forceinline__ void attn_join_rows(const AttnShare &c, uint32_t sums, int sharers, __nv_bfloat16 *dst, long long ld, int rows, int cols, const Weight &weight)
{
    constexpr int PIECES = D / 8;  // of a row: eight columns each
    const int row0 = c.rank * c.rows;
    for (int i = static_cast<int>(threadIdx.x); i < c.rows * PIECES; i += THREADS) {
        const int row = row0 + i / PIECES, piece = i % PIECES;
        if (row >= rows || piece * 8 >= cols) continue;
        float o[8] = {};
        for (int q = 0; q < sharers; ++q) {
            const int slot = c.slot(q, row);
            const float w = weight(q, row);
            float4 a, b;
            ptx::ld_shared_f32x4(sums + slot * (D * 4) + (((2 * piece) ^ (slot & 7)) << 4), a);
            ptx::ld_shared_f32x4(sums + slot * (D * 4) + (((2 * piece + 1) ^ (slot & 7)) << 4), b);
            const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(w, v[e], o[e]);
        }
        *reinterpret_cast<uint4 *>(dst + row * ld + piece * 8) =
            make_uint4(ptx::pack_bf16x2(o[0], o[1]), ptx::pack_bf16x2(o[2], o[3]), ptx::pack_bf16x2(o[4], o[5]), ptx::pack_bf16x2(o[6], o[7]));
    }
}

// A tile of ROWS rows, in boxes of 64 columns, from row `row` on.
template <int D, int ROWS = 128>
__device__ __forceinline__ void attn_load(uint32_t dst, const CUtensorMap *m, uint32_t bar, int head, int row)
{
#pragma unroll
    for (int c = 0; c < D / 64; ++c) ptx::tma_load_3d(dst + c * ROWS * 128, m, bar, c * 64, head, row);
}
// Rows [from, to) of a tile in shared memory are set to zero by one warp.
template <int D, int ROWS = 128>
__device__ __forceinline__ void attn_zero_rows(uint32_t tile, int from, int to)
{
    const int lane = static_cast<int>(threadIdx.x & 31);
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
        for (int i = lane; i < (to - from) * 8; i += 32) ptx::st_shared_v4(tile + c * ROWS * 128 + from * 128 + i * 16, 0, 0, 0, 0);
}
// Rows [from, to) of a tile become its row from - 1, by one warp. (A row's pieces of 16 bytes stand where the swizzle puts them.)
template <int D, int ROWS>
__device__ __forceinline__ void attn_repeat_row(uint32_t tile, int from, int to)
{
    const int lane = static_cast<int>(threadIdx.x & 31);
    auto at = [&](int row, int piece) { return tile + static_cast<uint32_t>(row * 128 + ((piece ^ (row & 7)) << 4)); };
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
        for (int i = lane; i < (to - from) * 8; i += 32) {
            uint32_t v[4];
            ptx::ld_shared_v4(at(from - 1, i & 7) + c * ROWS * 128, v[0], v[1], v[2], v[3]);
            ptx::st_shared_v4(at(from + (i >> 3), i & 7) + c * ROWS * 128, v[0], v[1], v[2], v[3]);
        }
}

// D[128, N] = A B^T over `steps` pieces of 16 columns, tiles A (128 rows) and B (N rows) with the summed index contiguous (boxes of 64 columns).
template <int N = 128>
__device__ __forceinline__ void attn_mma_kk(uint32_t d_tmem, uint32_t a, uint32_t b, uint32_t idesc, int steps)
{
    const uint64_t ad = make_smem_desc(a, 16, 1024), bd = make_smem_desc(b, 16, 1024);
    for (int k = 0; k < steps; ++k)
        ptx::umma_bf16<1>(d_tmem, ad + static_cast<uint64_t>((k >> 2) * (kAttnBox >> 4) + (k & 3) * (32 >> 4)),
                          bd + static_cast<uint64_t>((k >> 2) * (N * 128 >> 4) + (k & 3) * (32 >> 4)), idesc, k > 0 ? 1u : 0u);
}
// D[128, N] (+)= A B, A [128, 16 steps] in tensor memory (piece k of 16 columns at a_tmem + 8 k, or, SPLIT, the second 64 columns of A
// 64 columns of tensor memory after the first), B's rows the summed index (a tile of ROWS rows).
template <bool SPLIT = false, int ROWS = 128>
__device__ __forceinline__ void attn_mma_tn(uint32_t d_tmem, uint32_t a_tmem, uint32_t b, uint32_t idesc, int steps, bool accumulate)
{
    const uint64_t bd = make_smem_desc(b, ROWS * 128, 1024);
    for (int k = 0; k < steps; ++k)
        ptx::umma_bf16_ts(d_tmem, a_tmem + (SPLIT ? (k >> 2) * 64 + (k & 3) * 8 : k * 8), bd + static_cast<uint64_t>(k * (2048 >> 4)), idesc,
                          accumulate || k > 0 ? 1u : 0u);
}

// A row of W columns per lane from the fp32 accumulator at `acc` to bf16 in global memory, 32 bytes at a time where rows allow it (`wide`: address, D and
// ld are multiples of 32 bytes). `in`: the lane has a row; pieces from `cols` on are left out.
template <int W>
__device__ __forceinline__ void attn_store_row(uint32_t acc, float factor, __nv_bfloat16 *dst, bool in, int cols, bool wide)
{
#pragma unroll
    for (int c = 0; c < W; c += 32) {
        if (c >= cols) break;  // the same for all lanes
        uint32_t o[32];
        __syncwarp();
        ptx::tmem_ld_32x32_wait(acc + c, o);
        if (in) {
#pragma unroll
            for (int k = 0; k < 32; k += 16) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = ptx::pack_bf16x2(__uint_as_float(o[k + 2 * i]) * factor, __uint_as_float(o[k + 2 * i + 1]) * factor);
                if (wide) {
                    if (c + k < cols) ptx::st_global_v8(dst + c + k, w);
                } else {
                    if (c + k < cols) *reinterpret_cast<uint4 *>(dst + c + k) = make_uint4(w[0], w[1], w[2], w[3]);
                    if (c + k + 8 < cols) *reinterpret_cast<uint4 *>(dst + c + k + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                }
            }
        }
    }
    __syncwarp();
}

}  // namespace nb
