// Attention backward, in two passes without atomics (results do not depend on the order in which blocks run):
//
//   P = exp(scale Q K^T - lse)    delta = sum over a row of dout out    dS = P (dO V^T - delta)
//   dQ = scale dS K               (items of 128 queries of a head, over the keys that they see)
//   dV = P^T dO   dK = scale dS^T Q   (items of 128 keys of a head, over the queries that see them and all heads that share the keys)
//
// Both form P and dS themselves: seven products of tiles in place of five, for which no gradient crosses memory in fp32 and
// none is added up by atomics. The second pass works on transposed tiles (S^T = K Q^T, dP^T = V dO^T), so that P^T and dS^T stand in tensor
// memory as the A operands of its sums. P is rounded to bf16 for them (half an ulp, 2^-8 at most); all sums are fp32. A row of dS adds up to next to
// nothing, so what the keys have in common cancels in dQ while the roundings of dS do not, and much the same holds for dK: dS is given in two pieces of
// bf16, the second what the first left out, at the price of a product more in each pass. (With one piece dQ of keys that share half their length
// was 2.7e-3 off and dK up to 2.6e-3, of which their own rounding to bf16 is 1.7e-3.)
//
// What bounds it: of wide heads the products (nine with the second pieces, tensor core busy 49 % in dQ's pass, 64 % in dK and dV's, the latencies from one to the next
// filling the rest), of narrow ones the latencies of a tile's chain, and that products of 64 columns take as long as ones of 96. Measured, causal, both passes: 16 x 1024
// rows, 12 heads of 64: 89 + 107 us (328 TFLOP/s of the five products); 23 sequences in 8000 rows, 16 heads of 128 on 8: 124 + 124 us (468); 8192 rows: 0.87 to 1.02 ms
// (790 TFLOP/s in a burst, 675 under the power cap).
//
// A thread has 64 values of a row of a tile: heads of up to 64 columns take tiles of 64 columns with one warpgroup, two blocks to an SM, which fill
// each other's gaps; wider heads have no tensor memory for that and take tiles of 128 with two warpgroups, as narrow ones do in passes of few items. While these turn dP into dS, the
// tensor core works on what P was ready for, and the other way round. A block that is done with its item takes another (attention_sm100.cuh), whose tiles
// and first products come while the last gradients are being stored.
// Few items with much to walk over (one head of keys for many of queries: a block has all their tiles) are shared by the blocks of a cluster as in the forward
// pass (SPLIT), which add up their sums in a fixed order.
//
// Passes that fill the GPU follow one another, and that of dQ leaves delta behind. Where both together do not, delta has a kernel of its own, and dQ and dK, dV run side by side.
#pragma once
#include "attention_sm100.cuh"

namespace nb {

template <int D_, int WGS_>
struct AttnBwdCfg {
    static constexpr int D = D_, WGS = WGS_, ROWS = 64 * WGS_;  // warpgroups on scores, rows of the streamed tiles
    static constexpr int THREADS = 128 * WGS_ + 128, BLOCKS = 3 - WGS_;
    static constexpr uint32_t TMEM = 512 / BLOCKS;
    static constexpr uint32_t OWN = 128 * D_ * 2, TILE = ROWS * D_ * 2;
    static constexpr int STAGES = D_ == 64 ? 8 : 5;
    static constexpr uint32_t OFF_OWN = 0;          // the item's own tiles: Q, dO or K, V
    static constexpr uint32_t OFF_RING = 2 * OWN;   // the others, in turn
    static constexpr uint32_t OFF_BAR = OFF_RING + STAGES * TILE;
    static constexpr uint32_t OFF_ROWS = OFF_BAR + 384;  // dK, dV: lse and delta of two tiles of queries
    static constexpr uint32_t SMEM = OFF_ROWS + 2048;
    static constexpr int REGS_ROWS = WGS_ == 1 ? 184 : 208, REGS_OTHER = WGS_ == 1 ? 72 : 88;
    static_assert(WGS_ * REGS_ROWS + REGS_OTHER <= (WGS_ + 1) * (WGS_ == 1 ? 128 : 168), "registers");
    static_assert(SMEM <= (BLOCKS == 2 ? 113 * 1024 : 232448), "shared memory");
    static_assert(2 * ROWS + 2 * D_ <= TMEM && 3 * ROWS + D_ <= TMEM, "tensor memory");
};

// Two numbers in two pieces of bf16: rounded, and what that left out, rounded
__device__ __forceinline__ void split_bf16x2(ptx::f2 v, uint32_t &hi, uint32_t &lo)
{
    float a, b;
    ptx::split_f2(v, a, b);
    hi = ptx::pack_bf16x2(a, b);
    ptx::split_f2(ptx::fma2(ptx::make_f2_bits(hi << 16, hi & 0xffff0000u), ptx::make_f2(-1.0f, -1.0f), v), a, b);
    lo = ptx::pack_bf16x2(a, b);
}

__device__ __forceinline__ float dot_bf16x8(uint4 x, uint4 y)
{
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sum = fmaf(ptx::bf16_lo(xs[e]), ptx::bf16_lo(ys[e]), sum);
        sum = fmaf(ptx::bf16_hi(xs[e]), ptx::bf16_hi(ys[e]), sum);
    }
    return sum;
}

// ------------------------------------------------------------------------------------------------ delta
// For both passes, where they run side by side. Lanes that follow one another read what follows one another: D / 8 of them (rounded up) have a row of a head, and the
// next ones the row of the next head. All rows are read, whether they are of a sequence or not.
template <int D>
__global__ void __launch_bounds__(256)
attn_backward_delta_kernel(const AttnBackward b)
{
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    const AttnParams &p = b.a;
    const int piece = static_cast<int>(threadIdx.x) % LANES;
    const int i = static_cast<int>(blockIdx.x * ROWS + threadIdx.x / LANES), row = i / p.heads, head = i - row * p.heads;
    float sum = 0.0f;
    if (row < p.T && piece * 8 < p.D) {
        const uint4 x = ptx::ld_global_v4(static_cast<const __nv_bfloat16 *>(b.dout) + row * b.ld_dout + head * p.D + piece * 8);
        const uint4 y = ptx::ld_global_v4(static_cast<const __nv_bfloat16 *>(p.out) + row * p.ld_out + head * p.D + piece * 8);
        sum = dot_bf16x8(x, y);
    }
#pragma unroll
    for (int e = LANES / 2; e > 0; e /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, e);
    if (row < p.T && piece == 0) b.delta[static_cast<long long>(head) * p.T + row] = sum;
}

// Side by side: the first pass lets the second start when delta and all inputs are there, the second waits for the first at its end, so that what follows waits for both.
// The second starts when every block of the first has either said so, which each does after its own wait for all that came before the passes (delta's kernel, and through its
// wait what it waited for: their writes are in L2 then), or has been taken off the grid. Nothing else orders the second's reads behind those writes, so all of them go to L2:
// tiles by TMA, lse, delta and cu_seqlens by __ldcg. Neither pass reads through L1, whose lines may be of a time before.
__device__ __forceinline__ void attn_backward_begin(int side)
{
    if (side != kAttnFirst) ptx::grid_launch_dependents();
    if (side != kAttnSecond) ptx::grid_dependency_wait();
    if (side == kAttnFirst) ptx::grid_launch_dependents();
}
__device__ __forceinline__ void attn_backward_end(int side)
{
    if (side == kAttnSecond) ptx::grid_dependency_wait();
}

// ------------------------------------------------------------------------------------------------ dQ
template <class Cfg, bool SPLIT>
__global__ void __launch_bounds__(Cfg::THREADS, Cfg::BLOCKS)
attn_backward_q_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmDO, const __grid_constant__ CUtensorMap tmK,
   const __grid_constant__ CUtensorMap tmV, const AttnBackward b)
{
    constexpr int D = Cfg::D, WGS = Cfg::WGS, ROWS = Cfg::ROWS, STAGES = Cfg::STAGES, LOAD = 4 * WGS, MMA = LOAD + 1, LEAST = 2;
    const AttnParams &p = b.a;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t smem = ptx::smem_u32(smem_raw);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = static_cast<int>(threadIdx.x & 31);
    const bool smem_ok = (smem & 1023u) == 0;
    if (!smem_ok && threadIdx.x == 0 && atomicCAS(p.status, 0, kStatusBadSmem) == 0) p.status[2] = static_cast<int>(blockIdx.x);

    const uint32_t bar0 = smem + Cfg::OFF_BAR;
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
    auto named = [&](int i) { return bar0 + 8u * (2 * STAGES + i); };
    // the item's tiles; even and odd tiles of scores; dP; dS; the item's dQ; the item's tiles have been used; a tile that ends inside
    const uint32_t q_bar = named(0), do_bar = named(1), dp_bar = named(4), ds_bar = named(5), done_bar = named(6), own_bar = named(7), part_bar = named(8);
    auto s_bar = [&](uint32_t r) { return named(2 + (r & 1)); };
    const AttnItems items{named(9), bar0 + 304};
    const uint32_t tmem_slot = bar0 + 352, abort_addr = bar0 + 356;
    static_assert(8 * (2 * STAGES + 9 + AttnItems::kBars) <= 304, "barriers");
    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    const WaitCtx wctx2{abort_addr, p.status, 2 * p.timeout_ns};  // a round of work: the wait closest to a stall's cause is reported

    if (warp == LOAD) {
        if (lane < STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        }
        if (lane < 9) ptx::mbar_init(named(lane), lane == 5 ? 4 * WGS : lane == 7 ? 4 * WGS + 1 : 1);
        items.init(lane, 4 * WGS + 1);
        if (lane == 31) ptx::st_shared_u32_volatile(abort_addr, 0);
        ptx::fence_barrier_init();
        if (lane == 30) {
            ptx::prefetch_tmap(&tmQ);
            ptx::prefetch_tmap(&tmDO);
            ptx::prefetch_tmap(&tmK);
            ptx::prefetch_tmap(&tmV);
        }
        __syncwarp();
    }
    if (warp == MMA) {
        ptx::tmem_alloc<1>(tmem_slot, Cfg::TMEM);
        ptx::tmem_relinquish<1>();
    }
    if (warp == LOAD) {  // has no use for tensor memory: its first loads need not wait for it
        ptx::named_bar_arrive(2, Cfg::THREADS);
    } else {
        ptx::tc_fence_before();
        ptx::named_bar_sync(2, Cfg::THREADS);
        ptx::tc_fence_after();
    }
    const uint32_t tmem = ptx::ld_shared_u32_volatile(tmem_slot);
    attn_backward_begin(b.side);
    const uint32_t dp_tm = tmem + 2 * ROWS, dq_tm = tmem + 3 * ROWS;  // scores: two tiles from 0 on
    auto tiles_of = [&](const AttnItem &m) {  // tiles of keys that an item's queries see
        const int tiles = (m.len + ROWS - 1) / ROWS;
        return p.causal ? min(tiles, (m.block + 1) * (128 / ROWS)) : tiles;
    };
    auto part_of = [&](const AttnItem &m) { return attn_part<SPLIT, LEAST>(p.parts, tiles_of(m)); };  // this block's

    if (!smem_ok) {
        // nothing to do
    } else if (warp >= LOAD) {
        ptx::setmaxnreg_dec<Cfg::REGS_OTHER>();
        if (warp == LOAD) {
            // ------------------------------------------------------------ items, and their loads
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0, parts = 0, asked = 0;
            AttnOrder order;
            order.load(p);
            for (int k = 0, at = static_cast<int>(SPLIT ? blockIdx.x / p.parts : blockIdx.x); ok;) {
                AttnItem m{0, 0, -1, 0};
                if (at >= 0) {
                    const AttnSpan s = order.item(p, at / p.heads, false);
                    m = {s.start, s.len, s.block, at % p.heads};
                }
                if (SPLIT || at < 0 || m.block >= 0) {  // slots without a block are passed over
                    ok = items.put(wctx2, k, m);
                    if (!ok || m.block < 0) break;
                    const AttnPart own = part_of(m);
                    const int kv_head = m.head / p.group;
                    for (int i = 0; i < 2 * own.n && ok; ++i) {
                        const int j = own.first + (i >> 1);
                        if (i == 0) {
                            ok = warp_wait(wctx2, own_bar, (static_cast<uint32_t>(k) & 1u) ^ 1u, 130);
                            if (!ok) break;
                            if (ptx::elect_one()) {
                                ptx::mbar_expect_tx(q_bar, Cfg::OWN);
                                attn_load<D>(smem + Cfg::OFF_OWN, &tmQ, q_bar, m.head, m.start + m.block * 128);
                                ptx::mbar_expect_tx(do_bar, Cfg::OWN);
                                attn_load<D>(smem + Cfg::OFF_OWN + Cfg::OWN, &tmDO, do_bar, m.head, m.start + m.block * 128);
                            }
                            __syncwarp();
                        }
                        ok = warp_wait(wctx2, empty_bar(stage), phase ^ 1u, 100 + stage);
                        if (!ok) break;
                        const uint32_t dst = smem + Cfg::OFF_RING + stage * Cfg::TILE;
                        const int valid = m.len - j * ROWS, up = (valid + 15) & ~15;
                        const bool part = valid < ROWS && valid < up;
                        if (ptx::elect_one()) {
                            const uint32_t bar = part ? part_bar : full_bar(stage);
                            ptx::mbar_expect_tx(bar, Cfg::TILE + p.withhold);
                            attn_load<D, ROWS>(dst, (i & 1) ? &tmV : &tmK, bar, kv_head, m.start + j * ROWS);
                        }
                        __syncwarp();
                        if (part) {  // the last tile's keys, then its values
                            ok = warp_wait(wctx, part_bar, parts++ & 1u, 150);
                            if (!ok) break;
                            attn_zero_rows<D, ROWS>(dst, valid, up);
                            ptx::fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(full_bar(stage));
                        }
                        if (++stage == STAGES) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                    if (!ok) break;
                    ++k;
                }
                if (SPLIT) at = -1;
                else ok = items.next(wctx2, asked, at);
            }
        } else if (warp == MMA) {
            // ------------------------------------------------------------ products
            const uint32_t idesc_s = make_idesc(128, ROWS, false, false);
            const int nd = (p.D + 15) & ~15, dsteps = nd / 16;
            const uint32_t idesc_q = make_idesc(128, nd, false, true);
            const uint32_t q_s = smem + Cfg::OFF_OWN, do_s = q_s + Cfg::OWN;
            if (ptx::elect_one()) {
                uint32_t done = 0;  // tiles before this item: 2 done of the ring
                auto stage = [&](uint32_t i) { return static_cast<int>((2 * done + i) % STAGES); };
                auto tile = [&](uint32_t i) { return smem + Cfg::OFF_RING + stage(i) * Cfg::TILE; };
                auto ready = [&](uint32_t i) { return wait_barrier(wctx, full_bar(stage(i)), ((2 * done + i) / STAGES) & 1u, 300 + stage(i)); };
                AttnItem m;
                for (int k = 0; items.take<false>(wctx2, k, m); ++k) {
                    const AttnPart own = part_of(m);
                    const int n = own.n;
                    if (SPLIT && n == 0) continue;
                    const uint32_t kpar = static_cast<uint32_t>(k) & 1u;
                    auto scores = [&](int j) {
                        if (!ready(2 * j)) return false;
                        ptx::tc_fence_after();
                        attn_mma_kk<ROWS>(tmem + ((done + j) & 1) * ROWS, q_s, tile(2 * j), idesc_s, dsteps);
                        ptx::umma_commit<1>(s_bar(done + j));
                        return true;
                    };
                    auto grads = [&](int j) {
                        if (!ready(2 * j + 1)) return false;
                        ptx::tc_fence_after();
                        attn_mma_kk<ROWS>(dp_tm, do_s, tile(2 * j + 1), idesc_s, dsteps);
                        ptx::umma_commit<1>(dp_bar);
                        ptx::umma_commit<1>(empty_bar(stage(2 * j + 1)));
                        if (j + 1 == n) ptx::umma_commit<1>(own_bar);
                        return true;
                    };
                    bool ok = wait_barrier(wctx, q_bar, kpar, 330) && scores(0) && wait_barrier(wctx, do_bar, kpar, 331) && grads(0);
                    for (int j = 0; j < n && ok; ++j) {
                        if (j + 1 < n) ok = scores(j + 1);
                        ok = ok && wait_barrier(wctx2, ds_bar, (done + j) & 1u, 350);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        if (j + 1 < n) ok = grads(j + 1);
                        if (!ok) break;
                        const uint32_t ds = tmem + ((done + j) & 1) * ROWS;
                        const int steps = (min(ROWS, m.len - (own.first + j) * ROWS) + 15) / 16;
                        attn_mma_tn<WGS == 2, ROWS>(dq_tm, ds, tile(2 * j), idesc_q, steps, j > 0);
                        attn_mma_tn<WGS == 2, ROWS>(dq_tm, ds + 32, tile(2 * j), idesc_q, steps, true);  // what the roundings left out
                        ptx::umma_commit<1>(empty_bar(stage(2 * j)));
                    }
                    if (!ok) break;
                    ptx::umma_commit<1>(done_bar);
                    done += n;
                }
            }
            __syncwarp();
        } else if (warp == MMA + 1 && blockIdx.x == 0 && p.cu) {
            attn_report_bounds(p.cu, p.n, p.T, p.status);
        }
    } else {
        // ------------------------------------------------------------ scores: 64 columns of a row per thread
        ptx::setmaxnreg_inc<Cfg::REGS_ROWS>();
        const int half = warp >> 2, q = warp & 3;
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const float sl = p.scale * kLog2e;
        const ptx::f2 sl2 = ptx::make_f2(sl, sl);
        const bool wide = attn_wide(b.dq, b.ld_dq, p.D);
        // A warp reads its 32 rows of out four (two, of wide heads) at a time, 16 bytes a lane, so that lanes that follow one another read what follows
        // one another: a row a lane took the loads eight times as long.
        constexpr int LANES = D / 8, AT_ONCE = 32 / LANES, READS = 32 / AT_ONCE;
        const int piece = lane % LANES, sub = lane / LANES;
        // Side by side delta is there already, and the pass may run before its own wait for what came earlier: nothing of out is read then (see attn_backward_begin).
        // Passes of one warpgroup are of many items, which never run so.
        const bool side = WGS == 2 && b.side != 0;
        uint4 y[READS];
        float l, given = 0.0f;
        // an item's rows of out (or delta) and lse, on their way while the item before is still being stored
        auto fetch = [&](const AttnItem &m) {
            const int row0 = m.block * 128 + q * 32;
            if (side) {
                if (row0 + lane < m.len) given = __ldcg(b.delta + static_cast<long long>(m.head) * p.T + m.start + row0 + lane);
            } else {
#pragma unroll
                for (int c = 0; c < READS; ++c) {
                    const int row = row0 + c * AT_ONCE + sub;
                    y[c] = make_uint4(0, 0, 0, 0);
                    if (row < m.len && piece * 8 < p.D)
                        y[c] = ptx::ld_global_v4(static_cast<const __nv_bfloat16 *>(p.out) + (m.start + row) * p.ld_out + m.head * p.D + piece * 8);
                }
            }
            l = row0 + lane < m.len ? __ldcg(p.lse + static_cast<long long>(m.head) * p.T + m.start + row0 + lane) : 0.0f;
        };
        uint32_t done = 0;  // tiles before this item
        AttnItem m, shared{0, 0, -1, 0};
        bool sums = false;  // of a shared item are there
        bool more = items.take<true>(wctx2, 0, m);
        if (more) fetch(m);
        for (int k = 0; more; ++k) {
            const AttnPart own = part_of(m);
            const int n = own.n;
            if (SPLIT) shared = m;
            if (SPLIT && n == 0) break;
            const int row = m.block * 128 + q * 32 + lane;  // of the sequence
            const long long at = m.start + row;
            float delta = 0.0f;
            const float nl = -kLog2e * l;
            // delta: out from memory, dout from the item's tile. Where two threads have a row, both form all of it: a meeting of theirs could not be left
            // when a wait has run out elsewhere
            if (!warp_wait(wctx2, do_bar, static_cast<uint32_t>(k) & 1u, 430)) break;
            if (side) {
                delta = given;
            } else {
                const uint32_t do_s = smem + Cfg::OFF_OWN + Cfg::OWN + (piece >> 3) * kAttnBox;
#pragma unroll
                for (int c = 0; c < READS; ++c) {
                    const uint32_t r = static_cast<uint32_t>(q * 32 + c * AT_ONCE + sub);
                    uint4 x;
                    ptx::ld_shared_v4(do_s + r * 128 + (((piece & 7) ^ (r & 7)) << 4), x.x, x.y, x.z, x.w);
                    float part = dot_bf16x8(x, y[c]);
#pragma unroll
                    for (int e = LANES / 2; e > 0; e /= 2) part += __shfl_xor_sync(0xffffffffu, part, e);
                    part = __shfl_sync(0xffffffffu, part, (lane % AT_ONCE) * LANES);  // row c AT_ONCE + i stands in the i-th group
                    if (lane / AT_ONCE == c) delta = part;
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(own_bar);  // this warp has read the item's tile
            if (row >= m.len) delta = 0.0f;  // dout may hold anything there
            else if (half == 0 && !side && (!SPLIT || own.first == 0)) b.delta[static_cast<long long>(m.head) * p.T + at] = delta;
            const ptx::f2 base = ptx::make_f2(nl, nl), nd2 = ptx::make_f2(-delta, -delta);
            // keys that all rows of the warp see, that this one sees. Of one key alone the gradient is zero (formed, it would be the rounding of dP - delta)
            const int seen_by_all = min(m.len, p.causal ? row - lane + 1 : m.len), sees = min(m.len, p.causal ? row + 1 : m.len), seen = sees == 1 ? 0 : sees;
            bool ok = true;
            for (int j = 0; j < n; ++j) {
                const uint32_t r = done + j, s_tm = tmem + lanes + (r & 1) * ROWS + half * 64;
                ok = warp_wait(wctx2, s_bar(r), (r >> 1) & 1u, 400);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t s[2][32];
                ptx::tmem_ld_32x32_x2_wait(s_tm, s_tm + 32, s[0], s[1]);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float x, y;
                        ptx::split_f2(ptx::fma2(ptx::make_f2_bits(s[c][i], s[c][i + 1]), sl2, base), x, y);
                        s[c][i] = __float_as_uint(ptx::ex2_approx(x));
                        s[c][i + 1] = __float_as_uint(ptx::ex2_approx(y));
                    }
                ok = warp_wait(wctx2, dp_bar, r & 1u, 410);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t g[2][32], hi[32], lo[32];
                ptx::tmem_ld_32x32_x2_wait(dp_tm + lanes + half * 64, dp_tm + lanes + half * 64 + 32, g[0], g[1]);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const ptx::f2 ds = ptx::mul2(ptx::add2(ptx::make_f2_bits(g[c][i], g[c][i + 1]), nd2), ptx::make_f2_bits(s[c][i], s[c][i + 1]));
                        split_bf16x2(ds, hi[c * 16 + (i >> 1)], lo[c * 16 + (i >> 1)]);
                    }
                if (seen_by_all - (own.first + j) * ROWS - half * 64 < 64) {  // columns that are not seen may hold anything
                    const int limit = seen - (own.first + j) * ROWS - half * 64;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const uint32_t keep = 2 * i + 1 < limit ? 0xffffffffu : 2 * i < limit ? 0xffffu : 0u;
                        hi[i] &= keep;
                        lo[i] &= keep;
                    }
                }
                ptx::tmem_st_32x32(s_tm, hi);
                ptx::tmem_st_32x32(s_tm + 32, lo);
                ptx::tmem_st_wait();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ds_bar);
            }
            if (!ok) break;
            AttnItem next;
            more = items.take<true>(wctx2, k + 1, next);
            if (more) fetch(next);
            if (!warp_wait(wctx2, done_bar, static_cast<uint32_t>(k) & 1u, 420)) break;
            done += n;
            ptx::tc_fence_after();
            constexpr int W = D / WGS;  // columns of a thread
            if (SPLIT) {
                sums = true;
                break;
            }
            attn_store_row<W>(dq_tm + lanes + half * W, p.scale, static_cast<__nv_bfloat16 *>(b.dq) + at * b.ld_dq + m.head * p.D + half * W, row < m.len,
                              p.D - half * W, wide);
            ptx::tc_fence_before();
            m = next;
        }
        ptx::tc_fence_before();
        if (SPLIT) {
            const AttnShare c(p.parts);
            ptx::cluster_sync();  // all blocks' products are done: their tiles' memory is free
            if (sums) attn_give_row<D / WGS, D>(c, dq_tm + lanes + half * (D / WGS), smem, q * 32 + lane, half * (D / WGS));
            const bool failed = c.failed(abort_addr);
            ptx::cluster_sync();
            if (shared.block >= 0 && !failed) {
                const int row0 = shared.block * 128;
                attn_join_rows<D, 128 * WGS>(c, smem, attn_sharers<LEAST>(p.parts, tiles_of(shared)),
                                             static_cast<__nv_bfloat16 *>(b.dq) + (shared.start + row0) * b.ld_dq + shared.head * p.D, b.ld_dq,
                                             min(128, shared.len - row0), p.D, [&](int, int) { return p.scale; });
            }
        }
    }
    if (SPLIT && (!smem_ok || warp >= LOAD)) {
        __syncwarp();
        ptx::cluster_sync();
        ptx::cluster_sync();
    }

    // ---------------------------------------------------------------- common exit
    if (ptx::ld_shared_u32_volatile(abort_addr) != 0) {  // a wait ran out: let copies and products in flight land
        const uint64_t t0 = ptx::globaltimer_ns();
        while (ptx::globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc<1>(tmem, Cfg::TMEM);
    }
    attn_backward_end(b.side);
}

// ------------------------------------------------------------------------------------------------ dK, dV
template <class Cfg, bool SPLIT>
__global__ void __launch_bounds__(Cfg::THREADS, Cfg::BLOCKS)
attn_backward_kv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmDO, const __grid_constant__ CUtensorMap tmK,
   const __grid_constant__ CUtensorMap tmV, const AttnBackward b)
{
    constexpr int D = Cfg::D, WGS = Cfg::WGS, ROWS = Cfg::ROWS, STAGES = Cfg::STAGES, LOAD = 4 * WGS, MMA = LOAD + 1, LEAST = 2;
    const AttnParams &p = b.a;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t smem = ptx::smem_u32(smem_raw);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = static_cast<int>(threadIdx.x & 31);
    const bool smem_ok = (smem & 1023u) == 0;
    if (!smem_ok && threadIdx.x == 0 && atomicCAS(p.status, 0, kStatusBadSmem) == 0) p.status[2] = static_cast<int>(blockIdx.x);

    const uint32_t bar0 = smem + Cfg::OFF_BAR;
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
    auto named = [&](int i) { return bar0 + 8u * (2 * STAGES + i); };
    // the item's tiles; scores, P, dP, dS; the item's gradients; the item's tiles have been used; a tile that ends inside
    const uint32_t k_bar = named(0), v_bar = named(1), s_bar = named(2), p_bar = named(3), dp_bar = named(4), ds_bar = named(5), done_bar = named(6),
                   own_bar = named(7), part_bar = named(8);
    auto rows_bar = [&](uint32_t r) { return named(9 + (r & 1)); };    // lse and delta of a tile of queries are there
    auto rfree_bar = [&](uint32_t r) { return named(11 + (r & 1)); };  // and have been read
    const AttnItems items{named(13), bar0 + 304};
    const uint32_t tmem_slot = bar0 + 352, abort_addr = bar0 + 356;
    static_assert(8 * (2 * STAGES + 13 + AttnItems::kBars) <= 304, "barriers");
    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    const WaitCtx wctx2{abort_addr, p.status, 2 * p.timeout_ns};  // a round of work: the wait closest to a stall's cause is reported

    if (warp == LOAD) {
        if (lane < STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        }
        if (lane < 13) ptx::mbar_init(named(lane), lane == 3 || lane == 5 || lane >= 11 ? 4 * WGS : 1);
        items.init(lane, 4 * WGS + 2);
        if (lane == 31) ptx::st_shared_u32_volatile(abort_addr, 0);
        ptx::fence_barrier_init();
        if (lane == 30) {
            ptx::prefetch_tmap(&tmQ);
            ptx::prefetch_tmap(&tmDO);
            ptx::prefetch_tmap(&tmK);
            ptx::prefetch_tmap(&tmV);
        }
        __syncwarp();
    }
    if (warp == MMA) {
        ptx::tmem_alloc<1>(tmem_slot, Cfg::TMEM);
        ptx::tmem_relinquish<1>();
    }
    if (warp == LOAD) {  // has no use for tensor memory: its first loads need not wait for it
        ptx::named_bar_arrive(2, Cfg::THREADS);
    } else {
        ptx::tc_fence_before();
        ptx::named_bar_sync(2, Cfg::THREADS);
        ptx::tc_fence_after();
    }
    const uint32_t tmem = ptx::ld_shared_u32_volatile(tmem_slot);
    attn_backward_begin(b.side);
    const int kv_heads = p.heads / p.group;
    const uint32_t s_tm = tmem, dp_tm = tmem + ROWS, dv_tm = tmem + 2 * ROWS, dk_tm = dv_tm + D;
    // tiles of queries that see an item's keys: from first_of on, per head
    auto first_of = [&](const AttnItem &m) { return p.causal ? m.block * (128 / ROWS) : 0; };
    auto tiles_of = [&](const AttnItem &m) { return (m.len + ROWS - 1) / ROWS - first_of(m); };
    auto part_of = [&](const AttnItem &m) { return attn_part<SPLIT, LEAST>(p.parts, tiles_of(m) * p.group); };  // this block's, of all heads' tiles

    if (!smem_ok) {
        // nothing to do
    } else if (warp >= LOAD) {
        ptx::setmaxnreg_dec<Cfg::REGS_OTHER>();
        if (warp == LOAD) {
            // ------------------------------------------------------------ items, and their loads
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0, parts = 0, asked = 0;
            AttnOrder order;
            order.load(p);
            for (int k = 0, at = static_cast<int>(SPLIT ? blockIdx.x / p.parts : blockIdx.x); ok;) {
                AttnItem m{0, 0, -1, 0};
                if (at >= 0) {
                    const AttnSpan s = order.item(p, at / kv_heads, true);
                    m = {s.start, s.len, s.block, at % kv_heads};
                }
                if (SPLIT || at < 0 || m.block >= 0) {  // slots without a block are passed over
                    ok = items.put(wctx2, k, m);
                    if (!ok || m.block < 0) break;
                    ok = warp_wait(wctx2, own_bar, (static_cast<uint32_t>(k) & 1u) ^ 1u, 130);
                    if (!ok) break;
                    const int first = first_of(m), per_head = tiles_of(m);
                    const AttnPart own = part_of(m);
                    if (own.n > 0 && ptx::elect_one()) {
                        ptx::mbar_expect_tx(k_bar, Cfg::OWN);
                        attn_load<D>(smem + Cfg::OFF_OWN, &tmK, k_bar, m.head, m.start + m.block * 128);
                        ptx::mbar_expect_tx(v_bar, Cfg::OWN);
                        attn_load<D>(smem + Cfg::OFF_OWN + Cfg::OWN, &tmV, v_bar, m.head, m.start + m.block * 128);
                    }
                    __syncwarp();
                    int t = own.first % per_head, head = m.head * p.group + own.first / per_head;
                    for (int i = 0; i < 2 * own.n && ok; ++i) {
                        ok = warp_wait(wctx2, empty_bar(stage), phase ^ 1u, 100 + stage);
                        if (!ok) break;
                        const uint32_t dst = smem + Cfg::OFF_RING + stage * Cfg::TILE;
                        const int row = (first + t) * ROWS, valid = m.len - row, up = (valid + 15) & ~15;
                        const bool part = valid < ROWS && valid < up;
                        if (ptx::elect_one()) {
                            const uint32_t bar = part ? part_bar : full_bar(stage);
                            ptx::mbar_expect_tx(bar, Cfg::TILE + p.withhold);
                            attn_load<D, ROWS>(dst, (i & 1) ? &tmDO : &tmQ, bar, head, m.start + row);
                        }
                        __syncwarp();
                        if (part) {  // the last tile of each head's queries, then of their gradients
                            ok = warp_wait(wctx, part_bar, parts++ & 1u, 150);
                            if (!ok) break;
                            // Queries are filled up with the last one: a key with a score of -infinity for all of them has P = 0 there too (with
                            // queries of zeros its infinity would make NaN)
                            if (i & 1) attn_zero_rows<D, ROWS>(dst, valid, up);
                            else attn_repeat_row<D, ROWS>(dst, valid, up);
                            ptx::fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(full_bar(stage));
                        }
                        if (++stage == STAGES) {
                            stage = 0;
                            phase ^= 1u;
                        }
                        if ((i & 1) && ++t == per_head) {
                            t = 0;
                            ++head;
                        }
                    }
                    if (!ok) break;
                    ++k;
                }
                if (SPLIT) at = -1;
                else ok = items.next(wctx2, asked, at);
            }
        } else if (warp == MMA) {
            // ------------------------------------------------------------ products
            const uint32_t idesc_s = make_idesc(128, ROWS, false, false);
            const int nd = (p.D + 15) & ~15, dsteps = nd / 16;
            const uint32_t idesc_d = make_idesc(128, nd, false, true);
            const uint32_t k_s = smem + Cfg::OFF_OWN, v_s = k_s + Cfg::OWN;
            if (ptx::elect_one()) {
                uint32_t done = 0;  // tiles before this item: 2 done of the ring
                auto stage = [&](uint32_t i) { return static_cast<int>((2 * done + i) % STAGES); };
                auto tile = [&](uint32_t i) { return smem + Cfg::OFF_RING + stage(i) * Cfg::TILE; };
                auto ready = [&](uint32_t i) { return wait_barrier(wctx, full_bar(stage(i)), ((2 * done + i) / STAGES) & 1u, 300 + stage(i)); };
                AttnItem m;
                for (int k = 0; items.take<false>(wctx2, k, m); ++k) {
                    const int first = first_of(m), per_head = tiles_of(m);
                    const AttnPart own = part_of(m);
                    const int n = own.n;
                    if (SPLIT && n == 0) continue;
                    const uint32_t kpar = static_cast<uint32_t>(k) & 1u;
                    auto scores = [&](int i) {
                        if (!ready(2 * i)) return false;
                        ptx::tc_fence_after();
                        attn_mma_kk<ROWS>(s_tm, k_s, tile(2 * i), idesc_s, dsteps);
                        ptx::umma_commit<1>(s_bar);
                        return true;
                    };
                    auto grads = [&](int i) {
                        if (!ready(2 * i + 1)) return false;
                        ptx::tc_fence_after();
                        attn_mma_kk<ROWS>(dp_tm, v_s, tile(2 * i + 1), idesc_s, dsteps);
                        ptx::umma_commit<1>(dp_bar);
                        if (i + 1 == n) ptx::umma_commit<1>(own_bar);
                        return true;
                    };
                    bool ok = wait_barrier(wctx, k_bar, kpar, 330) && scores(0) && wait_barrier(wctx, v_bar, kpar, 331) && grads(0);
                    int t = own.first % per_head;
                    for (int i = 0; i < n && ok; ++i) {
                        const int steps = (min(ROWS, m.len - (first + t) * ROWS) + 15) / 16;
                        ok = wait_barrier(wctx2, p_bar, (done + i) & 1u, 350);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        attn_mma_tn<WGS == 2, ROWS>(dv_tm, s_tm, tile(2 * i + 1), idesc_d, steps, i > 0);
                        ptx::umma_commit<1>(empty_bar(stage(2 * i + 1)));
                        if (i + 1 < n) ok = scores(i + 1);
                        ok = ok && wait_barrier(wctx2, ds_bar, (done + i) & 1u, 360);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        attn_mma_tn<WGS == 2, ROWS>(dk_tm, dp_tm, tile(2 * i), idesc_d, steps, i > 0);
                        attn_mma_tn<WGS == 2, ROWS>(dk_tm, dp_tm + 32, tile(2 * i), idesc_d, steps, true);  // what the roundings left out
                        ptx::umma_commit<1>(empty_bar(stage(2 * i)));
                        if (i + 1 < n) ok = grads(i + 1);
                        if (++t == per_head) t = 0;
                    }
                    if (!ok) break;
                    ptx::umma_commit<1>(done_bar);
                    done += n;
                }
            }
            __syncwarp();
        } else if (warp == MMA + 1) {
            // ------------------------------------------------------------ lse and delta of the queries, negated, lse in units of log 2
            uint32_t r = 0;
            AttnItem m;
            for (int k = 0; items.take<true>(wctx2, k, m); ++k) {
                const int first = first_of(m), per_head = tiles_of(m);
                bool ok = true;
                const AttnPart own = part_of(m);
                int t = own.first % per_head, head = m.head * p.group + own.first / per_head;
                for (int i = 0; i < own.n && ok; ++i, ++r) {
                    const long long at = static_cast<long long>(head) * p.T + m.start + (first + t) * ROWS;
                    float l[ROWS / 32], d[ROWS / 32];
#pragma unroll
                    for (int e = 0; e < ROWS / 32; ++e) {
                        const int x = e * 32 + lane;
                        const bool in = (first + t) * ROWS + x < m.len;  // rows behind the last have no probability
                        l[e] = in ? -kLog2e * __ldcg(p.lse + at + x) : -INFINITY;
                        d[e] = in ? -__ldcg(b.delta + at + x) : 0.0f;
                    }
                    ok = warp_wait(wctx2, rfree_bar(r), ((r >> 1) & 1u) ^ 1u, 530);
                    if (!ok) break;
                    const uint32_t dst = smem + Cfg::OFF_ROWS + (r & 1) * 1024 + lane * 4;
#pragma unroll
                    for (int e = 0; e < ROWS / 32; ++e) {
                        ptx::st_shared_f32(dst + e * 128, l[e]);
                        ptx::st_shared_f32(dst + 512 + e * 128, d[e]);
                    }
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(rows_bar(r));
                    if (++t == per_head) {
                        t = 0;
                        ++head;
                    }
                }
                if (!ok) break;
            }
        } else if (warp == MMA + 2 && blockIdx.x == 0 && p.cu) {
            attn_report_bounds(p.cu, p.n, p.T, p.status);
        }
    } else {
        // ------------------------------------------------------------ scores: 64 columns (queries) of a row (a key) per thread
        ptx::setmaxnreg_inc<Cfg::REGS_ROWS>();
        const int half = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const float sl = p.scale * kLog2e;
        const ptx::f2 sl2 = ptx::make_f2(sl, sl);
        uint32_t it = 0;  // tiles so far
        AttnItem m, shared{0, 0, -1, 0};
        bool sums = false;  // of a shared item are there
        for (int k = 0; items.take<true>(wctx2, k, m); ++k) {
            const int first = first_of(m), per_head = tiles_of(m);
            const AttnPart own = part_of(m);
            const int n = own.n;
            if (SPLIT) shared = m;
            if (SPLIT && n == 0) continue;
            // the first key is all that the first query sees, and has no gradient from it
            const bool lonely = (p.causal || m.len == 1) && m.block == 0 && r == 0 && half == 0;
            bool ok = true;
            int t = own.first % per_head;
            for (int i = 0; i < n; ++i, ++it) {
                const uint32_t par = it & 1u;
                const uint32_t rows = smem + Cfg::OFF_ROWS + par * 1024 + half * 256;
                ok = warp_wait(wctx2, rows_bar(it), (it >> 1) & 1u, 540) && warp_wait(wctx2, s_bar, par, 400);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t s[2][32], pk[32];
                ptx::tmem_ld_32x32_x2_wait(s_tm + lanes + half * 64, s_tm + lanes + half * 64 + 32, s[0], s[1]);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float4 l;
                        ptx::ld_shared_f32x4(rows + (c * 32 + e) * 4, l);
                        float x[4];
                        ptx::split_f2(ptx::fma2(ptx::make_f2_bits(s[c][e], s[c][e + 1]), sl2, ptx::make_f2(l.x, l.y)), x[0], x[1]);
                        ptx::split_f2(ptx::fma2(ptx::make_f2_bits(s[c][e + 2], s[c][e + 3]), sl2, ptx::make_f2(l.z, l.w)), x[2], x[3]);
#pragma unroll
                        for (int v = 0; v < 4; ++v) s[c][e + v] = __float_as_uint(ptx::ex2_approx(x[v]));
                    }
                // a key is seen by queries from its own row on: columns below `hidden` are not
                const int hidden = p.causal ? m.block * 128 + r - (first + t) * ROWS - half * 64 : 0;
                const bool cut = p.causal && m.block * 128 + q * 32 + 31 > (first + t) * ROWS + half * 64;
                if (cut) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (c * 32 + e < hidden) s[c][e] = 0u;
                }
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) pk[c * 16 + (e >> 1)] = ptx::pack_bf16x2(__uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1]));
                ptx::tmem_st_32x32(s_tm + lanes + half * 64, pk);
                ptx::tmem_st_wait();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_bar);

                ok = warp_wait(wctx2, dp_bar, par, 410);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t g[2][32], lo[32];
                ptx::tmem_ld_32x32_x2_wait(dp_tm + lanes + half * 64, dp_tm + lanes + half * 64 + 32, g[0], g[1]);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float4 d;
                        ptx::ld_shared_f32x4(rows + 512 + (c * 32 + e) * 4, d);
#pragma unroll
                        for (int v = 0; v < 4; v += 2)
                            split_bf16x2(ptx::mul2(ptx::add2(ptx::make_f2_bits(g[c][e + v], g[c][e + v + 1]), v ? ptx::make_f2(d.z, d.w) : ptx::make_f2(d.x, d.y)),
                                                   ptx::make_f2_bits(s[c][e + v], s[c][e + v + 1])),
                                         pk[c * 16 + ((e + v) >> 1)], lo[c * 16 + ((e + v) >> 1)]);
                    }
                if (cut) {  // what is not seen may hold anything
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const uint32_t keep = 2 * e >= hidden ? 0xffffffffu : 2 * e + 1 >= hidden ? 0xffff0000u : 0u;
                        pk[e] &= keep;
                        lo[e] &= keep;
                    }
                }
                if (lonely && first + t == 0) {
                    pk[0] &= 0xffff0000u;
                    lo[0] &= 0xffff0000u;
                }
                ptx::tmem_st_32x32(dp_tm + lanes + half * 64, pk);
                ptx::tmem_st_32x32(dp_tm + lanes + half * 64 + 32, lo);
                ptx::tmem_st_wait();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(ds_bar);
                    ptx::mbar_arrive(rfree_bar(it));
                }
                if (++t == per_head) t = 0;
            }
            if (ok) ok = warp_wait(wctx2, done_bar, static_cast<uint32_t>(k) & 1u, 420);
            if (!ok) break;
            ptx::tc_fence_after();
            if (SPLIT) {
                sums = true;
                break;
            }
            const int row = m.block * 128 + r;
            const long long at = m.start + row;
            if (WGS == 1 || half == 0)
                attn_store_row<D>(dv_tm + lanes, 1.0f, static_cast<__nv_bfloat16 *>(b.dv) + at * b.ld_dv + m.head * p.D, row < m.len, p.D,
                                  attn_wide(b.dv, b.ld_dv, p.D));
            if (WGS == 1 || half == 1)
                attn_store_row<D>(dk_tm + lanes, p.scale, static_cast<__nv_bfloat16 *>(b.dk) + at * b.ld_dk + m.head * p.D, row < m.len, p.D,
                                  attn_wide(b.dk, b.ld_dk, p.D));
            ptx::tc_fence_before();
        }
        ptx::tc_fence_before();
        if (SPLIT) {
            const AttnShare c(p.parts);
            const uint32_t of_dk = smem + 128 * D * 4;
            ptx::cluster_sync();  // all blocks' products are done: their tiles' memory is free
            if (sums && (WGS == 1 || half == 0)) attn_give_row<D, D>(c, dv_tm + lanes, smem, r, 0);
            if (sums && (WGS == 1 || half == 1)) attn_give_row<D, D>(c, dk_tm + lanes, of_dk, r, 0);
            const bool failed = c.failed(abort_addr);
            ptx::cluster_sync();
            if (shared.block >= 0 && !failed) {
                const int row0 = shared.block * 128, sharers = attn_sharers<LEAST>(p.parts, tiles_of(shared) * p.group), rows = min(128, shared.len - row0);
                const long long at = shared.start + row0;
                attn_join_rows<D, 128 * WGS>(c, smem, sharers, static_cast<__nv_bfloat16 *>(b.dv) + at * b.ld_dv + shared.head * p.D, b.ld_dv, rows, p.D,
                                             [](int, int) { return 1.0f; });
                attn_join_rows<D, 128 * WGS>(c, of_dk, sharers, static_cast<__nv_bfloat16 *>(b.dk) + at * b.ld_dk + shared.head * p.D, b.ld_dk, rows, p.D,
                                             [&](int, int) { return p.scale; });
            }
        }
    }
    if (SPLIT && (!smem_ok || warp >= LOAD)) {
        __syncwarp();
        ptx::cluster_sync();
        ptx::cluster_sync();
    }

    // ---------------------------------------------------------------- common exit
    if (ptx::ld_shared_u32_volatile(abort_addr) != 0) {  // a wait ran out: let copies and products in flight land
        const uint64_t t0 = ptx::globaltimer_ns();
        while (ptx::globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc<1>(tmem, Cfg::TMEM);
    }
    attn_backward_end(b.side);
}

}  // namespace nb
