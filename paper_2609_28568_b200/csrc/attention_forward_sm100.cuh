// Attention forward, on items of 128 rows of a sequence and head, two blocks to an SM.
//
// A thread of a warpgroup owns a query: scores come from tensor memory, 64 keys at a time, the running maximum and sum stay in
// registers, probabilities go back to tensor memory as bf16, over the scores, and are the A operand of the product with V. With two tiles of
// scores the next one is formed while the exponentials of this one run.
//
// What bounds it are the exponentials (16 a clock and SM) and the latencies of a step (scores, maximum, exponentials, the way back); the two
// blocks of an SM fill each other's gaps. Two tiles of queries in one block that share keys and values took as long on one long sequence and a fifth longer
// on packed ones; 128 keys at a time took the same, and more registers. A quarter of the exponentials formed by a polynomial, on the multipliers, saved
// nothing: those instructions wait in the same line. Measured, causal: 16 x 1024 rows, 12 heads of 64: 55 us (469 TFLOP/s of what is seen, tensor core busy 27 %);
// 23 sequences in 8000 rows, 16 heads of 128: 70 us (708 TFLOP/s, 49 %); 16384 rows: 0.85 to 1.02 ms (1.29 PFLOP/s in a burst, 1.08 under the power cap).
//
// Items differ in work by the length of their sequence and their place in it, and are short beside what a block costs to start (first loads, first
// products: 2 to 3 us). So a block that is done with its item takes another off the grid (the hardware hands out blocks that have not
// started), asks for it when its own loads are on their way, and its loads and first scores come while the last output is still being stored.
//
// Few items with many keys are shared (SPLIT): the blocks of a cluster have a part of the keys each, with a maximum and a sum of its own, and every block joins an equal share of the
// rows from what the others write into its shared memory, the parts in their order. That costs 4 us, and halves a long item (nb_linear.cu has what it measured).
//
// The output accumulator in tensor memory is rescaled only when a row's maximum has grown by more than 2^8 since the last
// rescaling: until then probabilities up to 2^8 are summed against the old maximum, which changes no bit of their relative precision.
// Probabilities are rounded to bf16 for the tensor core (half an ulp, 2^-8 of each at most); their sum takes them unrounded.
#pragma once
#include "attention_sm100.cuh"

namespace nb {

template <int D_>
struct AttnFwdCfg {
    static constexpr int D = D_, KEYS = 64;  // keys of a tile
    static constexpr int THREADS = 256, BLOCKS = 2;
    static constexpr uint32_t TMEM = 256, TM_O = 2 * KEYS;  // scores from 0 on
    static constexpr uint32_t Q_BYTES = 128 * D_ * 2, TILE = KEYS * D_ * 2;
    static constexpr uint32_t MOST = 113 * 1024;  // of shared memory: 228 KB of an SM less 1 KB a block
    static constexpr int STAGES = (MOST - Q_BYTES - 512) / TILE < 8 ? (MOST - Q_BYTES - 512) / TILE : 8;  // keys and values in turn
    static constexpr uint32_t OFF_Q = 0;
    static constexpr uint32_t OFF_KV = Q_BYTES;
    static constexpr uint32_t OFF_BAR = OFF_KV + STAGES * TILE;
    static constexpr uint32_t SMEM = OFF_BAR + 512;
    // registers of a thread after they have been divided anew: within the 128 that the block is launched with
    static constexpr int REGS_ROWS = 192, REGS_OTHER = 64;
    static_assert(REGS_ROWS + REGS_OTHER <= 2 * 128, "registers");
    static_assert(TMEM >= TM_O + D_ && STAGES >= 4 && SMEM <= MOST, "memory");
    static_assert(128 * D_ * 4 + 1024 <= OFF_BAR, "a part's sums, maxima");
};

template <class Cfg, bool SPLIT>
__global__ void __launch_bounds__(Cfg::THREADS, Cfg::BLOCKS)
attn_forward_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                    const AttnParams p)
{
    constexpr int D = Cfg::D, KEYS = Cfg::KEYS, STAGES = Cfg::STAGES, LOAD = 4, MMA = 5, LEAST = 4;
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
    const uint32_t q_bar = named(0), qfree_bar = named(1);    // queries are there, and have been used
    // of even and odd tiles, since a warpgroup may be two of them ahead of the products
    auto s_bar = [&](uint32_t r) { return named(2 + (r & 1)); };  // scores are there
    auto p_bar = [&](uint32_t r) { return named(4 + (r & 1)); };  // probabilities are there
    auto o_bar = [&](uint32_t r) { return named(6 + (r & 1)); };  // their product with V is done
    auto half = [](uint32_t r) { return (r >> 1) & 1u; };         // parity of the r-th tile in them
    const uint32_t part_bar = named(8);  // values of a sequence's last tile have landed
    const AttnItems items{named(9), bar0 + 400};
    static_assert(8 * (2 * STAGES + 9 + AttnItems::kBars) <= 400, "barriers");
    const uint32_t tmem_slot = bar0 + 480, abort_addr = bar0 + 484;

    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    // The waits for a whole round of work have twice the limit, so that the wait closest to the cause of a stall is reported.
    const WaitCtx wctx2{abort_addr, p.status, 2 * p.timeout_ns};
    auto tiles_of = [&](const AttnItem &m) {  // tiles of keys that an item's queries see
        const int tiles = (m.len + KEYS - 1) / KEYS;
        return p.causal ? min(tiles, (m.block + 1) * (128 / KEYS)) : tiles;
    };
    auto part_of = [&](const AttnItem &m) { return attn_part<SPLIT, LEAST>(p.parts, tiles_of(m)); };  // this block's

    if (warp == LOAD) {
        if (lane < STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        }
        if (lane < 9) ptx::mbar_init(named(lane), lane == 4 || lane == 5 ? 4 : 1);
        items.init(lane, 5);
        if (lane == 31) ptx::st_shared_u32_volatile(abort_addr, 0);
        ptx::fence_barrier_init();
        if (lane == 30) {
            ptx::prefetch_tmap(&tmQ);
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
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();

    if (!smem_ok) {
        // nothing to do
    } else if (warp >= LOAD) {
        ptx::setmaxnreg_dec<Cfg::REGS_OTHER>();
        if (warp == LOAD) {
            // ------------------------------------------------------------ items, and their loads: keys of a tile, its values
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0, parts = 0, asked = 0, used = 0;
            AttnOrder order;
            order.load(p);
            for (int k = 0, at = static_cast<int>(SPLIT ? blockIdx.x / p.parts : blockIdx.x); ok;) {
                AttnItem m{0, 0, -1, 0};
                if (at >= 0) {
                    const AttnSpan s = order.item(p, at / p.heads, false);
                    m = {s.start, s.len, s.block, at % p.heads};
                }
                if (SPLIT || at < 0 || m.block >= 0) {  // slots without a block are passed over
                    ok = items.put(wctx2, k++, m);
                    if (!ok || m.block < 0) break;
                    const AttnPart own = part_of(m);
                    const int kv_head = m.head / p.group;
                    for (int i = 0; i < 2 * own.n && ok; ++i) {
                        const int j = own.first + (i >> 1);
                        ok = warp_wait(wctx2, empty_bar(stage), phase ^ 1u, 100 + stage);
                        if (!ok) break;
                        const uint32_t dst = smem + Cfg::OFF_KV + stage * Cfg::TILE;
                        const int valid = m.len - j * KEYS, up = (valid + 15) & ~15;
                        const bool part = (i & 1) && valid < KEYS && valid < up;
                        if (ptx::elect_one()) {
                            const uint32_t bar = part ? part_bar : full_bar(stage);
                            ptx::mbar_expect_tx(bar, Cfg::TILE + p.withhold);
                            attn_load<D, KEYS>(dst, (i & 1) ? &tmV : &tmK, bar, kv_head, m.start + j * KEYS);
                        }
                        __syncwarp();
                        if (part) {
                            ok = warp_wait(wctx, part_bar, parts++ & 1u, 150);
                            if (!ok) break;
                            attn_zero_rows<D, KEYS>(dst, valid, up);
                            ptx::fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(full_bar(stage));
                        }
                        if (++stage == STAGES) {
                            stage = 0;
                            phase ^= 1u;
                        }
                        if (i == 0) {  // the queries after the first keys: these may be waiting for the item before
                            ok = warp_wait(wctx2, qfree_bar, (used++ & 1u) ^ 1u, 130);
                            if (ok && ptx::elect_one()) {
                                ptx::mbar_expect_tx(q_bar, Cfg::Q_BYTES);
                                attn_load<D>(smem + Cfg::OFF_Q, &tmQ, q_bar, m.head, m.start + m.block * 128);
                            }
                            __syncwarp();
                        }
                    }
                    if (!ok) break;
                }
                if (SPLIT) at = -1;
                else ok = items.next(wctx2, asked, at);
            }
        } else if (warp == MMA) {
            // ------------------------------------------------------------ products
            const uint32_t idesc_s = make_idesc(128, KEYS, false, false);
            const int nd = (p.D + 15) & ~15, dsteps = nd / 16;
            const uint32_t idesc_o = make_idesc(128, nd, false, true);
            if (ptx::elect_one()) {
                uint32_t done = 0;  // tiles before this item: 2 done of the ring
                auto stage = [&](uint32_t i) { return static_cast<int>((2 * done + i) % STAGES); };
                auto tile = [&](uint32_t i) { return smem + Cfg::OFF_KV + stage(i) * Cfg::TILE; };
                auto ready = [&](uint32_t i) { return wait_barrier(wctx, full_bar(stage(i)), ((2 * done + i) / STAGES) & 1u, 300 + stage(i)); };
                AttnItem m;
                for (int k = 0; items.take<false>(wctx2, k, m); ++k) {
                    const AttnPart own = part_of(m);
                    const int n = own.n;
                    if (SPLIT && n == 0) continue;
                    auto scores = [&](int j) {
                        if (!ready(2 * j)) return false;
                        ptx::tc_fence_after();
                        attn_mma_kk<KEYS>(tmem + ((done + j) & 1) * KEYS, smem + Cfg::OFF_Q, tile(2 * j), idesc_s, dsteps);
                        ptx::umma_commit<1>(s_bar(done + j));
                        ptx::umma_commit<1>(empty_bar(stage(2 * j)));
                        if (j + 1 == n) ptx::umma_commit<1>(qfree_bar);
                        return true;
                    };
                    bool ok = wait_barrier(wctx, q_bar, static_cast<uint32_t>(k) & 1u, 330) && scores(0);
                    for (int j = 0; j < n && ok; ++j) {
                        if (j + 1 < n) ok = scores(j + 1);
                        ok = ok && ready(2 * j + 1) && wait_barrier(wctx2, p_bar(done + j), half(done + j), 350);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        attn_mma_tn<false, KEYS>(tmem + Cfg::TM_O, tmem + ((done + j) & 1) * KEYS, tile(2 * j + 1), idesc_o,
                                                 (min(KEYS, m.len - (own.first + j) * KEYS) + 15) / 16, j > 0);
                        ptx::umma_commit<1>(o_bar(done + j));
                        ptx::umma_commit<1>(empty_bar(stage(2 * j + 1)));
                    }
                    if (!ok) break;
                    done += n;
                }
            }
            __syncwarp();
        } else if (warp == MMA + 1 && blockIdx.x == 0 && p.cu) {
            attn_report_bounds(p.cu, p.n, p.T, p.status);
        }
    } else {
        // ------------------------------------------------------------ scores: a row per thread
        ptx::setmaxnreg_inc<Cfg::REGS_ROWS>();
        const uint32_t tm = tmem + (static_cast<uint32_t>(warp * 32) << 16), o_tm = tm + Cfg::TM_O;
        const float sl = p.scale * kLog2e;
        const ptx::f2 sl2 = ptx::make_f2(sl, sl);
        const bool wide = attn_wide(p.out, p.ld_out, p.D);
        uint32_t done = 0;  // tiles before this item
        AttnItem m, shared{0, 0, -1, 0};
        bool sums = false;  // of a shared item are there
        float top = 0.0f, total = 0.0f;  // the maximum that the sums refer to (of unscaled scores), the sum
        for (int k = 0; items.take<true>(wctx2, k, m); ++k) {
            const AttnPart own = part_of(m);
            const int n = own.n;
            if (SPLIT) shared = m;
            if (SPLIT && n == 0) continue;
            const int first = m.block * 128 + warp * 32, row = first + lane;  // of the sequence
            // keys that some row of the warp sees, all of them, this one
            const int seen_by_one = min(m.len, p.causal ? first + 32 : m.len), seen_by_all = min(m.len, p.causal ? first + 1 : m.len),
                      seen = min(m.len, p.causal ? row + 1 : m.len);
            total = 0.0f;
            bool ok = true;
            for (int j = 0; j < n; ++j) {
                const uint32_t r = done + j, s_tm = tm + (r & 1) * KEYS;
                ok = warp_wait(wctx2, s_bar(r), half(r), 400);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t s[2][32];
                ptx::tmem_ld_32x32_x2_wait(s_tm, s_tm + 32, s[0], s[1]);
                const int key = (own.first + j) * KEYS, one = seen_by_one - key;
                if (seen_by_all - key < KEYS) {
                    const int limit = seen - key;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c * 32 + i >= limit) s[c][i] = 0xff800000u;
                }
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaxf(__uint_as_float(s[0][e]), __uint_as_float(s[1][e]));
#pragma unroll
                for (int i = 8; i < 32; i += 8)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = ptx::max3(x[e], __uint_as_float(s[0][i + e]), __uint_as_float(s[1][i + e]));
                const float now = ptx::max3(ptx::max3(x[0], x[1], x[2]), ptx::max3(x[3], x[4], x[5]), fmaxf(x[6], x[7]));
                if (j == 0) {
                    top = now;
                } else {
                    // only rows that grew that much: a row's bits do not depend on the others of its warp
                    const bool grown = (now - top) * sl > 8.0f;
                    if (__any_sync(0xffffffffu, grown)) {
                        const float f = grown ? ptx::ex2_approx((top - now) * sl) : 1.0f;
                        total *= f;
                        if (grown) top = now;
                        ok = warp_wait(wctx2, o_bar(r - 1), half(r - 1), 410);
                        if (!ok) break;
                        ptx::tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            ptx::tmem_ld_32x16_wait(o_tm + c, o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            ptx::tmem_st_32x16(o_tm + c, o);
                        }
                    }
                }
                const float shift = top == -INFINITY ? 0.0f : -top * sl;  // nothing but infinities so far: no probability yet
                const ptx::f2 base = ptx::make_f2(shift, shift);
                ptx::f2 sum[2] = {ptx::make_f2(0.0f, 0.0f), ptx::make_f2(0.0f, 0.0f)};
                uint32_t pk[32];
                if (one <= 0) {  // no row of the warp sees these keys
#pragma unroll
                    for (int i = 0; i < 32; ++i) pk[i] = 0;
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const ptx::f2 y = ptx::fma2(ptx::make_f2_bits(s[i >> 4][2 * (i & 15)], s[i >> 4][2 * (i & 15) + 1]), sl2, base);
                        float a, b;
                        ptx::split_f2(y, a, b);
                        a = ptx::ex2_approx(a);
                        b = ptx::ex2_approx(b);
                        sum[i & 1] = ptx::add2(sum[i & 1], ptx::make_f2(a, b));
                        pk[i] = ptx::pack_bf16x2(a, b);
                    }
                }
                ptx::tmem_st_32x32(s_tm, pk);
                ptx::tmem_st_wait();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_bar(r));
                float a, b;
                ptx::split_f2(ptx::add2(sum[0], sum[1]), a, b);
                total += a + b;
            }
            if (ok) ok = warp_wait(wctx2, o_bar(done + n - 1), half(done + n - 1), 420);
            if (!ok) break;
            done += n;
            ptx::tc_fence_after();
            if (SPLIT) {
                sums = true;
                break;
            }
            attn_store_row<D>(o_tm, 1.0f / total, static_cast<__nv_bfloat16 *>(p.out) + (m.start + row) * p.ld_out + m.head * p.D, row < m.len, p.D, wide);
            if (p.lse && row < m.len) p.lse[static_cast<long long>(m.head) * p.T + m.start + row] = top * p.scale + logf(total);
            ptx::tc_fence_before();
        }
        ptx::tc_fence_before();
        if (SPLIT) {
            const AttnShare c(p.parts);
            const uint32_t stats = smem + Cfg::OFF_BAR - 1024;  // maximum and sum, in the rows' order
            ptx::cluster_sync();  // all blocks' products are done: their tiles' memory is free
            if (sums) {
                const int row = warp * 32 + lane;
                attn_give_row<D, D>(c, o_tm, smem, row, 0);
                ptx::st_cluster_v2(ptx::mapa(stats + c.slot(c.rank, row) * 8, c.owner(row)), __float_as_uint(top), __float_as_uint(total));
            }
            const bool failed = c.failed(abort_addr);
            ptx::cluster_sync();
            if (shared.block >= 0 && !failed) {
                const int sharers = attn_sharers<LEAST>(p.parts, tiles_of(shared)), row0 = shared.block * 128;
                const int rows = min(128, shared.len - row0), tid = static_cast<int>(threadIdx.x);
                const long long at = shared.start + row0;
                // weights: a part's sums refer to its own maximum. Of a row with nothing but infinities they are 0 / 0, as its result is without parts
                if (tid < c.rows) {
                    const int row = c.rank * c.rows + tid;
                    float2 v[kAttnParts];
                    float all = -INFINITY, sum = 0.0f;
#pragma unroll
                    for (int q = 0; q < kAttnParts; ++q)
                        if (q < sharers) {
                            v[q] = make_float2(ptx::ld_shared_f32(stats + c.slot(q, row) * 8), ptx::ld_shared_f32(stats + c.slot(q, row) * 8 + 4));
                            all = fmaxf(all, v[q].x);
                        }
#pragma unroll
                    for (int q = 0; q < kAttnParts; ++q)
                        if (q < sharers) {
                            const float w = v[q].x == -INFINITY ? 0.0f : ptx::ex2_approx((v[q].x - all) * sl);
                            sum += w * v[q].y;
                            v[q].x = w;
                        }
#pragma unroll
                    for (int q = 0; q < kAttnParts; ++q)
                        if (q < sharers) ptx::st_shared_f32(stats + c.slot(q, row) * 8, v[q].x / sum);
                    if (p.lse && row < rows) p.lse[static_cast<long long>(shared.head) * p.T + at + row] = all * p.scale + logf(sum);
                }
                ptx::named_bar_sync(3, 128);
                attn_join_rows<D, 128>(c, smem, sharers, static_cast<__nv_bfloat16 *>(p.out) + at * p.ld_out + shared.head * p.D, p.ld_out, rows, p.D,
                                       [&](int q, int row) { return ptx::ld_shared_f32(stats + c.slot(q, row) * 8); });
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
}

}  // namespace nb
