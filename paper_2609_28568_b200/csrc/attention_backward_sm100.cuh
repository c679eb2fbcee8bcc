// Attention backward, in two passes without atomics (results do not depend on the order in which blocks run):
//
//   P = exp(scale Q K^T - lse)    delta = sum over a row of dout out    dS = P (dO V^T - delta)
//   dQ = scale dS K               (a block per 128 queries of a head, over the keys that they see)
//   dV = P^T dO   dK = scale dS^T Q   (a block per 128 keys of a head, over the queries that see them and all heads that share the keys)
//
// Both form P and dS themselves: seven products of tiles in place of five, for which no gradient crosses memory in fp32 and
// none is added up by atomics. The second pass works on transposed tiles (S^T = K Q^T, dP^T = V dO^T), so that P^T and dS^T stand in tensor
// memory as the A operands of its sums. P and dS are rounded to bf16 for them (half an ulp, 2^-9 of each); all sums are fp32.
//
// A thread has 64 values of a row of a tile: heads of up to 64 columns take tiles of 64 columns with one warpgroup, two blocks to an SM, which fill
// each other's gaps; wider heads have no tensor memory for that and take tiles of 128 with two warpgroups. While these turn dP into dS, the
// tensor core works on what P was ready for, and the other way round.
#pragma once
#include "attention_sm100.cuh"

namespace nb {

template <int D_, int WGS_>
struct AttnBwdCfg {
    static constexpr int D = D_, WGS = WGS_, ROWS = 64 * WGS_;  // warpgroups on scores, rows of the streamed tiles
    static constexpr int THREADS = 128 * WGS_ + 128, BLOCKS = 3 - WGS_;
    static constexpr uint32_t TMEM = 512 / BLOCKS;
    static constexpr uint32_t OWN = 128 * D_ * 2, TILE = ROWS * D_ * 2;
    static constexpr int STAGES = D_ == 64 ? 8 : 4;
    static constexpr uint32_t OFF_OWN = 0;          // the block's own tiles: Q, dO or K, V
    static constexpr uint32_t OFF_RING = 2 * OWN;   // the others, in turn
    static constexpr uint32_t OFF_BAR = OFF_RING + STAGES * TILE;
    static constexpr uint32_t OFF_ROWS = OFF_BAR + 256;  // dQ: halves of delta; dK, dV: lse and delta of two tiles of queries
    static constexpr uint32_t SMEM_Q = OFF_ROWS + 1024;
    static constexpr uint32_t SMEM_KV = OFF_ROWS + 2048;
    static constexpr int REGS_ROWS = WGS_ == 1 ? 192 : 208, REGS_OTHER = WGS_ == 1 ? 64 : 88;
    static_assert(WGS_ * REGS_ROWS + REGS_OTHER <= (WGS_ + 1) * (WGS_ == 1 ? 128 : 168), "registers");
    static_assert(SMEM_KV <= (BLOCKS == 2 ? 113 * 1024 : 232448), "shared memory");
    static_assert(2 * ROWS + 2 * D_ <= TMEM && 3 * ROWS + D_ <= TMEM, "tensor memory");
};

// ------------------------------------------------------------------------------------------------ dQ
template <class Cfg>
__global__ void __launch_bounds__(Cfg::THREADS, Cfg::BLOCKS)
attn_backward_q_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmDO, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const AttnBackward b)
{
    constexpr int D = Cfg::D, WGS = Cfg::WGS, ROWS = Cfg::ROWS, STAGES = Cfg::STAGES, LOAD = 4 * WGS, MMA = LOAD + 1;
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
    const uint32_t q_bar = named(0), do_bar = named(1), dp_bar = named(4), ds_bar = named(5), done_bar = named(6), part_bar = named(7);
    auto s_bar = [&](int i) { return named(2 + i); };
    const uint32_t tmem_slot = bar0 + 232, abort_addr = bar0 + 236, span_addr = bar0 + 240;
    static_assert(8 * (2 * STAGES + 8) <= 232, "barriers");

    if (warp == LOAD) {
        if (lane < STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        }
        if (lane < 8) ptx::mbar_init(named(lane), lane == 5 ? 4 * WGS : 1);
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
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int head = static_cast<int>(blockIdx.x) % p.heads;
    if (warp == 0) {
        const AttnSpan s = attn_span(p, static_cast<int>(blockIdx.x) / p.heads, 128, true);
        if (lane == 0) {
            ptx::st_shared_u32(span_addr, static_cast<uint32_t>(s.start));
            ptx::st_shared_u32(span_addr + 4, static_cast<uint32_t>(s.len));
            ptx::st_shared_u32(span_addr + 8, static_cast<uint32_t>(s.block));
        }
    }
    if (warp == MMA + 2 && blockIdx.x == 0 && p.cu) attn_report_bounds(p.cu, p.n, p.T, p.status);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ptx::ld_shared_u32_volatile(tmem_slot);
    const int start = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr)), len = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr + 4)),
              block = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr + 8));
    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    const WaitCtx wctx2{abort_addr, p.status, 2 * p.timeout_ns};  // a round of work: the wait closest to a stall's cause is reported
    const int tiles = (len + ROWS - 1) / ROWS, n = p.causal ? min(tiles, (block + 1) * (128 / ROWS)) : tiles;
    const uint32_t dp_tm = tmem + 2 * ROWS, dq_tm = tmem + 3 * ROWS;  // scores: two tiles from 0 on

    if (!smem_ok || block < 0) {
        // nothing to do
    } else if (warp >= LOAD) {
        ptx::setmaxnreg_dec<Cfg::REGS_OTHER>();
        if (warp == LOAD) {
            // ------------------------------------------------------------ loads
            const int kv_head = head / p.group;
            if (ptx::elect_one()) {
                ptx::mbar_expect_tx(q_bar, Cfg::OWN);
                attn_load<D>(smem + Cfg::OFF_OWN, &tmQ, q_bar, head, start + block * 128);
                ptx::mbar_expect_tx(do_bar, Cfg::OWN);
                attn_load<D>(smem + Cfg::OFF_OWN + Cfg::OWN, &tmDO, do_bar, head, start + block * 128);
            }
            __syncwarp();
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0;
            for (int i = 0; i < 2 * n && ok; ++i) {
                const int j = i >> 1;
                ok = warp_wait(wctx2, empty_bar(stage), phase ^ 1u, 100 + stage);
                if (!ok) break;
                const uint32_t dst = smem + Cfg::OFF_RING + stage * Cfg::TILE;
                const int valid = len - j * ROWS, up = (valid + 15) & ~15;
                const bool part = valid < ROWS && valid < up;
                if (ptx::elect_one()) {
                    const uint32_t bar = part ? part_bar : full_bar(stage);
                    ptx::mbar_expect_tx(bar, Cfg::TILE + p.withhold);
                    attn_load<D, ROWS>(dst, (i & 1) ? &tmV : &tmK, bar, kv_head, start + j * ROWS);
                }
                __syncwarp();
                if (part) {  // the last tile's keys, then its values
                    ok = warp_wait(wctx, part_bar, static_cast<uint32_t>(i) & 1u, 150);
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
        } else if (warp == MMA) {
            // ------------------------------------------------------------ products
            const uint32_t idesc_s = make_idesc(128, ROWS, false, false);
            const int nd = (p.D + 15) & ~15, dsteps = nd / 16;
            const uint32_t idesc_q = make_idesc(128, nd, false, true);
            const uint32_t q_s = smem + Cfg::OFF_OWN, do_s = q_s + Cfg::OWN;
            if (ptx::elect_one()) {
                auto tile = [&](int i) { return smem + Cfg::OFF_RING + (i % STAGES) * Cfg::TILE; };
                auto ready = [&](int i) { return wait_barrier(wctx, full_bar(i % STAGES), static_cast<uint32_t>(i / STAGES) & 1u, 300 + i % STAGES); };
                auto scores = [&](int j) {
                    if (!ready(2 * j)) return false;
                    ptx::tc_fence_after();
                    attn_mma_kk<ROWS>(tmem + (j & 1) * ROWS, q_s, tile(2 * j), idesc_s, dsteps);
                    ptx::umma_commit<1>(s_bar(j & 1));
                    return true;
                };
                auto grads = [&](int j) {
                    if (!ready(2 * j + 1)) return false;
                    ptx::tc_fence_after();
                    attn_mma_kk<ROWS>(dp_tm, do_s, tile(2 * j + 1), idesc_s, dsteps);
                    ptx::umma_commit<1>(dp_bar);
                    ptx::umma_commit<1>(empty_bar((2 * j + 1) % STAGES));
                    return true;
                };
                bool ok = wait_barrier(wctx, q_bar, 0, 330) && scores(0) && wait_barrier(wctx, do_bar, 0, 331) && grads(0);
                for (int j = 0; j < n && ok; ++j) {
                    if (j + 1 < n) ok = scores(j + 1);
                    ok = ok && wait_barrier(wctx2, ds_bar, static_cast<uint32_t>(j) & 1u, 350);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    if (j + 1 < n) ok = grads(j + 1);
                    if (!ok) break;
                    attn_mma_tn<WGS == 2, ROWS>(dq_tm, tmem + (j & 1) * ROWS, tile(2 * j), idesc_q, (min(ROWS, len - j * ROWS) + 15) / 16, j > 0);
                    ptx::umma_commit<1>(empty_bar((2 * j) % STAGES));
                }
                if (ok) ptx::umma_commit<1>(done_bar);
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------ scores: half a row per thread
        ptx::setmaxnreg_inc<Cfg::REGS_ROWS>();
        const int half = warp >> 2, q = warp & 3;
        const int row = block * 128 + q * 32 + lane;  // of the sequence
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const float sl = p.scale * kLog2e;
        const ptx::f2 sl2 = ptx::make_f2(sl, sl);
        float delta = 0.0f, nl = 0.0f;
        {   // delta: a half of the row each where two threads have one
            const int cols = p.D / 8, mid = WGS == 2 ? (cols + 1) / 2 : cols, c0 = half ? mid : 0, c1 = half ? cols : mid;
            if (row < len) {
                const long long at = start + row;
                const __nv_bfloat16 *g = static_cast<const __nv_bfloat16 *>(b.dout) + at * b.ld_dout + head * p.D,
                                    *o = static_cast<const __nv_bfloat16 *>(p.out) + at * p.ld_out + head * p.D;
                for (int c = c0; c < c1; ++c) {
                    const uint4 x = ptx::ld_global_v4(g + c * 8), y = ptx::ld_global_v4(o + c * 8);
                    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        delta = fmaf(ptx::bf16_lo(xs[k]), ptx::bf16_lo(ys[k]), delta);
                        delta = fmaf(ptx::bf16_hi(xs[k]), ptx::bf16_hi(ys[k]), delta);
                    }
                }
                nl = -kLog2e * p.lse[static_cast<long long>(head) * p.T + at];
            }
            if (WGS == 2) {
                const uint32_t mine = smem + Cfg::OFF_ROWS + (q * 32 + lane) * 4;
                ptx::st_shared_f32(mine + half * 512, delta);
                ptx::named_bar_sync(1, 256);
                delta += ptx::ld_shared_f32(mine + (half ^ 1) * 512);
            }
            if (half == 0 && row < len) b.delta[static_cast<long long>(head) * p.T + start + row] = delta;
        }
        const ptx::f2 base = ptx::make_f2(nl, nl), nd2 = ptx::make_f2(-delta, -delta);
        // keys that all rows of the warp see, that this one sees
        const int seen_by_all = min(len, p.causal ? row - lane + 1 : len), seen = min(len, p.causal ? row + 1 : len);
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const uint32_t s_tm = tmem + lanes + (j & 1) * ROWS + half * 64;
            ok = warp_wait(wctx2, s_bar(j & 1), static_cast<uint32_t>(j >> 1) & 1u, 400);
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
            ok = warp_wait(wctx2, dp_bar, static_cast<uint32_t>(j) & 1u, 410);
            if (!ok) break;
            ptx::tc_fence_after();
            uint32_t g[2][32], pk[32];
            ptx::tmem_ld_32x32_x2_wait(dp_tm + lanes + half * 64, dp_tm + lanes + half * 64 + 32, g[0], g[1]);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    const ptx::f2 ds = ptx::mul2(ptx::add2(ptx::make_f2_bits(g[c][i], g[c][i + 1]), nd2), ptx::make_f2_bits(s[c][i], s[c][i + 1]));
                    float x, y;
                    ptx::split_f2(ds, x, y);
                    pk[c * 16 + (i >> 1)] = ptx::pack_bf16x2(x, y);
                }
            if (seen_by_all - j * ROWS - half * 64 < 64) {  // columns that are not seen may hold anything
                const int limit = seen - j * ROWS - half * 64;
#pragma unroll
                for (int i = 0; i < 32; ++i) pk[i] = 2 * i + 1 < limit ? pk[i] : 2 * i < limit ? pk[i] & 0xffffu : 0u;
            }
            ptx::tmem_st_32x32(s_tm, pk);
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ds_bar);
        }
        if (ok) ok = warp_wait(wctx2, done_bar, 0, 420);
        if (ok) {
            ptx::tc_fence_after();
            constexpr int W = D / WGS;  // columns of a thread
            attn_store_row<W>(dq_tm + lanes + half * W, p.scale, static_cast<__nv_bfloat16 *>(b.dq) + (start + row) * b.ld_dq + head * p.D + half * W, row < len,
                              p.D - half * W, attn_wide(b.dq, b.ld_dq, p.D));
        }
        ptx::tc_fence_before();
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

// ------------------------------------------------------------------------------------------------ dK, dV
template <class Cfg>
__global__ void __launch_bounds__(Cfg::THREADS, Cfg::BLOCKS)
attn_backward_kv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmDO, const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CUtensorMap tmV, const AttnBackward b)
{
    constexpr int D = Cfg::D, WGS = Cfg::WGS, ROWS = Cfg::ROWS, STAGES = Cfg::STAGES, LOAD = 4 * WGS, MMA = LOAD + 1;
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
    const uint32_t k_bar = named(0), v_bar = named(1), s_bar = named(2), p_bar = named(3), dp_bar = named(4), ds_bar = named(5), done_bar = named(6),
                   part_bar = named(7);
    auto rows_bar = [&](int i) { return named(8 + i); };   // lse and delta of a tile of queries are there
    auto rfree_bar = [&](int i) { return named(10 + i); };  // and have been read
    const uint32_t tmem_slot = bar0 + 232, abort_addr = bar0 + 236, span_addr = bar0 + 240;
    static_assert(8 * (2 * STAGES + 12) <= 232, "barriers");

    if (warp == LOAD) {
        if (lane < STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        }
        if (lane < 12) ptx::mbar_init(named(lane), lane == 3 || lane == 5 || lane >= 10 ? 4 * WGS : 1);
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
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int kv_heads = p.heads / p.group, kv_head = static_cast<int>(blockIdx.x) % kv_heads;
    if (warp == 0) {
        const AttnSpan s = attn_span(p, static_cast<int>(blockIdx.x) / kv_heads, 128, false);
        if (lane == 0) {
            ptx::st_shared_u32(span_addr, static_cast<uint32_t>(s.start));
            ptx::st_shared_u32(span_addr + 4, static_cast<uint32_t>(s.len));
            ptx::st_shared_u32(span_addr + 8, static_cast<uint32_t>(s.block));
        }
    }
    if (warp == MMA + 2 && blockIdx.x == 0 && p.cu) attn_report_bounds(p.cu, p.n, p.T, p.status);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ptx::ld_shared_u32_volatile(tmem_slot);
    const int start = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr)), len = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr + 4)),
              block = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr + 8));
    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    const WaitCtx wctx2{abort_addr, p.status, 2 * p.timeout_ns};
    const int tiles = (len + ROWS - 1) / ROWS, first_tile = p.causal ? block * (128 / ROWS) : 0;  // tiles of queries that see these keys: from first_tile on
    const int per_head = tiles - first_tile, n = per_head * p.group;
    const uint32_t s_tm = tmem, dp_tm = tmem + ROWS, dv_tm = tmem + 2 * ROWS, dk_tm = dv_tm + D;

    if (!smem_ok || block < 0) {
        // nothing to do
    } else if (warp >= LOAD) {
        ptx::setmaxnreg_dec<Cfg::REGS_OTHER>();
        if (warp == LOAD) {
            // ------------------------------------------------------------ loads
            if (ptx::elect_one()) {
                ptx::mbar_expect_tx(k_bar, Cfg::OWN);
                attn_load<D>(smem + Cfg::OFF_OWN, &tmK, k_bar, kv_head, start + block * 128);
                ptx::mbar_expect_tx(v_bar, Cfg::OWN);
                attn_load<D>(smem + Cfg::OFF_OWN + Cfg::OWN, &tmV, v_bar, kv_head, start + block * 128);
            }
            __syncwarp();
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0, parts = 0;
            for (int i = 0; i < 2 * n && ok; ++i) {
                const int g = (i >> 1) / per_head, t = first_tile + (i >> 1) - g * per_head;
                ok = warp_wait(wctx2, empty_bar(stage), phase ^ 1u, 100 + stage);
                if (!ok) break;
                const uint32_t dst = smem + Cfg::OFF_RING + stage * Cfg::TILE;
                const int valid = len - t * ROWS, up = (valid + 15) & ~15;
                const bool part = valid < ROWS && valid < up;
                if (ptx::elect_one()) {
                    const uint32_t bar = part ? part_bar : full_bar(stage);
                    ptx::mbar_expect_tx(bar, Cfg::TILE + p.withhold);
                    attn_load<D, ROWS>(dst, (i & 1) ? &tmDO : &tmQ, bar, kv_head * p.group + g, start + t * ROWS);
                }
                __syncwarp();
                if (part) {  // the last tile of each head's queries, then of their gradients
                    ok = warp_wait(wctx, part_bar, parts & 1u, 150);
                    if (!ok) break;
                    ++parts;
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
        } else if (warp == MMA) {
            // ------------------------------------------------------------ products
            const uint32_t idesc_s = make_idesc(128, ROWS, false, false);
            const int nd = (p.D + 15) & ~15, dsteps = nd / 16;
            const uint32_t idesc_d = make_idesc(128, nd, false, true);
            const uint32_t k_s = smem + Cfg::OFF_OWN, v_s = k_s + Cfg::OWN;
            if (ptx::elect_one()) {
                auto tile = [&](int i) { return smem + Cfg::OFF_RING + (i % STAGES) * Cfg::TILE; };
                auto ready = [&](int i) { return wait_barrier(wctx, full_bar(i % STAGES), static_cast<uint32_t>(i / STAGES) & 1u, 300 + i % STAGES); };
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
                    return true;
                };
                bool ok = wait_barrier(wctx, k_bar, 0, 330) && scores(0) && wait_barrier(wctx, v_bar, 0, 331) && grads(0);
                int t = first_tile;
                for (int i = 0; i < n && ok; ++i) {
                    const int steps = (min(ROWS, len - t * ROWS) + 15) / 16;
                    ok = wait_barrier(wctx2, p_bar, static_cast<uint32_t>(i) & 1u, 350);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    attn_mma_tn<WGS == 2, ROWS>(dv_tm, s_tm, tile(2 * i + 1), idesc_d, steps, i > 0);
                    ptx::umma_commit<1>(empty_bar((2 * i + 1) % STAGES));
                    if (i + 1 < n) ok = scores(i + 1);
                    ok = ok && wait_barrier(wctx2, ds_bar, static_cast<uint32_t>(i) & 1u, 360);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    attn_mma_tn<WGS == 2, ROWS>(dk_tm, dp_tm, tile(2 * i), idesc_d, steps, i > 0);
                    ptx::umma_commit<1>(empty_bar((2 * i) % STAGES));
                    if (i + 1 < n) ok = grads(i + 1);
                    if (++t == tiles) t = first_tile;
                }
                if (ok) ptx::umma_commit<1>(done_bar);
            }
            __syncwarp();
        } else if (warp == MMA + 1) {
            // ------------------------------------------------------------ lse and delta of the queries, negated, in units of log 2
            bool ok = true;
            for (int i = 0; i < n && ok; ++i) {
                const int g = i / per_head, t = first_tile + i - g * per_head;
                const long long at = static_cast<long long>(kv_head * p.group + g) * p.T + start + t * ROWS;
                float l[ROWS / 32], d[ROWS / 32];
#pragma unroll
                for (int k = 0; k < ROWS / 32; ++k) {
                    const int r = k * 32 + lane;
                    const bool in = t * ROWS + r < len;  // rows behind the last have no probability
                    l[k] = in ? -kLog2e * __ldcg(p.lse + at + r) : -INFINITY;
                    d[k] = in ? -__ldcg(b.delta + at + r) : 0.0f;
                }
                ok = warp_wait(wctx2, rfree_bar(i & 1), (static_cast<uint32_t>(i >> 1) & 1u) ^ 1u, 500);
                if (!ok) break;
                const uint32_t dst = smem + Cfg::OFF_ROWS + (i & 1) * 1024 + lane * 4;
#pragma unroll
                for (int k = 0; k < ROWS / 32; ++k) {
                    ptx::st_shared_f32(dst + k * 128, l[k]);
                    ptx::st_shared_f32(dst + 512 + k * 128, d[k]);
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(rows_bar(i & 1));
            }
        }
    } else {
        // ------------------------------------------------------------ scores: half a row (of keys) per thread
        ptx::setmaxnreg_inc<Cfg::REGS_ROWS>();
        const int half = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const float sl = p.scale * kLog2e;
        const ptx::f2 sl2 = ptx::make_f2(sl, sl);
        bool ok = true;
        int t = first_tile;
        for (int i = 0; i < n; ++i) {
            const uint32_t par = static_cast<uint32_t>(i) & 1u;
            const uint32_t rows = smem + Cfg::OFF_ROWS + par * 1024 + half * 256;
            ok = warp_wait(wctx2, rows_bar(i & 1), static_cast<uint32_t>(i >> 1) & 1u, 510) && warp_wait(wctx2, s_bar, par, 400);
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
                    for (int k = 0; k < 4; ++k) s[c][e + k] = __float_as_uint(ptx::ex2_approx(x[k]));
                }
            // a key is seen by queries from its own row on: columns below `hidden` are not
            const int hidden = p.causal ? block * 128 + r - t * ROWS - half * 64 : 0;
            const bool cut = p.causal && block * 128 + q * 32 + 31 > t * ROWS + half * 64;
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
            uint32_t g[2][32];
            ptx::tmem_ld_32x32_x2_wait(dp_tm + lanes + half * 64, dp_tm + lanes + half * 64 + 32, g[0], g[1]);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    float4 d;
                    ptx::ld_shared_f32x4(rows + 512 + (c * 32 + e) * 4, d);
                    float x[4];
                    ptx::split_f2(ptx::mul2(ptx::add2(ptx::make_f2_bits(g[c][e], g[c][e + 1]), ptx::make_f2(d.x, d.y)), ptx::make_f2_bits(s[c][e], s[c][e + 1])),
                                  x[0], x[1]);
                    ptx::split_f2(ptx::mul2(ptx::add2(ptx::make_f2_bits(g[c][e + 2], g[c][e + 3]), ptx::make_f2(d.z, d.w)),
                                            ptx::make_f2_bits(s[c][e + 2], s[c][e + 3])),
                                  x[2], x[3]);
                    pk[c * 16 + (e >> 1)] = ptx::pack_bf16x2(x[0], x[1]);
                    pk[c * 16 + (e >> 1) + 1] = ptx::pack_bf16x2(x[2], x[3]);
                }
            if (cut) {  // what is not seen may hold anything
#pragma unroll
                for (int e = 0; e < 32; ++e) pk[e] = 2 * e >= hidden ? pk[e] : 2 * e + 1 >= hidden ? pk[e] & 0xffff0000u : 0u;
            }
            ptx::tmem_st_32x32(dp_tm + lanes + half * 64, pk);
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive(ds_bar);
                ptx::mbar_arrive(rfree_bar(i & 1));
            }
            if (++t == tiles) t = first_tile;
        }
        if (ok) ok = warp_wait(wctx2, done_bar, 0, 420);
        if (ok) {
            ptx::tc_fence_after();
            const int row = block * 128 + r;
            if (WGS == 1 || half == 0)
                attn_store_row<D>(dv_tm + lanes, 1.0f, static_cast<__nv_bfloat16 *>(b.dv) + (start + row) * b.ld_dv + kv_head * p.D, row < len, p.D,
                                  attn_wide(b.dv, b.ld_dv, p.D));
            if (WGS == 1 || half == 1)
                attn_store_row<D>(dk_tm + lanes, p.scale, static_cast<__nv_bfloat16 *>(b.dk) + (start + row) * b.ld_dk + kv_head * p.D, row < len, p.D,
                                  attn_wide(b.dk, b.ld_dk, p.D));
        }
        ptx::tc_fence_before();
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
