// Attention forward: one block per 256 rows of a sequence and head.
//
// Two tiles of 128 queries share the keys and values that stream through shared memory. A thread of a warpgroup owns a row of its
// tile: scores come from tensor memory, the running maximum and sum stay in registers, probabilities go back to tensor
// memory as bf16 (over the scores) and are the A operand of the product with V. While one warpgroup works on its scores,
// the tensor core works for the other.
//
// The output accumulator in tensor memory is rescaled only when a row's maximum has grown by more than 2^8 since the last
// rescaling: until then probabilities up to 2^8 are summed against the old maximum, which changes no bit of their relative precision.
// Probabilities are rounded to bf16 for the tensor core (half an ulp, 2^-9 of each); their sum takes them unrounded.
#pragma once
#include "attention_sm100.cuh"

namespace nb {

template <int D_>
struct AttnFwdCfg {
    static constexpr int D = D_;
    static constexpr uint32_t TILE = 128 * D_ * 2;
    static constexpr int STAGES = D_ == 64 ? 8 : 4;  // keys and values in turn
    static constexpr uint32_t OFF_Q = 0;
    static constexpr uint32_t OFF_KV = 2 * TILE;
    static constexpr uint32_t OFF_BAR = OFF_KV + STAGES * TILE;
    static constexpr uint32_t SMEM = OFF_BAR + 256;
    static_assert(SMEM <= 232448, "shared memory");
};

template <int D>
__global__ void __launch_bounds__(kAttnThreads, 1)
attn_forward_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                    const AttnParams p)
{
    using Cfg = AttnFwdCfg<D>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t smem = ptx::smem_u32(smem_raw);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = static_cast<int>(threadIdx.x & 31);
    const bool smem_ok = (smem & 1023u) == 0;
    if (!smem_ok && threadIdx.x == 0 && atomicCAS(p.status, 0, kStatusBadSmem) == 0) p.status[2] = static_cast<int>(blockIdx.x);

    const uint32_t bar0 = smem + Cfg::OFF_BAR;
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (Cfg::STAGES + s); };
    auto named = [&](int i) { return bar0 + 8u * (2 * Cfg::STAGES + i); };
    auto q_bar = [&](int t) { return named(t); };
    auto s_bar = [&](int t) { return named(2 + t); };  // scores are there (and the product before them is done)
    auto p_bar = [&](int t) { return named(4 + t); };  // probabilities are there
    auto o_bar = [&](int t) { return named(6 + t); };  // the output is complete
    const uint32_t part_bar = named(8);                // values of a sequence's last tile have landed
    const uint32_t tmem_slot = bar0 + 232, abort_addr = bar0 + 236, span_addr = bar0 + 240;
    static_assert(8 * (2 * Cfg::STAGES + 9) <= 232, "barriers");

    if (warp == 8) {
        if (lane < Cfg::STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        }
        if (lane < 9) ptx::mbar_init(named(lane), lane == 4 || lane == 5 ? 4 : 1);
        if (lane == 31) ptx::st_shared_u32_volatile(abort_addr, 0);
        ptx::fence_barrier_init();
        if (lane == 30) {
            ptx::prefetch_tmap(&tmQ);
            ptx::prefetch_tmap(&tmK);
            ptx::prefetch_tmap(&tmV);
        }
        __syncwarp();
    }
    if (warp == 9) {
        ptx::tmem_alloc<1>(tmem_slot, 512);
        ptx::tmem_relinquish<1>();
    }
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int head = static_cast<int>(blockIdx.x) % p.heads;
    if (warp == 0) {
        const AttnSpan s = attn_span(p, static_cast<int>(blockIdx.x) / p.heads, 256, true);
        if (lane == 0) {
            ptx::st_shared_u32(span_addr, static_cast<uint32_t>(s.start));
            ptx::st_shared_u32(span_addr + 4, static_cast<uint32_t>(s.len));
            ptx::st_shared_u32(span_addr + 8, static_cast<uint32_t>(s.block));
        }
    }
    if (warp == 11 && blockIdx.x == 0 && p.cu) attn_report_bounds(p.cu, p.n, p.T, p.status);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ptx::ld_shared_u32_volatile(tmem_slot);
    const int start = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr)), len = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr + 4)),
              block = static_cast<int>(ptx::ld_shared_u32_volatile(span_addr + 8));
    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    // The waits for a whole round of work have twice the limit, so that the wait closest to the cause of a stall is reported.
    const WaitCtx wctx2{abort_addr, p.status, 2 * p.timeout_ns};

    const int q0 = block * 256;
    const int kv_tiles = (len + 127) / 128;
    auto tiles_of = [&](int t) {  // tiles of keys that queries' tile t sees
        const int row = q0 + t * 128;
        return row >= len ? 0 : p.causal ? min(kv_tiles, row / 128 + 1) : kv_tiles;
    };
    const int n0 = tiles_of(0), n1 = tiles_of(1), nkv = max(n0, n1);

    if (!smem_ok || block < 0) {
        // nothing to do
    } else if (warp >= 8) {
        ptx::setmaxnreg_dec<64>();
        if (warp == 8) {
            // ------------------------------------------------------------ loads
            const int kv_head = head / p.group;
            if (ptx::elect_one()) {
                ptx::mbar_expect_tx(q_bar(0), Cfg::TILE);
                attn_load<D>(smem + Cfg::OFF_Q, &tmQ, q_bar(0), head, start + q0);
                if (n1 > 0) {
                    ptx::mbar_expect_tx(q_bar(1), Cfg::TILE);
                    attn_load<D>(smem + Cfg::OFF_Q + Cfg::TILE, &tmQ, q_bar(1), head, start + q0 + 128);
                }
            }
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0;
            for (int i = 0; i < 2 * nkv && ok; ++i) {
                const int j = i >> 1;
                ok = warp_wait(wctx2, empty_bar(stage), phase ^ 1u, 100 + stage);
                if (!ok) break;
                const uint32_t dst = smem + Cfg::OFF_KV + stage * Cfg::TILE;
                const int valid = len - j * 128, up = (valid + 15) & ~15;
                const bool part = (i & 1) && valid < 128 && valid < up;
                if (ptx::elect_one()) {
                    const uint32_t bar = part ? part_bar : full_bar(stage);
                    ptx::mbar_expect_tx(bar, Cfg::TILE + p.withhold);
                    attn_load<D>(dst, (i & 1) ? &tmV : &tmK, bar, kv_head, start + j * 128);
                }
                __syncwarp();
                if (part) {
                    ok = warp_wait(wctx, part_bar, 0, 150);
                    if (!ok) break;
                    attn_zero_rows<D>(dst, valid, up);
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(full_bar(stage));
                }
                if (++stage == Cfg::STAGES) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        } else if (warp == 9) {
            // ------------------------------------------------------------ products
            const uint32_t idesc_s = make_idesc(128, 128, false, false);
            const int nd = (p.D + 15) & ~15, dsteps = nd / 16;
            const uint32_t idesc_o = make_idesc(128, nd, false, true);
            const uint32_t q_s[2] = {smem + Cfg::OFF_Q, smem + Cfg::OFF_Q + Cfg::TILE};
            if (ptx::elect_one()) {
                int stage = 0;
                uint32_t phase = 0;
                auto next = [&] {
                    if (++stage == Cfg::STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                };
                auto tile = [&](int s) { return smem + Cfg::OFF_KV + s * Cfg::TILE; };
                const int nt[2] = {n0, n1};
                bool ok = wait_barrier(wctx, full_bar(0), 0, 300);
                for (int t = 0; t < 2 && ok; ++t) {
                    if (nt[t] == 0) continue;
                    ok = wait_barrier(wctx, q_bar(t), 0, 330 + t);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    attn_mma_kk(tmem + t * 128, q_s[t], tile(0), idesc_s, dsteps);
                    ptx::umma_commit<1>(s_bar(t));
                }
                if (ok) ptx::umma_commit<1>(empty_bar(0));
                next();
                for (int j = 0; j < nkv && ok; ++j) {
                    const int vs = stage;
                    ok = wait_barrier(wctx, full_bar(vs), phase, 300 + vs);
                    if (!ok) break;
                    next();
                    const int ks = stage;
                    const uint32_t kphase = phase;
                    if (j + 1 < nkv) next();
                    const int steps = (min(128, len - j * 128) + 15) / 16;
                    for (int t = 0; t < 2 && ok; ++t) {
                        if (j >= nt[t]) continue;
                        ok = wait_barrier(wctx2, p_bar(t), static_cast<uint32_t>(j) & 1u, 350 + t);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        attn_mma_tn(tmem + 256 + t * D, tmem + t * 128, tile(vs), idesc_o, steps, j > 0);
                        if (j + 1 < nt[t]) {
                            ok = wait_barrier(wctx, full_bar(ks), kphase, 300 + ks);
                            if (!ok) break;
                            ptx::tc_fence_after();
                            attn_mma_kk(tmem + t * 128, q_s[t], tile(ks), idesc_s, dsteps);
                            ptx::umma_commit<1>(s_bar(t));
                        } else {
                            ptx::umma_commit<1>(o_bar(t));
                        }
                    }
                    if (!ok) break;
                    ptx::umma_commit<1>(empty_bar(vs));
                    if (j + 1 < nkv) ptx::umma_commit<1>(empty_bar(ks));
                }
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------ scores: a row per thread
        ptx::setmaxnreg_inc<216>();
        const int t = warp >> 2, nt = t == 0 ? n0 : n1;
        const int row = q0 + t * 128 + (warp & 3) * 32 + lane;  // of the sequence
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_tm = tmem + lanes + t * 128, o_tm = tmem + lanes + 256 + t * D;
        const float sl = p.scale * kLog2e;
        const ptx::f2 sl2 = ptx::make_f2(sl, sl);
        float top = 0.0f, total = 0.0f;  // the maximum that the sums refer to (of unscaled scores), the sum
        bool ok = true;
        for (int j = 0; j < nt; ++j) {
            ok = warp_wait(wctx2, s_bar(t), static_cast<uint32_t>(j) & 1u, 400 + t);
            if (!ok) break;
            ptx::tc_fence_after();
            uint32_t s[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) ptx::tmem_ld_32x32_issue(s_tm + c * 32, s[c]);
            ptx::tmem_ld_wait_32(s[0]);
            ptx::reg_fence_32(s[1]);
            ptx::reg_fence_32(s[2]);
            ptx::reg_fence_32(s[3]);
            int limit = len - j * 128;  // columns below it are seen
            if (p.causal) limit = min(limit, row + 1 - j * 128);
            if (__any_sync(0xffffffffu, limit < 128)) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c * 32 + i >= limit) s[c][i] = 0xff800000u;
            }
            float m[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                m[c] = __uint_as_float(s[c][0]);
#pragma unroll
                for (int i = 1; i < 32; ++i) m[c] = fmaxf(m[c], __uint_as_float(s[c][i]));
            }
            const float now = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
            if (j == 0) {
                top = now;
            } else if (__any_sync(0xffffffffu, (now - top) * sl > 8.0f)) {
                // only rows that grew that much: a row's bits do not depend on its neighbours
                const bool grown = (now - top) * sl > 8.0f;
                const float f = grown ? ptx::ex2_approx((top - now) * sl) : 1.0f;
                total *= f;
                if (grown) top = now;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    ptx::tmem_ld_32x32_wait(o_tm + c * 32, o);
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                    ptx::tmem_st_32x32(o_tm + c * 32, o);
                }
            }
            const ptx::f2 base = ptx::make_f2(-top * sl, -top * sl);
            ptx::f2 sum[2] = {ptx::make_f2(0.0f, 0.0f), ptx::make_f2(0.0f, 0.0f)};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t pk[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const int c = 2 * h + (i >> 4), e = (2 * i) & 31;
                    const ptx::f2 x = ptx::fma2(ptx::make_f2_bits(s[c][e], s[c][e + 1]), sl2, base);
                    float a, b;
                    ptx::split_f2(x, a, b);
                    a = ptx::ex2_approx(a);
                    b = ptx::ex2_approx(b);
                    sum[i & 1] = ptx::add2(sum[i & 1], ptx::make_f2(a, b));
                    pk[i] = ptx::pack_bf16x2(a, b);
                }
                ptx::tmem_st_32x32(s_tm + h * 32, pk);
            }
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(p_bar(t));
            float a, b;
            ptx::split_f2(ptx::add2(sum[0], sum[1]), a, b);
            total += a + b;
        }
        if (ok && nt > 0) ok = warp_wait(wctx2, o_bar(t), 0, 420 + t);
        if (ok && nt > 0) {
            ptx::tc_fence_after();
            // through where this warp's queries were: all products that read them are done
            const int first = row - lane;
            attn_store_rows<D>(o_tm, 1.0f / total, smem + Cfg::OFF_Q + t * Cfg::TILE + (warp & 3) * 32 * D * 2,
                               static_cast<__nv_bfloat16 *>(p.out) + (start + first) * p.ld_out + head * p.D, p.ld_out, len - first, p.D);
            if (p.lse && row < len) p.lse[static_cast<long long>(head) * p.T + start + row] = top * p.scale + logf(total);
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
    if (warp == 9) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc<1>(tmem, 512);
    }
}

}  // namespace nb
