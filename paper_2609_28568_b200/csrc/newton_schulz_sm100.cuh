// Products of the Newton-Schulz iteration for a batch of matrices of one shape, on tcgen05:
//
//   S = X X^T (or X^T X for tall X)    P = a I + b S + c S S    X <- P X (or X P)
//
// with m = min(R, C): S and P are symmetric [m, m], so only the tiles on and below the diagonal are computed and each is stored twice, as it is and
// transposed. a X is inside P X: the update is a plain product.
//
// Operands are fp16, accumulators fp32. X, S and P hold values of the order of one and below, and what the iteration amplifies is the
// rounding of its operands: fp16's eleven bits leave the update 1.1e-3 off (2-norm, gradients with a spectrum as of training), bf16's eight
// leave it 9e-3 off, at the same speed. Its narrow range is met by powers of two: X is stored times 2^12, S and P times 2^10.
//
// The kernel is a persistent one in the manner of gemm_kernel: warp 0 loads tiles by TMA, warp 1 issues the MMAs into one of two accumulators,
// warps 2..9 run the epilogue of the tile before. Every operand comes as boxes of 64 x 64 elements of one matrix of the batch (3-D
// maps: what lies outside the matrix reads as zero and is not written), K-major or MN-major by which of the matrix's axes is summed.
#pragma once
#include <cuda_fp16.h>

#include "gemm_sm100.cuh"
#include "muon.cuh"

namespace nb {

enum NsEpi : int {
    kNsGram = 0,  // D = alpha acc, symmetric
    kNsPoly = 1,  // D = alpha acc + beta aux + diag I, symmetric; aux is the operand itself
    kNsStep = 2,  // D = alpha acc
    kNsLast = 3   // out (bf16, the caller's) = alpha acc
};
constexpr float kNsScaleX = 4096.0f, kNsScaleS = 1024.0f;

struct NsParams {
    int M, N;              // of D, per matrix
    int tiles_m, tiles_n;
    int tiles;             // per matrix: all, or those on and below the diagonal
    int units;             // tiles of the batch
    int kblocks;
    float alpha, beta, diag;
    const __half *aux;     // kNsPoly: S, [n, M, M]
    int *status;
    unsigned long long timeout_ns;
    void *out[kMuonBatch];  // kNsLast
};

template <int CG_, int BLOCK_N_, bool A_MN_, bool B_MN_, int EPI_>
struct NsCfg {
    static constexpr int CG = CG_;
    static constexpr int TILE_M = kBlockM * CG_;
    static constexpr int BLOCK_N = BLOCK_N_;
    static constexpr bool A_MN = A_MN_;
    static constexpr bool B_MN = B_MN_;
    static constexpr int EPI = EPI_;
    static constexpr bool SYM = EPI_ == kNsGram || EPI_ == kNsPoly;
    static constexpr uint32_t A_BYTES = kBlockM * kBlockK * 2;
    static constexpr int B_ROWS = BLOCK_N / CG_;
    static constexpr uint32_t B_BYTES = B_ROWS * kBlockK * 2;
    static constexpr uint32_t BOX_BYTES = 32 * 128;  // 32 rows of 64 elements, or 64 of 32
    static constexpr uint32_t STG_BYTES = kEpiWarps * BOX_BYTES * (SYM ? 2 : 1);
    static constexpr int STAGES = SYM ? 5 : 6;
    static constexpr uint32_t OFF_B = STAGES * A_BYTES;
    static constexpr uint32_t OFF_STG = STAGES * (A_BYTES + B_BYTES);
    static constexpr uint32_t OFF_BAR = OFF_STG + STG_BYTES;
    static constexpr uint32_t SMEM_BYTES = OFF_BAR + 256;
    static constexpr uint32_t TMEM_COLS = 2 * BLOCK_N;
    static constexpr int STEPS = BLOCK_N / 128;  // pieces of 64 columns per epilogue warp
    static_assert(BLOCK_N == 128 || BLOCK_N == 256, "two accumulators, a power of two of TMEM columns");
    static_assert(!SYM || TILE_M == BLOCK_N, "tiles below the diagonal mirror onto tiles above it");
    static_assert(SMEM_BYTES <= 232448, "shared memory budget");
};

// 3-D forms of the tile copies: z is the matrix of the batch.
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *m, uint32_t bar, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap *m, uint32_t bar, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *m, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(m)), "r"(src), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Tile t of a matrix: (row, column) tile. Symmetric results: t runs through the lower triangle row by row.
template <bool SYM>
__device__ __forceinline__ void ns_tile(const NsParams &p, int t, int &m_blk, int &n_blk)
{
    if (SYM) {
        int i = static_cast<int>((sqrtf(8.0f * static_cast<float>(t) + 1.0f) - 1.0f) * 0.5f);
        while ((i + 1) * (i + 2) / 2 <= t) ++i;  // the root is off by at most one
        while (i * (i + 1) / 2 > t) --i;
        m_blk = i;
        n_blk = t - i * (i + 1) / 2;
    } else {
        n_blk = t / p.tiles_m;
        m_blk = t - n_blk * p.tiles_m;
    }
}

template <class Cfg>
__global__ void __launch_bounds__(kNumThreads, 1)
newton_schulz_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                     const __grid_constant__ CUtensorMap tmD, const __grid_constant__ CUtensorMap tmT,
                     const __grid_constant__ NsParams p)
{
    constexpr int BLOCK_N = Cfg::BLOCK_N;
    constexpr int STAGES = Cfg::STAGES;
    constexpr int EPI = Cfg::EPI;
    constexpr int CG = Cfg::CG;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t smem = ptx::smem_u32(smem_raw);
    const int warp = static_cast<int>(threadIdx.x >> 5);
    const int lane = static_cast<int>(threadIdx.x & 31);
    const uint32_t rank = (CG == 2) ? (blockIdx.x & 1u) : 0u;
    const int first_unit = static_cast<int>(blockIdx.x) / CG;
    const int unit_stride = static_cast<int>(gridDim.x) / CG;

    const bool smem_ok = (smem & 1023u) == 0;
    if (!smem_ok && threadIdx.x == 0 && atomicCAS(p.status, 0, kStatusBadSmem) == 0)
        p.status[2] = static_cast<int>(blockIdx.x);

    const uint32_t bar0 = smem + Cfg::OFF_BAR;
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
    auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + b); };
    auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * STAGES + 2 + b); };
    const uint32_t tmem_slot = bar0 + 240;
    const uint32_t abort_addr = bar0 + 244;
    const uint32_t epi_abort_addr = bar0 + 248;
    static_assert(8 * (2 * STAGES + 4) <= 240, "barrier region");

    if (warp == 0) {
        if (lane < STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        } else if (lane < STAGES + 2) {
            ptx::mbar_init(tfull_bar(lane - STAGES), 1);
            ptx::mbar_init(tempty_bar(lane - STAGES), kEpiWarps * CG);
        }
        if (lane == 31) {
            ptx::st_shared_u32_volatile(abort_addr, 0);
            ptx::st_shared_u32_volatile(epi_abort_addr, 0);
        }
        ptx::fence_barrier_init();
        if (lane == 30) {
            ptx::prefetch_tmap(&tmA);
            ptx::prefetch_tmap(&tmB);
            if (EPI != kNsLast) ptx::prefetch_tmap(&tmD);
            if (Cfg::SYM) ptx::prefetch_tmap(&tmT);
        }
        __syncwarp();
    }
    if (warp == 1) {
        ptx::tmem_alloc<CG>(tmem_slot, Cfg::TMEM_COLS);
        ptx::tmem_relinquish<CG>();
    }
    ptx::tc_fence_before();
    if (CG == 2) ptx::cluster_sync();
    else __syncthreads();
    ptx::tc_fence_after();
    // what is above touched this CTA's own memory only and may run while the launch before still drains
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const uint32_t tmem_base = ptx::ld_shared_u32_volatile(tmem_slot);
    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    const WaitCtx wctx_epi{abort_addr, p.status, 2 * p.timeout_ns};

    auto load = [&](uint32_t dst, const CUtensorMap *m, uint32_t bar, int x, int y, int z) {
        if (CG == 2) tma_load_3d_pair(dst, m, bar, x, y, z);
        else tma_load_3d(dst, m, bar, x, y, z);
    };

    if (!smem_ok) {
        // fall through to the common exit
    } else if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (every CTA)
        if (ptx::elect_one()) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int u = first_unit; u < p.units && ok; u += unit_stride) {
                const int z = u / p.tiles;
                int m_blk, n_blk;
                ns_tile<Cfg::SYM>(p, u - z * p.tiles, m_blk, n_blk);
                const int m0 = m_blk * Cfg::TILE_M + static_cast<int>(rank) * kBlockM;
                const int n0 = n_blk * BLOCK_N + static_cast<int>(rank) * Cfg::B_ROWS;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    ok = wait_barrier(wctx, empty_bar(stage), phase ^ 1u, 100 + stage);
                    if (!ok) break;
                    const uint32_t fb = (CG == 2) ? ptx::mapa(full_bar(stage), 0) : full_bar(stage);
                    if (rank == 0) ptx::mbar_expect_tx(full_bar(stage), CG * (Cfg::A_BYTES + Cfg::B_BYTES));
                    const uint32_t sa = smem + stage * Cfg::A_BYTES;
                    const uint32_t sb = smem + Cfg::OFF_B + stage * Cfg::B_BYTES;
                    const int k0 = kb * kBlockK;
#pragma unroll
                    for (int j = 0; j < kBlockM / 64; ++j)
                        load(sa + j * 8192u, &tmA, fb, Cfg::A_MN ? m0 + j * 64 : k0, Cfg::A_MN ? k0 : m0 + j * 64, z);
#pragma unroll
                    for (int j = 0; j < Cfg::B_ROWS / 64; ++j)
                        load(sb + j * 8192u, &tmB, fb, Cfg::B_MN ? n0 + j * 64 : k0, Cfg::B_MN ? k0 : n0 + j * 64, z);
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (leader CTA only)
        if (rank == 0 && ptx::elect_one()) {
            // bits 7 and 10 clear: both operands fp16
            constexpr uint32_t idesc = make_idesc(Cfg::TILE_M, BLOCK_N, Cfg::A_MN, Cfg::B_MN) & ~((1u << 7) | (1u << 10));
            int stage = 0;
            uint32_t phase = 0;
            int acc = 0;
            uint32_t acc_phase = 0;
            bool ok = true;
            for (int u = first_unit; u < p.units && ok; u += unit_stride) {
                ok = wait_barrier(wctx, tempty_bar(acc), acc_phase ^ 1u, 200 + acc);
                if (!ok) break;
                ptx::tc_fence_after();
                const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * BLOCK_N);
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    ok = wait_barrier(wctx, full_bar(stage), phase, 300 + stage);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    const uint32_t sa = smem + stage * Cfg::A_BYTES;
                    const uint32_t sb = smem + Cfg::OFF_B + stage * Cfg::B_BYTES;
                    const uint64_t adesc = Cfg::A_MN ? make_smem_desc(sa, 8192, 1024) : make_smem_desc(sa, 16, 1024);
                    const uint64_t bdesc = Cfg::B_MN ? make_smem_desc(sb, 8192, 1024) : make_smem_desc(sb, 16, 1024);
                    constexpr uint32_t a_step = Cfg::A_MN ? (2048u >> 4) : (32u >> 4);
                    constexpr uint32_t b_step = Cfg::B_MN ? (2048u >> 4) : (32u >> 4);
#pragma unroll
                    for (int k = 0; k < kBlockK / kUmmaK; ++k)
                        ptx::umma_bf16<CG>(d_tmem, adesc + static_cast<uint64_t>(k * a_step),
                                           bdesc + static_cast<uint64_t>(k * b_step), idesc, (kb > 0 || k > 0) ? 1u : 0u);
                    ptx::umma_commit<CG>(empty_bar(stage));
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (!ok) break;
                ptx::umma_commit<CG>(tfull_bar(acc));
                if (++acc == 2) {
                    acc = 0;
                    acc_phase ^= 1u;
                }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue (warps 2..9), warp by warp
        // A warp owns 32 rows (its TMEM lane quarter) and half of the tile's columns, 64 columns at a time.
        const int q = warp & 3;
        const int hf = (warp - 2) >> 2;
        const int ew = warp - 2;
        const uint32_t stg = smem + Cfg::OFF_STG + static_cast<uint32_t>(ew) * Cfg::BOX_BYTES * (Cfg::SYM ? 2 : 1);
        const uint32_t stgT = stg + Cfg::BOX_BYTES;
        const uint32_t sw = static_cast<uint32_t>(lane & 7);
        const ptx::f2 al = ptx::make_f2(p.alpha, p.alpha);
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int u = first_unit; u < p.units; u += unit_stride) {
            if (ptx::ld_shared_u32_volatile(epi_abort_addr) != 0) break;
            const int z = u / p.tiles;
            int m_blk, n_blk;
            ns_tile<Cfg::SYM>(p, u - z * p.tiles, m_blk, n_blk);
            const int y0 = m_blk * Cfg::TILE_M + static_cast<int>(rank) * kBlockM + q * 32;  // the warp's first row
            const int x00 = n_blk * BLOCK_N + hf * (BLOCK_N / 2);                            // and first column
            const int row = y0 + lane;
            bool ok = true;
            if (lane == 0) ok = wait_barrier(wctx_epi, tfull_bar(acc), acc_phase, 400 + acc);
            ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
            if (!ok) ptx::st_shared_u32_volatile(epi_abort_addr, 1);
            ptx::tc_fence_after();
            const uint32_t t_acc = tmem_base + (static_cast<uint32_t>(q * 32) << 16) +
                                   static_cast<uint32_t>(acc * BLOCK_N + hf * (BLOCK_N / 2));
#pragma unroll
            for (int step = 0; step < Cfg::STEPS; ++step) {
                const int x0 = x00 + step * 64;
                uint32_t r[2][32];
                ptx::tmem_ld_32x32_issue(t_acc + static_cast<uint32_t>(step * 64), r[0]);
                ptx::tmem_ld_32x32_issue(t_acc + static_cast<uint32_t>(step * 64 + 32), r[1]);
                uint4 aux[EPI == kNsPoly ? 8 : 1];
                if constexpr (EPI == kNsPoly) {
                    const __half *src = p.aux + (static_cast<long long>(z) * p.M + row) * p.N + x0;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        aux[j] = row < p.M && x0 + j * 8 < p.N ? ptx::ld_global_v4(src + j * 8) : make_uint4(0, 0, 0, 0);
                }
                ptx::tmem_ld_wait_32(r[0]);
                ptx::reg_fence_32(r[1]);
                if (step == Cfg::STEPS - 1) {  // the accumulator's last column is in registers
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (CG == 2) ptx::mbar_arrive_cluster(ptx::mapa(tempty_bar(acc), 0));
                        else ptx::mbar_arrive(tempty_bar(acc));
                    }
                    __syncwarp();
                }
                // the staging boxes are free once the copies of the step before have read them
                ptx::bulk_wait_group_read<0>();
                __syncwarp();
                const bool mirror = Cfg::SYM && m_blk != n_blk;
#pragma unroll
                for (int j = 0; j < 8; ++j) {  // eight columns
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int c = j * 8 + 2 * k;
                        ptx::f2 v = ptx::make_f2_bits(r[c >> 5][c & 31], r[c >> 5][(c & 31) + 1]);
                        float lo, hi;
                        if constexpr (EPI == kNsPoly) {
                            const uint32_t a2 = k == 0 ? aux[j].x : k == 1 ? aux[j].y : k == 2 ? aux[j].z : aux[j].w;
                            const float2 s = __half22float2(*reinterpret_cast<const __half2 *>(&a2));
                            v = ptx::fma2(v, al, ptx::make_f2(s.x * p.beta + (row == x0 + c ? p.diag : 0.0f),
                                                              s.y * p.beta + (row == x0 + c + 1 ? p.diag : 0.0f)));
                        } else {
                            v = ptx::mul2(v, al);
                        }
                        ptx::split_f2(v, lo, hi);
                        w[k] = EPI == kNsLast ? ptx::pack_bf16x2(lo, hi) : pack_f16x2(lo, hi);
                    }
                    ptx::st_shared_v4(stg + static_cast<uint32_t>(lane) * 128u + ((static_cast<uint32_t>(j) ^ sw) << 4), w[0], w[1],
                                      w[2], w[3]);
                    if (mirror) {
                        // transposed: 64 rows (the columns) of 32 elements. Neighbouring lanes swap halves, so that each stores
                        // two rows' values of one column as a word: even lanes of column c, odd lanes of column c + 1.
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t other = __shfl_xor_sync(0xffffffffu, w[k], 1);
                            const uint32_t word = (lane & 1) ? __byte_perm(other, w[k], 0x7632) : __byte_perm(w[k], other, 0x5410);
                            const uint32_t col = static_cast<uint32_t>(j * 8 + 2 * k + (lane & 1));
                            ptx::st_shared_u32(stgT + col * 64u + static_cast<uint32_t>(lane & 30) * 2u, word);
                        }
                    }
                }
                if constexpr (EPI == kNsLast) {
                    __syncwarp();
                    // eight lanes to a row: whole 128-byte pieces of the caller's rows
                    uint4 *out = static_cast<uint4 *>(p.out[z]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int rr = i * 4 + (lane >> 3), cc = lane & 7;
                        uint32_t w[4];
                        ptx::ld_shared_v4(stg + static_cast<uint32_t>(rr) * 128u +
                                              ((static_cast<uint32_t>(cc) ^ static_cast<uint32_t>(rr & 7)) << 4),
                                          w[0], w[1], w[2], w[3]);
                        if (ok && y0 + rr < p.M && x0 + cc * 8 < p.N)
                            out[(static_cast<long long>(y0 + rr) * p.N + x0) / 8 + cc] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    __syncwarp();
                } else {
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (ptx::elect_one()) {
                        if (ok && y0 < p.M && x0 < p.N) {
                            tma_store_3d(&tmD, stg, x0, y0, z);
                            if (mirror) tma_store_3d(&tmT, stgT, y0, x0, z);
                        }
                        ptx::bulk_commit_group();
                    }
                    __syncwarp();
                }
            }
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
            }
        }
        ptx::bulk_wait_group<0>();
        __syncwarp();
    }

    // ---------------------------------------------------------------- common exit
    if (ptx::ld_shared_u32_volatile(abort_addr) != 0 || ptx::ld_shared_u32_volatile(epi_abort_addr) != 0) {
        const uint64_t t0 = ptx::globaltimer_ns();  // copies and MMAs in flight land first
        while (ptx::globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    __syncwarp();
    ptx::tc_fence_before();
    if (CG == 2) ptx::cluster_sync();
    else __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc<CG>(tmem_base, Cfg::TMEM_COLS);
    }
}

}  // namespace nb
