// Products of the Newton-Schulz iteration for a batch of matrices of one shape, on tcgen05, in one launch:
//
//   S = X X^T (or X^T X for tall X)    P = a I + b S + c S S    X <- P X (or X P)
//
// with m = min(R, C): S and P are symmetric [m, m], so only their tiles on and below the diagonal are computed and stored. A consumer
// that needs a tile above it reads the mirrored one in the other major order, which the tensor core takes as it takes the first: no transposed
// copy exists. a X is inside P X: the update is a plain product.
//
// Operands are fp16, accumulators fp32. X, S and P hold values of the order of one and below, and what the iteration amplifies is the
// rounding of its operands: fp16's eleven bits leave the update 1.1e-3 off (2-norm, gradients with a spectrum as of training), bf16's eight
// leave it 9e-3 off, at the same speed. Its narrow range is met by powers of two: X is stored times 2^12, S and P times 2^10.
//
// The work of all steps is one list of tiles, phase by phase (S of every matrix, P of every matrix, X of every matrix, ...), which
// the CTAs (or CTA pairs) of a cooperative launch walk with the stride of the grid. A matrix's tiles of one phase wait for its tiles of
// the phase before, counted in global memory; other matrices are not waited for. Inside a CTA it is gemm_kernel's division: warp 0 loads tiles by
// TMA, warp 1 issues the MMAs into one of two accumulators, the others run the epilogue of the tile before. Every operand comes as
// boxes of 64 x 64 elements of one matrix of the batch (3-D maps: what lies outside the matrix reads as zero).
//
// As fifteen launches (three per step) each phase cost 2.5 us more: the drain and the start of a launch.
#pragma once
#include <cuda_fp16.h>

#include "gemm_sm100.cuh"
#include "muon.cuh"

namespace nb {

constexpr float kNsScaleX = 4096.0f, kNsScaleS = 1024.0f;

struct NsParams {
    int R, C, m, n;
    int steps;
    int tiles_r;             // of X, down its rows
    int sym_tiles, x_tiles;  // tiles per matrix of S or P, of X
    int kb_gram, kb_m;     // k-blocks of S = X X^T, and of the other two products
    int units;             // tiles of all steps and matrices
    float gram_alpha, poly_alpha, poly_beta, poly_diag, step_alpha, last_alpha;
    __half *x[2], *s, *p;  // [n, R, ldx], [n, m, lds]
    int ldx, lds;          // of whole 128-byte pieces: rows of 776 as they are straddle the lines that their boxes are read from
    unsigned *done;        // [n], kMuonCountPitch apart: CTAs that have stored their part of a tile, over all phases
    unsigned *failed;      // raised by a block that gives up: what the others wait for will not come
    void *out[kMuonBatch];
    int withhold;          // nb_debug_muon_timeout only: tiles that P's tiles wait for beside those that come; else 0
    int *status;
    unsigned long long timeout_ns;
};

template <int CG_, int EDGE_>
struct NsCfg {
    static constexpr int CG = CG_;
    static constexpr int EDGE = EDGE_;       // tiles are square, so those above the diagonal mirror those below
    static constexpr int ROWS = EDGE / CG_;  // of either operand in one CTA
    static constexpr uint32_t OP_BYTES = ROWS * kBlockK * 2;
    // Epilogue: a warp reads the TMEM lanes of its quarter, which hold a quarter of the CTA's rows (64-row tiles: in the first 16 of 32
    // lanes), and half of the columns, or all of a 64-column tile, in pieces of 64.
    static constexpr int EPI_WARPS = EDGE_ == 64 ? 4 : 8;
    static constexpr int WARP_ROWS = ROWS / 4;
    static constexpr int WARP_COLS = EDGE_ / (EPI_WARPS / 4);
    static constexpr int PIECES = WARP_COLS / 64;
    static constexpr int THREADS = (2 + EPI_WARPS) * 32;
    static constexpr uint32_t BOX_BYTES = WARP_ROWS * 128;  // a piece in staging
    static constexpr uint32_t STG_BYTES = EPI_WARPS * PIECES * BOX_BYTES;
    static constexpr int FIT = static_cast<int>((232448 - 512 - STG_BYTES) / (2 * OP_BYTES));
    static constexpr int STAGES = FIT < 12 ? FIT : 12;
    static constexpr uint32_t OFF_B = STAGES * OP_BYTES;
    static constexpr uint32_t OFF_STG = 2 * STAGES * OP_BYTES;
    static constexpr uint32_t OFF_BAR = OFF_STG + STG_BYTES;
    static constexpr uint32_t SMEM_BYTES = OFF_BAR + 512;
    static constexpr uint32_t TMEM_COLS = 2 * EDGE;
    static_assert((CG_ == 2 && EDGE_ == 256) || (CG_ == 1 && (EDGE_ == 128 || EDGE_ == 64)), "tile");
    static_assert(SMEM_BYTES <= 232448, "shared memory budget");
};

// 3-D forms of the tile load: z is the matrix of the batch.
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
// from L2: what another SM wrote during this launch may lie stale in L1
__device__ __forceinline__ uint4 ld_global_cg_v4(const void *p)
{
    uint4 v;
    asm volatile("ld.global.cg.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ unsigned ld_acquire_gpu(const unsigned *p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void red_release_gpu(unsigned *p, unsigned v)
{
    asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t atom_add_acq_rel_shared(uint32_t addr, uint32_t v)
{
    uint32_t old;
    asm volatile("atom.acq_rel.cta.shared::cta.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(addr), "r"(v) : "memory");
    return old;
}
// between plain accesses to global memory and those of the TMA unit, in either direction
__device__ __forceinline__ void fence_proxy_async_global()
{
    asm volatile("fence.proxy.async.global;" ::: "memory");
}

enum NsPhase : int { kNsGram = 0, kNsPoly = 1, kNsStep = 2 };

// What a unit of the list is: a tile of one phase of one matrix in one step.
struct NsUnit {
    int step, phase, z, m_blk, n_blk;
    unsigned need;  // tiles of this matrix that come before
};
__device__ __forceinline__ NsUnit ns_unit(const NsParams &p, int u)
{
    NsUnit t;
    const int sym = p.n * p.sym_tiles, per_step = 2 * sym + p.n * p.x_tiles;
    t.step = u / per_step;
    int r = u - t.step * per_step;
    t.need = static_cast<unsigned>(t.step) * (2 * p.sym_tiles + p.x_tiles);
    if (r < 2 * sym) {
        t.phase = r < sym ? kNsGram : kNsPoly;
        if (t.phase == kNsPoly) {
            r -= sym;
            t.need += p.sym_tiles + p.withhold;
        }
        t.z = r / p.sym_tiles;
        const int k = r - t.z * p.sym_tiles;  // through the lower triangle row by row
        int i = static_cast<int>((sqrtf(8.0f * static_cast<float>(k) + 1.0f) - 1.0f) * 0.5f);
        while ((i + 1) * (i + 2) / 2 <= k) ++i;  // the root is off by at most one
        while (i * (i + 1) / 2 > k) --i;
        t.m_blk = i;
        t.n_blk = k - i * (i + 1) / 2;
    } else {
        t.phase = kNsStep;
        t.need += 2 * p.sym_tiles;
        r -= 2 * sym;
        t.z = r / p.x_tiles;
        const int k = r - t.z * p.x_tiles;
        t.n_blk = k / p.tiles_r;
        t.m_blk = k - t.n_blk * p.tiles_r;
    }
    return t;
}
// Whether an operand's box of k-block kb is read MN-major. X: by the side that is summed. S, P: where the box lies in a block above the
// diagonal and its mirror is read.
template <class Cfg>
__device__ __forceinline__ bool ns_a_mn(const NsParams &p, const NsUnit &t, int kb)
{
    if (t.phase == kNsGram) return p.R > p.C;
    if (t.phase == kNsStep && p.R > p.C) return false;  // X's rows
    return kb * kBlockK / Cfg::EDGE > t.m_blk;
}
template <class Cfg>
__device__ __forceinline__ bool ns_b_mn(const NsParams &p, const NsUnit &t, int kb)
{
    if (t.phase == kNsGram) return p.R > p.C;
    if (t.phase == kNsStep && p.R <= p.C) return true;  // X's columns
    return kb * kBlockK / Cfg::EDGE > t.n_blk;
}

// Whether both operands are the same rows of the same matrix, as on the diagonal of S and P: they are then fetched once.
__device__ __forceinline__ bool ns_same_operand(const NsUnit &t)
{
    return t.phase != kNsStep && t.m_blk == t.n_blk;
}

// Waits, for a limited time, until `need` tile parts of a matrix are stored. Another block's failure ends this one too. It is told by a
// word of this launch: the device's status word is written by other launches, and cleared by the host, while this one runs.
__device__ __forceinline__ bool ns_wait_done(const WaitCtx &w, const unsigned *failed, const unsigned *done, unsigned need, int where)
{
    if (ld_acquire_gpu(done) >= need) return true;
    const uint64_t t0 = ptx::globaltimer_ns();
    for (uint32_t it = 1;; ++it) {
        if (ld_acquire_gpu(done) >= need) return true;
        if ((it & 15u) == 0) {
            if (ptx::ld_shared_u32_volatile(w.abort_addr) != 0 || ld_acquire_gpu(failed) != 0) {
                ptx::st_shared_u32_volatile(w.abort_addr, 1);
                return false;
            }
            if (ptx::globaltimer_ns() - t0 > w.timeout_ns) {
                ptx::st_shared_u32_volatile(w.abort_addr, 1);
                if (atomicCAS(w.status, 0, kStatusTimeout) == 0) {
                    w.status[1] = where;
                    w.status[2] = static_cast<int>(blockIdx.x);
                }
                return false;
            }
        }
    }
}

// The same for a word in shared memory that another warp of the block raises.
__device__ __forceinline__ bool ns_wait_word(const WaitCtx &w, uint32_t word, uint32_t need, int where)
{
    bool ok = true;
    if (ptx::ld_shared_u32_volatile(word) < need) {
        const uint64_t t0 = ptx::globaltimer_ns();
        for (uint32_t it = 1; ptx::ld_shared_u32_volatile(word) < need; ++it) {
            if ((it & 63u) != 0) continue;
            ok = ptx::ld_shared_u32_volatile(w.abort_addr) == 0;
            if (ok && ptx::globaltimer_ns() - t0 > w.timeout_ns) {
                ok = false;
                ptx::st_shared_u32_volatile(w.abort_addr, 1);
                if (atomicCAS(w.status, 0, kStatusTimeout) == 0) {
                    w.status[1] = where;
                    w.status[2] = static_cast<int>(blockIdx.x);
                }
            }
            if (!ok) break;
        }
    }
    __threadfence_block();
    return ok;
}

template <class Cfg>
__global__ void __launch_bounds__(Cfg::THREADS, 1)
newton_schulz_kernel(const __grid_constant__ CUtensorMap tmX0, const __grid_constant__ CUtensorMap tmX1,
                     const __grid_constant__ CUtensorMap tmS, const __grid_constant__ CUtensorMap tmP,
                     const __grid_constant__ CUtensorMap tmX0out, const __grid_constant__ CUtensorMap tmX1out,
                     const __grid_constant__ CUtensorMap tmSout, const __grid_constant__ CUtensorMap tmPout,
                     const __grid_constant__ NsParams p)
{
    constexpr int STAGES = Cfg::STAGES;
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
    // Epilogue warps that have stored tile i. Four words in turn: a warp comes to tile i + 3 at the earliest when all have released the
    // accumulator of tile i + 1, and so are done with tile i.
    auto stored_word = [&](uint32_t i) { return bar0 + 256u + 4u * (i & 3u); };
    // Tiles whose predecessors the producer has seen done; it only grows, as the producer may be many short tiles ahead.
    const uint32_t ready_word = bar0 + 272u;
    static_assert(8 * (2 * STAGES + 4) <= 240, "barrier region");

    if (warp == 0) {
        if (lane < STAGES) {
            ptx::mbar_init(full_bar(lane), 1);
            ptx::mbar_init(empty_bar(lane), 1);
        } else if (lane < STAGES + 2) {
            ptx::mbar_init(tfull_bar(lane - STAGES), 1);
            ptx::mbar_init(tempty_bar(lane - STAGES), Cfg::EPI_WARPS * CG);
        }
        if (lane < 4) ptx::st_shared_u32_volatile(stored_word(static_cast<uint32_t>(lane)), 0);
        if (lane == 4) ptx::st_shared_u32_volatile(ready_word, 0);
        if (lane == 31) {
            ptx::st_shared_u32_volatile(abort_addr, 0);
            ptx::st_shared_u32_volatile(epi_abort_addr, 0);
        }
        ptx::fence_barrier_init();
        if (lane == 30) {
            ptx::prefetch_tmap(&tmX0);
            ptx::prefetch_tmap(&tmX1);
            ptx::prefetch_tmap(&tmS);
            ptx::prefetch_tmap(&tmP);
            ptx::prefetch_tmap(&tmX0out);
            ptx::prefetch_tmap(&tmX1out);
            ptx::prefetch_tmap(&tmSout);
            ptx::prefetch_tmap(&tmPout);
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
    const uint32_t tmem_base = ptx::ld_shared_u32_volatile(tmem_slot);
    // the wait nearest the cause of a stall is the one that runs out: the producer's for other blocks, then the issuer's, then the epilogue's
    const WaitCtx wctx{abort_addr, p.status, p.timeout_ns};
    const WaitCtx wctx_mma{abort_addr, p.status, 2 * p.timeout_ns};
    const WaitCtx wctx_epi{abort_addr, p.status, 3 * p.timeout_ns};

    auto load = [&](uint32_t dst, const CUtensorMap *m, uint32_t bar, int x, int y, int z) {
        if (CG == 2) tma_load_3d_pair(dst, m, bar, x, y, z);
        else ptx::tma_load_3d(dst, m, bar, x, y, z);
    };

    if (!smem_ok) {
        // fall through to the common exit
    } else if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (every CTA)
        if (ptx::elect_one()) {
            int stage = 0;
            uint32_t phase = 0, tile = 0;
            bool ok = true;
            for (int u = first_unit; u < p.units && ok; u += unit_stride) {
                const NsUnit t = ns_unit(p, u);
                const CUtensorMap *x = (t.step & 1) ? &tmX1 : &tmX0;
                const bool tall = p.R > p.C;
                const CUtensorMap *mapA = t.phase == kNsGram ? x : t.phase == kNsPoly ? &tmS : tall ? x : &tmP;
                const CUtensorMap *mapB = t.phase == kNsGram ? x : t.phase == kNsPoly ? &tmS : tall ? &tmP : x;
                const int m0 = t.m_blk * Cfg::EDGE + static_cast<int>(rank) * Cfg::ROWS;
                const int n0 = t.n_blk * Cfg::EDGE + static_cast<int>(rank) * Cfg::ROWS;
                const int kblocks = t.phase == kNsGram ? p.kb_gram : p.kb_m;
                const bool same = ns_same_operand(t);
                ok = ns_wait_done(wctx, p.failed, p.done + t.z * kMuonCountPitch, t.need * CG, 700 + t.phase);
                if (!ok) break;
                __threadfence_block();
                ptx::st_shared_u32_volatile(ready_word, ++tile);
                fence_proxy_async_global();  // the first X was stored by plain stores
                for (int kb = 0; kb < kblocks; ++kb) {
                    ok = wait_barrier(wctx, empty_bar(stage), phase ^ 1u, 100 + stage);
                    if (!ok) break;
                    const uint32_t fb = (CG == 2) ? ptx::mapa(full_bar(stage), 0) : full_bar(stage);
                    if (rank == 0) ptx::mbar_expect_tx(full_bar(stage), CG * Cfg::OP_BYTES * (same ? 1u : 2u));
                    const uint32_t sa = smem + stage * Cfg::OP_BYTES;
                    const uint32_t sb = smem + Cfg::OFF_B + stage * Cfg::OP_BYTES;
                    const int k0 = kb * kBlockK;
                    const bool a_mn = ns_a_mn<Cfg>(p, t, kb), b_mn = ns_b_mn<Cfg>(p, t, kb);
#pragma unroll
                    for (int j = 0; j < Cfg::ROWS / 64; ++j)
                        load(sa + j * 8192u, mapA, fb, a_mn ? m0 + j * 64 : k0, a_mn ? k0 : m0 + j * 64, t.z);
                    if (!same)
#pragma unroll
                        for (int j = 0; j < Cfg::ROWS / 64; ++j)
                            load(sb + j * 8192u, mapB, fb, b_mn ? n0 + j * 64 : k0, b_mn ? k0 : n0 + j * 64, t.z);
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
            constexpr uint32_t idesc0 = make_idesc(Cfg::EDGE, Cfg::EDGE, false, false) & ~((1u << 7) | (1u << 10));
            int stage = 0;
            uint32_t phase = 0;
            int acc = 0;
            uint32_t acc_phase = 0;
            bool ok = true;
            for (int u = first_unit; u < p.units && ok; u += unit_stride) {
                const NsUnit t = ns_unit(p, u);
                const int kblocks = t.phase == kNsGram ? p.kb_gram : p.kb_m;
                const bool same = ns_same_operand(t);
                ok = wait_barrier(wctx_mma, tempty_bar(acc), acc_phase ^ 1u, 200 + acc);
                if (!ok) break;
                ptx::tc_fence_after();
                const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * Cfg::EDGE);
                for (int kb = 0; kb < kblocks; ++kb) {
                    ok = wait_barrier(wctx_mma, full_bar(stage), phase, 300 + stage);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    const uint32_t sa = smem + stage * Cfg::OP_BYTES;
                    const uint32_t sb = same ? sa : smem + Cfg::OFF_B + stage * Cfg::OP_BYTES;
                    const bool a_mn = ns_a_mn<Cfg>(p, t, kb), b_mn = ns_b_mn<Cfg>(p, t, kb);
                    // K-major: 8-row groups 1024 B apart, 16 k = 32 B inside the swizzle row.
                    // MN-major: 64-wide chunks 8192 B apart, 8-k groups 1024 B apart, 16 k = 2048 B.
                    const uint64_t adesc = make_smem_desc(sa, a_mn ? 8192 : 16, 1024);
                    const uint64_t bdesc = make_smem_desc(sb, b_mn ? 8192 : 16, 1024);
                    const uint32_t a_step = a_mn ? (2048u >> 4) : (32u >> 4);
                    const uint32_t b_step = b_mn ? (2048u >> 4) : (32u >> 4);
                    const uint32_t idesc = idesc0 | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
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
        // ------------------------------------------------------------ epilogue, warp by warp
        // A warp's pieces have a staging box each, which it stores by TMA copies of its own.
        const int q = warp & 3;
        const int ew = warp - 2;
        const int column = (ew >> 2) * Cfg::WARP_COLS;  // the warp's first, in the tile
        constexpr int WR = Cfg::WARP_ROWS;
        constexpr int PIECES = Cfg::PIECES;
        const uint32_t stg = smem + Cfg::OFF_STG + static_cast<uint32_t>(ew * PIECES) * Cfg::BOX_BYTES;
        const uint32_t mine = stg + static_cast<uint32_t>(lane) * 128u;  // this lane's row
        const uint32_t sw = static_cast<uint32_t>(lane & 7);
        const bool has_row = lane < WR;
        const int rr0 = lane >> 3, cc = lane & 7;  // eight lanes to 64 columns of a row where memory is accessed
        const uint32_t flat = stg + static_cast<uint32_t>(rr0) * 128u;
        int acc = 0;
        uint32_t acc_phase = 0, tile = 0;
        for (int u = first_unit; u < p.units; u += unit_stride) {
            if (ptx::ld_shared_u32_volatile(epi_abort_addr) != 0) break;
            const NsUnit t = ns_unit(p, u);
            const int y0 = t.m_blk * Cfg::EDGE + static_cast<int>(rank) * Cfg::ROWS + q * WR;  // the warp's first row
            const int x0 = t.n_blk * Cfg::EDGE + column;                           // and first column
            const bool poly = t.phase == kNsPoly, last = t.phase == kNsStep && t.step == p.steps - 1;
            const int M = t.phase == kNsStep ? p.R : p.m, N = t.phase == kNsStep ? p.C : p.m;
            const float alpha = t.phase == kNsGram ? p.gram_alpha : poly ? p.poly_alpha : last ? p.last_alpha : p.step_alpha;
            const ptx::f2 al = ptx::make_f2(alpha, alpha);
            bool ok = true;
            auto in_row = [&](int i) { return y0 + rr0 + i * 4 < M; };
            if (poly) {  // b S is added: the tile's part of S comes into staging while the product is formed
                if (lane == 0) ok = ns_wait_word(wctx_epi, ready_word, tile + 1, 710);
                __syncwarp();
                // the lane's first 16 bytes; its rows lie 4 lds apart
                const __half *src = p.s + (static_cast<long long>(t.z) * M + y0 + rr0) * p.lds + x0 + cc * 8;
#pragma unroll 1
                for (int piece = 0; piece < PIECES; ++piece) {
                    const bool in_col = x0 + piece * 64 + cc * 8 < N;
                    uint4 v[WR / 4];
#pragma unroll
                    for (int i = 0; i < WR / 4; ++i)
                        v[i] = in_row(i) && in_col ? ld_global_cg_v4(src + static_cast<long long>(i) * 4 * p.lds + piece * 64)
                                                   : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < WR / 4; ++i)
                        ptx::st_shared_v4(flat + piece * Cfg::BOX_BYTES + i * 512u +
                                              (static_cast<uint32_t>(cc ^ ((rr0 + i * 4) & 7)) << 4), v[i].x, v[i].y, v[i].z, v[i].w);
                }
                __syncwarp();
            }
            if (lane == 0) ok = wait_barrier(wctx_epi, tfull_bar(acc), acc_phase, 400 + acc) && ok;
            ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
            if (!ok) ptx::st_shared_u32_volatile(epi_abort_addr, 1);
            ptx::tc_fence_after();
            const uint32_t t_acc = tmem_base + (static_cast<uint32_t>(q * 32) << 16) +
                                   static_cast<uint32_t>(acc * Cfg::EDGE + column);
            uint32_t r[2 * PIECES][32];
#pragma unroll
            for (int i = 0; i < 2 * PIECES; ++i) ptx::tmem_ld_32x32_issue(t_acc + static_cast<uint32_t>(i * 32), r[i]);
            ptx::tmem_ld_wait_32(r[0]);
#pragma unroll
            for (int i = 1; i < 2 * PIECES; ++i) ptx::reg_fence_32(r[i]);
            ptx::tc_fence_before();  // the accumulator is in registers
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) ptx::mbar_arrive_cluster(ptx::mapa(tempty_bar(acc), 0));
                else ptx::mbar_arrive(tempty_bar(acc));
            }
            const CUtensorMap *out = t.phase == kNsGram ? &tmSout : poly ? &tmPout : (t.step & 1) ? &tmX0out : &tmX1out;
#pragma unroll
            for (int piece = 0; piece < PIECES; ++piece) {
                const uint32_t box = mine + piece * Cfg::BOX_BYTES;
                // eight columns at a time: f gives their words from their pairs
                auto convert = [&](auto &&f) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t (&rj)[32] = r[2 * piece + (j >> 2)];
                        uint32_t w[4];
                        f(j, w, [&](int k) { return ptx::make_f2_bits(rj[(j & 3) * 8 + 2 * k], rj[(j & 3) * 8 + 2 * k + 1]); });
                        if (WR == 32 || has_row) ptx::st_shared_v4(box + ((static_cast<uint32_t>(j) ^ sw) << 4), w[0], w[1], w[2], w[3]);
                    }
                };
                if (poly) {
                    convert([&](int j, uint32_t (&w)[4], auto &&pair) {
                        uint32_t a4[4];
                        a4[0] = a4[1] = a4[2] = a4[3] = 0;
                        if (WR == 32 || has_row) ptx::ld_shared_v4(box + ((static_cast<uint32_t>(j) ^ sw) << 4), a4[0], a4[1], a4[2], a4[3]);
                        const int d = y0 + lane - (x0 + piece * 64 + j * 8);  // the diagonal's place among the eight
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float2 s = __half22float2(*reinterpret_cast<const __half2 *>(&a4[k]));
                            const ptx::f2 add = ptx::make_f2(fmaf(s.x, p.poly_beta, d == 2 * k ? p.poly_diag : 0.0f),
                                                             fmaf(s.y, p.poly_beta, d == 2 * k + 1 ? p.poly_diag : 0.0f));
                            float lo, hi;
                            ptx::split_f2(ptx::fma2(pair(k), al, add), lo, hi);
                            w[k] = pack_f16x2(lo, hi);
                        }
                    });
                } else if (last) {
                    convert([&](int, uint32_t (&w)[4], auto &&pair) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] = pack_f2_bf16x2(ptx::mul2(pair(k), al));
                    });
                } else {
                    convert([&](int, uint32_t (&w)[4], auto &&pair) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float lo, hi;
                            ptx::split_f2(ptx::mul2(pair(k), al), lo, hi);
                            w[k] = pack_f16x2(lo, hi);
                        }
                    });
                }
                if (!last) {
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (ptx::elect_one()) {
                        if (ok && y0 < M && x0 + piece * 64 < N) tma_store_3d(out, stg + piece * Cfg::BOX_BYTES, x0 + piece * 64, y0, t.z);
                        ptx::bulk_commit_group();
                    }
                    __syncwarp();
                    continue;
                }
                // The results: whole pieces of the caller's rows, by plain stores.
                __syncwarp();
                uint4 *d4 = static_cast<uint4 *>(p.out[t.z]) + (static_cast<long long>(y0 + rr0) * N + x0) / 8 + cc;
                const bool in_col = ok && x0 + piece * 64 + cc * 8 < N;
#pragma unroll
                for (int i = 0; i < WR / 4; ++i) {
                    uint32_t w[4];
                    ptx::ld_shared_v4(flat + piece * Cfg::BOX_BYTES + i * 512u + (static_cast<uint32_t>(cc ^ ((rr0 + i * 4) & 7)) << 4),
                                      w[0], w[1], w[2], w[3]);
                    if (in_col && in_row(i)) d4[static_cast<long long>(i) * (N / 2) + piece * 8] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            ptx::bulk_wait_group<0>();  // in memory; every lane: only the one that issued copies has any to wait for
            __syncwarp();
            // The warp that is the last to have its part of the tile in memory counts it for the others; nobody waits for the results.
            if (lane == 0 && atom_add_acq_rel_shared(stored_word(tile), 1) == Cfg::EPI_WARPS - 1) {
                ptx::st_shared_u32_volatile(stored_word(tile), 0);
                if (!last && ptx::ld_shared_u32_volatile(epi_abort_addr) == 0) red_release_gpu(p.done + t.z * kMuonCountPitch, 1);
            }
            __syncwarp();
            ++tile;
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
            }
        }
    }

    // ---------------------------------------------------------------- common exit
    if (ptx::ld_shared_u32_volatile(abort_addr) != 0 || ptx::ld_shared_u32_volatile(epi_abort_addr) != 0) {
        if (lane == 0) atomicExch(p.failed, 1u);
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
