// Layer norm with the residual add in front of it, forward and backward, for rows of C elements.
//
//   s = round(x + branch)   mean = sum_j s_j / C   rstd = 1 / sqrt(sum_j (s_j - mean)^2 / C + eps)
//   out_j = (s_j - mean) rstd w_j + b_j
//
//   xh = (s - mean) rstd    g = dout w    dinp = dres + rstd (g - mean(g) - xh mean(g xh))
//   dweight = sum over rows of dout xh    dbias = sum over rows of dout
//
// A team of T threads owns a row (NV vectors of eight elements per thread), so the deviations are summed from the mean itself
// and every tensor crosses the memory bus once. At a training batch the forward pass is bound by HBM (16384 x 768 bf16: 17.8 us, 15.4 at
// the measured rate), and so is the backward pass of fp32 rows (5001 x 4096: 58 us, 50 at that rate). The backward pass of bf16 rows is short of
// warps to hide its instructions' latency (16384 x 768: 19.4 us of the same 15.4), and the sums over the rows' blocks add a launch to it
// (22.9 in all, in a captured chain). Teams walk the rows with the stride of the grid. All links of the dependent-launch chain: no read-only loads (ptx::ld_global_*).
#pragma once
#include "elementwise.cuh"

namespace nb {

// Eight elements of the residual stream as they lie in memory (bf16 or fp32).
template <bool F32>
struct Raw8 {
    uint4 q[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ Raw8<F32> load8(const void *base, long long vec)
{
    Raw8<F32> r;
    const uint4 *p = static_cast<const uint4 *>(base) + vec * (F32 ? 2 : 1);
    r.q[0] = ptx::ld_global_v4(p);
    if constexpr (F32) r.q[1] = ptx::ld_global_v4(p + 1);
    return r;
}
// Eight values as four packed pairs: these kernels are short of instructions before they are short of bandwidth (one value at a
// time the forward took 526 per warp and row of 768, the backward 760, at half an instruction per cycle and scheduler).
struct Pairs {
    ptx::f2 v[4];
};
__device__ __forceinline__ Pairs unpack_bf16(const uint4 &q)
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    Pairs r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r.v[k] = ptx::make_f2_bits(w[k] << 16, w[k] & 0xffff0000u);
    return r;
}
template <bool F32>
__device__ __forceinline__ Pairs unpack8(const Raw8<F32> &q)
{
    if constexpr (F32) {
        Pairs r;
        r.v[0] = ptx::make_f2_bits(q.q[0].x, q.q[0].y);
        r.v[1] = ptx::make_f2_bits(q.q[0].z, q.q[0].w);
        r.v[2] = ptx::make_f2_bits(q.q[1].x, q.q[1].y);
        r.v[3] = ptx::make_f2_bits(q.q[1].z, q.q[1].w);
        return r;
    } else {
        return unpack_bf16(q.q[0]);
    }
}
__device__ __forceinline__ uint4 pack_bf16(const Pairs &a)
{
    return make_uint4(pack_f2_bf16x2(a.v[0]), pack_f2_bf16x2(a.v[1]), pack_f2_bf16x2(a.v[2]), pack_f2_bf16x2(a.v[3]));
}
template <bool F32>
__device__ __forceinline__ Raw8<F32> pack8(const Pairs &a)
{
    Raw8<F32> r;
    if constexpr (F32) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) ptx::split_f2(a.v[k], f[2 * k], f[2 * k + 1]);
        r.q[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        r.q[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    } else {
        r.q[0] = pack_bf16(a);
    }
    return r;
}
// Stream + branch, rounded to the stream's type. bf16: the packed addition, whose one rounding is that of the fp32 sum rounded to bf16 (the
// fp32 sum is inexact only where one addend is below 2^-16 of the other, and both then round to that other).
template <bool F32>
__device__ __forceinline__ Raw8<F32> add_branch(const Raw8<F32> &x, const uint4 &b)
{
    if constexpr (F32) {
        Pairs s = unpack8<true>(x);
        const Pairs a = unpack_bf16(b);
#pragma unroll
        for (int k = 0; k < 4; ++k) s.v[k] = ptx::add2(s.v[k], a.v[k]);
        return pack8<true>(s);
    } else {
        Raw8<F32> r;
        auto add = [](uint32_t u, uint32_t v) {
            uint32_t w;
            asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(w) : "r"(u), "r"(v));
            return w;
        };
        r.q[0] = make_uint4(add(x.q[0].x, b.x), add(x.q[0].y, b.y), add(x.q[0].z, b.z), add(x.q[0].w, b.w));
        return r;
    }
}
__device__ __forceinline__ float sum2(ptx::f2 a)
{
    float lo, hi;
    ptx::split_f2(a, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ ptx::f2 both(float a) { return ptx::make_f2(a, a); }
template <bool F32>
__device__ __forceinline__ void store8(void *base, long long vec, const Raw8<F32> &r)
{
    uint4 *p = static_cast<uint4 *>(base) + vec * (F32 ? 2 : 1);
    p[0] = r.q[0];
    if constexpr (F32) p[1] = r.q[1];
}

// Consecutive bytes into shared memory, counted on an mbarrier. Both addresses and the size are multiples of 16.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

template <int T>
__device__ __forceinline__ void team_sync(int team)
{
    if (T == 32) __syncwarp();
    else ptx::named_bar_sync(1u + static_cast<uint32_t>(team), T);
}

// Sums two values over the team; every thread gets both sums, added in the same order on every call. Teams of several warps meet at ONE
// barrier: the slots alternate by `turn`, so a slot is rewritten only after the barrier behind its last read.
template <int T>
__device__ __forceinline__ float2 team_sum(float2 v, float2 (*slots)[T / 32], int turn, int team)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if constexpr (T > 32) {
        float2 *s = slots[turn & 1];
        if ((threadIdx.x & 31) == 0) s[threadIdx.x % T / 32] = v;
        team_sync<T>(team);
        v = s[0];
#pragma unroll
        for (int i = 1; i < T / 32; ++i) {
            v.x += s[i].x;
            v.y += s[i].y;
        }
    }
    return v;
}

constexpr int kNormMaxSlots = 4;
constexpr int kNormMaxThreads = 512;  // of a block; half of that in the DIRECT forms

// What the passes share: rows come into shared memory by bulk copies, up to kNormMaxSlots per team under way, whatever registers the
// arithmetic needs. (By loads into registers, with the next row's ahead, a backward row of 768 took 218 registers and one of
// 1024 forward 158: one block of eight warps on an SM, 28.7 us for 16384 x 768 and 32.7 us for 16384 x 1024.)
struct NormRing {
    uint32_t at, bar, row_bytes;
    int slots, slot;
    uint32_t phase;
    __device__ __forceinline__ uint32_t row() const { return at + static_cast<uint32_t>(slot) * row_bytes; }
    __device__ __forceinline__ uint32_t full() const { return bar + 8u * static_cast<uint32_t>(slot); }
    __device__ __forceinline__ void next()
    {
        if (++slot == slots) {
            slot = 0;
            phase ^= 1u;
        }
    }
};
template <bool F32>
__device__ __forceinline__ Raw8<F32> shared8(uint32_t base, int vec)
{
    Raw8<F32> r;
    const uint32_t at = base + static_cast<uint32_t>(vec) * (F32 ? 32u : 16u);
    ptx::ld_shared_v4(at, r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w);
    if constexpr (F32) ptx::ld_shared_v4(at + 16u, r.q[1].x, r.q[1].y, r.q[1].z, r.q[1].w);
    return r;
}

// Waits for a row's copy; not again once a thread of the block gave up. A team that gave up goes on through its rows, since its threads
// meet at barriers, but no slot is filled again: its barrier may not have come to the end of its phase. (The failure held in a
// variable over the rows instead: 29.6 us against 29.0 for 4096 x 4096 bf16 backward, 47.1 against 43.9 for 4096 x 8192 forward.)
__device__ __forceinline__ bool norm_wait(const WaitCtx &w, const NormRing &ring, int where)
{
    return ptx::mbar_try_wait(ring.full(), ring.phase) ||
           (ptx::ld_shared_u32_volatile(w.abort_addr) == 0 && wait_barrier(w, ring.full(), ring.phase, where));
}
// Where a wait ran out: copies that are still under way write the block's shared memory, so it stays until they have landed.
__device__ __forceinline__ void norm_leave()
{
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
}

struct NormForward {
    void *out;           // bf16
    void *sum;           // stream's type, or null where there is no branch
    float *mean, *rstd;  // or both null
    const void *inp;     // stream's type
    const void *branch;  // bf16, or null
    const void *weight;  // bf16
    const void *bias;    // bf16, or null
    long long BT;
    int nvec;            // C / 8
    int slots;           // rows that a team has in shared memory
    float inv_c, eps;
    int withhold;        // nb_debug_layernorm_timeout only: bytes that every row waits for and that never come; else 0
    int *status;
    unsigned long long timeout_ns;  // 0: the usual limit
};
// Shared memory of a row of the forward pass: inp, branch (if there is one).
__host__ __device__ constexpr int norm_forward_row_bytes(bool f32, int nvec, bool has_branch) { return nvec * ((f32 ? 32 : 16) + (has_branch ? 16 : 0)); }

// DIRECT: no team has more than one row, which it loads into registers instead, in blocks of half as many warps: through shared memory a call
// on few rows takes 0.3 to 1.6 us longer (captured chains, forward: 8 x 768 bf16 1.95 against 2.29 us, 1184 x 768 2.10 against 2.92, 1003 x 776 fp32
// 3.2 against 4.8).
template <bool F32, int T, int NV, bool DIRECT>
__global__ void __launch_bounds__(DIRECT ? kNormMaxThreads / 2 : kNormMaxThreads, 1)
layernorm_forward_kernel(const NormForward p)
{
    extern __shared__ __align__(128) uint8_t norm_smem[];  // the teams' rows
    __shared__ __align__(8) unsigned long long bars[kNormMaxThreads / T * kNormMaxSlots];
    __shared__ float2 sums[kNormMaxThreads / T][2][T / 32];
    __shared__ uint32_t abort_flag;
    const int t = static_cast<int>(threadIdx.x) % T;
    const int team = threadIdx.x / T, teams = static_cast<int>(blockDim.x) / T;
    const bool has_branch = p.branch != nullptr;
    const uint32_t branch_bytes = static_cast<uint32_t>(p.nvec) * 16u, x_bytes = branch_bytes * (F32 ? 2u : 1u);
    const uint32_t row_bytes = static_cast<uint32_t>(norm_forward_row_bytes(F32, p.nvec, has_branch));
    NormRing ring{ptx::smem_u32(norm_smem) + static_cast<uint32_t>(team * p.slots) * row_bytes,
                  ptx::smem_u32(bars) + 8u * static_cast<uint32_t>(team * kNormMaxSlots), row_bytes, p.slots, 0, 0};
    if constexpr (!DIRECT) {
        if (t < p.slots) ptx::mbar_init(ring.bar + 8u * t, 1);
        if (threadIdx.x == 0) abort_flag = 0;
        ptx::fence_barrier_init();
        __syncthreads();
    }
    chained_start();
    const WaitCtx wctx{ptx::smem_u32(&abort_flag), p.status, p.timeout_ns};
    auto gave_up = [&] { return ptx::ld_shared_u32_volatile(wctx.abort_addr) != 0; };
    const long long stride = static_cast<long long>(gridDim.x) * teams;
    const long long first = static_cast<long long>(blockIdx.x) * teams + team;
    auto fetch = [&](long long row, int slot) {  // one thread of the team
        const uint32_t dst = ring.at + static_cast<uint32_t>(slot) * row_bytes, b = ring.bar + 8u * slot;
        ptx::mbar_expect_tx(b, row_bytes + static_cast<uint32_t>(p.withhold));
        bulk_load(dst, static_cast<const uint8_t *>(p.inp) + row * x_bytes, x_bytes, b);
        if (has_branch) bulk_load(dst + x_bytes, static_cast<const uint8_t *>(p.branch) + row * branch_bytes, branch_bytes, b);
    };
    Raw8<F32> xd[DIRECT ? NV : 1];
    uint4 bd[DIRECT ? NV : 1];
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            if (j >= p.nvec || first >= p.BT) continue;
            xd[i] = load8<F32>(p.inp, first * p.nvec + j);
            if (has_branch) bd[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.branch) + first * p.nvec + j);
        }
    } else if (t == 0)
        for (int i = 0; i < p.slots && first + i * stride < p.BT; ++i) fetch(first + i * stride, i);
    uint4 w[NV], b[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = t + i * T;
        w[i] = b[i] = make_uint4(0, 0, 0, 0);
        if (j < p.nvec) {
            w[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.weight) + j);
            if (p.bias) b[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.bias) + j);
        }
    }
    int turn = 0;
    for (long long row = first; row < p.BT; row += stride) {
        bool ok = true;
        if constexpr (!DIRECT) ok = norm_wait(wctx, ring, 811);
        Pairs v[NV];
        ptx::f2 sum = both(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            v[i] = Pairs{{both(0.0f), both(0.0f), both(0.0f), both(0.0f)}};
            if (j >= p.nvec) continue;
            Raw8<F32> x;
            if constexpr (DIRECT) x = xd[i];
            else x = shared8<F32>(ring.row(), j);
            if (has_branch) {
                if constexpr (DIRECT) x = add_branch<F32>(x, bd[i]);
                else x = add_branch<F32>(x, shared8<false>(ring.row() + x_bytes, j).q[0]);
                if (ok) store8<F32>(p.sum, row * p.nvec + j, x);
            }
            v[i] = unpack8<F32>(x);  // the norm is that of the stored sum
            sum = ptx::add2(sum, ptx::add2(ptx::add2(v[i].v[0], v[i].v[1]), ptx::add2(v[i].v[2], v[i].v[3])));
        }
        const float mean = team_sum<T>(make_float2(sum2(sum), 0.0f), sums[team], turn++, team).x * p.inv_c;
        if constexpr (!DIRECT) {
            if (T == 32) __syncwarp();
            // the whole team has read the slot
            if (t == 0 && row + p.slots * stride < p.BT && ok && !gave_up()) fetch(row + p.slots * stride, ring.slot);
            ring.next();
        }
        const ptx::f2 minus = both(-mean);
        ptx::f2 sq = both(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (t + i * T >= p.nvec) continue;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[i].v[k] = ptx::add2(v[i].v[k], minus);
                sq = ptx::fma2(v[i].v[k], v[i].v[k], sq);
            }
        }
        const float var = team_sum<T>(make_float2(sum2(sq), 0.0f), sums[team], turn++, team).x * p.inv_c;
        const float rstd = 1.0f / sqrtf(var + p.eps);
        const ptx::f2 rs = both(rstd);
        if (!ok) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (t + i * T >= p.nvec) continue;
            const Pairs wf = unpack_bf16(w[i]), bf = unpack_bf16(b[i]);
            Pairs o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o.v[k] = ptx::fma2(ptx::mul2(v[i].v[k], rs), wf.v[k], bf.v[k]);
            static_cast<uint4 *>(p.out)[row * p.nvec + t + i * T] = pack_bf16(o);
        }
        if (t == 0 && p.mean) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
        }
    }
    if constexpr (!DIRECT) {
        if (gave_up()) norm_leave();
    }
}

struct NormBackward {
    void *dinp;           // stream's type
    void *dbranch;        // bf16 copy of dinp, or null
    float *part;          // [gridDim.x][2 C] sums of this block's rows (dweight, then dbias), or null
    const void *dout;     // bf16
    const void *dres;     // stream's type, or null
    const void *inp;      // stream's type: what the forward normed
    const float *mean, *rstd;
    const void *weight;   // bf16
    long long BT;
    int nvec;
    int slots;            // rows that a team has in shared memory
    float inv_c;
    int withhold;         // as in the forward pass
    int *status;
    unsigned long long timeout_ns;
};

// Shared memory of a row of the backward pass: dout, inp, dres (if there is one).
__host__ __device__ constexpr int norm_row_bytes(bool f32, int nvec, bool has_res) { return nvec * (16 + (f32 ? 32 : 16) * (has_res ? 2 : 1)); }

// A row is read twice from shared memory: once for its two sums and for the columns' sums, which stay in registers, and once for dinp.
// DIRECT: as in the forward pass; the row stays in registers.
template <bool F32, int T, int NV, bool DIRECT>
__global__ void __launch_bounds__(DIRECT ? kNormMaxThreads / 2 : kNormMaxThreads, 1)
layernorm_backward_kernel(const NormBackward p)
{
    extern __shared__ __align__(128) uint8_t norm_smem[];  // the teams' rows; then, of several teams, their sums [teams][2 C]
    __shared__ __align__(8) unsigned long long bars[kNormMaxThreads / T * kNormMaxSlots];
    __shared__ float2 sums[kNormMaxThreads / T][2][T / 32];
    __shared__ uint32_t abort_flag;
    const int t = static_cast<int>(threadIdx.x) % T;
    const int team = threadIdx.x / T, teams = static_cast<int>(blockDim.x) / T;
    const bool has_res = p.dres != nullptr;
    const uint32_t row_bytes = static_cast<uint32_t>(norm_row_bytes(F32, p.nvec, has_res));
    NormRing ring{ptx::smem_u32(norm_smem) + static_cast<uint32_t>(team * p.slots) * row_bytes,
                  ptx::smem_u32(bars) + 8u * static_cast<uint32_t>(team * kNormMaxSlots), row_bytes, p.slots, 0, 0};
    if constexpr (!DIRECT) {
        if (t < p.slots) ptx::mbar_init(ring.bar + 8u * t, 1);
        if (threadIdx.x == 0) abort_flag = 0;
        ptx::fence_barrier_init();
        __syncthreads();
    }
    chained_start();
    const WaitCtx wctx{ptx::smem_u32(&abort_flag), p.status, p.timeout_ns};
    auto gave_up = [&] { return ptx::ld_shared_u32_volatile(wctx.abort_addr) != 0; };
    const uint32_t dout_bytes = static_cast<uint32_t>(p.nvec) * 16u, x_bytes = dout_bytes * (F32 ? 2u : 1u);

    const long long stride = static_cast<long long>(gridDim.x) * teams;
    const long long first = static_cast<long long>(blockIdx.x) * teams + team;
    auto fetch = [&](long long row, int slot) {  // one thread of the team
        const uint32_t dst = ring.at + static_cast<uint32_t>(slot) * row_bytes, b = ring.bar + 8u * slot;
        ptx::mbar_expect_tx(b, row_bytes + static_cast<uint32_t>(p.withhold));
        bulk_load(dst, static_cast<const uint8_t *>(p.dout) + row * dout_bytes, dout_bytes, b);
        bulk_load(dst + dout_bytes, static_cast<const uint8_t *>(p.inp) + row * x_bytes, x_bytes, b);
        if (has_res) bulk_load(dst + dout_bytes + x_bytes, static_cast<const uint8_t *>(p.dres) + row * x_bytes, x_bytes, b);
    };
    uint4 dd[DIRECT ? NV : 1];
    Raw8<F32> xd[DIRECT ? NV : 1], rd[DIRECT ? NV : 1];
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            if (j >= p.nvec || first >= p.BT) continue;
            dd[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.dout) + first * p.nvec + j);
            xd[i] = load8<F32>(p.inp, first * p.nvec + j);
            if (has_res) rd[i] = load8<F32>(p.dres, first * p.nvec + j);
        }
    } else if (t == 0)
        for (int i = 0; i < p.slots && first + i * stride < p.BT; ++i) fetch(first + i * stride, i);

    uint4 w[NV];
    Pairs dw[NV], db[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        w[i] = make_uint4(0, 0, 0, 0);
        if (t + i * T < p.nvec) w[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.weight) + t + i * T);
#pragma unroll
        for (int k = 0; k < 4; ++k) dw[i].v[k] = db[i].v[k] = both(0.0f);
    }
    float mean = 0.0f, rstd = 0.0f;
    if (first < p.BT) {
        mean = __ldcg(p.mean + first);
        rstd = __ldcg(p.rstd + first);
    }
    int turn = 0;
    for (long long row = first; row < p.BT; row += stride) {
        bool ok = true;
        const float mu = mean, rs = rstd;
        if (row + stride < p.BT) {
            mean = __ldcg(p.mean + row + stride);
            rstd = __ldcg(p.rstd + row + stride);
        }
        if constexpr (!DIRECT) ok = norm_wait(wctx, ring, 810);
        const uint32_t src = ring.row();
        auto get_dout = [&](int i) {
            if constexpr (DIRECT) return dd[i];
            else return shared8<false>(src, t + i * T).q[0];
        };
        auto get_inp = [&](int i) {
            if constexpr (DIRECT) return xd[i];
            else return shared8<F32>(src + dout_bytes, t + i * T);
        };
        const ptx::f2 minus = both(-mu), rs2 = both(rs);
        ptx::f2 s1 = both(0.0f), s2 = both(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            if (j >= p.nvec) continue;
            const Pairs d = unpack_bf16(get_dout(i)), x = unpack8<F32>(get_inp(i)),
                        wf = unpack_bf16(w[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const ptx::f2 xh = ptx::mul2(ptx::add2(x.v[k], minus), rs2), g = ptx::mul2(d.v[k], wf.v[k]);
                dw[i].v[k] = ptx::fma2(d.v[k], xh, dw[i].v[k]);
                db[i].v[k] = ptx::add2(db[i].v[k], d.v[k]);
                s1 = ptx::add2(s1, g);
                s2 = ptx::fma2(g, xh, s2);
            }
        }
        const float2 s = team_sum<T>(make_float2(sum2(s1), sum2(s2)), sums[team], turn++, team);
        const ptx::f2 c1 = both(-(s.x * p.inv_c)), c2 = both(-(s.y * p.inv_c));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            if (j >= p.nvec) continue;
            const Pairs d = unpack_bf16(get_dout(i)), x = unpack8<F32>(get_inp(i)),
                        wf = unpack_bf16(w[i]);
            Pairs o;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const ptx::f2 xh = ptx::mul2(ptx::add2(x.v[k], minus), rs2);
                o.v[k] = ptx::fma2(xh, c2, ptx::fma2(d.v[k], wf.v[k], c1));
            }
            if (has_res) {
                Raw8<F32> raw;
                if constexpr (DIRECT) raw = rd[i];
                else raw = shared8<F32>(src + dout_bytes + x_bytes, j);
                const Pairs res = unpack8<F32>(raw);
#pragma unroll
                for (int k = 0; k < 4; ++k) o.v[k] = ptx::fma2(o.v[k], rs2, res.v[k]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) o.v[k] = ptx::mul2(o.v[k], rs2);
            }
            if (ok) {
                store8<F32>(p.dinp, row * p.nvec + j, pack8<F32>(o));
                if (p.dbranch) static_cast<uint4 *>(p.dbranch)[row * p.nvec + j] = pack_bf16(o);
            }
        }
        if constexpr (DIRECT) break;
        team_sync<T>(team);  // the slot has been read
        if (t == 0 && row + p.slots * stride < p.BT && ok && !gave_up()) fetch(row + p.slots * stride, ring.slot);
        ring.next();
    }
    if constexpr (!DIRECT) {
        if (gave_up()) norm_leave();
    }
    if (p.part == nullptr) return;
    __syncthreads();  // every row has been read: the same memory holds the sums now
    float4 *part = reinterpret_cast<float4 *>(p.part) + static_cast<long long>(blockIdx.x) * 4 * p.nvec;
    float4 *mine = teams > 1 ? reinterpret_cast<float4 *>(norm_smem) + team * 4 * p.nvec : part;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = t + i * T;
        if (j >= p.nvec) continue;
        const Raw8<true> a = pack8<true>(dw[i]), b = pack8<true>(db[i]);
        uint4 *m = reinterpret_cast<uint4 *>(mine);
        m[2 * j] = a.q[0];
        m[2 * j + 1] = a.q[1];
        m[2 * p.nvec + 2 * j] = b.q[0];
        m[2 * p.nvec + 2 * j + 1] = b.q[1];
    }
    if (teams > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < 4 * p.nvec; c += blockDim.x) {
            const float4 *all = reinterpret_cast<const float4 *>(norm_smem);
            float4 a = all[c];
            for (int k = 1; k < teams; ++k) {
                const float4 v = all[k * 4 * p.nvec + c];
                a.x += v.x;
                a.y += v.y;
                a.z += v.z;
                a.w += v.w;
            }
            part[c] = a;
        }
    }
}

// dweight[c] (+)= sum over the blocks' sums, dbias likewise, in a fixed order: results do not depend on which block ended
// first. A block owns 16 columns of [dweight | dbias], half a warp every 32nd part, all of them (five at most) loaded at once, as is what
// the result is added to: one trip to memory.
constexpr int kNormMaxBlocks = 148, kNormReduceCols = 16;
__global__ void __launch_bounds__(512)
layernorm_reduce_kernel(float *dweight, float *dbias, const float *part, int parts, int C, int accumulate)
{
    constexpr int N = (kNormMaxBlocks + 31) / 32;
    __shared__ float s[32][kNormReduceCols];
    chained_start();
    const int column = threadIdx.x % kNormReduceCols, group = threadIdx.x / kNormReduceCols;
    const int c = blockIdx.x * kNormReduceCols + column;  // 2 C is a multiple of 16
    float *dst = c < C ? dweight : dbias;
    if (dst != nullptr) dst += c < C ? c : c - C;
    const float old = group == 0 && accumulate && dst != nullptr ? __ldcg(dst) : 0.0f;
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int k = group + 32 * i;
        v[i] = dst != nullptr && k < parts ? __ldcg(part + static_cast<long long>(k) * 2 * C + c) : 0.0f;
    }
    float a = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) a += v[i];
    s[group][column] = a;
    __syncthreads();
    if (group != 0 || dst == nullptr) return;
#pragma unroll
    for (int k = 1; k < 32; ++k) a += s[k][column];
    *dst = old + a;
}

}  // namespace nb
