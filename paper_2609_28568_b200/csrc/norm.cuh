// Layer norm with the residual add in front of it, forward and backward, for rows of C elements.
//
//   s = round(x + branch)   mean = sum_j s_j / C   rstd = 1 / sqrt(sum_j (s_j - mean)^2 / C + eps)
//   out_j = (s_j - mean) rstd w_j + b_j
//
//   xh = (s - mean) rstd    g = dout w    dinp = dres + rstd (g - mean(g) - xh mean(g xh))
//   dweight = sum over rows of dout xh    dbias = sum over rows of dout
//
// A team of T threads owns a row and holds it in registers (NV vectors of eight elements per thread), so the
// deviations are summed from the mean itself and every tensor crosses the memory bus once: both passes are bound by
// HBM. Teams walk the rows with the stride of the grid; the next row's loads are issued as soon as this
// row's have been unpacked. All links of the dependent-launch chain: no read-only loads (ptx::ld_global_*).
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
__device__ __forceinline__ void unpack_bf16(const uint4 &q, float (&v)[8])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[2 * k] = ptx::bf16_lo(w[k]);
        v[2 * k + 1] = ptx::bf16_hi(w[k]);
    }
}
template <bool F32>
__device__ __forceinline__ void unpack8(const Raw8<F32> &r, float (&v)[8])
{
    if constexpr (F32) {
        const uint32_t w[8] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w, r.q[1].x, r.q[1].y, r.q[1].z, r.q[1].w};
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[k]);
    } else {
        unpack_bf16(r.q[0], v);
    }
}
__device__ __forceinline__ uint4 pack_bf16(const float (&v)[8])
{
    return make_uint4(ptx::pack_bf16x2(v[0], v[1]), ptx::pack_bf16x2(v[2], v[3]), ptx::pack_bf16x2(v[4], v[5]),
                      ptx::pack_bf16x2(v[6], v[7]));
}
template <bool F32>
__device__ __forceinline__ Raw8<F32> pack8(const float (&v)[8])
{
    Raw8<F32> r;
    if constexpr (F32) {
        r.q[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        r.q[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else {
        r.q[0] = pack_bf16(v);
    }
    return r;
}
template <bool F32>
__device__ __forceinline__ void store8(void *base, long long vec, const Raw8<F32> &r)
{
    uint4 *p = static_cast<uint4 *>(base) + vec * (F32 ? 2 : 1);
    p[0] = r.q[0];
    if constexpr (F32) p[1] = r.q[1];
}

// Threads of a block: eight teams of a warp, or one team.
template <int T>
constexpr int kNormThreads = T == 32 ? 256 : T;

// Sums two values over the team; every thread gets both sums, added in the same order on every call. Teams of several warps meet at ONE
// barrier: the slots alternate by `turn`, so a slot is rewritten only after the barrier behind its last read.
template <int T>
__device__ __forceinline__ float2 team_sum(float2 v, float2 (*slots)[T / 32], int turn)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if constexpr (T > 32) {
        float2 *s = slots[turn & 1];
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int i = 1; i < T / 32; ++i) {
            v.x += s[i].x;
            v.y += s[i].y;
        }
    }
    return v;
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
    float inv_c, eps;
};

template <bool F32, int T, int NV>
__global__ void __launch_bounds__(kNormThreads<T>)
layernorm_forward_kernel(const NormForward p)
{
    __shared__ float2 slots[2][T / 32];
    chained_start();
    const int t = static_cast<int>(threadIdx.x) % T;
    constexpr int TEAMS = kNormThreads<T> / T;
    const long long stride = static_cast<long long>(gridDim.x) * TEAMS;
    long long row = static_cast<long long>(blockIdx.x) * TEAMS + threadIdx.x / T;
    const bool has_branch = p.branch != nullptr;
    Raw8<F32> x[NV];
    uint4 br[NV], w[NV], b[NV];
    auto load = [&](long long r) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            x[i] = Raw8<F32>{};
            br[i] = make_uint4(0, 0, 0, 0);
            if (j < p.nvec) {
                x[i] = load8<F32>(p.inp, r * p.nvec + j);
                if (has_branch) br[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.branch) + r * p.nvec + j);
            }
        }
    };
    if (row < p.BT) load(row);
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
    for (; row < p.BT; row += stride) {
        float v[NV][8];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            unpack8<F32>(x[i], v[i]);
            if (has_branch) {
                float a[8];
                unpack_bf16(br[i], a);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[i][k] += a[k];
                const Raw8<F32> s = pack8<F32>(v[i]);
                if (t + i * T < p.nvec) store8<F32>(p.sum, row * p.nvec + t + i * T, s);
                unpack8<F32>(s, v[i]);  // the norm is that of the stored sum
            }
            sum += ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3])) + ((v[i][4] + v[i][5]) + (v[i][6] + v[i][7]));
        }
        if (row + stride < p.BT) load(row + stride);
        const float mean = team_sum<T>(make_float2(sum, 0.0f), slots, turn++).x * p.inv_c;
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (t + i * T >= p.nvec) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[i][k] -= mean;
                sq = fmaf(v[i][k], v[i][k], sq);
            }
        }
        const float var = team_sum<T>(make_float2(sq, 0.0f), slots, turn++).x * p.inv_c;
        const float rstd = 1.0f / sqrtf(var + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (t + i * T >= p.nvec) continue;
            float wf[8], bf[8], o[8];
            unpack_bf16(w[i], wf);
            unpack_bf16(b[i], bf);
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = fmaf(v[i][k] * rstd, wf[k], bf[k]);
            static_cast<uint4 *>(p.out)[row * p.nvec + t + i * T] = pack_bf16(o);
        }
        if (t == 0 && p.mean) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
        }
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
    float inv_c;
};

template <bool F32, int T, int NV>
__global__ void __launch_bounds__(kNormThreads<T>)
layernorm_backward_kernel(const NormBackward p)
{
    extern __shared__ float4 norm_smem[];  // T == 32: the warps' sums, [8][2 C]
    __shared__ float2 slots[2][T / 32];
    chained_start();
    const int t = static_cast<int>(threadIdx.x) % T;
    constexpr int TEAMS = kNormThreads<T> / T;
    const long long stride = static_cast<long long>(gridDim.x) * TEAMS;
    long long row = static_cast<long long>(blockIdx.x) * TEAMS + threadIdx.x / T;
    const bool has_res = p.dres != nullptr;
    uint4 dy[NV], w[NV];
    Raw8<F32> x[NV], res[NV];
    float mean = 0.0f, rstd = 0.0f;
    float dw[NV][8], db[NV][8];
    auto load = [&](long long r) {
        mean = __ldcg(p.mean + r);
        rstd = __ldcg(p.rstd + r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            if (j < p.nvec) {
                dy[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.dout) + r * p.nvec + j);
                x[i] = load8<F32>(p.inp, r * p.nvec + j);
                if (has_res) res[i] = load8<F32>(p.dres, r * p.nvec + j);
            }
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        dy[i] = w[i] = make_uint4(0, 0, 0, 0);
        x[i] = res[i] = Raw8<F32>{};
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[i][k] = db[i][k] = 0.0f;
    }
    if (row < p.BT) load(row);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * T < p.nvec) w[i] = ptx::ld_global_v4(static_cast<const uint4 *>(p.weight) + t + i * T);
    int turn = 0;
    for (; row < p.BT; row += stride) {
        float xh[NV][8], g[NV][8];
        float2 s = make_float2(0.0f, 0.0f);
        const float rs = rstd;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float wf[8], d[8];
            unpack8<F32>(x[i], xh[i]);
            unpack_bf16(dy[i], d);
            unpack_bf16(w[i], wf);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                xh[i][k] = (xh[i][k] - mean) * rs;
                g[i][k] = d[k] * wf[k];
                // vectors past the end of the row: d = 0 and g = 0, so they add nothing to any sum
                dw[i][k] = fmaf(d[k], xh[i][k], dw[i][k]);
                db[i][k] += d[k];
                s.x += g[i][k];
                s.y = fmaf(g[i][k], xh[i][k], s.y);
            }
        }
        Raw8<F32> cur[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) cur[i] = res[i];
        if (row + stride < p.BT) load(row + stride);
        s = team_sum<T>(s, slots, turn++);
        const float c1 = s.x * p.inv_c, c2 = s.y * p.inv_c;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + i * T;
            if (j >= p.nvec) continue;
            float o[8];
            unpack8<F32>(cur[i], o);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float dx = rs * (g[i][k] - c1 - xh[i][k] * c2);
                o[k] = has_res ? dx + o[k] : dx;
            }
            store8<F32>(p.dinp, row * p.nvec + j, pack8<F32>(o));
            if (p.dbranch) static_cast<uint4 *>(p.dbranch)[row * p.nvec + j] = pack_bf16(o);
        }
    }
    if (p.part == nullptr) return;
    float4 *part = reinterpret_cast<float4 *>(p.part) + static_cast<long long>(blockIdx.x) * 4 * p.nvec;
    float4 *mine = T == 32 ? norm_smem + (threadIdx.x / 32) * 4 * p.nvec : part;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = t + i * T;
        if (j >= p.nvec) continue;
        mine[2 * j] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
        mine[2 * j + 1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
        mine[2 * p.nvec + 2 * j] = make_float4(db[i][0], db[i][1], db[i][2], db[i][3]);
        mine[2 * p.nvec + 2 * j + 1] = make_float4(db[i][4], db[i][5], db[i][6], db[i][7]);
    }
    if constexpr (T == 32) {
        __syncthreads();
        for (int c = threadIdx.x; c < 4 * p.nvec; c += 256) {
            float4 a = norm_smem[c];
#pragma unroll
            for (int k = 1; k < 8; ++k) {
                const float4 v = norm_smem[k * 4 * p.nvec + c];
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
// first. A block owns 32 columns of [dweight | dbias], a warp every eighth part; they meet in shared memory.
__global__ void __launch_bounds__(256)
layernorm_reduce_kernel(float *dweight, float *dbias, const float *part, int parts, int C, int accumulate)
{
    __shared__ float s[8][32];
    chained_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float a = 0.0f;
    if (c < 2 * C) {
        int k = warp;
        for (; k + 24 < parts; k += 32) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __ldcg(part + (k + 8ll * i) * 2 * C + c);
            a += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; k < parts; k += 8) a += __ldcg(part + static_cast<long long>(k) * 2 * C + c);
    }
    s[warp][lane] = a;
    __syncthreads();
    if (warp == 0 && c < 2 * C) {
        float *dst = c < C ? dweight + c : dbias + (c - C);
        if ((c < C ? dweight : dbias) == nullptr) return;
#pragma unroll
        for (int k = 1; k < 8; ++k) a += s[k][lane];
        *dst = accumulate ? *dst + a : a;
    }
}

}  // namespace nb
