// The elementwise ends of the weight update by orthogonalised momentum: what is read ahead of the products, and the
// application of their result. Many matrices of one shape per launch: blockIdx.y is the matrix. Links of the
// dependent-launch chain.
#pragma once
#include <cuda_fp16.h>

#include "elementwise.cuh"

namespace nb {

constexpr int kMuonBatch = 32;  // matrices per launch: their addresses are kernel parameters

struct MuonApply {
    float *master[kMuonBatch];
    void *weight[kMuonBatch];  // bf16, or all null
    const void *update[kMuonBatch];
    long long count;
    float decay, step;
};

__device__ __forceinline__ float muon_apply_one(float m, float u, float decay, float step)
{
    return fmaf(-step, u, decay * m);
}

// master <- decay master - step update, weight <- bf16(master); 12 bytes per element, bound by HBM. Two vectors of eight per thread are in
// flight at a time.
__global__ void __launch_bounds__(256)
muon_apply_kernel(const __grid_constant__ MuonApply p)
{
    chained_start();
    float *master = p.master[blockIdx.y];
    uint4 *weight = static_cast<uint4 *>(p.weight[blockIdx.y]);
    const uint4 *update = static_cast<const uint4 *>(p.update[blockIdx.y]);
    const long long nvec = p.count / 8;
    const long long stride = static_cast<long long>(gridDim.x) * 256;
    const long long t0 = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    for (long long i0 = t0; i0 < nvec; i0 += 2 * stride) {
        float4 m[2][2];
        uint4 u[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long long i = i0 + h * stride;
            if (i >= nvec) continue;
            m[h][0] = ptx::ld_global_f32x4(master + 8 * i);
            m[h][1] = ptx::ld_global_f32x4(master + 8 * i + 4);
            u[h] = ptx::ld_global_v4(update + i);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long long i = i0 + h * stride;
            if (i >= nvec) continue;
            const uint32_t uw[4] = {u[h].x, u[h].y, u[h].z, u[h].w};
            float o[8] = {m[h][0].x, m[h][0].y, m[h][0].z, m[h][0].w, m[h][1].x, m[h][1].y, m[h][1].z, m[h][1].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                o[2 * k] = muon_apply_one(o[2 * k], ptx::bf16_lo(uw[k]), p.decay, p.step);
                o[2 * k + 1] = muon_apply_one(o[2 * k + 1], ptx::bf16_hi(uw[k]), p.decay, p.step);
            }
            float4 *d = reinterpret_cast<float4 *>(master + 8 * i);
            d[0] = make_float4(o[0], o[1], o[2], o[3]);
            d[1] = make_float4(o[4], o[5], o[6], o[7]);
            if (weight)
                weight[i] = make_uint4(ptx::pack_bf16x2(o[0], o[1]), ptx::pack_bf16x2(o[2], o[3]),
                                       ptx::pack_bf16x2(o[4], o[5]), ptx::pack_bf16x2(o[6], o[7]));
        }
    }
    const long long i = nvec * 8 + t0;  // at most seven elements
    if (i < p.count) {
        const float u = __uint_as_float(ptx::ld_global_u16(reinterpret_cast<const unsigned short *>(update) + i) << 16);
        const float o = muon_apply_one(master[i], u, p.decay, p.step);
        master[i] = o;
        if (weight) reinterpret_cast<__nv_bfloat16 *>(weight)[i] = __float2bfloat16_rn(o);
    }
}

// What comes ahead of the products: m <- mu m + g (fp32, in place; without momentum the gradient itself is taken), v = g + mu m (nesterov)
// or m, and |v|^2 per matrix. Squares are summed in 64 bits, which hold those of every fp32 value: a gradient of
// 1e-30 or 1e30 is normalised like any other. In a fixed order: one partial sum per block, added up by whoever needs the norm.
struct MuonPrepare {
    const void *grad[kMuonBatch];  // fp32 or bf16
    float *momentum[kMuonBatch];   // or all null
    void *out[kMuonBatch];         // muon_normalise_kernel with no step to follow: bf16 results
    double *part;                  // [n][parts]
    unsigned *done;                // [n], zeroed for the products' counts
    __half *x;                     // [n][count], times `scale`
    long long nvec;                // elements / 8
    int parts;
    int nesterov;
    float mu, scale;
    double eps;
};

template <bool G32>
__device__ __forceinline__ void muon_load_grad(const void *grad, long long i, float (&g)[8])
{
    if constexpr (G32) {
        const float4 a = ptx::ld_global_f32x4(static_cast<const float4 *>(grad) + 2 * i);
        const float4 b = ptx::ld_global_f32x4(static_cast<const float4 *>(grad) + 2 * i + 1);
        g[0] = a.x, g[1] = a.y, g[2] = a.z, g[3] = a.w, g[4] = b.x, g[5] = b.y, g[6] = b.z, g[7] = b.w;
    } else {
        const uint4 a = ptx::ld_global_v4(static_cast<const uint4 *>(grad) + i);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            g[2 * k] = ptx::bf16_lo(w[k]);
            g[2 * k + 1] = ptx::bf16_hi(w[k]);
        }
    }
}
// Sum over the block's 256 threads, in a fixed order; every thread gets it.
__device__ __forceinline__ double block_sum_256(double v)
{
    __shared__ double s[8];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
}

template <bool G32>
__global__ void __launch_bounds__(256)
muon_momentum_kernel(const __grid_constant__ MuonPrepare p)
{
    chained_start();
    const void *grad = p.grad[blockIdx.y];
    float *mom = p.momentum[blockIdx.y];
    double sq = 0.0;
    for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < p.nvec; i += 256ll * gridDim.x) {
        float v[8];
        if (mom) {
            float4 m0 = ptx::ld_global_f32x4(mom + 8 * i), m1 = ptx::ld_global_f32x4(mom + 8 * i + 4);
            muon_load_grad<G32>(grad, i, v);
            float m[8] = {m0.x, m0.y, m0.z, m0.w, m1.x, m1.y, m1.z, m1.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                m[k] = fmaf(p.mu, m[k], v[k]);
                v[k] = p.nesterov ? fmaf(p.mu, m[k], v[k]) : m[k];
            }
            float4 *dst = reinterpret_cast<float4 *>(mom + 8 * i);
            dst[0] = make_float4(m[0], m[1], m[2], m[3]);
            dst[1] = make_float4(m[4], m[5], m[6], m[7]);
        } else {
            muon_load_grad<G32>(grad, i, v);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sq = fma(static_cast<double>(v[k]), static_cast<double>(v[k]), sq);
    }
    sq = block_sum_256(sq);
    if (threadIdx.x == 0) {
        p.part[static_cast<long long>(blockIdx.y) * p.parts + blockIdx.x] = sq;
        if (blockIdx.x == 0) p.done[blockIdx.y] = 0;
    }
}

// x = fp16(scale v / (|v| + eps)); v from the momentum as the launch before left it. The division is by a 64-bit factor, so that it neither
// overflows nor vanishes for gradients at either end of fp32.
template <bool G32, bool LAST>
__global__ void __launch_bounds__(256)
muon_normalise_kernel(const __grid_constant__ MuonPrepare p)
{
    chained_start();
    const void *grad = p.grad[blockIdx.y];
    const float *mom = p.momentum[blockIdx.y];
    const double *part = p.part + static_cast<long long>(blockIdx.y) * p.parts;
    const double sq = block_sum_256(static_cast<int>(threadIdx.x) < p.parts ? __ldcg(part + threadIdx.x) : 0.0);
    const double f = static_cast<double>(LAST ? 1.0f : p.scale) / (sqrt(sq) + p.eps);
    uint4 *dst = LAST ? static_cast<uint4 *>(p.out[blockIdx.y])
                      : reinterpret_cast<uint4 *>(p.x) + static_cast<long long>(blockIdx.y) * p.nvec;
    for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < p.nvec; i += 256ll * gridDim.x) {
        float v[8];
        if (mom) {
            const float4 m0 = ptx::ld_global_f32x4(mom + 8 * i), m1 = ptx::ld_global_f32x4(mom + 8 * i + 4);
            const float m[8] = {m0.x, m0.y, m0.z, m0.w, m1.x, m1.y, m1.z, m1.w};
            if (p.nesterov) muon_load_grad<G32>(grad, i, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p.nesterov ? fmaf(p.mu, m[k], v[k]) : m[k];
        } else {
            muon_load_grad<G32>(grad, i, v);
        }
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float lo = static_cast<float>(static_cast<double>(v[2 * k]) * f);
            const float hi = static_cast<float>(static_cast<double>(v[2 * k + 1]) * f);
            if constexpr (LAST) {
                w[k] = ptx::pack_bf16x2(lo, hi);
            } else {
                const __half2 h = __floats2half2_rn(lo, hi);
                w[k] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

}  // namespace nb
