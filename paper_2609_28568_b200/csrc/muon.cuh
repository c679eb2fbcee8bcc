// The elementwise ends of the weight update by orthogonalised momentum: what is read ahead of the products, and the
// application of their result. Many matrices of one shape per launch: blockIdx.y is the matrix. Links of the
// dependent-launch chain.
#pragma once
#include <cuda_fp16.h>

#include "elementwise.cuh"

namespace nb {

constexpr int kMuonCountPitch = 32;  // words between the counts of two matrices: a line of L2 each
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
// or m, and |v|^2 per matrix. Squares are summed in 64 bits, which hold those of every fp32 value: the norm of a gradient of 1e-30 or
// 1e30 is as exact as any other's. In a fixed order: one partial sum per block, added up by whoever needs the norm.
struct MuonPrepare {
    const void *grad[kMuonBatch];  // fp32 or bf16
    float *momentum[kMuonBatch];   // or all null
    void *out[kMuonBatch];         // muon_normalise_kernel with no step to follow: bf16 results
    double *part;                  // [n][parts]
    unsigned *done;                // [n + 1], zeroed: the products' counts, and the word that says that one of their blocks failed
    __half *x;                     // [n][rows][8 pitch], times `scale`
    long long nvec;                // elements / 8
    int row_vec, pitch;            // vectors of eight in a row, and from one row of x to the next
    int parts;
    int nesterov;
    float mu, scale;
    double eps;
};

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

// v of vector i, from the gradient's and the momentum's eight values as they were loaded.
template <bool G32>
struct MuonVec {
    float4 m[2];
    uint4 g[G32 ? 2 : 1];
    __device__ __forceinline__ void load_grad(const void *grad, long long i)
    {
        g[0] = ptx::ld_global_v4(static_cast<const uint4 *>(grad) + i * (G32 ? 2 : 1));
        if constexpr (G32) g[1] = ptx::ld_global_v4(static_cast<const uint4 *>(grad) + i * 2 + 1);
    }
    __device__ __forceinline__ void load_momentum(const float *mom, long long i)
    {
        m[0] = ptx::ld_global_f32x4(mom + 8 * i);
        m[1] = ptx::ld_global_f32x4(mom + 8 * i + 4);
    }
    __device__ __forceinline__ void momentum(float (&v)[8]) const
    {
        v[0] = m[0].x, v[1] = m[0].y, v[2] = m[0].z, v[3] = m[0].w, v[4] = m[1].x, v[5] = m[1].y, v[6] = m[1].z, v[7] = m[1].w;
    }
    __device__ __forceinline__ void grad(float (&v)[8]) const
    {
        if constexpr (G32) {
            const uint32_t w[8] = {g[0].x, g[0].y, g[0].z, g[0].w, g[1].x, g[1].y, g[1].z, g[1].w};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[k]);
        } else {
            const uint32_t w[4] = {g[0].x, g[0].y, g[0].z, g[0].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = ptx::bf16_lo(w[k]);
                v[2 * k + 1] = ptx::bf16_hi(w[k]);
            }
        }
    }
};
constexpr int kMuonUnroll = 2;  // vectors of a thread under way at once

template <bool G32>
__global__ void __launch_bounds__(256)
muon_momentum_kernel(const __grid_constant__ MuonPrepare p)
{
    chained_start();
    const void *grad = p.grad[blockIdx.y];
    float *mom = p.momentum[blockIdx.y];
    double sq = 0.0;
    const long long stride = 256ll * gridDim.x;
    for (long long i0 = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i0 < p.nvec; i0 += kMuonUnroll * stride) {
        MuonVec<G32> x[kMuonUnroll];
#pragma unroll
        for (int h = 0; h < kMuonUnroll; ++h) {
            const long long i = i0 + h * stride;
            if (i >= p.nvec) continue;
            x[h].load_grad(grad, i);
            if (mom) x[h].load_momentum(mom, i);
        }
#pragma unroll
        for (int h = 0; h < kMuonUnroll; ++h) {
            const long long i = i0 + h * stride;
            if (i >= p.nvec) continue;
            float v[8];
            x[h].grad(v);
            if (mom) {
                float m[8];
                x[h].momentum(m);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    m[k] = fmaf(p.mu, m[k], v[k]);
                    v[k] = p.nesterov ? fmaf(p.mu, m[k], v[k]) : m[k];
                }
                float4 *dst = reinterpret_cast<float4 *>(mom + 8 * i);
                dst[0] = make_float4(m[0], m[1], m[2], m[3]);
                dst[1] = make_float4(m[4], m[5], m[6], m[7]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sq = fma(static_cast<double>(v[k]), static_cast<double>(v[k]), sq);
        }
    }
    sq = block_sum_256(sq);
    if (threadIdx.x == 0) {
        p.part[static_cast<long long>(blockIdx.y) * p.parts + blockIdx.x] = sq;
        if (blockIdx.x == 0) p.done[blockIdx.y * kMuonCountPitch] = 0;
        if (blockIdx.x == 0 && blockIdx.y == 0) p.done[gridDim.y * kMuonCountPitch] = 0;
    }
}

// x = fp16(scale v / (|v| + eps)); v from the momentum as the launch before left it. The division is by a 64-bit factor, so that it neither
// overflows nor vanishes for gradients at either end of fp32. The scale is fixed: where eps exceeds |v| by so much that the values of x come below
// 2^-14 / scale, fp16 holds them to 2^-25 / scale and no closer.
template <bool G32, bool LAST>
__global__ void __launch_bounds__(256)
muon_normalise_kernel(const __grid_constant__ MuonPrepare p)
{
    chained_start();
    const void *grad = p.grad[blockIdx.y];
    const float *mom = p.momentum[blockIdx.y];
    const bool with_grad = !mom || p.nesterov;
    const long long stride = 256ll * gridDim.x;
    double f = 0.0;
    uint4 *dst = LAST ? static_cast<uint4 *>(p.out[blockIdx.y])
                      : reinterpret_cast<uint4 *>(p.x) + static_cast<long long>(blockIdx.y) * (p.nvec / p.row_vec) * p.pitch;
    const double *part = p.part + static_cast<long long>(blockIdx.y) * p.parts;
    const double share = static_cast<int>(threadIdx.x) < p.parts ? __ldcg(part + threadIdx.x) : 0.0;
    bool first = true;
    const long long start = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    // every thread goes through the first round: the norm is added up while its values are on their way
    for (long long i0 = start; first || i0 < p.nvec; i0 += kMuonUnroll * stride) {
        MuonVec<G32> x[kMuonUnroll];
#pragma unroll
        for (int h = 0; h < kMuonUnroll; ++h) {
            const long long i = i0 + h * stride;
            if (i >= p.nvec) continue;
            if (with_grad) x[h].load_grad(grad, i);
            if (mom) x[h].load_momentum(mom, i);
        }
        if (first) {
            f = static_cast<double>(LAST ? 1.0f : p.scale) / (sqrt(block_sum_256(share)) + p.eps);
            first = false;
        }
#pragma unroll
        for (int h = 0; h < kMuonUnroll; ++h) {
            const long long i = i0 + h * stride;
            if (i >= p.nvec) continue;
            float v[8];
            if (with_grad) x[h].grad(v);
            if (mom) {
                float m[8];
                x[h].momentum(m);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = p.nesterov ? fmaf(p.mu, m[k], v[k]) : m[k];
            }
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float lo = static_cast<float>(static_cast<double>(v[2 * k]) * f);
                const float hi = static_cast<float>(static_cast<double>(v[2 * k + 1]) * f);
                if constexpr (LAST) {
                    w[k] = ptx::pack_bf16x2(lo, hi);
                } else {
                    const __half2 h2 = __floats2half2_rn(lo, hi);
                    w[k] = *reinterpret_cast<const uint32_t *>(&h2);
                }
            }
            const uint32_t row = static_cast<uint32_t>(i) / static_cast<uint32_t>(p.row_vec);  // i is below 2^27
            const long long to = LAST ? i : i + static_cast<long long>(row) * (p.pitch - p.row_vec);
            dst[to] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

}  // namespace nb
