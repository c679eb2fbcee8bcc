// The elementwise ends of the weight update by orthogonalised momentum: what is read ahead of the products, and the
// application of their result. Many matrices of one shape per launch: blockIdx.y is the matrix. Links of the
// dependent-launch chain.
#pragma once
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

}  // namespace nb
