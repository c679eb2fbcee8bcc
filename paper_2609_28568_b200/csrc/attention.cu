// The attention kernels, in a translation unit of their own; nb_linear.cu checks arguments and launches them.
#include "attention.h"

#include "attention_backward_sm100.cuh"
#include "attention_forward_sm100.cuh"

namespace nb {

template <class Cfg>
static AttnKernel forward_kernel()
{
    return {reinterpret_cast<const void *>(&attn_forward_kernel<Cfg>), Cfg::THREADS, Cfg::SMEM, 128, Cfg::KEYS};
}
AttnKernel attn_forward(int D) { return D <= 64 ? forward_kernel<AttnFwdCfg<64>>() : forward_kernel<AttnFwdCfg<128>>(); }
AttnKernel attn_backward_q(int D)
{
    if (D <= 64) return {reinterpret_cast<const void *>(&attn_backward_q_kernel<64>), kAttnThreads, AttnBwdCfg<64>::SMEM_Q, 128, 128};
    return {reinterpret_cast<const void *>(&attn_backward_q_kernel<128>), kAttnThreads, AttnBwdCfg<128>::SMEM_Q, 128, 128};
}
AttnKernel attn_backward_kv(int D)
{
    if (D <= 64) return {reinterpret_cast<const void *>(&attn_backward_kv_kernel<64>), kAttnThreads, AttnBwdCfg<64>::SMEM_KV, 128, 128};
    return {reinterpret_cast<const void *>(&attn_backward_kv_kernel<128>), kAttnThreads, AttnBwdCfg<128>::SMEM_KV, 128, 128};
}

}  // namespace nb
