// The attention kernels, in a translation unit of their own; nb_linear.cu checks arguments and launches them.
#include "attention.h"

#include "attention_backward_sm100.cuh"
#include "attention_forward_sm100.cuh"

namespace nb {

AttnKernel attn_forward(int D)
{
    if (D <= 64) return {reinterpret_cast<const void *>(&attn_forward_kernel<64>), AttnFwdCfg<64>::SMEM};
    return {reinterpret_cast<const void *>(&attn_forward_kernel<128>), AttnFwdCfg<128>::SMEM};
}

AttnKernel attn_backward_q(int D)
{
    if (D <= 64) return {reinterpret_cast<const void *>(&attn_backward_q_kernel<64>), AttnBwdCfg<64>::SMEM_Q};
    return {reinterpret_cast<const void *>(&attn_backward_q_kernel<128>), AttnBwdCfg<128>::SMEM_Q};
}
AttnKernel attn_backward_kv(int D)
{
    if (D <= 64) return {reinterpret_cast<const void *>(&attn_backward_kv_kernel<64>), AttnBwdCfg<64>::SMEM_KV};
    return {reinterpret_cast<const void *>(&attn_backward_kv_kernel<128>), AttnBwdCfg<128>::SMEM_KV};
}

}  // namespace nb
