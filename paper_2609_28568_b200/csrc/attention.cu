// The attention kernels, in a translation unit of their own; nb_linear.cu checks arguments and launches them.
#include "attention.h"

#include "attention_forward_sm100.cuh"

namespace nb {

AttnKernel attn_forward(int D)
{
    if (D <= 64) return {reinterpret_cast<const void *>(&attn_forward_kernel<64>), AttnFwdCfg<64>::SMEM};
    return {reinterpret_cast<const void *>(&attn_forward_kernel<128>), AttnFwdCfg<128>::SMEM};
}

}  // namespace nb
