// The attention kernels, in a translation unit of their own; nb_linear.cu checks arguments and launches them.
#include "attention.h"

#include "attention_backward_sm100.cuh"
#include "attention_forward_sm100.cuh"

namespace nb {

template <class Cfg, bool SPLIT>
static AttnKernel forward_kernel()
{
    return {reinterpret_cast<const void *>(&attn_forward_kernel<Cfg, SPLIT>), Cfg::THREADS, Cfg::SMEM, 128, Cfg::KEYS};
}
AttnKernel attn_forward(int D, bool split)
{
    if (split) return D <= 64 ? forward_kernel<AttnFwdCfg<64>, true>() : forward_kernel<AttnFwdCfg<128>, true>();
    return D <= 64 ? forward_kernel<AttnFwdCfg<64>, false>() : forward_kernel<AttnFwdCfg<128>, false>();
}
template <class Cfg, bool SPLIT>
static AttnKernel backward_q_kernel()
{
    return {reinterpret_cast<const void *>(&attn_backward_q_kernel<Cfg, SPLIT>), Cfg::THREADS, Cfg::SMEM, 128, Cfg::ROWS};
}
template <class Cfg, bool SPLIT>
static AttnKernel backward_kv_kernel()
{
    return {reinterpret_cast<const void *>(&attn_backward_kv_kernel<Cfg, SPLIT>), Cfg::THREADS, Cfg::SMEM, 128, Cfg::ROWS};
}
AttnKernel attn_backward_delta(int D)
{
    return {reinterpret_cast<const void *>(D <= 64 ? &attn_backward_delta_kernel<64> : &attn_backward_delta_kernel<128>), 256, 0, 256 / (D <= 64 ? 8 : 16), 0};
}
AttnKernel attn_backward_q(int D, bool few, bool split)
{
    if (split) return D > 64 ? backward_q_kernel<AttnBwdCfg<128, 2>, true>() : backward_q_kernel<AttnBwdCfg<64, 2>, true>();
    return D > 64 ? backward_q_kernel<AttnBwdCfg<128, 2>, false>() : few ? backward_q_kernel<AttnBwdCfg<64, 2>, false>() : backward_q_kernel<AttnBwdCfg<64, 1>, false>();
}
AttnKernel attn_backward_kv(int D, bool few, bool split)
{
    if (split) return D > 64 ? backward_kv_kernel<AttnBwdCfg<128, 2>, true>() : backward_kv_kernel<AttnBwdCfg<64, 2>, true>();
    return D > 64 ? backward_kv_kernel<AttnBwdCfg<128, 2>, false>() : few ? backward_kv_kernel<AttnBwdCfg<64, 2>, false>() : backward_kv_kernel<AttnBwdCfg<64, 1>, false>();
}

}  // namespace nb
