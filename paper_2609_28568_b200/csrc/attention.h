// What nb_linear.cu launches of attention.cu.
#pragma once
#include <stdint.h>

namespace nb {

constexpr int kAttnTile = 128;
constexpr int kAttnThreads = 384;  // two warpgroups on scores, warp 8: loads, warp 9: products
constexpr int kStatusBadSequences = 6;

struct AttnParams {
    int T, n, heads, group;  // group: queries' heads per head of keys
    int D;
    int causal;
    const int *cu;           // [n + 1] or null: T / n rows each
    float scale;
    long long ld_out;        // elements between rows of what threads store (forward: out)
    void *out;
    float *lse;              // [heads, T]; forward: or null
    int *status;
    unsigned long long timeout_ns;
};

// A kernel for heads of D columns and its dynamic shared memory. Parameters: its tensor maps, then AttnParams.
struct AttnKernel {
    const void *fn;
    uint32_t smem;
};
AttnKernel attn_forward(int D);

}  // namespace nb
