// What nb_linear.cu launches of attention.cu.
#pragma once
#include <stdint.h>

namespace nb {

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
    int withhold;            // nb_debug_attention_timeout only: bytes that a tile of the ring waits for beyond what its copies bring
};

struct AttnBackward {
    AttnParams a;            // a.out: the forward pass's output, a.ld_out its ld; a.lse: read
    float *delta;            // [heads, T]: sum over a row of dout out, written by the pass of dq, read by that of dk and dv
    const void *dout;
    void *dq, *dk, *dv;
    long long ld_dout, ld_dq, ld_dk, ld_dv;
};

// A kernel for heads of D columns, its threads, its dynamic shared memory, the rows of a block and those of the tiles that it walks over. Parameters: its tensor maps (forward: q, k, v), then AttnParams or AttnBackward.
struct AttnKernel {
    const void *fn;
    int threads;
    uint32_t smem;
    int rows, streamed;
};
AttnKernel attn_forward(int D);
AttnKernel attn_backward_q(int D);   // maps: q, dout, k, v
AttnKernel attn_backward_kv(int D);  // the same

}  // namespace nb
