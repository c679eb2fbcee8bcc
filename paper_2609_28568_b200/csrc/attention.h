// What nb_linear.cu launches of attention.cu.
#pragma once
#include <stdint.h>

namespace nb {

constexpr int kStatusBadSequences = 6;
constexpr int kAttnFirst = 1, kAttnSecond = 2;  // AttnBackward::side

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
    int parts;               // blocks of an item's cluster, which share its tiles (1: a block to an item)
    int withhold;            // nb_debug_attention_timeout only: bytes that a tile of the ring waits for beyond what its copies bring
};

struct AttnBackward {
    AttnParams a;            // a.out: the forward pass's output, a.ld_out its ld; a.lse: read
    float *delta;            // [heads, T]: sum over a row of dout out, for the pass of dk and dv (side by side: for both)
    int side;                // 0, or the pass's place among two that run side by side: delta is there before either of them
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
AttnKernel attn_forward(int D, bool split);
AttnKernel attn_backward_delta(int D);         // no maps; a block has `rows` of all rows of all heads, fewer than 2^31
AttnKernel attn_backward_q(int D, bool few, bool split);   // maps: q, dout, k, v; few: a block to an SM in place of two (D <= 64); split: few too
AttnKernel attn_backward_kv(int D, bool few, bool split);  // the same

}  // namespace nb
