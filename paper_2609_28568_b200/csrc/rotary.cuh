// Rotary positions: pairs (a, b) of a head's first R columns are turned by an angle that grows with the token's position,
//
//   a' = s (a cos t - b sin t)    b' = s (b cos t + a sin t)    t = position * freq_j    (inverse: -t)
//
// with the pairs (j, j + R / 2) or (2 j, 2 j + 1). The angle is formed in 64 bits in units of a turn and whole turns are taken off before it is
// rounded to fp32, so that far positions are as exact as near ones (a rounded product of 32 bits would be off by 2e-3 radians at position 32768).
// Bound by HBM: every element is read and written once (16384 rows, 24 heads of 128: 36 us, 5.6 TB/s; 85 % of a copy's rate). A block takes some tokens at a time: their cosines and sines are formed once, in shared
// memory, for all heads; then its threads walk the tokens' vectors of eight elements.
#pragma once
#include "attention.h"
#include "elementwise.cuh"

namespace nb {

constexpr int kRotaryThreads = 256;
constexpr int kRotaryMaxPairs = 64;  // R / 2
constexpr int kRotaryTokens = 8;     // of a block at a time

struct RotaryParams {
    const void *in[2];  // queries, keys (or null)
    void *out[2];
    long long ld_in[2], ld_out[2];
    int heads[2];
    int T, n, D, R;
    float scale, sign;     // sign -1: inverse
    const double *freq;    // radians per position, R / 2 of them
    const int *positions;  // [T] or null
    const int *cu;         // [n + 1] or null: n sequences of T / n
    int *status;
};

// The position of a row, if it is in a sequence. The search stays within [0, n] whatever cu holds.
__device__ __forceinline__ int rotary_position(const RotaryParams &p, int row, bool &in_sequence)
{
    in_sequence = p.cu == nullptr || (p.cu[0] <= row && p.cu[p.n] > row);
    if (!in_sequence) return 0;
    if (p.positions) return p.positions[row];
    if (p.cu == nullptr) return row % (p.T / p.n);
    int lo = 0, hi = p.n;  // the last i with cu[i] <= row lies in [lo, hi)
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (p.cu[mid] <= row) lo = mid;
        else hi = mid;
    }
    return row - max(p.cu[lo], 0);
}

// One thread's piece of a head: two vectors of eight that hold eight pairs, or, where the columns are no multiples of 16, one that holds four or is only copied. (Pieces of two
// where they are: 16384 rows of 12 heads of 80, 32 columns turned: 16.2 us, of one 18.4; 8192 of 24 of 128, 64 turned: 20.6, 25.0.)
struct RotaryItem {
    uint4 a, b;
    __nv_bfloat16 *out;  // null: it stays as it is
};

// TWO: pieces that are copied or hold neighbours are of two vectors (where the numbers of columns allow it)
template <bool HALF, bool TWO>
__global__ void __launch_bounds__(kRotaryThreads, 5)
rotary_kernel(const RotaryParams p, int tokens)
{
    // (cos, sin) of a token's pairs, two to a piece of 16 bytes; piece u stands at u ^ (u >> 3), so that eight threads that read theirs of
    // 64 or 32 bytes meet no bank twice
    __shared__ __align__(16) float2 turn[kRotaryTokens][kRotaryMaxPairs];
    __shared__ int position[kRotaryTokens];
    __shared__ bool in_sequence[kRotaryTokens];
    chained_start();
    const int tid = static_cast<int>(threadIdx.x);
    const int row0 = static_cast<int>(blockIdx.x) * tokens, count = min(tokens, p.T - row0);
    const int pairs = p.R / 2, H = p.heads[0] + p.heads[1];
    // pieces of a head: a thread keeps its own, and walks the heads of the block's tokens with the others that have the same
    constexpr int vectors = TWO ? 2 : 1;
    const int turned = p.R / (HALF ? 16 : 8 * vectors), per = turned + (p.D - p.R) / (8 * vectors);
    const int it = tid % per, stride = kRotaryThreads / per;
    const bool turns = it < turned;
    const int col = HALF && turns ? it * 8 : turns ? it * 8 * vectors : p.R + (it - turned) * 8 * vectors;
    const int second = HALF && turns ? pairs : TWO ? 8 : 0;  // columns from the first vector to the second; 0: there is none
    int tok = 0, h = tid / per;
    bool more = h < stride;
    auto settle = [&] {
        while (h >= H) {
            h -= H;
            ++tok;
        }
        more = more && tok < count;
    };
    auto load = [&](RotaryItem &x) {
        const int t = h < p.heads[0] ? 0 : 1, hh = t ? h - p.heads[0] : h;
        const long long row = row0 + tok;
        const auto *in = static_cast<const __nv_bfloat16 *>(t ? p.in[1] : p.in[0]) + row * (t ? p.ld_in[1] : p.ld_in[0]) + hh * p.D + col;
        x.out = static_cast<__nv_bfloat16 *>(t ? p.out[1] : p.out[0]) + row * (t ? p.ld_out[1] : p.ld_out[0]) + hh * p.D + col;
        if (!turns && in == x.out) x.out = nullptr;
        if (TWO && !x.out) return;
        x.a = ptx::ld_global_v4(in);
        if (second) x.b = ptx::ld_global_v4(in + second);
    };
    RotaryItem x;
    settle();
    if (more) load(x);  // under way while the angles are formed

    if (tid < count) {
        bool in;
        position[tid] = rotary_position(p, row0 + tid, in);
        in_sequence[tid] = in;
    }
    if (blockIdx.x == 0 && p.cu)  // reported, not relied on
        for (int i = tid; i <= p.n; i += kRotaryThreads)
            if (p.cu[i] < (i ? p.cu[i - 1] : 0) || p.cu[i] > p.T)
                if (atomicCAS(p.status, 0, kStatusBadSequences) == 0) p.status[1] = i;
    __syncthreads();
    for (int i = tid; i < count * pairs; i += kRotaryThreads) {
        const int t = i / pairs, j = i - t * pairs;
        double turned_by = position[t] * (p.freq[j] * 0.15915494309189535);  // whole turns and a part, 1 / (2 pi)
        turned_by -= rint(turned_by);
        float sn, cs;
        sincospif(static_cast<float>(2.0 * turned_by), &sn, &cs);
        const int u = j >> 1;
        turn[t][((u ^ (u >> 3)) << 1) | (j & 1)] = make_float2(cs * p.scale, sn * p.scale * p.sign);
    }
    __syncthreads();

    while (more) {
        const int now = tok;
        RotaryItem y = x;
        h += stride;
        settle();
        if (more) load(x);
        if (!in_sequence[now] || !y.out) continue;
        if (!turns) {
            *reinterpret_cast<uint4 *>(y.out) = y.a;
            if (TWO) *reinterpret_cast<uint4 *>(y.out + 8) = y.b;
            continue;
        }
        const uint32_t a[4] = {y.a.x, y.a.y, y.a.z, y.a.w}, b[4] = {y.b.x, y.b.y, y.b.z, y.b.w};
        uint32_t oa[4], ob[4];
        const float4 *cs = reinterpret_cast<const float4 *>(turn[now]);
        if constexpr (HALF) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int u = 4 * it + k;
                const float4 c = cs[u ^ (u >> 3)];
                const float a0 = ptx::bf16_lo(a[k]), a1 = ptx::bf16_hi(a[k]), b0 = ptx::bf16_lo(b[k]), b1 = ptx::bf16_hi(b[k]);
                oa[k] = ptx::pack_bf16x2(a0 * c.x - b0 * c.y, a1 * c.z - b1 * c.w);
                ob[k] = ptx::pack_bf16x2(b0 * c.x + a0 * c.y, b1 * c.z + a1 * c.w);
            }
            *reinterpret_cast<uint4 *>(y.out) = make_uint4(oa[0], oa[1], oa[2], oa[3]);
            *reinterpret_cast<uint4 *>(y.out + pairs) = make_uint4(ob[0], ob[1], ob[2], ob[3]);
        } else {
            auto turn4 = [&](const uint32_t *v, uint32_t *o, int first) {
#pragma unroll
                for (int k = 0; k < 4; k += 2) {
                    const int u = first + (k >> 1);
                    const float4 c = cs[u ^ (u >> 3)];
                    const float a0 = ptx::bf16_lo(v[k]), b0 = ptx::bf16_hi(v[k]), a1 = ptx::bf16_lo(v[k + 1]), b1 = ptx::bf16_hi(v[k + 1]);
                    o[k] = ptx::pack_bf16x2(a0 * c.x - b0 * c.y, b0 * c.x + a0 * c.y);
                    o[k + 1] = ptx::pack_bf16x2(a1 * c.z - b1 * c.w, b1 * c.z + a1 * c.w);
                }
            };
            turn4(a, oa, 2 * it * vectors);
            *reinterpret_cast<uint4 *>(y.out) = make_uint4(oa[0], oa[1], oa[2], oa[3]);
            if (TWO) {
                turn4(b, ob, 2 * it * vectors + 2);
                *reinterpret_cast<uint4 *>(y.out + 8) = make_uint4(ob[0], ob[1], ob[2], ob[3]);
            }
        }
    }
}

}  // namespace nb
