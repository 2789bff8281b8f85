// Dropout's draws: 16 bits of a Philox4x32-10 word per element, eight elements to a block (include/qbp.h, qbp_dropout).
#pragma once

#include <cmath>

#include "qbp_real.cuh"

namespace qbp {

constexpr uint32_t kDropoutWord = 0xFFFFFFFFu;       // last counter word: the stochastic quantisers' and ternarisers' are below it

// What a kernel is told of a dropout: elements whose draw is below `threshold` go, the others are multiplied by `factor`.
struct DropoutParams { uint32_t threshold; float factor; uint32_t tensor_id; uint64_t block0; };
inline DropoutParams dropout_params(float p, uint32_t tensor_id, uint64_t index_base)
{
    DropoutParams d;
    d.threshold = (uint32_t)std::floor((double)p * 65536.0 + 0.5);
    d.factor = d.threshold < 65536u ? (float)(65536.0 / (65536.0 - (double)d.threshold)) : 0.0f;
    d.tensor_id = tensor_id;
    d.block0 = index_base / 8;
    return d;
}

#ifdef __CUDACC__

__device__ __forceinline__ uint4 dropout_block(const DropoutParams &d, const PhiloxKeys &keys, uint64_t block)
{
    const uint64_t b = d.block0 + block;
    return philox4x32_10(make_uint4((uint32_t)b, (uint32_t)(b >> 32), d.tensor_id, kDropoutWord), keys);
}
__device__ __forceinline__ uint32_t draw_of(const uint4 &w, int k)
{
    const uint32_t v = k < 2 ? w.x : k < 4 ? w.y : k < 6 ? w.z : w.w;
    return (k & 1) ? v >> 16 : v & 0xFFFFu;
}
// The draws of eight elements from element `first` (counted from index_base) on, as one block's words would hold them.
__device__ __forceinline__ uint4 dropout_draws8(const DropoutParams &d, const PhiloxKeys &keys, uint64_t first)
{
    const uint4 a = dropout_block(d, keys, first >> 3);
    const uint32_t o = (uint32_t)first & 7u;
    if (o == 0) return a;
    const uint4 b = dropout_block(d, keys, (first >> 3) + 1);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int s = 2; s >= 1; s >>= 1) {
        const bool by = ((o >> 1) & (uint32_t)s) != 0;
#pragma unroll
        for (int k = 0; k + s < 8; ++k) w[k] = by ? w[k + s] : w[k];
    }
    if (o & 1u) return make_uint4(__funnelshift_r(w[0], w[1], 16), __funnelshift_r(w[1], w[2], 16), __funnelshift_r(w[2], w[3], 16), __funnelshift_r(w[3], w[4], 16));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

#endif  // __CUDACC__
}  // namespace qbp
