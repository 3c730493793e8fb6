// What the kernels of the gated delta rule share: arguments, the chunks of packed sequences, gates.
#pragma once
#include "../../include/deltaops.h"
#include "seq_common.hpp"

namespace dwc {

struct GdArgs {
    int T, H, K, V, key_heads, sequences, length;   // length: of equal sequences (0 where starts are given)
    int softplus, sigmoid, norm;
    float scale, eps;
    long long q_stride, k_stride, v_stride, a_stride, b_stride, y_stride;
    const void *q, *k, *v, *a, *b;
    const float *A, *a_bias;
    const int32_t *starts;
};

// What the gate makes of a and b: the logarithm of the decay, and the rate
__device__ __forceinline__ float gd_raw(const GdArgs &g, float a, int h) { return a + (g.a_bias ? g.a_bias[h] : 0.f); }
__device__ __forceinline__ float gd_soft(const GdArgs &g, float raw)
{
    return !g.softplus || raw > 20.f ? raw : log1pf(expf(raw));
}
constexpr float GD_LEAST = -256.f;                  // e^-256 is zero in fp32, and sums of 64 such keep their parts in 64 bits
__device__ __forceinline__ float gd_log_decay(const GdArgs &g, float raw, float A)
{
    const float d = A * gd_soft(g, raw);
    return d < GD_LEAST ? GD_LEAST : d;
}
__device__ __forceinline__ float gd_rate(const GdArgs &g, float b) { return g.sigmoid ? 1.f / (1.f + expf(-b)) : b; }

}  // namespace dwc
