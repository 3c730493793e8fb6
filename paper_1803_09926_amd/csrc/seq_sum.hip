// The second stage of the sums over tokens: partials of workgroups, added in 64 bits in a fixed order.
#include "seq_common.hpp"

namespace dwc {

// A block adds 64 neighbouring columns; its four wavefronts take every fourth partial each, and wavefront 0 adds their sums.  Bound by the read of
// the partials, a few per cent of what the first stage reads.
__global__ __launch_bounds__(256) void k_sum_partials(const float *__restrict__ partials, int parts, long long n0, long long n1, long long n, float *out0,
                                                      float *out1, float *out2)
{
    __shared__ double sums[3][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const long long i = (long long)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (i < n) {
        const float *p = partials + i;
        int k = wv;
        for (; k + 28 < parts; k += 32) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[(k + 4 * j) * n];
#pragma unroll
            for (int j = 0; j < 8; ++j) s += (double)v[j];
        }
        for (; k < parts; k += 4) s += (double)p[k * n];
    }
    if (wv) sums[wv - 1][lane] = s;
    __syncthreads();
    if (wv || i >= n) return;
    const float total = (float)((s + sums[0][lane]) + (sums[1][lane] + sums[2][lane]));
    if (i < n0) { if (out0) out0[i] = total; }
    else if (i < n1) { if (out1) out1[i - n0] = total; }
    else if (out2) out2[i - n1] = total;
}

hipError_t launch_sum_partials(const float *partials, int parts, long long n0, long long n1, long long n, float *out0, float *out1, float *out2,
                               hipStream_t stream)
{
    if (n == 0) return hipSuccess;
    const long long blocks = (n + 63) / 64;
    if (!launchable(blocks, 256)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_sum_partials, dim3((unsigned)blocks), dim3(256), 0, stream, partials, parts, n0, n1, n, out0, out1, out2);
    return hipGetLastError();
}

}  // namespace dwc
