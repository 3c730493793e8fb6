// The second stage of the sums over tokens: partials of workgroups, added in 64 bits in a fixed order.
#include "seq_common.hpp"

namespace dwc {

namespace {

// A block adds COLUMNS neighbouring columns, block 0 those from column `first` on; 64 / COLUMNS * WAVES rows of lanes take every so many partials each, and their sums are added in LDS in turn.
// Bound by the latency of the reads, which are a few per cent of what the first stage reads: many partials take many lanes a column (the
// 1024 of a norm of 1536 channels: 13.8 us with four lanes a column, 6.2 with 64; its 512 now 4.7).
template <int COLUMNS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_sum_partials(const float *__restrict__ partials, int parts, long long first, long long n0, long long n1,
                                                             long long n, float *out0, float *out1, float *out2)
{
    constexpr int ROWS = 64 / COLUMNS * WAVES;
    __shared__ double sums[ROWS][COLUMNS];
    const int row = threadIdx.x / COLUMNS, col = threadIdx.x % COLUMNS;
    const long long i = first + (long long)blockIdx.x * COLUMNS + col;
    double s = 0.0;
    if (i < n) {
        const float *p = partials + i;
        int k = row;
        for (; k + 7 * ROWS < parts; k += 8 * ROWS) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[(k + j * ROWS) * n];
#pragma unroll
            for (int j = 0; j < 8; ++j) s += (double)v[j];
        }
        for (; k < parts; k += ROWS) s += (double)p[k * n];
    }
    sums[row][col] = s;
    for (int half = ROWS / 2; half > 0; half /= 2) {
        __syncthreads();
        if (row < half) sums[row][col] += sums[row + half][col];
    }
    if (row || i >= n) return;
    const float total = (float)sums[0][col];
    if (i < n0) { if (out0) out0[i] = total; }
    else if (i < n1) { if (out1) out1[i - n0] = total; }
    else if (out2) out2[i - n1] = total;
}

}  // namespace

hipError_t launch_sum_partials(const float *partials, int parts, long long n0, long long n1, long long n, float *out0, float *out1, float *out2,
                               hipStream_t stream)
{
    if (n == 0) return hipSuccess;
    const bool many = parts >= 128;
    const int columns = many ? 16 : 64, threads = many ? 1024 : 256;
    const long long blocks = (n + columns - 1) / columns, most = most_blocks(threads);
    for (long long b = 0; b < blocks; b += most) {
        const unsigned now = (unsigned)(blocks - b < most ? blocks - b : most);
        const long long first = b * columns;
        if (many) hipLaunchKernelGGL((k_sum_partials<16, 16>), dim3(now), dim3(threads), 0, stream, partials, parts, first, n0, n1, n, out0, out1, out2);
        else hipLaunchKernelGGL((k_sum_partials<64, 4>), dim3(now), dim3(threads), 0, stream, partials, parts, first, n0, n1, n, out0, out1, out2);
    }
    return hipGetLastError();
}

}  // namespace dwc
