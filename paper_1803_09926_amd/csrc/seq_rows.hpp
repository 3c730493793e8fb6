// What the norms of whole rows share: a row held in the registers of a team of lanes (a wavefront, or a block of 2 to 16 of them), V consecutive channels a vector and
// NV vectors a lane.
#pragma once
#include "seq_common.hpp"

namespace dwc {

namespace {

// The sum over a team of two values at a time, in every lane.  `lds` holds 2 floats a wavefront and is free again after the caller's next barrier.
template <int TEAM> __device__ __forceinline__ void team_sum2(float &a, float &b, float *lds)
{
    a = lanes_sum(a);
    b = lanes_sum(b);
    if constexpr (TEAM > 64) {
        constexpr int WAVES = TEAM / 64;
        const int wv = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) { lds[2 * wv] = a; lds[2 * wv + 1] = b; }
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) { a += lds[2 * i]; b += lds[2 * i + 1]; }
    }
}
template <int TEAM> __device__ __forceinline__ float team_sum(float a, float *lds)
{
    a = lanes_sum(a);
    if constexpr (TEAM > 64) {
        constexpr int WAVES = TEAM / 64;
        const int wv = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) lds[wv] = a;
        __syncthreads();
        a = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) a += lds[i];
    }
    return a;
}

// V channels of a row from channel c on.  WHOLE: C is a multiple of V and rows are aligned: loads and stores through a view of the row, in which what lies
// behind its end reads zero and is not written, without a branch.  Otherwise each vector is looked at.
template <typename T, int V, bool WHOLE> struct Part;
template <typename T, int V> struct Part<T, V, true> {
    Ahead<T, V, true> v;
    __device__ __forceinline__ void load(const T *row, int C, int c) { v.load(BufView(row, (uint32_t)C * (uint32_t)sizeof(T)), (uint32_t)c * (uint32_t)sizeof(T), 1); }
    __device__ __forceinline__ float at(int i) const { return v.at(i); }
    static __device__ __forceinline__ void store(T *row, int C, int c, const float (&r)[V])
    {
        // (past the end of the last 16 bytes of a vector that starts inside there is nothing: a whole vector is inside or outside)
        store_late<T, V, true>(BufView(row, (uint32_t)C * (uint32_t)sizeof(T)), (uint32_t)c * (uint32_t)sizeof(T), 1, r);
    }
};
template <typename T, int V> struct Part<T, V, false> {
    Some<T, V> v;
    __device__ __forceinline__ void load(const T *row, int C, int c) { v.load(row + c, C - c); }
    __device__ __forceinline__ float at(int i) const { return v.at(i); }
    static __device__ __forceinline__ void store(T *row, int C, int c, const float (&r)[V])
    {
        Some<T, V> p;
        p.set(r);
        p.store(row + c, C - c);
    }
};

// How many lanes share a row, and how many of its channels a lane has.
struct Team { int lanes, channels; };
constexpr int block_of(int lanes) { return lanes == 64 ? 256 : lanes; }

// f(lanes, vectors a lane) with the numbers as types
template <int LANES, int NV> struct Shape { static constexpr int TEAM = LANES, VECTORS = NV, BLOCK = block_of(LANES); };
template <int V, int LANES, int CHANNELS, typename F> bool shape_is(const Team &t, F f)
{
    if (t.lanes != LANES || t.channels != CHANNELS) return false;
    f(Shape<LANES, CHANNELS / V>());
    return true;
}

}  // namespace

}  // namespace dwc
