// What the two walks over a sequence's chunks share: columns of the state in registers.
#pragma once
#include "gdelta_tile.hpp"
#include "gdelta_launch.hpp"

namespace dwc {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

// The columns of a lane: NT neighbours, one in each of its NT result tiles, so that its numbers of a row lie beside each other
template <int NT> struct Columns {
    int c;                                        // the first
    __device__ __forceinline__ Columns(int block) : c((block * WAVES + (int)(threadIdx.x >> 6)) * 16 * NT + (int)(threadIdx.x & 15) * NT) {}
    // NT numbers of a row, of which those below `width` are there
    template <typename T> __device__ __forceinline__ void load(const T *row, int width, bool there, float (&x)[NT]) const
    {
#pragma unroll
        for (int i = 0; i < NT; ++i) x[i] = there && c + i < width ? ldf(row + c + i) : 0.f;
    }
    template <typename T> __device__ __forceinline__ void store(T *row, int width, bool there, const float (&x)[NT]) const
    {
#pragma unroll
        for (int i = 0; i < NT; ++i)
            if (there && c + i < width) stf(row + c + i, x[i]);
    }
};

// rows 16 mt + 4 q + r of a tile of tokens
__device__ __forceinline__ int row_of(int mt, int r) { return mt * 16 + 4 * (int)((threadIdx.x & 63) >> 4) + r; }
__device__ __forceinline__ float4 four(const float *v, int mt) { return *reinterpret_cast<const float4 *>(v + row_of(mt, 0)); }
__device__ __forceinline__ v4f_t times(const v4f_t &a, const float4 &b) { return v4f_t{a[0] * b.x, a[1] * b.y, a[2] * b.z, a[3] * b.w}; }

// result tiles of 64 rows as operands that are contracted over them
template <int N, int NT> __device__ __forceinline__ void split_rows(const v4f_t (&x)[4][NT], Frag (&f)[2][NT][N])
{
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) split_tiles<N>(x[2 * ks][nt], x[2 * ks + 1][nt], f[ks][nt]);
}

template <typename T, int KP, bool SHARE> struct Walk {
    static constexpr int RAW = PartsOf<T>::RAW, INNER = PartsOf<T>::INNER, LD = KP + PAD;
    static constexpr size_t TILE = (size_t)RAW * CHUNK * LD * 2, MATRIX = (size_t)INNER * CHUNK * LDM * 2;
    static constexpr size_t LDS = (SHARE ? 1 : 2) * TILE + 2 * MATRIX + 2 * 256 * 4;
};
// Whether the tiles of keys and queries share their place in LDS: where both do not fit
template <typename T, int KP> constexpr bool shares() { return Walk<T, KP, false>::LDS > 160 * 1024; }

}  // namespace

}  // namespace dwc
