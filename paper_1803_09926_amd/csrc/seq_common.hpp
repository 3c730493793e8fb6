// What the kernels over token sequences share: rows of any alignment, sums over lanes, the sequences of packed tokens, and the sum of partials.
#pragma once
#include "../../include/seqops.h"
#include "common.hpp"
#include "bounds.hpp"

namespace dwc {

// ---- rows ----------------------------------------------------------------------------------------
// 8 and 16 bytes that lie anywhere: one load or store each, as the alignment that the types promise is an element's.
typedef uint32_t u2any_t __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u4any_t __attribute__((ext_vector_type(4), aligned(2)));

// V consecutive elements of a row, of which the first n are there (the others are zero, and are neither read nor written).
// They stay as stored until they are used: bf16 takes half the registers.
template <typename T, int V> struct Some {
    static constexpr int WORDS = (int)(V * sizeof(T)) / 4;
    static_assert(V * sizeof(T) % 8 == 0, "whole pairs of 32-bit words");
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= V) {
            const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
            constexpr int W4 = WORDS / 4 * 4;
#pragma unroll
            for (int i = 0; i < W4; i += 4) {
                const u4any_t v = *reinterpret_cast<const u4any_t *>(q + 2 * i);
                w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
            }
            if constexpr (WORDS % 4 == 2) {
                const u2any_t v = *reinterpret_cast<const u2any_t *>(q + 2 * W4);
                w[W4] = v.x; w[W4 + 1] = v.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = 0;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < n) {
                    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint((float)p[i]);
                    else w[i / 2] |= (uint32_t)p[i] << (i % 2 * 16);
                }
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void get(float (&r)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = at(i);
    }
    // rounded to nearest-even where T is bf16
    __device__ __forceinline__ void set(const float (&r)[V])
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(r[i]);
            else w[i] = pack2_bf16(r[2 * i], r[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void store(T *p, int n) const
    {
        if (n >= V) {
            uint16_t *q = reinterpret_cast<uint16_t *>(p);
            constexpr int W4 = WORDS / 4 * 4;
#pragma unroll
            for (int i = 0; i < W4; i += 4) {
                const u4any_t v = {w[i], w[i + 1], w[i + 2], w[i + 3]};
                *reinterpret_cast<u4any_t *>(q + 2 * i) = v;
            }
            if constexpr (WORDS % 4 == 2) {
                const u2any_t v = {w[W4], w[W4 + 1]};
                *reinterpret_cast<u2any_t *>(q + 2 * W4) = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < n) {
                    if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(p)[i] = w[i];
                    else p[i] = (T)(w[i / 2] >> (i % 2 * 16));
                }
        }
    }
};
// V consecutive elements that are asked for early and used late.  The loads go through a view of the rows, in which a lane that is to have zeros asks for what
// lies outside: no branch, and so nothing that waits for them before they are used.  WHOLE: V elements are all there or none of them, and aligned to their
// bytes; otherwise each is a load of its own, STEP elements from the one before, and those less than n from the first are there.
template <typename T, int V, bool WHOLE, int STEP = 1> struct Ahead {
    static_assert(STEP == 1 || !WHOLE, "vectors are of neighbours");
    static constexpr int BYTES = V * (int)sizeof(T), WORDS = WHOLE ? (BYTES + 3) / 4 : V;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const BufView &rows, uint32_t off, int n)
    {
        if constexpr (WHOLE) {
            const uint32_t at = n > 0 ? off : BufView::OUTSIDE;
            if constexpr (BYTES == 2) w[0] = rows.b16(at, 0);
            else if constexpr (BYTES == 4) w[0] = rows.b32(at, 0);
            else if constexpr (BYTES == 8) { const u2raw_t v = rows.b64(at, 0); w[0] = v.x; w[1] = v.y; }
            else {
                static_assert(BYTES % 16 == 0, "vectors of 2, 4, 8 and 16 bytes");
#pragma unroll
                for (int i = 0; i < BYTES / 16; ++i) {
                    const u4raw_t v = rows.b128(n > i * (16 / (int)sizeof(T)) ? off + 16 * i : BufView::OUTSIDE, 0);
                    w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t at = n > i * STEP ? off + i * STEP * (uint32_t)sizeof(T) : BufView::OUTSIDE;
                if constexpr (sizeof(T) == 2) w[i] = rows.b16(at, 0);
                else w[i] = rows.b32(at, 0);
            }
        }
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (!WHOLE || V == 1) return __uint_as_float(w[i] << 16);
        else return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};
// The counterpart for stores, rounded where T is bf16: what is not there is stored outside the view, which does nothing.  No branch here either: the loads
// behind it would have to wait for all stores, and not for those only that come before them.
template <typename T, int V, bool WHOLE, int STEP = 1>
__device__ __forceinline__ void store_late(const BufView &rows, uint32_t off, int n, const float (&r)[V])
{
    constexpr int BYTES = V * (int)sizeof(T);
    if constexpr (WHOLE && BYTES >= 4) {
        const uint32_t at = n > 0 ? off : BufView::OUTSIDE;
        uint32_t w[BYTES / 4];
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(r[i]);
            else w[i] = pack2_bf16(r[2 * i], r[2 * i + 1]);
        }
        if constexpr (BYTES == 4) rows.st32<false>(w[0], at, 0);
        else if constexpr (BYTES == 8) { const u2raw_t v = {w[0], w[1]}; rows.st64<false>(v, at, 0); }
        else {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const u4raw_t v = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
                rows.st128<false>(v, n > i * (16 / (int)sizeof(T)) ? off + 16 * i : BufView::OUTSIDE, 0);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t at = n > i * STEP ? off + i * STEP * (uint32_t)sizeof(T) : BufView::OUTSIDE;
            if constexpr (sizeof(T) == 4) rows.st32<false>(__float_as_uint(r[i]), at, 0);
            else __builtin_amdgcn_raw_buffer_store_b16(f32_to_bf16(r[i]), rows.rsrc, (int)at, 0, 0);
        }
    }
}
constexpr uint32_t VIEW_BYTES = 0x7fffffffu;   // of a view whose lanes ask for nothing that is not there, or for BufView::OUTSIDE

// ---- sums over lanes -------------------------------------------------------------------------------
// Data moves inside the vector registers (lane permutations as operand modifiers, row swaps of gfx950), not through LDS.
template <int CTRL> __device__ __forceinline__ float lane_move(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140, DPP_ROR8 = 0x128;
// a in the lower and b in the upper half of each pair of rows (of 16 lanes), each added to what the other half held of it
__device__ __forceinline__ float rows_join(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// the same for the lower and upper 32 lanes
__device__ __forceinline__ float halves_join(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// the sum over the 64 lanes, in every lane; the order of additions is fixed by the lane numbers
__device__ __forceinline__ float lanes_sum(float v)
{
    v += lane_move<DPP_XOR1>(v);
    v += lane_move<DPP_XOR2>(v);
    v += lane_move<DPP_HALF_MIRROR>(v);
    v += lane_move<DPP_MIRROR>(v);
    v = rows_join(v, v);
    return halves_join(v, v);
}

// ---- sequences of packed tokens --------------------------------------------------------------------
// starts may hold anything: an index that comes out of it lies in 0 .. n - 1, and no token comes out of it that is not clamped where it is used.
struct Sequences {
    const int32_t *starts;   // n + 1 of them, or NULL: equal lengths
    int n, length, T;
    __device__ __forceinline__ int start(int s) const
    {
        // (the last one of equal lengths is T, and no product passes it)
        return starts ? starts[s] : s * length;
    }
    // the last sequence that starts at or before t: the one that holds t
    __device__ __forceinline__ int of(int t) const
    {
        if (!starts) return length > 0 ? min(t / length, n - 1) : 0;
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (starts[mid] <= t) lo = mid;
            else hi = mid;
        }
        return lo;
    }
    // the same for a t that is the same in a wavefront's 64 lanes, all of which are here: one load for 64 sequences, two for 4096
    __device__ __forceinline__ int of_one(int t) const
    {
        if (!starts) return of(t);
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int step = (hi - lo + 63) / 64;
            const long long at = lo + (long long)step * ((threadIdx.x & 63) + 1);
            lo += step * __popcll(__ballot(at < hi && starts[at < hi ? at : lo] <= t));
            hi = hi - lo > step ? lo + step : hi;
        }
        return lo;
    }
};

// ---- elementwise -----------------------------------------------------------------------------------
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }   // one instruction, 1 ulp, results below 2^-126 are zero
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + exp2_fast(-LOG2E * v)); }

// ---- sum of partials (seq_sum.hip) -----------------------------------------------------------------
// The sum over p < parts of partials[p * n + i], added in 64 bits in a fixed order, for the n columns i of up to three outputs that lie one after
// the other: the first ends before column n0, the second before n1, the third before n.  An output that is NULL is skipped.
hipError_t launch_sum_partials(const float *partials, int parts, long long n0, long long n1, long long n, float *out0, float *out1, float *out2,
                               hipStream_t stream);

// ---- host ------------------------------------------------------------------------------------------
// The most blocks of one launch, which has fewer than 2^32 lanes.  What takes more of them goes in several launches.
constexpr long long most_blocks(int threads) { return ((1ll << 32) - 1) / threads; }
inline bool unaligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool unaligned_to(const void *p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == DWCONV_F32 ? 3u : 1u)) != 0; }
inline bool unaligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

}  // namespace dwc
