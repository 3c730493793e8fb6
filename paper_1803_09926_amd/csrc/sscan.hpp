// Shared by the forward, backward and step kernels of the selective state space scan.
//
// Layout of the work.  A lane holds 4 states of one channel, LPC neighbouring lanes hold a channel's up to 4 * LPC states, and a block of 256 lanes
// holds 256 / LPC channels of one group: the sum over the states is a few moves between neighbouring lanes, one exponential and four multiply-adds a state
// stay in one lane's registers, and a launch of C channels has LPC times the wavefronts that a channel a lane would have.
// A block walks its tokens in tiles.  What is elementwise in a token and channel (the step size and its softplus, the gate, rounding) is done once for
// a tile by lanes that take neighbouring channels of a token, in vectors; the recurrence reads it from LDS.
#pragma once
#include "seq_common.hpp"

namespace dwc {

constexpr int KEPT_EVERY = 16;   // tokens between two states that the forward pass keeps for the backward pass

struct Scan {
    int C, N, groups, per_group, blocks_of_group;   // per_group: channels of a group
    int softplus, part, parts;                      // tokens of a part; parts of the launch
    long long xs, dts, zs, bs, cs, ys;              // row strides
    Sequences seq;
};

// Which channels and which part of the tokens a block has: blocks of neighbouring channels are neighbours, then groups, then parts.
struct ScanBlock { int group, block, part; };
__device__ __forceinline__ ScanBlock scan_block(const Scan &g)
{
    const unsigned id = blockIdx.x, per = (unsigned)g.blocks_of_group, rest = id / per;
    return {(int)(rest % (unsigned)g.groups), (int)(id % per), (int)(rest / (unsigned)g.groups)};
}

// log(1 + e) for 0 <= e <= 1 as 2 atanh(s), s = e / (2 + e) <= 1/3: the odd series in s (its first nine terms leave 3^-19 / 19 at s = 1/3) keeps its relative
// accuracy down to e = 0, where log of the rounded 1 + e has none.
__device__ __forceinline__ float log1p_unit(float e)
{
    const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
    float p = 1.f / 17.f;
    p = fmaf(p, q, 1.f / 15.f);
    p = fmaf(p, q, 1.f / 13.f);
    p = fmaf(p, q, 1.f / 11.f);
    p = fmaf(p, q, 1.f / 9.f);
    p = fmaf(p, q, 1.f / 7.f);
    p = fmaf(p, q, 1.f / 5.f);
    p = fmaf(p, q, 1.f / 3.f);
    p = fmaf(p, q, 1.f);
    return 2.f * s * p;
}
// max(v, 0) + log(1 + exp(-|v|)); NaN stays NaN, by way of the exponential
__device__ __forceinline__ float softplus_of(float v)
{
    const float e = exp2_fast(-LOG2E * fabsf(v));
    return fmaxf(v, 0.f) + log1p_unit(e);
}
__device__ __forceinline__ float step_size(const Scan &g, float raw) { return g.softplus ? softplus_of(raw) : raw; }

// Of L neighbouring lanes, lane q gets the sum over all of them of v[q].  L - 1 moves of one register each: at each step a lane keeps one half of its values
// and adds its partner's of the same half (the partner of a step differs in that step's bit of the lane number).
template <int L> __device__ __forceinline__ float transpose_sum(float (&v)[L], int q)
{
    if constexpr (L >= 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) { const float keep = q & 8 ? v[j + 8] : v[j], give = q & 8 ? v[j] : v[j + 8]; v[j] = keep + lane_move<DPP_ROR8>(give); }
    }
    if constexpr (L >= 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) { const float keep = q & 4 ? v[j + 4] : v[j], give = q & 4 ? v[j] : v[j + 4]; v[j] = keep + lane_move<DPP_HALF_MIRROR>(give); }
    }
    if constexpr (L >= 4) {
#pragma unroll
        for (int j = 0; j < 2; ++j) { const float keep = q & 2 ? v[j + 2] : v[j], give = q & 2 ? v[j] : v[j + 2]; v[j] = keep + lane_move<DPP_XOR2>(give); }
    }
    const float keep = q & 1 ? v[1] : v[0], give = q & 1 ? v[0] : v[1];
    return keep + lane_move<DPP_XOR1>(give);
}

// The tokens of t0 .. t0 + n - 1 (n <= 32) that are the first of their sequence, a bit each; the same in every lane.
__device__ __forceinline__ uint32_t first_tokens(const Sequences &seq, int t0, int n, int end)
{
    const int lane = threadIdx.x & 63, t = t0 + lane;
    const bool first = lane < n && t < end && seq.start(seq.of(t)) == t;
    return (uint32_t)__ballot(first);
}
__device__ __forceinline__ bool first_token(const Sequences &seq, int t) { return seq.start(seq.of(t)) == t; }

// ---- host (sscan.hip) ----------------------------------------------------------------------------
// The parts that the tokens are split into: few channel blocks alone do not fill the card.  `carry`: whether a pass over the parts comes first, which
// finds the state at each part's head.  `packed`: `starts` is given.
struct ScanPlan { int lanes, channel_blocks, part, parts; bool carry; };
ScanPlan plan_sscan_fwd(const sscan_desc *d, bool packed);
ScanPlan plan_sscan_bwd(const sscan_desc *d, bool packed);
Scan sscan_geometry(const sscan_desc *d, const ScanPlan &p, const void *starts);
inline int state_lanes(int N) { return N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }

hipError_t launch_sscan_fwd(const sscan_desc *d, const sscan_tensors *t, float *workspace, hipStream_t stream);
hipError_t launch_sscan_bwd(const sscan_desc *d, const sscan_tensors *t, float *workspace, hipStream_t stream);
hipError_t launch_sscan_step(const sscan_desc *d, const sscan_tensors *t, hipStream_t stream);

// Floats of the workspaces, in the order in which they lie there, each a multiple of 4.
struct FwdSpace { size_t ends, sums, total; };                              // states at the parts' ends [parts][C][4 LPC], sums of step sizes [parts][C]
FwdSpace sscan_fwd_space(const sscan_desc *d, const ScanPlan &p);
struct BwdSpace { size_t ends, sums, dA, shared, total; };                  // as above; [parts][C * N + 2 C]; [channel blocks][T][8 LPC]
BwdSpace sscan_bwd_space(const sscan_desc *d, const ScanPlan &p);

// f(the number of lanes of a channel) for the states of d
template <typename F> hipError_t with_state_lanes(int lanes, F f)
{
    switch (lanes) {
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    case 16: f(std::integral_constant<int, 16>()); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace dwc
