// Shared by the forward, backward and step kernels of the selective state space scan.
//
// Layout of the work.  A lane holds 4 states of one channel, LPC neighbouring lanes hold a channel's up to 4 * LPC states, and a block of 256 lanes
// holds 256 / LPC channels of one group: the sum over the states is a few moves between neighbouring lanes, one exponential and four multiply-adds a state
// stay in one lane's registers, and a launch of C channels has LPC times the wavefronts that a channel a lane would have.
// A block walks its tokens in tiles.  What is elementwise in a token and channel (the step size and its softplus, the gate, rounding) is done once for
// a tile by lanes that take neighbouring channels of a token, in vectors; the recurrence reads it from LDS.
#pragma once
#include "seq_common.hpp"
#include <initializer_list>

namespace dwc {

constexpr int KEPT_EVERY = 16;   // tokens between two states that the forward pass keeps for the backward pass

struct Scan {
    int C, N, groups, per_group, blocks_of_group;   // per_group: channels of a group
    int copies, twice, by_n, by_twice;              // of a channel's states, see state_of; 2^16 / N and 2^16 / twice, rounded up
    float share;                                    // 1 / copies
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

// Which state a channel's slot k < 4 * LPC has.  Where N is less than the slots, those behind the first N have states once more: each state is there `copies` times,
// the largest power of two for which there is room, and the first `twice` of them two times that.  Zeros in these slots would make NaN of an infinite x or step size
// beside them; a copy has what its state has.  A copy's C is divided by the number of copies, which is exact, and so the sums over slots are those over states.
// (k % N, and behind the N * copies slots that this reaches, what is left % twice; exact for numbers below 2^8.  Products of 24 bits are one instruction, and as
// many states as slots are a scalar branch: these lines stand before the first load)
__device__ __forceinline__ int state_of(const Scan &g, int k)
{
    if (g.N * g.copies + g.twice == g.N) return k;
    const int left = k - g.N * g.copies;
    return left < 0 ? k - __mul24(__mul24(k, g.by_n) >> 16, g.N) : left - __mul24(__mul24(left, g.by_twice) >> 16, g.twice);
}
__device__ __forceinline__ float share_of(const Scan &g, int state) { return state < g.twice ? 0.5f * g.share : g.share; }   // of C, in each of its slots

// log(1 + e) for 0 <= e <= 1: the logarithm of the rounded sum, one instruction, and to first order what the rounding took, which is most of the result where
// e is small.  Within 2e-7 of the result over 2^-30 <= e <= 1, measured; a series in e / (2 + e) of that accuracy takes twice the instructions.
__device__ __forceinline__ float log1p_unit(float e)
{
    const float u = 1.f + e;
    return fmaf(__builtin_amdgcn_logf(u), LN2, e - (u - 1.f));
}
// max(v, 0), in one instruction, + log(1 + exp(-|v|)); NaN stays NaN, by way of the exponential
__device__ __forceinline__ float softplus_of(float v)
{
    const float e = exp2_fast(-LOG2E * fabsf(v));
    return __builtin_amdgcn_fmed3f(v, 0.f, __builtin_inff()) + log1p_unit(e);
}
// the step sizes of V elements
template <int V> __device__ __forceinline__ void step_sizes(const Scan &g, float (&v)[V])
{
    if (g.softplus) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = softplus_of(v[i]);
    }
}

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

// The sum over a channel's L lanes, in each of them.
template <int L> __device__ __forceinline__ float states_sum(float v)
{
    v += lane_move<DPP_XOR1>(v);
    if constexpr (L >= 4) v += lane_move<DPP_XOR2>(v);
    if constexpr (L >= 8) v += lane_move<DPP_HALF_MIRROR>(v);
    if constexpr (L >= 16) v += lane_move<DPP_MIRROR>(v);
    return v;
}

// The tokens of t0 .. t0 + n - 1 (n <= 32) that are the first of their sequence, a bit each; the same in every lane.  `of` gets the token's sequence in the
// lane of its number from t0, and that of the token before t0 in the last lane: a search in each token's turn costs a chain of loads for each.
__device__ __forceinline__ uint32_t first_tokens(const Sequences &seq, int t0, int n, int end, int &of)
{
    const int lane = threadIdx.x & 63, t = lane == 63 ? t0 - 1 : t0 + lane;
    const bool there = t >= 0 && t < end && (lane < n || lane == 63);
    of = there ? seq.of(t) : 0;
    return (uint32_t)__ballot(there && lane < n && seq.start(of) == t);
}
__device__ __forceinline__ int sequence_of(int of, int t) { return __builtin_amdgcn_readlane(of, t & 63); }   // of token t from t0, -1 the one before it
__device__ __forceinline__ bool first_token(const Sequences &seq, int t) { return seq.start(seq.of_one(t)) == t; }

// What `count` parts from `first` on (in the direction of `step`) leave at the end of a row of them: v = e[first] + decay(first) * (e[next] + ...), with the
// decay over a part exp(A * its sum of step sizes), from the farthest part on.
template <int LPC, bool WIDE>
__device__ __forceinline__ void gather_parts_as(float (&v)[4], const float (&a2)[4], const float *ends, const float *sums, int C, int chan, int q, bool valid,
                                                int first, int step, int count)
{
    constexpr int AHEAD = WIDE ? 1 : 6;                               // parts asked for at a time: eight take registers that the kernel behind it wants
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = 0.f;
    for (int k = count - 1; k >= 0; k -= AHEAD) {
        float4 e[AHEAD];
        float sum[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const long long at = (long long)(first + step * (k - i)) * C + chan;
            const bool there = valid && k >= i;
            e[i] = there ? *reinterpret_cast<const float4 *>(ends + at * (4 * LPC) + 4 * q) : make_float4(0.f, 0.f, 0.f, 0.f);
            sum[i] = there && k - i < count - 1 ? sums[at] : 0.f;     // (nothing comes through the farthest, whose first tokens may be another sequence's)
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (k < i) break;
            const float u[4] = {e[i].x, e[i].y, e[i].z, e[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (WIDE) {
                    const float root = exp2_fast(__builtin_amdgcn_fmed3f(0.5f * a2[j] * sum[i], -126.f, 127.f));
                    v[j] = fmaf(v[j] * root, root, u[j]);
                } else {
                    v[j] = fmaf(v[j], exp2_fast(a2[j] * sum[i]), u[j]);
                }
            }
        }
    }
}
// A decay over a whole part may pass the range of a float on either side where the state that it meets brings it back: a zero that grows stays zero, a small number may grow
// to an ordinary one, an infinity that decays stays one.  Where that happens the sum comes out as no finite number, and is taken once more with each decay as the
// square of its root, which is held inside the range.
template <int LPC>
__device__ __forceinline__ void gather_parts(float (&v)[4], const float (&a2)[4], const float *ends, const float *sums, int C, int chan, int q, bool valid,
                                             int first, int step, int count)
{
    gather_parts_as<LPC, false>(v, a2, ends, sums, C, chan, q, valid, first, step, count);
    if (!(fabsf(v[0]) + fabsf(v[1]) + fabsf(v[2]) + fabsf(v[3]) <= 3.4e38f))
        gather_parts_as<LPC, true>(v, a2, ends, sums, C, chan, q, valid, first, step, count);
}

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

// Whether lanes that take `each` neighbouring channels of a group find these, or 16 bytes of them where they are more, all there or none of them, in rows
// aligned to that.
template <typename T> bool whole_vectors(int each, int per_group, std::initializer_list<const void *> rows, std::initializer_list<long long> strides)
{
    const int most = 16 / (int)sizeof(T), unit = each < most ? each : most;
    if (per_group % unit) return false;
    for (const void *p : rows)
        if (reinterpret_cast<uintptr_t>(p) % (unit * sizeof(T))) return false;
    for (const long long s : strides)
        if (s % unit) return false;
    return true;
}

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
