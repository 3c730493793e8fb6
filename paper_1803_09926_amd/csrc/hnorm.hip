// The RMS norm of each head with a gate, forward and backward.  The contract stands in include/deltaops.h.
//
// A run of D channels is held by a team of TL = 4 to 64 lanes of one wavefront, 16 bytes a vector and NV vectors a lane; its sum is taken inside the vector
// registers, so that a run is read once and written once and nothing waits at a barrier.  Both passes are bound by memory: 9999 tokens of 12 runs of 100 in fp32 20.6 us (96 MB,
// 4.7 TB/s), the gradients of 16384 tokens of 8 runs of 128 in bf16 with a gate 33 us (168 MB, 5.1 TB/s) and 4.6 for the sum of the partials.
//
// The weight's gradient is a sum over tokens and heads: each lane keeps the sums of its channels over all runs that its team walks, the teams of a wavefront add
// theirs between lanes, the wavefronts of a block in LDS, and the blocks' partials meet in seq_sum.hip.
#include "../../include/deltaops.h"
#include "seq_common.hpp"
#include <initializer_list>

namespace dwc {

namespace {

struct HnormArgs {
    long long runs;            // T * H
    int H, D, silu;
    float eps, inv_d;
    long long x_stride, z_stride, y_stride;
};

// the sum over the TL lanes of a team, in every lane of it
template <int TL> __device__ __forceinline__ float team_sum(float v)
{
    v += lane_move<DPP_XOR1>(v);
    v += lane_move<DPP_XOR2>(v);
    if constexpr (TL >= 8) v += lane_move<DPP_HALF_MIRROR>(v);
    if constexpr (TL >= 16) v += lane_move<DPP_MIRROR>(v);
    if constexpr (TL >= 32) v = rows_join(v, v);
    if constexpr (TL >= 64) v = halves_join(v, v);
    return v;
}

// the token of a run, and its head
__device__ __forceinline__ void place_of(long long run, const HnormArgs &a, long long &t, int &h)
{
    if (a.runs <= 0xffffffffll) {
        const uint32_t r = (uint32_t)run, q = r / (uint32_t)a.H;
        t = q;
        h = (int)(r - q * (uint32_t)a.H);
    } else {
        t = run / a.H;
        h = (int)(run - t * a.H);
    }
}

constexpr int BLOCK = 256;

template <typename T, int TL, int NV>
__global__ __launch_bounds__(BLOCK) void k_hnorm_fwd(HnormArgs a, const T *__restrict__ x, const T *__restrict__ z, const T *__restrict__ w,
                                                     T *__restrict__ y, float *__restrict__ rstd)
{
    constexpr int V = 16 / (int)sizeof(T), TEAMS = BLOCK / TL;
    typedef Some<T, V> P;
    const int lane = threadIdx.x % TL;
    P wr[NV];
    if (w) {
#pragma unroll
        for (int j = 0; j < NV; ++j) wr[j].load(w + (j * TL + lane) * V, a.D - (j * TL + lane) * V);
    }
    for (long long first = (long long)blockIdx.x * TEAMS; first < a.runs; first += (long long)gridDim.x * TEAMS) {
        const long long run = first + threadIdx.x / TL;
        const bool here = run < a.runs;          // (the sums are over all lanes of a wavefront's teams)
        long long t;
        int h;
        place_of(here ? run : first, a, t, h);
        const int D = here ? a.D : 0;
        P in[NV], gate[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TL + lane) * V;
            in[j].load(x + t * a.x_stride + (long long)h * a.D + c, D - c);
            if (z) gate[j].load(z + t * a.z_stride + (long long)h * a.D + c, D - c);
        }
        float squares = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) squares += in[j].at(i) * in[j].at(i);
        const float r = 1.f / sqrtf(team_sum<TL>(squares) * a.inv_d + a.eps);
        if (rstd && here && lane == 0) rstd[run] = r;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TL + lane) * V;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                o[i] = in[j].at(i) * r;
                if (w) o[i] *= wr[j].at(i);
                if (z) {
                    const float zz = gate[j].at(i);
                    o[i] *= a.silu ? zz * sigmoid(zz) : sigmoid(zz);
                }
            }
            P out;
            out.set(o);
            out.store(y + t * a.y_stride + (long long)h * a.D + c, D - c);
        }
    }
}

// partials: [blocks][D], or NULL where the weight's gradient is not asked for
template <typename T, int TL, int NV>
__global__ __launch_bounds__(BLOCK) void k_hnorm_bwd(HnormArgs a, const T *__restrict__ x, const T *__restrict__ z, const T *__restrict__ w,
                                                     const float *__restrict__ rstd, const T *__restrict__ dy, T *__restrict__ dx, T *__restrict__ dz,
                                                     float *__restrict__ partials)
{
    constexpr int V = 16 / (int)sizeof(T), TEAMS = BLOCK / TL, WAVES = BLOCK / 64;
    typedef Some<T, V> P;
    const int lane = threadIdx.x % TL;
    P wr[NV];
    float gw[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (w) wr[j].load(w + (j * TL + lane) * V, a.D - (j * TL + lane) * V);
#pragma unroll
        for (int i = 0; i < V; ++i) gw[j][i] = 0.f;
    }
    struct Run { P x[NV], z[NV], dy[NV]; float r; long long t; int h; } ahead;
    auto load = [&](long long first) {
        const long long run = first + threadIdx.x / TL;
        const bool here = run < a.runs;
        place_of(here ? run : first, a, ahead.t, ahead.h);
        ahead.r = here ? rstd[run] : 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TL + lane) * V, n = here ? a.D - c : 0;
            ahead.x[j].load(x + ahead.t * a.x_stride + (long long)ahead.h * a.D + c, n);
            ahead.dy[j].load(dy + ahead.t * a.y_stride + (long long)ahead.h * a.D + c, n);
            if (z) ahead.z[j].load(z + ahead.t * a.z_stride + (long long)ahead.h * a.D + c, n);
        }
    };
    const long long stride = (long long)gridDim.x * TEAMS;
    long long first = (long long)blockIdx.x * TEAMS;
    if (first < a.runs) load(first);
    for (; first < a.runs; first += stride) {
        const Run r = ahead;
        if (first + stride < a.runs) load(first + stride);
        const bool here = first + threadIdx.x / TL < a.runs;
        float m = 0.f, g[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TL + lane) * V;
            float oz[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n = r.x[j].at(i) * r.r, d = r.dy[j].at(i), wn = w ? n * wr[j].at(i) : n;
                float act = 1.f;
                oz[i] = 0.f;
                if (z) {
                    const float zz = r.z[j].at(i), q = sigmoid(zz);
                    act = a.silu ? zz * q : q;
                    oz[i] = d * wn * (a.silu ? q * (1.f + zz * (1.f - q)) : q * (1.f - q));
                }
                const float da = d * act;
                gw[j][i] += da * n;
                m += da * wn;
                g[j][i] = w ? da * wr[j].at(i) : da;
            }
            if (z) {
                P out;
                out.set(oz);
                out.store(dz + r.t * a.z_stride + (long long)r.h * a.D + c, here ? a.D - c : 0);
            }
        }
        m = team_sum<TL>(m) * a.inv_d;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TL + lane) * V;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = r.r * (g[j][i] - r.x[j].at(i) * r.r * m);
            P out;
            out.set(o);
            out.store(dx + r.t * a.x_stride + (long long)r.h * a.D + c, here ? a.D - c : 0);
        }
    }
    if (!partials) return;
    __shared__ float sums[WAVES][TL * NV * V];
    const int wv = threadIdx.x / 64;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float s = gw[j][i];
            for (int off = 32; off >= TL; off >>= 1) s += __shfl_xor(s, off, 64);
            if ((threadIdx.x & 63) < TL) sums[wv][(j * TL + lane) * V + i] = s;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += BLOCK) partials[(long long)blockIdx.x * a.D + c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
}

int validate(const hnorm_desc *d)
{
    if (!d) return DWCONV_ERR_NULL;
    if (d->dtype != DWCONV_F32 && d->dtype != DWCONV_BF16) return DWCONV_ERR_BAD_ENUM;
    if ((d->silu | 1) != 1) return DWCONV_ERR_BAD_ENUM;
    if (d->T < 0 || d->H < 1 || d->D < 1 || !(d->eps >= 0.f)) return DWCONV_ERR_BAD_DIM;
    if (d->D > HNORM_MAX_D) return DWCONV_ERR_UNSUPPORTED;
    const long long width = (long long)d->H * d->D;
    if (d->T > SEQOPS_MAX_T || width > SEQOPS_MAX_C || d->x_stride > SEQOPS_MAX_STRIDE || d->z_stride > SEQOPS_MAX_STRIDE || d->y_stride > SEQOPS_MAX_STRIDE)
        return DWCONV_ERR_TOO_LARGE;
    if (d->T > 1 && (d->x_stride < width || d->z_stride < width || d->y_stride < width)) return DWCONV_ERR_BAD_DIM;
    return DWCONV_OK;
}

// lanes of a team: as many as a run has vectors, at most a wavefront
int team_lanes(const hnorm_desc *d)
{
    const int vectors = cdiv(d->D, d->dtype == DWCONV_F32 ? 4 : 8);
    int lanes = 4;
    while (lanes < vectors && lanes < 64) lanes *= 2;
    return lanes;
}
long long blocks_for(const hnorm_desc *d, long long most)
{
    const int teams = BLOCK / team_lanes(d);
    const long long runs = (long long)d->T * d->H, need = (runs + teams - 1) / teams;
    return need < most ? need : most;
}
// Blocks of the backward pass; each leaves partials that are read again (16384 tokens of 8 runs of 128 in bf16, with their sum: 512 blocks 37.1 us, 1024 39.8, 2048 41.8).
long long bwd_blocks(const hnorm_desc *d) { return blocks_for(d, 512); }

HnormArgs args_of(const hnorm_desc *d)
{
    return {(long long)d->T * d->H, d->H, d->D, d->silu, d->eps, 1.f / (float)d->D, d->x_stride, d->z_stride, d->y_stride};
}

template <int TL, int NV> struct Lanes { static constexpr int LANES = TL, VECTORS = NV; };
// f with the team's lanes and vectors a lane as types
template <typename T, typename F> void with_team(const hnorm_desc *d, F f)
{
    constexpr int V = 16 / (int)sizeof(T);
    switch (team_lanes(d)) {
    case 4: return f(Lanes<4, 1>());
    case 8: return f(Lanes<8, 1>());
    case 16: return f(Lanes<16, 1>());
    case 32: return f(Lanes<32, 1>());
    default:
        if (d->D <= 64 * V) return f(Lanes<64, 1>());
        if (d->D <= 128 * V) return f(Lanes<64, 2>());
        if constexpr (V == 4) return f(Lanes<64, 4>());
    }
}

template <typename T> hipError_t launch_fwd(const hnorm_desc *d, const hnorm_tensors *t, hipStream_t stream)
{
    with_team<T>(d, [&](auto team) {
        typedef decltype(team) S;
        hipLaunchKernelGGL((k_hnorm_fwd<T, S::LANES, S::VECTORS>), dim3((unsigned)blocks_for(d, most_blocks(BLOCK))), dim3(BLOCK), 0, stream, args_of(d),
                           (const T *)t->x, (const T *)t->z, (const T *)t->w, (T *)t->y, (float *)t->rstd);
    });
    return hipGetLastError();
}

template <typename T> hipError_t launch_bwd(const hnorm_desc *d, const hnorm_tensors *t, float *partials, hipStream_t stream)
{
    with_team<T>(d, [&](auto team) {
        typedef decltype(team) S;
        hipLaunchKernelGGL((k_hnorm_bwd<T, S::LANES, S::VECTORS>), dim3((unsigned)bwd_blocks(d)), dim3(BLOCK), 0, stream, args_of(d), (const T *)t->x,
                           (const T *)t->z, (const T *)t->w, (const float *)t->rstd, (const T *)t->dy, (T *)t->dx, (T *)t->dz, partials);
    });
    return hipGetLastError();
}

}  // namespace

}  // namespace dwc

using namespace dwc;

extern "C" {

int hnorm_fwd(const hnorm_desc *desc, const hnorm_tensors *t, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t) return DWCONV_ERR_NULL;
    if (desc->T == 0) return DWCONV_OK;
    if (!t->x || !t->y) return DWCONV_ERR_NULL;
    for (const void *p : {t->x, t->z, t->w, (const void *)t->y})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    if (unaligned4(t->rstd)) return DWCONV_ERR_ALIGN;
    const hipError_t e = desc->dtype == DWCONV_F32 ? launch_fwd<float>(desc, t, (hipStream_t)stream) : launch_fwd<bf16_t>(desc, t, (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

size_t hnorm_bwd_workspace_bytes(const hnorm_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    return (size_t)bwd_blocks(desc) * (size_t)desc->D * sizeof(float);
}

int hnorm_bwd(const hnorm_desc *desc, const hnorm_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t) return DWCONV_ERR_NULL;
    if (desc->T > 0 && (!t->x || !t->rstd || !t->dy || !t->dx || !t->z != !t->dz)) return DWCONV_ERR_NULL;
    for (const void *p : {t->x, t->z, t->w, t->dy, (const void *)t->dx, (const void *)t->dz})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    if (unaligned4(t->rstd) || unaligned4(t->dw)) return DWCONV_ERR_ALIGN;
    const size_t need = hnorm_bwd_workspace_bytes(desc);
    if (t->dw && need) {
        if (!workspace || workspace_bytes < need) return DWCONV_ERR_WORKSPACE;
        if (unaligned16(workspace)) return DWCONV_ERR_ALIGN;
    }
    float *const partials = t->dw ? (float *)workspace : nullptr;
    hipError_t e = hipSuccess;
    if (desc->T > 0)
        e = desc->dtype == DWCONV_F32 ? launch_bwd<float>(desc, t, partials, (hipStream_t)stream) : launch_bwd<bf16_t>(desc, t, partials, (hipStream_t)stream);
    if (e == hipSuccess && t->dw)
        e = launch_sum_partials(partials, (int)bwd_blocks(desc), desc->D, desc->D, desc->D, (float *)t->dw, nullptr, nullptr, (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

}  // extern "C"
