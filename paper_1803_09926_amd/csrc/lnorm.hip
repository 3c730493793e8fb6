// Layer norm over the channels of each token, forward and backward.  The contract stands in include/seqops.h.
//
// A team of lanes (a wavefront, or a block of 4 or 16 of them) holds a row in registers, V consecutive channels a vector and NV vectors a lane, so
// that the row is read once, the variance is taken about the mean that is already known (two sums over the team, no cancellation), and all is written once.
// Both passes are bound by memory.
//
// The weight's gradient is a sum over rows: each lane keeps the sums of its own channels over all rows that its team walks, the teams of a block add
// theirs in LDS one after the other, and the blocks' partials meet in seq_sum.hip.
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

template <typename T, int TEAM, int V, int NV, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_lnorm_fwd(int rows, int C, float eps, float inv_c, const T *__restrict__ x, const T *__restrict__ residual,
                                                     const T *__restrict__ w, const T *__restrict__ b, T *__restrict__ y, T *__restrict__ total,
                                                     float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    __shared__ float lds[2][TEAM / 64];
    const int lane = threadIdx.x % TEAM;
    const long long row = (long long)blockIdx.x * (BLOCK / TEAM) + threadIdx.x / TEAM;
    if (row >= rows) return;   // (whole teams: a block of one team is always inside)
    const T *xr = x + row * C;
    Some<T, V> in[NV], more[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) in[j].load(xr + (j * TEAM + lane) * V, C - (j * TEAM + lane) * V);
    float s[NV][V], sum = 0.f;
    if (residual) {
#pragma unroll
        for (int j = 0; j < NV; ++j) more[j].load(residual + row * C + (j * TEAM + lane) * V, C - (j * TEAM + lane) * V);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] = in[j].at(i) + more[j].at(i);
            more[j].set(s[j]);
            more[j].store(total + row * C + (j * TEAM + lane) * V, C - (j * TEAM + lane) * V);
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) in[j].get(s[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) sum += s[j][i];
    const float mean = team_sum<TEAM>(sum, lds[0]) * inv_c;
    float squares = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[j][i] = (j * TEAM + lane) * V + i < C ? s[j][i] - mean : 0.f;
            squares += s[j][i] * s[j][i];
        }
    const float var = team_sum<TEAM>(squares, lds[1]) * inv_c, rstd = 1.f / sqrtf(var + eps);
    if (mean_out && lane == 0) { mean_out[row] = mean; rstd_out[row] = rstd; }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TEAM + lane) * V, n = C - c;
        if (n <= 0) break;
        float o[V];
        Some<T, V> p;
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = s[j][i] * rstd;
        if (w) {
            p.load(w + c, n);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] *= p.at(i);
        }
        if (b) {
            p.load(b + c, n);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] += p.at(i);
        }
        p.set(o);
        p.store(y + row * C + c, n);
    }
}

// Rows are dealt out to the teams of the whole launch in turn.  partials: [blocks][2][C], or NULL where the weight's gradient is not asked for.
template <typename T, int TEAM, int V, int NV, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_lnorm_bwd(int rows, int C, float inv_c, const T *__restrict__ x, const T *__restrict__ w,
                                                     const float *__restrict__ mean_in, const float *__restrict__ rstd_in, const T *__restrict__ dy,
                                                     const T *__restrict__ dtotal, T *__restrict__ dx, float *__restrict__ partials)
{
    constexpr int TEAMS = BLOCK / TEAM;
    __shared__ float lds[2][2 * TEAM / 64];
    extern __shared__ float sums[];            // [2][C], where a block has more than one team
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    Some<T, V> wr[NV];
    float gw[NV][V], gb[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (w) wr[j].load(w + (j * TEAM + lane) * V, C - (j * TEAM + lane) * V);
#pragma unroll
        for (int i = 0; i < V; ++i) gw[j][i] = gb[j][i] = 0.f;
    }
    int turn = 0;
    for (long long row = (long long)blockIdx.x * TEAMS + team; row < rows; row += (long long)gridDim.x * TEAMS, turn ^= 1) {
        Some<T, V> xr[NV], gr[NV], ar[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TEAM + lane) * V;
            xr[j].load(x + row * C + c, C - c);
            gr[j].load(dy + row * C + c, C - c);
        }
        if (dtotal) {
#pragma unroll
            for (int j = 0; j < NV; ++j) ar[j].load(dtotal + row * C + (j * TEAM + lane) * V, C - (j * TEAM + lane) * V);
        }
        const float mean = mean_in[row], rstd = rstd_in[row];
        float m1 = 0.f, m2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                // beyond the row dy is zero, and so are all products with it
                const float xhat = (xr[j].at(i) - mean) * rstd, g = gr[j].at(i), gx = g * xhat;
                gb[j][i] += g;
                gw[j][i] += gx;
                m1 += w ? g * wr[j].at(i) : g;
                m2 += w ? gx * wr[j].at(i) : gx;
            }
        team_sum2<TEAM>(m1, m2, lds[turn]);
        m1 *= inv_c;
        m2 *= inv_c;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TEAM + lane) * V, n = C - c;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xhat = (xr[j].at(i) - mean) * rstd, g = w ? gr[j].at(i) * wr[j].at(i) : gr[j].at(i);
                o[i] = rstd * ((g - m1) - xhat * m2);
            }
            if (dtotal) {
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] += ar[j].at(i);
            }
            Some<T, V> p;
            p.set(o);
            p.store(dx + row * C + c, n);
        }
    }
    if (!partials) return;
    float *out = partials + (long long)blockIdx.x * 2 * C;
    if constexpr (TEAMS > 1) {
        for (int k = 0; k < TEAMS; ++k) {      // one team after the other: a fixed order
            if (team == k) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = (j * TEAM + lane) * V + i;
                        if (c >= C) continue;
                        sums[c] = k ? sums[c] + gw[j][i] : gw[j][i];
                        sums[C + c] = k ? sums[C + c] + gb[j][i] : gb[j][i];
                    }
            }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < 2 * C; i += BLOCK) out[i] = sums[i];
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (j * TEAM + lane) * V + i;
                if (c >= C) continue;
                out[c] = gw[j][i];
                out[C + c] = gb[j][i];
            }
    }
}

int validate(const lnorm_desc *d)
{
    if (!d) return DWCONV_ERR_NULL;
    if (d->dtype != DWCONV_F32 && d->dtype != DWCONV_BF16) return DWCONV_ERR_BAD_ENUM;
    if (d->T < 0 || d->C < 1 || !(d->eps >= 0.f)) return DWCONV_ERR_BAD_DIM;
    if (d->C > LNORM_MAX_C) return DWCONV_ERR_UNSUPPORTED;
    return DWCONV_OK;
}

// How many lanes share a row, and how many of its channels a lane has.  The backward pass has five values a channel in registers, the forward pass two.
struct Team { int lanes, channels; };
Team fwd_team(int C)
{
    if (C <= 512) return {64, 8};
    if (C <= 1024) return {64, 16};
    if (C <= 2048) return {64, 32};
    if (C <= 4096) return {256, 16};
    if (C <= 8192) return {256, 32};
    return {1024, 16};
}
Team bwd_team(int C)
{
    if (C <= 512) return {64, 8};
    if (C <= 1024) return {64, 16};
    if (C <= 2048) return {256, 8};
    if (C <= 4096) return {256, 16};
    if (C <= 8192) return {1024, 8};
    return {1024, 16};
}
constexpr int block_of(int lanes) { return lanes < 256 ? 256 : lanes; }

// Blocks of the backward pass: four on each of the 256 compute units, fewer where there are fewer rows.
int bwd_blocks(const lnorm_desc *d)
{
    const int lanes = bwd_team(d->C).lanes, teams = block_of(lanes) / lanes, most = lanes == 1024 ? 256 : 1024;
    const int need = d->T > 0 ? cdiv(d->T, teams) : 0;
    return need < most ? need : most;
}

// f(lanes, vectors a lane) with the numbers as types
template <int LANES, int NV> struct Shape { static constexpr int TEAM = LANES, VECTORS = NV, BLOCK = block_of(LANES); };
template <int V, int LANES, int CHANNELS, typename F> bool shape_is(const Team &t, F f)
{
    if (t.lanes != LANES || t.channels != CHANNELS) return false;
    f(Shape<LANES, CHANNELS / V>());
    return true;
}

template <typename T> hipError_t launch_fwd(const lnorm_desc *d, const lnorm_tensors *t, hipStream_t stream)
{
    constexpr int V = 16 / (int)sizeof(T);
    const Team team = fwd_team(d->C);
    auto launch = [&](auto shape) {
        typedef decltype(shape) S;
        hipLaunchKernelGGL((k_lnorm_fwd<T, S::TEAM, V, S::VECTORS, S::BLOCK>), dim3((unsigned)cdiv(d->T, S::BLOCK / S::TEAM)), dim3(S::BLOCK), 0, stream,
                           d->T, d->C, d->eps, 1.f / (float)d->C, (const T *)t->x, (const T *)t->residual, (const T *)t->w, (const T *)t->b, (T *)t->y,
                           (T *)t->total, (float *)t->mean, (float *)t->rstd);
    };
    const bool found = shape_is<V, 64, 8>(team, launch) || shape_is<V, 64, 16>(team, launch) || shape_is<V, 64, 32>(team, launch) ||
                       shape_is<V, 256, 16>(team, launch) || shape_is<V, 256, 32>(team, launch) || shape_is<V, 1024, 16>(team, launch);
    return found ? hipGetLastError() : hipErrorInvalidValue;
}

template <typename T> hipError_t launch_bwd(const lnorm_desc *d, const lnorm_tensors *t, float *partials, hipStream_t stream)
{
    constexpr int V = 16 / (int)sizeof(T);
    const Team team = bwd_team(d->C);
    auto launch = [&](auto shape) {
        typedef decltype(shape) S;
        const size_t lds = S::BLOCK > S::TEAM && partials ? 2 * (size_t)d->C * sizeof(float) : 0;
        hipLaunchKernelGGL((k_lnorm_bwd<T, S::TEAM, V, S::VECTORS, S::BLOCK>), dim3((unsigned)bwd_blocks(d)), dim3(S::BLOCK), lds, stream, d->T, d->C,
                           1.f / (float)d->C, (const T *)t->x, (const T *)t->w, (const float *)t->mean, (const float *)t->rstd, (const T *)t->dy,
                           (const T *)t->dtotal, (T *)t->dx, partials);
    };
    const bool found = shape_is<V, 64, 8>(team, launch) || shape_is<V, 64, 16>(team, launch) || shape_is<V, 256, 8>(team, launch) ||
                       shape_is<V, 256, 16>(team, launch) || shape_is<V, 1024, 8>(team, launch) || shape_is<V, 1024, 16>(team, launch);
    return found ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace

}  // namespace dwc

using namespace dwc;

extern "C" {

int lnorm_fwd(const lnorm_desc *desc, const lnorm_tensors *t, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t) return DWCONV_ERR_NULL;
    if (desc->T == 0) return DWCONV_OK;
    if (!t->x || !t->y || (t->residual && !t->total) || !t->mean != !t->rstd) return DWCONV_ERR_NULL;
    for (const void *p : {t->x, t->residual, t->w, t->b, (const void *)t->y, (const void *)t->total})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    if (unaligned4(t->mean) || unaligned4(t->rstd)) return DWCONV_ERR_ALIGN;
    const hipError_t e = desc->dtype == DWCONV_F32 ? launch_fwd<float>(desc, t, (hipStream_t)stream) : launch_fwd<bf16_t>(desc, t, (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

size_t lnorm_bwd_workspace_bytes(const lnorm_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    return (size_t)bwd_blocks(desc) * 2 * (size_t)desc->C * sizeof(float);
}

int lnorm_bwd(const lnorm_desc *desc, const lnorm_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || !t->dw != !t->db) return DWCONV_ERR_NULL;
    if (desc->T > 0 && (!t->x || !t->mean || !t->rstd || !t->dy || !t->dx)) return DWCONV_ERR_NULL;
    for (const void *p : {t->x, t->w, t->dy, t->dtotal, (const void *)t->dx})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    for (const void *p : {(const void *)t->mean, (const void *)t->rstd, (const void *)t->dw, (const void *)t->db})
        if (unaligned4(p)) return DWCONV_ERR_ALIGN;
    const size_t need = lnorm_bwd_workspace_bytes(desc);
    if (t->dw && need) {
        if (!workspace || workspace_bytes < need) return DWCONV_ERR_WORKSPACE;
        if (unaligned16(workspace)) return DWCONV_ERR_ALIGN;
    }
    float *const partials = t->dw ? (float *)workspace : nullptr;
    hipError_t e = hipSuccess;
    if (desc->T > 0)
        e = desc->dtype == DWCONV_F32 ? launch_bwd<float>(desc, t, partials, (hipStream_t)stream) : launch_bwd<bf16_t>(desc, t, partials, (hipStream_t)stream);
    if (e == hipSuccess && t->dw)
        e = launch_sum_partials(partials, bwd_blocks(desc), desc->C, 2ll * desc->C, 2ll * desc->C, (float *)t->dw, (float *)t->db, nullptr,
                                (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

}  // extern "C"
