// The RMS norms after a block and before the next one, with the block's gate, the residual's scale and sum between them, forward and backward.
// The contract stands in include/deltaops.h.
//
// A team of lanes holds a row in registers (seq_rows.hpp), so that everything is read once and written once: two sums over the team a row, one for each norm, the
// second of what the first one's channels become.  Both passes are bound by memory: 32768 rows of 1024 in bf16 52 us (269 MB, 5.1 TB/s), the gradients of 9999 rows of 1536 in bf16
// with all parts 55 us (246 MB, 4.5 TB/s) and 5.7 for the sums of the partials.
//
// The gradients of the three weights are sums over rows: each lane keeps those of its channels over all rows that its team walks, the teams of a block add
// theirs in LDS in turn, and the blocks' partials meet in seq_sum.hip.
#include "../../include/deltaops.h"
#include "seq_rows.hpp"
#include <initializer_list>
#include <math.h>

namespace dwc {

namespace {

struct RnormArgs {
    long long rows;
    int C, post, silu;
    float eps, inv_c, alpha;
    long long x_stride, z_stride;
};

// act(z) and its slope
__device__ __forceinline__ void gate_of(float z, bool silu, float &act, float &slope)
{
    const float q = sigmoid(z);
    if (silu) {
        act = z * q;
        slope = q * (1.f + z * (1.f - q));
    } else {
        act = q;
        slope = q * (1.f - q);
    }
}

template <typename T, int TEAM, int V, int NV, int BLOCK, bool WHOLE>
__global__ __launch_bounds__(BLOCK) void k_rnorm_fwd(RnormArgs a, const T *__restrict__ x, const T *__restrict__ z, const T *__restrict__ residual,
                                                     const T *__restrict__ w1, const T *__restrict__ scale, const T *__restrict__ w2, T *__restrict__ total,
                                                     T *__restrict__ y, float *__restrict__ rstd1, float *__restrict__ rstd2)
{
    typedef Part<T, V, WHOLE> P;
    __shared__ float lds[2][TEAM / 64];
    const int lane = threadIdx.x % TEAM, C = a.C;
    for (long long row = (long long)blockIdx.x * (BLOCK / TEAM) + threadIdx.x / TEAM; row < a.rows; row += (long long)gridDim.x * (BLOCK / TEAM)) {
        P in[NV], gate[NV], more[NV], p[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) in[j].load(x + row * a.x_stride, C, (j * TEAM + lane) * V);
        if (z) {
#pragma unroll
            for (int j = 0; j < NV; ++j) gate[j].load(z + row * a.z_stride, C, (j * TEAM + lane) * V);
        }
        if (residual) {
#pragma unroll
            for (int j = 0; j < NV; ++j) more[j].load(residual + row * C, C, (j * TEAM + lane) * V);
        }
        float s[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] = in[j].at(i);
        float factor = a.alpha;
        if (a.post) {
            float squares = 0.f;                 // (beyond the row all is zero)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) squares += s[j][i] * s[j][i];
            if constexpr (TEAM > 64) __syncthreads();   // the row before has read its sums
            const float r = 1.f / sqrtf(team_sum<TEAM>(squares, lds[0]) * a.inv_c + a.eps);
            if (rstd1 && lane == 0) rstd1[row] = r;
            factor *= r;
            if (w1) {
#pragma unroll
                for (int j = 0; j < NV; ++j) p[j].load(w1, C, (j * TEAM + lane) * V);
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) s[j][i] *= p[j].at(i);
            }
        }
        if (z) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float zz = gate[j].at(i);
                    s[j][i] *= a.silu ? zz * sigmoid(zz) : sigmoid(zz);
                }
        }
        if (scale) {
#pragma unroll
            for (int j = 0; j < NV; ++j) p[j].load(scale, C, (j * TEAM + lane) * V);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) s[j][i] *= p[j].at(i);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[j][i] *= factor;
                if (residual) s[j][i] += more[j].at(i);
            }
            P::store(total + row * C, C, (j * TEAM + lane) * V, s[j]);
        }
        if (!y && !rstd2) continue;
        float squares = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                // (a lane beyond the row has zeros times the row's factor there: no zero where that is infinite)
                s[j][i] = (j * TEAM + lane) * V + i < C ? s[j][i] : 0.f;
                squares += s[j][i] * s[j][i];
            }
        if constexpr (TEAM > 64) { if (!a.post) __syncthreads(); }
        const float r = 1.f / sqrtf(team_sum<TEAM>(squares, lds[1]) * a.inv_c + a.eps);
        if (rstd2 && lane == 0) rstd2[row] = r;
        if (!y) continue;
        if (w2) {
#pragma unroll
            for (int j = 0; j < NV; ++j) p[j].load(w2, C, (j * TEAM + lane) * V);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] *= w2 ? r * p[j].at(i) : r;
            P::store(y + row * C, C, (j * TEAM + lane) * V, s[j]);
        }
    }
}

// Rows are dealt out to the teams of the whole launch in turn; a team asks for its next row before it works on the one in hand.
// partials: [blocks][3][C] (dw1, dscale, dw2), or NULL where none of them is asked for.
template <typename T, int TEAM, int V, int NV, int BLOCK, bool WHOLE>
__global__ __launch_bounds__(BLOCK) void k_rnorm_bwd(RnormArgs a, const T *__restrict__ x, const T *__restrict__ z, const T *__restrict__ w1,
                                                     const T *__restrict__ scale, const T *__restrict__ w2, const T *__restrict__ total,
                                                     const float *__restrict__ rstd1, const float *__restrict__ rstd2, const T *__restrict__ dy,
                                                     const T *__restrict__ dtotal, T *__restrict__ dx, T *__restrict__ dz, T *__restrict__ dresidual,
                                                     float *__restrict__ partials)
{
    typedef Part<T, V, WHOLE> P;
    constexpr int TEAMS = BLOCK / TEAM;
    __shared__ float lds[4][TEAM / 64];
    extern __shared__ float sums[];            // [3][C], where a block has more than one team
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM, C = a.C;
    P w1r[NV], scaler[NV], w2r[NV];
    float g1[NV][V], gs[NV][V], g2[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (w1) w1r[j].load(w1, C, (j * TEAM + lane) * V);
        if (scale) scaler[j].load(scale, C, (j * TEAM + lane) * V);
        if (w2) w2r[j].load(w2, C, (j * TEAM + lane) * V);
#pragma unroll
        for (int i = 0; i < V; ++i) g1[j][i] = gs[j][i] = g2[j][i] = 0.f;
    }
    struct Row { P x[NV], z[NV], total[NV], dy[NV], add[NV]; float r1, r2; } ahead;
    auto load = [&](long long row) {
        if (x) {
#pragma unroll
            for (int j = 0; j < NV; ++j) ahead.x[j].load(x + row * a.x_stride, C, (j * TEAM + lane) * V);
        }
        if (z) {
#pragma unroll
            for (int j = 0; j < NV; ++j) ahead.z[j].load(z + row * a.z_stride, C, (j * TEAM + lane) * V);
        }
        if (dy) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                ahead.total[j].load(total + row * C, C, (j * TEAM + lane) * V);
                ahead.dy[j].load(dy + row * C, C, (j * TEAM + lane) * V);
            }
            ahead.r2 = rstd2[row];
        }
        if (dtotal) {
#pragma unroll
            for (int j = 0; j < NV; ++j) ahead.add[j].load(dtotal + row * C, C, (j * TEAM + lane) * V);
        }
        if (a.post) ahead.r1 = rstd1[row];
    };
    int turn = 0;
    const long long stride = (long long)gridDim.x * TEAMS;
    long long row = (long long)blockIdx.x * TEAMS + team;
    if (row < a.rows) load(row);
    for (; row < a.rows; row += stride, turn ^= 2) {
        const Row r = ahead;
        if (row + stride < a.rows) load(row + stride);
        float ds[NV][V];
        if (dy) {
            float m = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float n = r.total[j].at(i) * r.r2, gn = r.dy[j].at(i) * n;
                    g2[j][i] += gn;
                    m += w2 ? gn * w2r[j].at(i) : gn;
                }
            m = team_sum<TEAM>(m, lds[turn]) * a.inv_c;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float g = w2 ? r.dy[j].at(i) * w2r[j].at(i) : r.dy[j].at(i);
                    ds[j][i] = r.r2 * (g - r.total[j].at(i) * r.r2 * m);
                }
            if (dtotal) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) ds[j][i] += r.add[j].at(i);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) ds[j][i] = r.add[j].at(i);
        }
        if (dresidual) {
#pragma unroll
            for (int j = 0; j < NV; ++j) P::store(dresidual + row * C, C, (j * TEAM + lane) * V, ds[j]);
        }
        // from here on ds is the gradient of scale * p * act(z), then of p
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float oz[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float act = 1.f, slope = 0.f;
                if (z) gate_of(r.z[j].at(i), a.silu, act, slope);
                const float n = !x ? 0.f : a.post ? r.x[j].at(i) * r.r1 : r.x[j].at(i), p = w1 ? n * w1r[j].at(i) : n;
                float d = a.alpha * ds[j][i];
                gs[j][i] += d * p * act;
                if (scale) d *= scaler[j].at(i);
                oz[i] = d * p * slope;
                d *= act;
                g1[j][i] += d * n;
                if (w1) d *= w1r[j].at(i);
                m += d * n;
                ds[j][i] = d;
            }
            if (z) P::store(dz + row * a.z_stride, C, (j * TEAM + lane) * V, oz);
        }
        if (a.post) {
            m = team_sum<TEAM>(m, lds[turn + 1]) * a.inv_c;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) ds[j][i] = r.r1 * (ds[j][i] - r.x[j].at(i) * r.r1 * m);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) P::store(dx + row * a.x_stride, C, (j * TEAM + lane) * V, ds[j]);
        // A row's sums lie in two of four places, and its neighbours' in the others: a wavefront that is a row ahead has passed this row's barriers.  With one barrier
        // a row (one of the norms alone) that holds as well; with none nothing is summed.
    }
    if (!partials) return;
    float *out = partials + (long long)blockIdx.x * 3 * C;
    if constexpr (TEAMS > 1) {
        for (int k = 0; k < TEAMS; ++k) {      // one team after the other: a fixed order
            if (team == k) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = (j * TEAM + lane) * V + i;
                        if (c >= C) continue;
                        sums[c] = k ? sums[c] + g1[j][i] : g1[j][i];
                        sums[C + c] = k ? sums[C + c] + gs[j][i] : gs[j][i];
                        sums[2 * C + c] = k ? sums[2 * C + c] + g2[j][i] : g2[j][i];
                    }
            }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < 3 * C; i += BLOCK) out[i] = sums[i];
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (j * TEAM + lane) * V + i;
                if (c >= C) continue;
                out[c] = g1[j][i];
                out[C + c] = gs[j][i];
                out[2 * C + c] = g2[j][i];
            }
    }
}

int validate(const rnorm_desc *d)
{
    if (!d) return DWCONV_ERR_NULL;
    if (d->dtype != DWCONV_F32 && d->dtype != DWCONV_BF16) return DWCONV_ERR_BAD_ENUM;
    if ((d->post | 1) != 1 || (d->silu | 1) != 1 || d->reserved != 0) return DWCONV_ERR_BAD_ENUM;
    if (d->T < 0 || d->C < 1 || !(d->eps >= 0.f) || !isfinite(d->alpha)) return DWCONV_ERR_BAD_DIM;
    if (d->C > RNORM_MAX_C) return DWCONV_ERR_UNSUPPORTED;
    if (d->T > SEQOPS_MAX_T || d->x_stride > SEQOPS_MAX_STRIDE || d->z_stride > SEQOPS_MAX_STRIDE) return DWCONV_ERR_TOO_LARGE;
    if (d->T > 1 && (d->x_stride < d->C || d->z_stride < d->C)) return DWCONV_ERR_BAD_DIM;
    return DWCONV_OK;
}

// (32768 x 1024 in bf16: a wavefront a row 52.3 us, two 53.4)
Team fwd_team(int C)
{
    if (C <= 512) return {64, 8};
    if (C <= 1024) return {64, 16};
    if (C <= 2048) return {128, 16};
    if (C <= 4096) return {256, 16};
    return {512, 16};
}
Team bwd_team(int C)
{
    if (C <= 512) return {64, 8};
    if (C <= 1024) return {128, 8};
    if (C <= 2048) return {256, 8};
    if (C <= 4096) return {512, 8};
    return {1024, 8};
}
// Blocks of the backward pass, fewer where there are fewer rows; each leaves partials that are read again (9999 x 1536 in bf16, with their sums: 256 blocks 77 us, 512 59,
// 1024 72).
int bwd_blocks(const rnorm_desc *d)
{
    const int lanes = bwd_team(d->C).lanes, teams = block_of(lanes) / lanes, most = lanes == 1024 ? 256 : 512;
    const int need = d->T > 0 ? cdiv(d->T, teams) : 0;
    return need < most ? need : most;
}

// Whether rows are whole vectors of 16 bytes, each aligned to that
bool whole_rows(const rnorm_desc *d, std::initializer_list<const void *> rows, bool x, bool z)
{
    const int v = d->dtype == DWCONV_F32 ? 4 : 8;
    if (d->C % v || (x && d->T > 1 && d->x_stride % v) || (z && d->T > 1 && d->z_stride % v)) return false;
    for (const void *p : rows)
        if (unaligned16(p)) return false;
    return true;
}

RnormArgs args_of(const rnorm_desc *d)
{
    return {d->T, d->C, d->post, d->silu, d->eps, 1.f / (float)d->C, d->alpha, d->x_stride, d->z_stride};
}

template <typename T> hipError_t launch_fwd(const rnorm_desc *d, const rnorm_tensors *t, hipStream_t stream)
{
    constexpr int V = 16 / (int)sizeof(T);
    const Team team = fwd_team(d->C);
    auto launch = [&](auto shape) {
        typedef decltype(shape) S;
        constexpr int TEAMS = S::BLOCK / S::TEAM;
        const long long need = cdiv(d->T, TEAMS), most = most_blocks(S::BLOCK);
        auto run = [&](auto whole) {
            hipLaunchKernelGGL((k_rnorm_fwd<T, S::TEAM, V, S::VECTORS, S::BLOCK, decltype(whole)::value>), dim3((unsigned)(need < most ? need : most)),
                               dim3(S::BLOCK), 0, stream, args_of(d), (const T *)t->x, (const T *)t->z, (const T *)t->residual, (const T *)t->w1,
                               (const T *)t->scale, (const T *)t->w2, (T *)t->total, (T *)t->y, (float *)t->rstd1, (float *)t->rstd2);
        };
        if (whole_rows(d, {t->x, t->z, t->residual, t->w1, t->scale, t->w2, t->total, t->y}, true, t->z)) run(std::true_type());
        else run(std::false_type());
    };
    const bool found = shape_is<V, 64, 8>(team, launch) || shape_is<V, 64, 16>(team, launch) || shape_is<V, 128, 16>(team, launch) ||
                       shape_is<V, 256, 16>(team, launch) || shape_is<V, 512, 16>(team, launch);
    return found ? hipGetLastError() : hipErrorInvalidValue;
}

template <typename T> hipError_t launch_bwd(const rnorm_desc *d, const rnorm_tensors *t, float *partials, hipStream_t stream)
{
    constexpr int V = 16 / (int)sizeof(T);
    const Team team = bwd_team(d->C);
    // x is read where it is normalised, gated or scaled
    const void *x = d->post || t->z || t->scale ? t->x : nullptr;
    auto launch = [&](auto shape) {
        typedef decltype(shape) S;
        const size_t lds = S::BLOCK > S::TEAM && partials ? 3 * (size_t)d->C * sizeof(float) : 0;
        auto run = [&](auto whole) {
            hipLaunchKernelGGL((k_rnorm_bwd<T, S::TEAM, V, S::VECTORS, S::BLOCK, decltype(whole)::value>), dim3((unsigned)bwd_blocks(d)), dim3(S::BLOCK), lds,
                               stream, args_of(d), (const T *)x, (const T *)t->z, (const T *)t->w1, (const T *)t->scale, (const T *)t->w2, (const T *)t->total,
                               (const float *)t->rstd1, (const float *)t->rstd2, (const T *)t->dy, (const T *)t->dtotal, (T *)t->dx, (T *)t->dz,
                               (T *)t->dresidual, partials);
        };
        if (whole_rows(d, {x, t->z, t->w1, t->scale, t->w2, t->total, t->dy, t->dtotal, t->dx, t->dz, t->dresidual}, true, t->z)) run(std::true_type());
        else run(std::false_type());
    };
    const bool found = shape_is<V, 64, 8>(team, launch) || shape_is<V, 128, 8>(team, launch) || shape_is<V, 256, 8>(team, launch) ||
                       shape_is<V, 512, 8>(team, launch) || shape_is<V, 1024, 8>(team, launch);
    return found ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace

}  // namespace dwc

using namespace dwc;

extern "C" {

int rnorm_fwd(const rnorm_desc *desc, const rnorm_tensors *t, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t) return DWCONV_ERR_NULL;
    if (desc->T == 0) return DWCONV_OK;
    if (!t->x || !t->total || (t->w1 && !desc->post)) return DWCONV_ERR_NULL;
    for (const void *p : {t->x, t->z, t->residual, t->w1, t->scale, t->w2, (const void *)t->total, (const void *)t->y})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    if (unaligned4(t->rstd1) || unaligned4(t->rstd2)) return DWCONV_ERR_ALIGN;
    const hipError_t e = desc->dtype == DWCONV_F32 ? launch_fwd<float>(desc, t, (hipStream_t)stream) : launch_fwd<bf16_t>(desc, t, (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

size_t rnorm_bwd_workspace_bytes(const rnorm_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    return (size_t)bwd_blocks(desc) * 3 * (size_t)desc->C * sizeof(float);
}

int rnorm_bwd(const rnorm_desc *desc, const rnorm_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || (t->dw1 && !desc->post) || (t->w1 && !desc->post)) return DWCONV_ERR_NULL;
    if (desc->T > 0) {
        if (!t->dx || (!t->dy && !t->dtotal) || (t->dy && (!t->total || !t->rstd2)) || (desc->post && !t->rstd1)) return DWCONV_ERR_NULL;
        if (((desc->post || t->z || t->scale) && !t->x) || !t->z != !t->dz) return DWCONV_ERR_NULL;
        if ((t->dw2 && !t->dy) || (t->dscale && !t->scale)) return DWCONV_ERR_NULL;
    }
    for (const void *p : {t->x, t->z, t->w1, t->scale, t->w2, (const void *)t->total, t->dy, t->dtotal, (const void *)t->dx, (const void *)t->dz,
                          (const void *)t->dresidual})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    for (const void *p : {t->rstd1, t->rstd2, t->dw1, t->dscale, t->dw2})
        if (unaligned4(p)) return DWCONV_ERR_ALIGN;
    const bool sums = t->dw1 || t->dscale || t->dw2;
    const size_t need = rnorm_bwd_workspace_bytes(desc);
    if (sums && need) {
        if (!workspace || workspace_bytes < need) return DWCONV_ERR_WORKSPACE;
        if (unaligned16(workspace)) return DWCONV_ERR_ALIGN;
    }
    float *const partials = sums ? (float *)workspace : nullptr;
    hipError_t e = hipSuccess;
    if (desc->T > 0)
        e = desc->dtype == DWCONV_F32 ? launch_bwd<float>(desc, t, partials, (hipStream_t)stream) : launch_bwd<bf16_t>(desc, t, partials, (hipStream_t)stream);
    if (e == hipSuccess && sums)
        e = launch_sum_partials(partials, bwd_blocks(desc), desc->C, 2ll * desc->C, 3ll * desc->C, (float *)t->dw1, (float *)t->dscale, (float *)t->dw2,
                                (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

}  // extern "C"
