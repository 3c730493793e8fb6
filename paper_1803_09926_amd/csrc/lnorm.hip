// Layer norm over the channels of each token, forward and backward.  The contract stands in include/seqops.h.
//
// A team of lanes (a wavefront, or a block of 2 to 16 of them) holds a row in registers, V consecutive channels a vector and NV vectors a lane, so
// that the row is read once, the variance is taken about the mean that is already known (two sums over the team, no cancellation), and all is written once.
// Both passes are bound by memory: 32768 x 1024 in bf16 with a residual takes 47.1 us, 5.7 TB/s, where a large copy reaches 5.2; the backward pass at
// 9999 x 1536 in fp32 35 us, 5.3 TB/s, and 4.7 for the sum of its partials.  Above 8192 channels the backward pass is bound by spills instead: 16 channels a lane of
// 1024 lanes need more than the 128 registers there, and 4096 x 16384 takes 245 us in bf16 (1.6 TB/s) and 432 in fp32 (1.9).
//
// The weight's gradient is a sum over rows: each lane keeps the sums of its own channels over all rows that its team walks, the teams of a block add
// theirs in LDS one after the other, and the blocks' partials meet in seq_sum.hip.
#include "seq_common.hpp"
#include <initializer_list>

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

template <typename T, int TEAM, int V, int NV, int BLOCK, bool WHOLE>
__global__ __launch_bounds__(BLOCK) void k_lnorm_fwd(int rows, int C, float eps, float inv_c, const T *__restrict__ x, const T *__restrict__ residual,
                                                     const T *__restrict__ w, const T *__restrict__ b, T *__restrict__ y, T *__restrict__ total,
                                                     float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    typedef Part<T, V, WHOLE> P;
    __shared__ float lds[2][TEAM / 64];
    const int lane = threadIdx.x % TEAM;
    const long long row = (long long)blockIdx.x * (BLOCK / TEAM) + threadIdx.x / TEAM;
    if (row >= rows) return;   // (whole wavefronts; a block of one team is always inside)
    P in[NV], more[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) in[j].load(x + row * C, C, (j * TEAM + lane) * V);
    float s[NV][V], sum = 0.f;
    if (residual) {
#pragma unroll
        for (int j = 0; j < NV; ++j) more[j].load(residual + row * C, C, (j * TEAM + lane) * V);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] = in[j].at(i) + more[j].at(i);
            P::store(total + row * C, C, (j * TEAM + lane) * V, s[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] = in[j].at(i);
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
    P p[NV];
    if (w) {
#pragma unroll
        for (int j = 0; j < NV; ++j) p[j].load(w, C, (j * TEAM + lane) * V);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) s[j][i] *= w ? rstd * p[j].at(i) : rstd;
    if (b) {
#pragma unroll
        for (int j = 0; j < NV; ++j) p[j].load(b, C, (j * TEAM + lane) * V);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] += p[j].at(i);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) P::store(y + row * C, C, (j * TEAM + lane) * V, s[j]);
}

// Rows are dealt out to the teams of the whole launch in turn; a team asks for its next row before it works on the one in hand.
// partials: [blocks][2][C], or NULL where the weight's gradient is not asked for.
template <typename T, int TEAM, int V, int NV, int BLOCK, bool WHOLE>
__global__ __launch_bounds__(BLOCK) void k_lnorm_bwd(int rows, int C, float inv_c, const T *__restrict__ x, const T *__restrict__ w,
                                                     const float *__restrict__ mean_in, const float *__restrict__ rstd_in, const T *__restrict__ dy,
                                                     const T *__restrict__ dtotal, T *__restrict__ dx, float *__restrict__ partials)
{
    typedef Part<T, V, WHOLE> P;
    constexpr int TEAMS = BLOCK / TEAM;
    __shared__ float lds[2][2 * TEAM / 64];
    extern __shared__ float sums[];            // [2][C], where a block has more than one team
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    P wr[NV];
    float gw[NV][V], gb[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (w) wr[j].load(w, C, (j * TEAM + lane) * V);
#pragma unroll
        for (int i = 0; i < V; ++i) gw[j][i] = gb[j][i] = 0.f;
    }
    struct Row { P x[NV], dy[NV], add[NV]; float mean, rstd; } ahead;
    auto load = [&](long long row) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            ahead.x[j].load(x + row * C, C, (j * TEAM + lane) * V);
            ahead.dy[j].load(dy + row * C, C, (j * TEAM + lane) * V);
        }
        if (dtotal) {
#pragma unroll
            for (int j = 0; j < NV; ++j) ahead.add[j].load(dtotal + row * C, C, (j * TEAM + lane) * V);
        }
        ahead.mean = mean_in[row];
        ahead.rstd = rstd_in[row];
    };
    int turn = 0;
    const long long stride = (long long)gridDim.x * TEAMS;
    long long row = (long long)blockIdx.x * TEAMS + team;
    if (row < rows) load(row);
    for (; row < rows; row += stride, turn ^= 1) {
        const Row r = ahead;
        if (row + stride < rows) load(row + stride);
        float m1 = 0.f, m2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                // beyond the row dy is zero, and so are all products with it
                const float xhat = (r.x[j].at(i) - r.mean) * r.rstd, g = r.dy[j].at(i), gx = g * xhat;
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
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xhat = (r.x[j].at(i) - r.mean) * r.rstd, g = w ? r.dy[j].at(i) * wr[j].at(i) : r.dy[j].at(i);
                o[i] = r.rstd * ((g - m1) - xhat * m2);
            }
            if (dtotal) {
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] += r.add[j].at(i);
            }
            P::store(dx + row * C, C, (j * TEAM + lane) * V, o);
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
    if (d->T > SEQOPS_MAX_T) return DWCONV_ERR_TOO_LARGE;
    return DWCONV_OK;
}

// How many lanes share a row, and how many of its channels a lane has.  A wavefront alone needs no barrier; 16 channels a lane (8 in the backward pass, which
// holds seven values a channel) leave enough wavefronts on a compute unit: 2048 channels of bf16 by 64, 128, 256 lanes forward 26.0, 26.0, 29.1 us (16384
// rows); backward 67, 50, 47 us.  1536 channels of fp32 forward 27.7, 26.5, 25.4 us (9999 rows), backward 60, 41, 40 us.
struct Team { int lanes, channels; };
Team fwd_team(int C)
{
    if (C <= 512) return {64, 8};
    if (C <= 1024) return {64, 16};
    if (C <= 2048) return {128, 16};
    if (C <= 4096) return {256, 16};
    if (C <= 8192) return {512, 16};
    return {1024, 16};
}
// Few rows: a row a block of 128 lanes, 8 x 1024 in bf16 7.5 us, where four rows a block whose sums meet in LDS take 10.8; 600 rows 10.7 and 12.6 us.
constexpr int FEW_ROWS = 1024;
Team bwd_team(int C, int T)
{
    if (C <= 1024 && T <= FEW_ROWS) return {128, 8};
    if (C <= 512) return {64, 8};
    if (C <= 1024) return {64, 16};
    if (C <= 2048) return {256, 8};
    if (C <= 4096) return {512, 8};
    if (C <= 8192) return {1024, 8};
    return {1024, 16};
}
constexpr int block_of(int lanes) { return lanes == 64 ? 256 : lanes; }

// Blocks of the backward pass: two on each of the 256 compute units (one of 1024 lanes), fewer where there are fewer rows.  Each leaves partials that are read again:
// 256, 512, 1024 blocks take 63, 42, 46 us at 9999 x 1536 in fp32, and 61, 47, 57 at 32768 x 1024 in bf16.
int bwd_blocks(const lnorm_desc *d)
{
    const int lanes = bwd_team(d->C, d->T).lanes, teams = block_of(lanes) / lanes, most = lanes == 1024 ? 256 : 512;
    const int need = d->T > 0 ? cdiv(d->T, teams) : 0;
    return need < most ? need : most;
}

// Whether rows are whole vectors of 16 bytes, each aligned to that
bool whole_rows(const lnorm_desc *d, std::initializer_list<const void *> rows)
{
    if (d->C % (d->dtype == DWCONV_F32 ? 4 : 8)) return false;
    for (const void *p : rows)
        if (unaligned16(p)) return false;
    return true;
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
        constexpr int TEAMS = S::BLOCK / S::TEAM;
        constexpr long long MOST = most_blocks(S::BLOCK) * TEAMS;      // rows
        auto run = [&](auto whole) {
            for (long long row = 0; row < d->T; row += MOST) {
                const int rows = (int)(d->T - row < MOST ? d->T - row : MOST);
                auto at = [&](const void *p) { return p ? (const T *)p + row * d->C : nullptr; };
                hipLaunchKernelGGL((k_lnorm_fwd<T, S::TEAM, V, S::VECTORS, S::BLOCK, decltype(whole)::value>), dim3((unsigned)cdiv(rows, TEAMS)), dim3(S::BLOCK),
                                   0, stream, rows, d->C, d->eps, 1.f / (float)d->C, at(t->x), at(t->residual), (const T *)t->w, (const T *)t->b,
                                   (T *)at(t->y), (T *)at(t->total), t->mean ? (float *)t->mean + row : nullptr, t->rstd ? (float *)t->rstd + row : nullptr);
            }
        };
        if (whole_rows(d, {t->x, t->residual, t->w, t->b, t->y, t->total})) run(std::true_type());
        else run(std::false_type());
    };
    const bool found = shape_is<V, 64, 8>(team, launch) || shape_is<V, 64, 16>(team, launch) || shape_is<V, 128, 16>(team, launch) ||
                       shape_is<V, 256, 16>(team, launch) || shape_is<V, 512, 16>(team, launch) || shape_is<V, 1024, 16>(team, launch);
    return found ? hipGetLastError() : hipErrorInvalidValue;
}

template <typename T> hipError_t launch_bwd(const lnorm_desc *d, const lnorm_tensors *t, float *partials, hipStream_t stream)
{
    constexpr int V = 16 / (int)sizeof(T);
    const Team team = bwd_team(d->C, d->T);
    auto launch = [&](auto shape) {
        typedef decltype(shape) S;
        const size_t lds = S::BLOCK > S::TEAM && partials ? 2 * (size_t)d->C * sizeof(float) : 0;
        auto run = [&](auto whole) {
            hipLaunchKernelGGL((k_lnorm_bwd<T, S::TEAM, V, S::VECTORS, S::BLOCK, decltype(whole)::value>), dim3((unsigned)bwd_blocks(d)), dim3(S::BLOCK), lds,
                               stream, d->T, d->C, 1.f / (float)d->C, (const T *)t->x, (const T *)t->w, (const float *)t->mean, (const float *)t->rstd,
                               (const T *)t->dy, (const T *)t->dtotal, (T *)t->dx, partials);
        };
        if (whole_rows(d, {t->x, t->w, t->dy, t->dtotal, t->dx})) run(std::true_type());
        else run(std::false_type());
    };
    const bool found = shape_is<V, 128, 8>(team, launch) || shape_is<V, 64, 8>(team, launch) || shape_is<V, 64, 16>(team, launch) ||
                       shape_is<V, 256, 8>(team, launch) || shape_is<V, 512, 8>(team, launch) || shape_is<V, 1024, 8>(team, launch) ||
                       shape_is<V, 1024, 16>(team, launch);
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
