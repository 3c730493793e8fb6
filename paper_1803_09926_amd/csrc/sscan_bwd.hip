// Selective state space scan, backward.  See sscan.hpp for the layout of the work, include/seqops.h for the contract.
//
// With g the gradient that arrives at h[t] (from y[t], and from h[t+1] times its decay), v = y before the gate and dv its gradient:
//   g += dv * C[t];  dC[t] = sum_c dv * h[t];  dB[t] = sum_c g * delta * x;  dx = D * dv + delta * sum_n g * B[t]
//   r = g * decay * h[t-1];  ddelta = x * sum_n g * B[t] + sum_n r * A;  dA += r * delta;  then g *= decay for the token before
// A tile is the 16 tokens between two states that the forward pass kept: a lane computes its 16 decays and states again, keeps them in registers (decay *
// h[t-1] is exact that way; the difference h[t] - delta x B would cancel), and walks back through them.  The sums over channels (dB, dC) go through the
// lanes of a wavefront by row swaps and moves, two instructions for the first two halvings, then through LDS over the block's wavefronts, then over the
// blocks in a second kernel.  Bound by its vector instructions, about three times the forward pass's.
//
// Where the tokens are split, a first pass finds the gradient that each part hands to the state before it, as the forward pass does with the states.
#include "sscan.hpp"

namespace dwc {

namespace {

template <int LPC> struct BackTile {
    static constexpr int CHANNELS = 256 / LPC, TOKENS = KEPT_EVERY, EACH = TOKENS / LPC, STATES = 4 * LPC, LANES = 256 / TOKENS;
    static constexpr int SHARED = (TOKENS * STATES + 255) / 256;
};

struct BackIn {
    const void *x, *dt, *B, *C, *z, *dy;
    const float *A, *D, *dt_bias, *init, *kept;
};
struct BackOut {
    void *dx, *ddt, *dz;
    float *ends, *sums, *dA, *shared;    // as BwdSpace has them
};

// The first pass over the parts: from the last token of a part back to its first, the gradient that leaves the part, from zero, and the sum of step sizes.
template <typename T, int LPC>
__global__ __launch_bounds__(256) void k_sscan_bwd_carry(Scan g, BackIn in, BackOut out)
{
    constexpr int CHANNELS = 256 / LPC, TOKENS = LPC == 2 ? 16 : 32, EACH = TOKENS * CHANNELS / 256, STATES = 4 * LPC, LANES = 256 / TOKENS;
    constexpr int SHARED = (TOKENS * STATES + 255) / 256;
    __shared__ float2 du[TOKENS][CHANNELS];                          // step size, dv
    __shared__ float4 Cs[TOKENS][LPC];
    const ScanBlock at = scan_block(g);
    const int part = at.part + 1;                                    // (nothing comes before part 0)
    const int lane = threadIdx.x & 63, q = lane % LPC, wv = threadIdx.x >> 6;
    const int mine = wv * (64 / LPC) + lane / LPC, in_group = at.block * CHANNELS + mine, chan = at.group * g.per_group + in_group;
    const bool valid = in_group < g.per_group;
    const int row = threadIdx.x / LANES, col = threadIdx.x % LANES * EACH;
    const int first_chan = at.group * g.per_group + at.block * CHANNELS + col, n = g.per_group - at.block * CHANNELS - col;
    const int t0 = (int)((long long)part * g.part), t1 = g.seq.T - t0 < g.part ? g.seq.T : t0 + g.part;
    if (t1 <= t0) return;

    float a2[4], gr[4] = {0.f, 0.f, 0.f, 0.f}, bias[EACH];
#pragma unroll
    for (int i = 0; i < 4; ++i) a2[i] = valid && 4 * q + i < g.N ? in.A[(long long)chan * g.N + 4 * q + i] * LOG2E : 0.f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) bias[i] = in.dt_bias && i < n ? in.dt_bias[first_chan + i] : 0.f;

    Some<T, EACH> rdt, rz, rdy;
    float rc[SHARED];
    auto load = [&](int tile) {
        const int t = tile + row, m = t < t1 ? n : 0;
        rdt.load((const T *)in.dt + (long long)t * g.dts + first_chan, m);
        rdy.load((const T *)in.dy + (long long)t * g.ys + first_chan, m);
        if (in.z) rz.load((const T *)in.z + (long long)t * g.zs + first_chan, m);
#pragma unroll
        for (int i = 0; i < SHARED; ++i) {
            const int e = threadIdx.x + 256 * i, tb = tile + e / STATES, k = e % STATES;
            rc[i] = e < TOKENS * STATES && tb < t1 && k < g.N ? ldf((const T *)in.C + (long long)tb * g.cs + (long long)at.group * g.N + k) : 0.f;
        }
    };
    float total = 0.f;
    int tile = t0 + (t1 - t0 - 1) / TOKENS * TOKENS;
    load(tile);
    for (; tile >= t0; tile -= TOKENS) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float d = tile + row < t1 ? step_size(g, rdt.at(i) + bias[i]) : 0.f;
            float dv = rdy.at(i);
            if (in.z) { const float zv = rz.at(i); dv *= zv * sigmoid(zv); }
            du[row][col + i] = make_float2(d, dv);
        }
#pragma unroll
        for (int i = 0; i < SHARED; ++i) {
            const int e = threadIdx.x + 256 * i;
            if (e < TOKENS * STATES) reinterpret_cast<float *>(Cs)[e] = rc[i];
        }
        if (tile > t0) load(tile - TOKENS);
        __syncthreads();
        const int s = g.seq.of(tile);
        const bool any = g.seq.start(s) == tile || g.seq.start(s + 1) < tile + TOKENS;
        const uint32_t firsts = any ? first_tokens(g.seq, tile, TOKENS, t1) : 0u;
        auto walk = [&](auto special) {
#pragma unroll 4
            for (int t = TOKENS - 1; t >= 0; --t) {
                if constexpr (decltype(special)::value) {
                    if (tile + t >= t1) continue;
                }
                const float2 d = du[t][mine];
                const float4 c = Cs[t][q];
                const float cv[4] = {c.x, c.y, c.z, c.w};
                total += d.x;
#pragma unroll
                for (int i = 0; i < 4; ++i) gr[i] = fmaf(d.y, cv[i], gr[i]) * exp2_fast(d.x * a2[i]);
                if constexpr (decltype(special)::value) {
                    if (firsts >> t & 1) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) gr[i] = 0.f;
                    }
                }
            }
        };
        if (firsts || tile + TOKENS > t1) walk(std::true_type());
        else walk(std::false_type());
        __syncthreads();
    }
    if (valid) {
        *reinterpret_cast<float4 *>(out.ends + ((long long)part * g.C + chan) * STATES + 4 * q) = make_float4(gr[0], gr[1], gr[2], gr[3]);
        if (q == 0) out.sums[(long long)part * g.C + chan] = total;
    }
}

template <typename T, int LPC>
__global__ __launch_bounds__(256) void k_sscan_bwd(Scan g, BackIn in, BackOut out)
{
    typedef BackTile<LPC> S;
    __shared__ float4 slot[S::TOKENS][S::CHANNELS];                  // step size, step size * x, dv; then sum g B, sum r A, -, sum C h
    __shared__ float4 Bs[S::TOKENS][LPC], Cs[S::TOKENS][LPC];
    __shared__ float red[4][S::TOKENS][2 * S::STATES];               // dB and dC of each wavefront's channels
    const ScanBlock at = scan_block(g);
    const int lane = threadIdx.x & 63, q = lane % LPC, wv = threadIdx.x >> 6;
    const int mine = wv * (64 / LPC) + lane / LPC, in_group = at.block * S::CHANNELS + mine, chan = at.group * g.per_group + in_group;
    const bool valid = in_group < g.per_group;
    const int row = threadIdx.x / S::LANES, col = threadIdx.x % S::LANES * S::EACH;
    const int first_chan = at.group * g.per_group + at.block * S::CHANNELS + col, n = g.per_group - at.block * S::CHANNELS - col;
    const int t0 = (int)((long long)at.part * g.part), t1 = g.seq.T - t0 < g.part ? g.seq.T : t0 + g.part;
    if (t1 <= t0) return;

    float a2[4], gr[4] = {0.f, 0.f, 0.f, 0.f}, dA[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) a2[i] = valid && 4 * q + i < g.N ? in.A[(long long)chan * g.N + 4 * q + i] * LOG2E : 0.f;
    float bias[S::EACH], skip[S::EACH], dskip[S::EACH], dbias[S::EACH];
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) {
        bias[i] = in.dt_bias && i < n ? in.dt_bias[first_chan + i] : 0.f;
        skip[i] = in.D && i < n ? in.D[first_chan + i] : 0.f;
        dskip[i] = dbias[i] = 0.f;
    }

    if (out.ends && t1 < g.seq.T) {                                  // what the parts behind hand back to the sequence that goes on there
        const int end = g.seq.start(g.seq.of(t1 - 1) + 1);
        float decay[4] = {1.f, 1.f, 1.f, 1.f};
        for (int p = at.part + 1; p < g.parts && (long long)p * g.part < end; ++p) {
            if (!valid) continue;
            const float4 e = *reinterpret_cast<const float4 *>(out.ends + ((long long)p * g.C + chan) * S::STATES + 4 * q);
            const float sum = out.sums[(long long)p * g.C + chan];
            const float v[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                gr[i] = fmaf(decay[i], v[i], gr[i]);
                decay[i] *= exp2_fast(a2[i] * sum);
            }
        }
    }

    auto init_of = [&](int s, float (&h)[4]) {
        const float *p = in.init + ((long long)s * g.C + chan) * g.N + 4 * q;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = in.init && valid && 4 * q + i < g.N ? p[i] : 0.f;
    };

    Some<T, S::EACH> rx, rdt, rz, rdy;
    float rb[S::SHARED], rc[S::SHARED];
    float4 rh = make_float4(0.f, 0.f, 0.f, 0.f);
    auto load = [&](int tile) {
        const int t = tile + row, m = t < t1 ? n : 0;
        rx.load((const T *)in.x + (long long)t * g.xs + first_chan, m);
        rdt.load((const T *)in.dt + (long long)t * g.dts + first_chan, m);
        rdy.load((const T *)in.dy + (long long)t * g.ys + first_chan, m);
        if (in.z) rz.load((const T *)in.z + (long long)t * g.zs + first_chan, m);
#pragma unroll
        for (int i = 0; i < S::SHARED; ++i) {
            const int e = threadIdx.x + 256 * i, tb = tile + e / S::STATES, k = e % S::STATES;
            const bool inside = e < S::TOKENS * S::STATES && tb < t1 && k < g.N;
            rb[i] = inside ? ldf((const T *)in.B + (long long)tb * g.bs + (long long)at.group * g.N + k) : 0.f;
            rc[i] = inside ? ldf((const T *)in.C + (long long)tb * g.cs + (long long)at.group * g.N + k) : 0.f;
        }
        if (valid) rh = *reinterpret_cast<const float4 *>(in.kept + ((long long)(tile / KEPT_EVERY) * g.C + chan) * S::STATES + 4 * q);
    };

    int tile = t0 + (t1 - t0 - 1) / S::TOKENS * S::TOKENS;
    load(tile);
    for (; tile >= t0; tile -= S::TOKENS) {
        const Some<T, S::EACH> kx = rx, kdt = rdt, kz = rz, kdy = rdy;
        const float hin[4] = {rh.x, rh.y, rh.z, rh.w};
        const int m = tile + row < t1 ? n : 0;
        float delta[S::EACH];
#pragma unroll
        for (int i = 0; i < S::EACH; ++i) {
            delta[i] = m > 0 ? step_size(g, kdt.at(i) + bias[i]) : 0.f;
            float dv = kdy.at(i);
            if (in.z) { const float zv = kz.at(i); dv *= zv * sigmoid(zv); }
            slot[row][col + i] = make_float4(delta[i], delta[i] * kx.at(i), dv, 0.f);
        }
#pragma unroll
        for (int i = 0; i < S::SHARED; ++i) {
            const int e = threadIdx.x + 256 * i;
            if (e < S::TOKENS * S::STATES) {
                reinterpret_cast<float *>(Bs)[e] = rb[i];
                reinterpret_cast<float *>(Cs)[e] = rc[i];
            }
        }
        if (tile > t0) load(tile - S::TOKENS);
        __syncthreads();
        const int s = g.seq.of(tile);
        const bool any = g.seq.start(s) == tile || g.seq.start(s + 1) < tile + S::TOKENS;
        const uint32_t firsts = any ? first_tokens(g.seq, tile, S::TOKENS, t1) : 0u;

        auto walk = [&](auto special) {
            constexpr bool SPECIAL = decltype(special)::value;
            float decay[S::TOKENS][4], h[S::TOKENS][4], sums[LPC], more[LPC];
#pragma unroll
            for (int t = 0; t < S::TOKENS; ++t) {
                const float4 v = slot[t][mine], b = Bs[t][q], c = Cs[t][q];
                const float bv[4] = {b.x, b.y, b.z, b.w}, cv[4] = {c.x, c.y, c.z, c.w};
                float before[4], sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) before[i] = t ? h[t ? t - 1 : 0][i] : hin[i];
                if constexpr (SPECIAL) {
                    if (firsts >> t & 1) init_of(g.seq.of(tile + t), before);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    decay[t][i] = exp2_fast(v.x * a2[i]);
                    h[t][i] = fmaf(decay[t][i], before[i], v.y * bv[i]);
                    sum = fmaf(cv[i], h[t][i], sum);
                }
                sums[t % LPC] = sum;
                if (t % LPC == LPC - 1 && in.z) slot[t - (LPC - 1) + q][mine].w = transpose_sum<LPC>(sums, q);
            }
#pragma unroll
            for (int t = S::TOKENS - 1; t >= 0; --t) {
                if (SPECIAL && tile + t >= t1) {                     // behind the last token
                    sums[t % LPC] = more[t % LPC] = 0.f;
                } else {
                    const float4 v = slot[t][mine], b = Bs[t][q], c = Cs[t][q];
                    const float bv[4] = {b.x, b.y, b.z, b.w}, cv[4] = {c.x, c.y, c.z, c.w};
                    float before[4], db[4], dc[4], sg = 0.f, sa = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) before[i] = t ? h[t ? t - 1 : 0][i] : hin[i];
                    if constexpr (SPECIAL) {
                        if (firsts >> t & 1) init_of(g.seq.of(tile + t), before);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        gr[i] = fmaf(v.z, cv[i], gr[i]);
                        db[i] = gr[i] * v.y;
                        dc[i] = v.z * h[t][i];
                        sg = fmaf(gr[i], bv[i], sg);
                        const float r = gr[i] * (decay[t][i] * before[i]);
                        sa = fmaf(r, a2[i], sa);
                        dA[i] = fmaf(r, v.x, dA[i]);
                        gr[i] *= decay[t][i];
                    }
                    if constexpr (SPECIAL) {
                        if (firsts >> t & 1) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) gr[i] = 0.f;
                        }
                    }
                    sums[t % LPC] = sg;
                    more[t % LPC] = sa;
                    // over the wavefront's channels: after the halves (dB below, dC above) and the rows (state 2j below 2j + 1) a lane has two states' sums
                    const float w0 = rows_join(halves_join(db[0], dc[0]), halves_join(db[1], dc[1]));
                    const float w1 = rows_join(halves_join(db[2], dc[2]), halves_join(db[3], dc[3]));
                    float *const to = &red[wv][t][(lane >> 5) * S::STATES + 4 * q + (lane >> 4 & 1)];
                    if constexpr (LPC == 16) {
                        to[0] = w0;
                        to[2] = w1;
                    } else {
                        const float u0 = w0 + lane_move<DPP_ROR8>(w0), u1 = w1 + lane_move<DPP_ROR8>(w1);   // (every lane moves: no branch here)
                        float w = lane & 8 ? u1 : u0;
                        if constexpr (LPC <= 4) w += lane_move<0x104>(w);        // four lanes further up; used in the lower four of eight
                        if constexpr (LPC == 2) w += lane_move<DPP_XOR2>(w);
                        if ((lane & 7) < LPC) to[lane & 8 ? 2 : 0] = w;
                    }
                }
                if (t % LPC == 0) {
                    const float a = transpose_sum<LPC>(sums, q), b2 = transpose_sum<LPC>(more, q);
                    slot[t + q][mine].x = a;
                    slot[t + q][mine].y = b2 * LN2;
                }
            }
        };
        if (firsts || tile + S::TOKENS > t1) walk(std::true_type());
        else walk(std::false_type());
        __syncthreads();

        {
            float dx[S::EACH], dd[S::EACH], dz[S::EACH];
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) {
                const float4 v = slot[row][col + i];
                const float xv = kx.at(i), dout = kdy.at(i);
                float dv = dout;
                if (in.z) {
                    const float zv = kz.at(i), sz = sigmoid(zv);
                    dv *= zv * sz;
                    dz[i] = dout * fmaf(skip[i], xv, v.w) * (sz + zv * sz * (1.f - sz));
                }
                dx[i] = fmaf(skip[i], dv, delta[i] * v.x);
                dd[i] = fmaf(xv, v.x, v.y);
                if (g.softplus) dd[i] *= sigmoid(kdt.at(i) + bias[i]);
                if (m > 0) {
                    dskip[i] = fmaf(dv, xv, dskip[i]);
                    dbias[i] += dd[i];
                }
            }
            Some<T, S::EACH> o;
            o.set(dx);
            o.store((T *)out.dx + (long long)(tile + row) * g.xs + first_chan, m);
            o.set(dd);
            o.store((T *)out.ddt + (long long)(tile + row) * g.dts + first_chan, m);
            if (in.z) {
                o.set(dz);
                o.store((T *)out.dz + (long long)(tile + row) * g.zs + first_chan, m);
            }
            float *const to = out.shared + ((long long)(at.group * g.blocks_of_group + at.block) * g.seq.T + tile) * (2 * S::STATES);
            for (int e = threadIdx.x; e < S::TOKENS * 2 * S::STATES; e += 256) {
                const int t = e / (2 * S::STATES), k = e % (2 * S::STATES);
                if (tile + t < t1) to[e] = (red[0][t][k] + red[1][t][k]) + (red[2][t][k] + red[3][t][k]);
            }
        }
    }

    // the part's sums over tokens: [C,N] of A, then [C] of D and [C] of dt_bias
    float *const to = out.dA + (long long)at.part * ((long long)g.C * g.N + 2ll * g.C);
    if (valid) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * q + i < g.N) to[(long long)chan * g.N + 4 * q + i] = dA[i];
    }
    float2 *const sums = reinterpret_cast<float2 *>(&slot[0][0]);    // (a lane's own places: the ones that it has read)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) sums[row * S::CHANNELS + col + i] = make_float2(dskip[i], dbias[i]);
    __syncthreads();
    for (int c = threadIdx.x; c < S::CHANNELS; c += 256) {
        const int k = at.block * S::CHANNELS + c;
        if (k >= g.per_group) continue;
        float a = 0.f, b = 0.f;
        for (int r = 0; r < S::TOKENS; ++r) { a += sums[r * S::CHANNELS + c].x; b += sums[r * S::CHANNELS + c].y; }
        to[(long long)g.C * g.N + at.group * g.per_group + k] = a;
        to[(long long)g.C * g.N + g.C + at.group * g.per_group + k] = b;
    }
}

// dB and dC: the sum over a group's channel blocks, a lane a value, neighbours at neighbouring states.
template <typename T>
__global__ __launch_bounds__(256) void k_sscan_bwd_shared(Scan g, int states, const float *__restrict__ shared, T *__restrict__ dB, T *__restrict__ dC)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int k = (int)(id % (2 * g.N)), n = k % g.N, is_c = k / g.N;
    const long long rest = id / (2 * g.N), t = rest / g.groups;
    const int group = (int)(rest % g.groups);
    if (t >= g.seq.T) return;
    const long long step = (long long)g.seq.T * 2 * states;
    const float *p = shared + (long long)group * g.blocks_of_group * step + t * 2 * states + is_c * states + n;
    float sum = 0.f;
#pragma unroll 4
    for (int b = 0; b < g.blocks_of_group; ++b) sum += p[b * step];
    if (is_c) stf(dC + t * g.cs + (long long)group * g.N + n, sum);
    else stf(dB + t * g.bs + (long long)group * g.N + n, sum);
}

template <typename T> hipError_t launch(const sscan_desc *d, const sscan_tensors *t, float *workspace, hipStream_t stream)
{
    const ScanPlan p = plan_sscan_bwd(d, t->starts != nullptr);
    const BwdSpace space = sscan_bwd_space(d, p);
    const Scan g = sscan_geometry(d, p, t->starts);
    const long long values = (long long)d->C * d->N;
    if (d->T > 0) {
        const BackIn in = {t->x, t->dt, t->B, t->C, t->z, t->dy, (const float *)t->A, (const float *)t->D, (const float *)t->dt_bias,
                           (const float *)t->init, (const float *)t->kept};
        const BackOut out = {t->dx, t->ddt, t->dz, p.carry ? workspace + space.ends : nullptr, p.carry ? workspace + space.sums : nullptr,
                             workspace + space.dA, workspace + space.shared};
        const long long blocks = (long long)p.channel_blocks * p.parts, last = ((long long)d->T * d->groups * 2 * d->N + 255) / 256;
        if (!launchable(blocks, 256) || !launchable(last, 256)) return hipErrorInvalidValue;
        const hipError_t e = with_state_lanes(p.lanes, [&](auto lanes) {
            constexpr int LPC = decltype(lanes)::value;
            if (p.carry) hipLaunchKernelGGL((k_sscan_bwd_carry<T, LPC>), dim3((unsigned)(blocks - p.channel_blocks)), dim3(256), 0, stream, g, in, out);
            hipLaunchKernelGGL((k_sscan_bwd<T, LPC>), dim3((unsigned)blocks), dim3(256), 0, stream, g, in, out);
            hipLaunchKernelGGL(k_sscan_bwd_shared<T>, dim3((unsigned)last), dim3(256), 0, stream, g, 4 * LPC, workspace + space.shared, (T *)t->dB, (T *)t->dC);
        });
        if (e != hipSuccess) return e;
    }
    return launch_sum_partials(workspace + space.dA, d->T > 0 ? p.parts : 0, values, values + d->C, values + 2ll * d->C, (float *)t->dA, (float *)t->dD,
                               (float *)t->ddt_bias, stream);
}

}  // namespace

hipError_t launch_sscan_bwd(const sscan_desc *d, const sscan_tensors *t, float *workspace, hipStream_t stream)
{
    return d->dtype == DWCONV_F32 ? launch<float>(d, t, workspace, stream) : launch<bf16_t>(d, t, workspace, stream);
}

}  // namespace dwc
