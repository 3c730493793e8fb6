// Selective state space scan, forward, and one token at a time.  See sscan.hpp for the layout of the work, include/seqops.h for the contract.
//
// Each state costs a multiply, an exponential at a quarter of the vector rate, a multiply and two multiply-adds a token: 32 cycles of a SIMD for 64 of
// them, where the tensors move 8 bytes (bf16) for 16 states.  The kernel is bound by its vector instructions.
//
// Where there are few channels the tokens are split into parts.  A first pass finds each part's state at its end from zero and the sum of its step
// sizes (the decay over a part is exp(A * sum)); a block of the second pass then walks back over the parts before it, to the one that holds its sequence's first
// token, and starts from the state that they leave.
#include "sscan.hpp"

namespace dwc {

namespace {

template <int LPC> struct Tile {
    static constexpr int CHANNELS = 256 / LPC, TOKENS = LPC == 2 ? 16 : 32, EACH = TOKENS * CHANNELS / 256, STATES = 4 * LPC;
    static constexpr int LANES = 256 / TOKENS;                        // that share a token's channels, EACH of them a lane
    static constexpr int SHARED = (TOKENS * STATES + 255) / 256;      // values of B, and of C, that a lane brings
};

// ENDS: the first pass, which leaves the states at the parts' ends; otherwise the pass that writes y.
template <typename T, int LPC, bool ENDS>
__global__ __launch_bounds__(256) void k_sscan_fwd(Scan g, const T *__restrict__ x, const T *__restrict__ dt, const float *__restrict__ A,
                                                   const T *__restrict__ B, const T *__restrict__ Cm, const float *__restrict__ D,
                                                   const T *__restrict__ z, const float *__restrict__ dt_bias, const float *__restrict__ init,
                                                   T *__restrict__ y, float *__restrict__ final, float *__restrict__ kept, float *__restrict__ ends,
                                                   float *__restrict__ sums)
{
    typedef Tile<LPC> S;
    __shared__ float2 du[S::TOKENS][S::CHANNELS];                     // step size, step size * x; y takes the first's place
    __shared__ float4 Bs[S::TOKENS][LPC], Cs[ENDS ? 1 : S::TOKENS][LPC];
    const ScanBlock at = scan_block(g);
    const int lane = threadIdx.x & 63, q = lane % LPC, wv = threadIdx.x >> 6;
    // the lane's channel in the recurrence
    const int mine = wv * (64 / LPC) + lane / LPC, in_group = at.block * S::CHANNELS + mine, chan = at.group * g.per_group + in_group;
    const bool valid = in_group < g.per_group;
    // the lane's token and channels in what is elementwise
    const int row = threadIdx.x / S::LANES, col = threadIdx.x % S::LANES * S::EACH;
    const int first_chan = at.group * g.per_group + at.block * S::CHANNELS + col, n = g.per_group - at.block * S::CHANNELS - col;
    const int t0 = (int)((long long)at.part * g.part), t1 = g.seq.T - t0 < g.part ? g.seq.T : t0 + g.part;

    float a2[4], h[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) a2[i] = valid && 4 * q + i < g.N ? A[(long long)chan * g.N + 4 * q + i] * LOG2E : 0.f;
    float bias[S::EACH], skip[S::EACH];
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) {
        bias[i] = dt_bias && i < n ? dt_bias[first_chan + i] : 0.f;
        skip[i] = !ENDS && D && i < n ? D[first_chan + i] : 0.f;
    }

    auto put_state = [&](float *to, int s) {                          // a sequence's row of [sequences,C,N]
        if (!valid) return;
        float *p = to + ((long long)s * g.C + chan) * g.N + 4 * q;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * q + i < g.N) p[i] = h[i];
    };
    auto get_state = [&](int s) {
        const float *p = init + ((long long)s * g.C + chan) * g.N + 4 * q;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = init && valid && 4 * q + i < g.N ? p[i] : 0.f;
    };

    // an empty sequence hands on what it was given; 64 sequences are looked at together
    if (!ENDS && final && (g.seq.starts || g.seq.T == 0))
        for (long long e0 = (long long)at.part * 64; e0 < g.seq.n; e0 += (long long)g.parts * 64) {
            const long long e = e0 + lane;
            uint64_t empty = __ballot(e < g.seq.n && g.seq.start((int)e + 1) <= g.seq.start((int)e));
            for (; empty; empty &= empty - 1) {
                const int s = (int)e0 + __ffsll((unsigned long long)empty) - 1;
                get_state(s);
                put_state(final, s);
            }
        }
    if (t1 <= t0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = 0.f;

    if (!ENDS && ends) {                                              // the state that the parts before leave
        const int f = g.seq.start(g.seq.of(t0));
        if (f < t0) {
            const int least = (f < 0 ? 0 : f) / g.part;
            float decay[4] = {1.f, 1.f, 1.f, 1.f};
            for (int p = at.part - 1; p >= least; --p) {
                if (!valid) continue;
                const float4 e = *reinterpret_cast<const float4 *>(ends + ((long long)p * g.C + chan) * S::STATES + 4 * q);
                const float sum = sums[(long long)p * g.C + chan];
                const float v[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[i] = fmaf(decay[i], v[i], h[i]);
                    decay[i] *= exp2_fast(a2[i] * sum);
                }
            }
        }
    }

    Some<T, S::EACH> rx, rdt, rz;
    float rb[S::SHARED], rc[S::SHARED];
    auto load = [&](int tile) {
        const int t = tile + row, m = t < t1 ? n : 0;
        rx.load(x + (long long)t * g.xs + first_chan, m);
        rdt.load(dt + (long long)t * g.dts + first_chan, m);
        if (!ENDS && z) rz.load(z + (long long)t * g.zs + first_chan, m);
#pragma unroll
        for (int i = 0; i < S::SHARED; ++i) {
            const int e = threadIdx.x + 256 * i, tb = tile + e / S::STATES, k = e % S::STATES;
            const bool in = e < S::TOKENS * S::STATES && tb < t1 && k < g.N;
            rb[i] = in ? ldf(B + (long long)tb * g.bs + (long long)at.group * g.N + k) : 0.f;
            if (!ENDS) rc[i] = in ? ldf(Cm + (long long)tb * g.cs + (long long)at.group * g.N + k) : 0.f;
        }
    };
    load(t0);

    int s = g.seq.of(t0), next = g.seq.start(s + 1);
    float total = 0.f;
    for (int tile = t0; tile < t1; tile += S::TOKENS) {
        const Some<T, S::EACH> kx = rx, kz = rz;
        {
            float2 o[S::EACH];
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) {
                // beyond the last token the step size is zero: the state stays
                const float d = tile + row < t1 ? step_size(g, rdt.at(i) + bias[i]) : 0.f;
                o[i] = make_float2(d, d * rx.at(i));
            }
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) du[row][col + i] = o[i];
#pragma unroll
            for (int i = 0; i < S::SHARED; ++i) {
                const int e = threadIdx.x + 256 * i;
                if (e < S::TOKENS * S::STATES) {
                    reinterpret_cast<float *>(Bs)[e] = rb[i];
                    if (!ENDS) reinterpret_cast<float *>(Cs)[e] = rc[i];
                }
            }
        }
        if (tile + S::TOKENS < t1) load(tile + S::TOKENS);
        __syncthreads();

        if (tile >= next) { s = g.seq.of(tile); next = g.seq.start(s + 1); }
        const bool any = g.seq.start(s) == tile || next < tile + S::TOKENS;
        const uint32_t firsts = any ? first_tokens(g.seq, tile, S::TOKENS, t1) : 0u;

        auto walk = [&](auto special) {           // special: a sequence starts here, or the tokens end
            constexpr int GROUP = LPC < 4 ? 4 : LPC;
            for (int t = 0; t < S::TOKENS; t += GROUP) {
                float part[GROUP];
#pragma unroll
                for (int u = 0; u < GROUP; ++u) {
                    const int tt = t + u;
                    part[u] = 0.f;
                    if constexpr (decltype(special)::value) {
                        if (tile + tt >= t1) continue;
                        if (firsts >> tt & 1) {
                            if (!ENDS && final && tile + tt > t0) put_state(final, g.seq.of(tile + tt - 1));
                            get_state(g.seq.of(tile + tt));
                        }
                    }
                    if (!ENDS && kept && (tt % KEPT_EVERY) == 0 && valid) {
                        const float4 v = make_float4(h[0], h[1], h[2], h[3]);
                        *reinterpret_cast<float4 *>(kept + ((long long)((tile + tt) / KEPT_EVERY) * g.C + chan) * S::STATES + 4 * q) = v;
                    }
                    const float2 d = du[tt][mine];
                    const float4 b = Bs[tt][q];
                    const float bv[4] = {b.x, b.y, b.z, b.w};
                    if (ENDS) total += d.x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[i] = fmaf(exp2_fast(d.x * a2[i]), h[i], d.y * bv[i]);
                    if (!ENDS) {
                        const float4 c = Cs[tt][q];
                        part[u] = fmaf(c.x, h[0], fmaf(c.y, h[1], fmaf(c.z, h[2], c.w * h[3])));
                    }
                }
                if (!ENDS) {
#pragma unroll
                    for (int u = 0; u < GROUP; u += LPC) {
                        float v[LPC];
#pragma unroll
                        for (int j = 0; j < LPC; ++j) v[j] = part[u + j];
                        // (only this wavefront reads the place, and it has)
                        du[t + u + q][mine].x = transpose_sum<LPC>(v, q);
                    }
                }
            }
        };
        if (firsts || tile + S::TOKENS > t1) walk(std::true_type());
        else walk(std::false_type());
        __syncthreads();

        if (!ENDS) {
            float o[S::EACH];
            const int m = tile + row < t1 ? n : 0;
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) {
                o[i] = fmaf(skip[i], kx.at(i), du[row][col + i].x);
                if (z) { const float v = kz.at(i); o[i] *= v * sigmoid(v); }
            }
            Some<T, S::EACH> out;
            out.set(o);
            out.store(y + (long long)(tile + row) * g.ys + first_chan, m);
        }
    }
    if (ENDS) {
        if (valid) {
            *reinterpret_cast<float4 *>(ends + ((long long)at.part * g.C + chan) * S::STATES + 4 * q) = make_float4(h[0], h[1], h[2], h[3]);
            if (q == 0) sums[(long long)at.part * g.C + chan] = total;
        }
    } else if (final && (t1 == g.seq.T || first_token(g.seq, t1))) {
        put_state(final, g.seq.of(t1 - 1));
    }
}

template <typename T, int LPC>
__global__ __launch_bounds__(256) void k_sscan_step(Scan g, const T *__restrict__ x, const T *__restrict__ dt, const float *__restrict__ A,
                                                    const T *__restrict__ B, const T *__restrict__ Cm, const float *__restrict__ D,
                                                    const T *__restrict__ z, const float *__restrict__ dt_bias, const int32_t *__restrict__ slots,
                                                    float *__restrict__ state, T *__restrict__ y)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, which = id / LPC;
    const int q = (int)(id % LPC), t = (int)(which / g.C), c = (int)(which % g.C), n = g.N - 4 * q;
    if (t >= g.seq.T) return;                                          // (all lanes of a channel)
    const int slot = slots ? slots[t] : t;
    if (slot < 0 || slot >= g.seq.n) {
        if (q == 0) stf(y + (long long)t * g.ys + c, 0.f);
        return;
    }
    float *const st = state + ((long long)slot * g.C + c) * g.N + 4 * q;
    const long long shared = (long long)(c / g.per_group) * g.N + 4 * q;
    Some<float, 4> h, a;
    Some<T, 4> b, cc;
    h.load(st, n);
    a.load(A + (long long)c * g.N + 4 * q, n);
    b.load(B + (long long)t * g.bs + shared, n);
    cc.load(Cm + (long long)t * g.cs + shared, n);
    const float xv = ldf(x + (long long)t * g.xs + c), d = step_size(g, ldf(dt + (long long)t * g.dts + c) + (dt_bias ? dt_bias[c] : 0.f));
    float hv[4], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hv[i] = fmaf(exp2_fast(d * (a.at(i) * LOG2E)), h.at(i), d * xv * b.at(i));
        sum += cc.at(i) * (i < n ? hv[i] : 0.f);
    }
    h.set(hv);
    h.store(st, n);
    sum += lane_move<DPP_XOR1>(sum);
    if constexpr (LPC >= 4) sum += lane_move<DPP_XOR2>(sum);
    if constexpr (LPC >= 8) sum += lane_move<DPP_HALF_MIRROR>(sum);
    if constexpr (LPC >= 16) sum += lane_move<DPP_MIRROR>(sum);
    if (q) return;
    if (D) sum = fmaf(D[c], xv, sum);
    if (z) { const float v = ldf(z + (long long)t * g.zs + c); sum *= v * sigmoid(v); }
    stf(y + (long long)t * g.ys + c, sum);
}

template <typename T> hipError_t launch(const sscan_desc *d, const sscan_tensors *t, float *workspace, hipStream_t stream)
{
    const ScanPlan p = plan_sscan_fwd(d, t->starts != nullptr);
    const FwdSpace space = sscan_fwd_space(d, p);
    if (!launchable((long long)p.channel_blocks * p.parts, 256)) return hipErrorInvalidValue;
    const Scan g = sscan_geometry(d, p, t->starts);
    float *const ends = p.carry ? workspace + space.ends : nullptr, *const sums = p.carry ? workspace + space.sums : nullptr;
    return with_state_lanes(p.lanes, [&](auto lanes) {
        constexpr int LPC = decltype(lanes)::value;
        const unsigned blocks = (unsigned)p.channel_blocks * (unsigned)p.parts;
        auto run = [&](auto kernel, unsigned n) {
            hipLaunchKernelGGL(kernel, dim3(n), dim3(256), 0, stream, g, (const T *)t->x, (const T *)t->dt, (const float *)t->A, (const T *)t->B,
                               (const T *)t->C, (const float *)t->D, (const T *)t->z, (const float *)t->dt_bias, (const float *)t->init, (T *)t->y,
                               (float *)t->final, (float *)t->kept, ends, sums);
        };
        if (p.carry) run(k_sscan_fwd<T, LPC, true>, blocks - (unsigned)p.channel_blocks);   // (nothing follows the last part)
        run(k_sscan_fwd<T, LPC, false>, blocks);
    });
}

template <typename T> hipError_t launch_one(const sscan_desc *d, const sscan_tensors *t, hipStream_t stream)
{
    ScanPlan p = {state_lanes(d->N), 1, 1, 1, false};
    const Scan g = sscan_geometry(d, p, nullptr);
    const long long blocks = ((long long)d->T * d->C * p.lanes + 255) / 256;
    if (!launchable(blocks, 256)) return hipErrorInvalidValue;
    return with_state_lanes(p.lanes, [&](auto lanes) {
        hipLaunchKernelGGL((k_sscan_step<T, decltype(lanes)::value>), dim3((unsigned)blocks), dim3(256), 0, stream, g, (const T *)t->x, (const T *)t->dt,
                           (const float *)t->A, (const T *)t->B, (const T *)t->C, (const float *)t->D, (const T *)t->z, (const float *)t->dt_bias,
                           (const int32_t *)t->slots, (float *)t->state, (T *)t->y);
    });
}

}  // namespace

hipError_t launch_sscan_fwd(const sscan_desc *d, const sscan_tensors *t, float *workspace, hipStream_t stream)
{
    return d->dtype == DWCONV_F32 ? launch<float>(d, t, workspace, stream) : launch<bf16_t>(d, t, workspace, stream);
}
hipError_t launch_sscan_step(const sscan_desc *d, const sscan_tensors *t, hipStream_t stream)
{
    return d->dtype == DWCONV_F32 ? launch_one<float>(d, t, stream) : launch_one<bf16_t>(d, t, stream);
}

}  // namespace dwc
