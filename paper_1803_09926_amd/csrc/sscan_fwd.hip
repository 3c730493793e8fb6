// Selective state space scan, forward, and one token at a time.  See sscan.hpp for the layout of the work, include/seqops.h for the contract.
//
// Each state costs a multiply, an exponential at half the vector rate (8.1 cycles measured, 4.4 a multiply-add), a multiply and two multiply-adds a token: 24 cycles
// of a SIMD for 64 of them, where the tensors move 8 bytes (bf16) for 16 states.  The kernel is bound by its vector instructions: they are active in 78 % of its cycles,
// 92 % of those in which the compute units are busy, and the recurrence is three fifths of them (three quarters in the first pass).  16384 tokens of 1024
// channels of 16 states take 132 us (62 the first pass, 95 the second, each timed alone), 16383 of 2048 228 us, 2.4 states a ns; that many states at 24
// cycles each, and no first pass, would take 41 and 82.
//
// Where there are few channels the tokens are split into parts.  A first pass finds each part's state at its end from zero and the sum of its step
// sizes (the decay over a part is exp(A * sum)); a block of the second pass then walks back over the parts before it, to the one that holds its sequence's first
// token, and starts from the state that they leave.
#include "sscan.hpp"

namespace dwc {

namespace {

// A tile of the tokens: those between two states that are kept.
template <int LPC> struct Tile {
    static constexpr int CHANNELS = 256 / LPC, TOKENS = KEPT_EVERY, EACH = TOKENS * CHANNELS / 256, STATES = 4 * LPC;
    static constexpr int LANES = 256 / TOKENS;                        // that share a token's channels, EACH of them a lane
    static constexpr int SHARED = (TOKENS * STATES + 255) / 256;      // values of B, and of C, that a lane brings
    static constexpr int PLANE = CHANNELS + 64 / LPC;
    static constexpr int WAVES = LPC == 2 ? 3 : 5;                    // a SIMD: what the registers and 31 KB of LDS allow; 6 and 8 spill, and take 3 and 20 % longer
};

// WHOLE: a lane's channels are all there or none of them, in rows that are aligned to them.
// ENDS: the first pass, which leaves the states at the parts' ends; otherwise the pass that writes y.
template <typename T, int LPC, bool ENDS, bool WHOLE>
__global__ __launch_bounds__(256, Tile<LPC>::WAVES) void k_sscan_fwd(Scan g, const T *__restrict__ x, const T *__restrict__ dt, const float *__restrict__ A,
                                                   const T *__restrict__ B, const T *__restrict__ Cm, const float *__restrict__ D,
                                                   const T *__restrict__ z, const float *__restrict__ dt_bias, const float *__restrict__ init,
                                                   T *__restrict__ y, float *__restrict__ final, float *__restrict__ kept, float *__restrict__ ends,
                                                   float *__restrict__ sums)
{
    typedef Tile<LPC> S;
    // step sizes, and these times x.  Lanes write EACH neighbours, 16 bytes for 16 states: no two on one bank
    __shared__ __attribute__((aligned(16))) float steps[S::TOKENS][S::CHANNELS], gains[S::TOKENS][S::CHANNELS];
    __shared__ float4 Bs[S::TOKENS][LPC], Cs[ENDS ? 1 : S::TOKENS][LPC];
    // a token's and channel's y, a share from each of its lanes: added up by the lane that rounds and stores, in 3 additions for 16 states, where moves between
    // the lanes took 9 instructions for 4 tokens.  A plane of channels for each lane, 64 / LPC further on than the banks' turn
    __shared__ __attribute__((aligned(16))) float shares[ENDS ? 1 : S::TOKENS][LPC][ENDS ? 4 : S::PLANE];
    const ScanBlock at = scan_block(g);
    const int lane = threadIdx.x & 63, q = lane % LPC, wv = threadIdx.x >> 6;
    // the lane's channel in the recurrence
    const int mine = wv * (64 / LPC) + lane / LPC, in_group = at.block * S::CHANNELS + mine, chan = at.group * g.per_group + in_group;
    const bool valid = in_group < g.per_group;
    // the lane's token and channels in what is elementwise
    constexpr int STEP = WHOLE ? 1 : S::LANES;                         // between a lane's channels: alone they are loads of their own, next to other lanes'
    const int row = threadIdx.x / S::LANES, col = threadIdx.x % S::LANES * (WHOLE ? S::EACH : 1);
    const int first_chan = at.group * g.per_group + at.block * S::CHANNELS + col, n = g.per_group - at.block * S::CHANNELS - col;
    int t0 = (int)((long long)at.part * g.part);
    const int t1 = g.seq.T - t0 < g.part ? g.seq.T : t0 + g.part;
    if (ENDS) {                                                       // only what the next part goes on from is asked for
        const int f = g.seq.start(g.seq.of_one(t1));
        if (f == t1) return;
        if (f > t0 && f < t1) t0 += (f - t0) / S::TOKENS * S::TOKENS;
    }

    float a2[4], h[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) a2[i] = valid ? A[(long long)chan * g.N + state_of(g, 4 * q + i)] * LOG2E : 0.f;
    float bias[S::EACH], skip[S::EACH];
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) {
        bias[i] = dt_bias && i * STEP < n ? dt_bias[first_chan + i * STEP] : 0.f;
        skip[i] = !ENDS && D && i * STEP < n ? D[first_chan + i * STEP] : 0.f;
    }

    // a sequence's row of [sequences,C,N]; rare, so that its address is not to be held in registers meanwhile
    auto put_state = [&](float *to, int s) {
        if (!valid) return;
        int c = chan;
        asm volatile("" : "+v"(c));
        float *p = to + ((long long)s * g.C + c) * g.N + 4 * q;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * q + i < g.N) p[i] = h[i];
    };
    auto get_state = [&](int s) {
        int c = chan, k = 4 * q;
        asm volatile("" : "+v"(c), "+v"(k));
        const float *p = init + ((long long)s * g.C + c) * g.N;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = init && valid ? p[state_of(g, k + i)] : 0.f;
    };

    auto keep_state = [&](int tile) {
        if (valid)
            *reinterpret_cast<float4 *>(kept + ((long long)(tile / KEPT_EVERY) * g.C + chan) * S::STATES + 4 * q) = make_float4(h[0], h[1], h[2], h[3]);
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

    int s = g.seq.of_one(t0), head = g.seq.start(s), next = g.seq.start(s + 1);    // the sequence of the tile's first token
    if (!ENDS && ends && head < t0) {                                 // the state that the parts before leave
        const int least = (head < 0 ? 0 : head) / g.part;
        gather_parts<LPC>(h, a2, ends, sums, g.C, chan, q, valid, at.part - 1, -1, at.part - least);
    }

    // offsets in bytes from a tile's first row: at most 16 rows of SEQOPS_MAX_STRIDE
    constexpr uint32_t W = sizeof(T);
    const uint32_t ox = ((uint32_t)row * (uint32_t)g.xs + first_chan) * W, odt = ((uint32_t)row * (uint32_t)g.dts + first_chan) * W;
    const uint32_t oz = ((uint32_t)row * (uint32_t)g.zs + first_chan) * W, oy = ((uint32_t)row * (uint32_t)g.ys + first_chan) * W;
    Ahead<T, S::EACH, WHOLE, STEP> rx, rdt, rz;
    Ahead<T, 1, true> rb[S::SHARED], rc[S::SHARED];
    // the rows of the tile that is loaded next, moved on by additions: a product of 64 bits for each of them and tile took 60 scalar instructions
    const T *px = x + (long long)t0 * g.xs, *pdt = dt + (long long)t0 * g.dts, *pz = !ENDS && z ? z + (long long)t0 * g.zs : x;
    const T *pb = B + (long long)t0 * g.bs + (long long)at.group * g.N, *pc = ENDS ? pb : Cm + (long long)t0 * g.cs + (long long)at.group * g.N;
    T *py = ENDS ? nullptr : y + (long long)t0 * g.ys;
    uint32_t ob[S::SHARED], oc[S::SHARED];
    float share[S::SHARED];                                           // of C that a slot has
#pragma unroll
    for (int i = 0; i < S::SHARED; ++i) {
        const int e = threadIdx.x + 256 * i, r = e / S::STATES, k = state_of(g, e % S::STATES);
        ob[i] = ((uint32_t)r * (uint32_t)g.bs + k) * W;
        oc[i] = ((uint32_t)r * (uint32_t)g.cs + k) * W;
        share[i] = share_of(g, k);
    }
    auto load = [&](int tile) {
        const int left = t1 - tile, m = row < left ? n : 0;
        rx.load(BufView(px, VIEW_BYTES), ox, m);
        rdt.load(BufView(pdt, VIEW_BYTES), odt, m);
        if (!ENDS) rz.load(BufView(pz, VIEW_BYTES), oz, z ? m : 0);
        const BufView b(pb, VIEW_BYTES), c(pc, VIEW_BYTES);
#pragma unroll
        for (int i = 0; i < S::SHARED; ++i) {
            const int in = (int)(threadIdx.x + 256 * i) / S::STATES < (left < S::TOKENS ? left : S::TOKENS);    // (a lane without a value: a row behind the tile)
            rb[i].load(b, ob[i], in);
            if (!ENDS) rc[i].load(c, oc[i], in);
        }
        px += S::TOKENS * g.xs;
        pdt += S::TOKENS * g.dts;
        pz += S::TOKENS * g.zs;
        pb += S::TOKENS * g.bs;
        pc += S::TOKENS * g.cs;
    };
    load(t0);

    float total = 0.f;
    for (int tile = t0; tile < t1; tile += S::TOKENS) {
        float direct[ENDS ? 1 : S::EACH], gate[ENDS ? 1 : S::EACH];    // D * x, and what the gate lets through
        {
            float d[S::EACH];
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) d[i] = rdt.at(i) + bias[i];
            step_sizes(g, d);
            if (!ENDS) {
#pragma unroll
                for (int i = 0; i < S::EACH; ++i) { direct[ENDS ? 0 : i] = 0.f; gate[ENDS ? 0 : i] = 1.f; }
                if (D) {
#pragma unroll
                    for (int i = 0; i < S::EACH; ++i) direct[ENDS ? 0 : i] = skip[i] * rx.at(i);
                }
                if (z) {
#pragma unroll
                    for (int i = 0; i < S::EACH; ++i) { const float v = rz.at(i); gate[ENDS ? 0 : i] = v * sigmoid(v); }
                }
            }
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) { steps[row][col + i * STEP] = d[i]; gains[row][col + i * STEP] = d[i] * rx.at(i); }
#pragma unroll
            for (int i = 0; i < S::SHARED; ++i) {
                const int e = threadIdx.x + 256 * i;
                if (e < S::TOKENS * S::STATES) {
                    reinterpret_cast<float *>(Bs)[e] = rb[i].at(0);
                    if (!ENDS) reinterpret_cast<float *>(Cs)[e] = rc[i].at(0) * share[i];
                }
            }
        }
        if (tile >= next) { s = g.seq.of_one(tile); head = g.seq.start(s); next = g.seq.start(s + 1); }
        const bool any = head == tile || next < tile + S::TOKENS;
        int of = 0;
        const uint32_t firsts = any ? first_tokens(g.seq, tile, S::TOKENS, t1, of) : 0u;
        if (!ENDS && kept && !(firsts & 1)) keep_state(tile);
        if (tile + S::TOKENS < t1) load(tile + S::TOKENS);
        __syncthreads();

        auto token = [&](int t) {                                     // the state at token t; its share of y
            const float d = steps[t][mine], gain = gains[t][mine];
            const float4 b = Bs[t][q];
            const float bv[4] = {b.x, b.y, b.z, b.w};
            if (ENDS) total += d;
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = fmaf(exp2_fast(d * a2[i]), h[i], gain * bv[i]);
            if (ENDS) return 0.f;
            const float4 c = Cs[t][q];
            return fmaf(c.x, h[0], fmaf(c.y, h[1], fmaf(c.z, h[2], c.w * h[3])));
        };
        if (firsts || tile + S::TOKENS > t1) {                        // sequences start here, or the tokens end
#pragma unroll 1
            for (int t = 0; t < S::TOKENS && tile + t < t1; ++t) {
                if (firsts >> t & 1) {
                    if (!ENDS && final && tile + t > t0) put_state(final, sequence_of(of, t - 1));
                    get_state(sequence_of(of, t));
                    if (!ENDS && kept && t == 0) keep_state(tile);
                }
                const float share = token(t);
                if (!ENDS) shares[ENDS ? 0 : t][q][ENDS ? 0 : mine] = share;
            }
        } else {
#pragma unroll 8
            for (int t = 0; t < S::TOKENS; ++t) {
                const float share = token(t);
                if (!ENDS) shares[ENDS ? 0 : t][q][ENDS ? 0 : mine] = share;
            }
        }
        __syncthreads();

        if (!ENDS) {
            float o[S::EACH];
            const int m = tile + row < t1 ? n : 0;
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) o[i] = direct[ENDS ? 0 : i];
#pragma unroll
            for (int j = 0; j < LPC; ++j)
#pragma unroll
                for (int i = 0; i < S::EACH; ++i) o[i] += shares[ENDS ? 0 : row][j][ENDS ? 0 : col + i * STEP];
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) o[i] *= gate[ENDS ? 0 : i];
            store_late<T, S::EACH, WHOLE, STEP>(BufView(py, VIEW_BYTES), oy, m, o);
            py += S::TOKENS * g.ys;
        }
    }
    if (ENDS) {
        if (valid) {
            *reinterpret_cast<float4 *>(ends + ((long long)at.part * g.C + chan) * S::STATES + 4 * q) = make_float4(h[0], h[1], h[2], h[3]);
            if (q == 0) sums[(long long)at.part * g.C + chan] = total;
        }
    } else if (final && (t1 == g.seq.T || first_token(g.seq, t1))) {
        put_state(final, g.seq.of_one(t1 - 1));
    }
}

template <typename T, int LPC>
__global__ __launch_bounds__(256) void k_sscan_step(Scan g, const T *__restrict__ x, const T *__restrict__ dt, const float *__restrict__ A,
                                                    const T *__restrict__ B, const T *__restrict__ Cm, const float *__restrict__ D,
                                                    const T *__restrict__ z, const float *__restrict__ dt_bias, const int32_t *__restrict__ slots,
                                                    float *__restrict__ state, T *__restrict__ y)
{
    // a block takes neighbouring channels of one row: its slot is a scalar, and no lane divides
    const int t = (int)(blockIdx.x / (unsigned)g.blocks_of_group), q = threadIdx.x % LPC;
    const int c = (int)(blockIdx.x % (unsigned)g.blocks_of_group) * (256 / LPC) + threadIdx.x / LPC, n = g.N - 4 * q;
    if (c >= g.C) return;                                              // (all lanes of a channel)
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
    const float xv = ldf(x + (long long)t * g.xs + c);
    float step[1] = {ldf(dt + (long long)t * g.dts + c) + (dt_bias ? dt_bias[c] : 0.f)};
    step_sizes(g, step);
    const float d = step[0];
    float hv[4], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hv[i] = fmaf(exp2_fast(d * (a.at(i) * LOG2E)), h.at(i), d * xv * b.at(i));
        sum += cc.at(i) * (i < n ? hv[i] : 0.f);
    }
    h.set(hv);
    h.store(st, n);
    sum = states_sum<LPC>(sum);
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
        auto both = [&](auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            if (p.carry) run(k_sscan_fwd<T, LPC, true, WHOLE>, blocks - (unsigned)p.channel_blocks);   // (nothing follows the last part)
            run(k_sscan_fwd<T, LPC, false, WHOLE>, blocks);
        };
        constexpr int EACH = Tile<LPC>::EACH;
        const bool whole = whole_vectors<T>(EACH, g.per_group, {t->x, t->dt, t->z, t->y}, {g.xs, g.dts, g.zs, g.ys});
        if (whole) both(std::true_type());
        else both(std::false_type());
    });
}

template <typename T> hipError_t launch_one(const sscan_desc *d, const sscan_tensors *t, hipStream_t stream)
{
    ScanPlan p = {state_lanes(d->N), 1, 1, 1, false};
    Scan g = sscan_geometry(d, p, nullptr);
    g.blocks_of_group = cdiv(d->C, 256 / p.lanes);                     // here: of a row
    const long long most = most_blocks(256) / g.blocks_of_group;       // rows of one launch
    return with_state_lanes(p.lanes, [&](auto lanes) {
        for (long long row = 0; row < d->T; row += most) {
            const long long rows = d->T - row < most ? d->T - row : most, own = t->slots ? 0 : row;     // the first slot, where rows have their own number
            g.seq.n = d->sequences - (int)own;
            hipLaunchKernelGGL((k_sscan_step<T, decltype(lanes)::value>), dim3((unsigned)(rows * g.blocks_of_group)), dim3(256), 0, stream, g,
                               (const T *)t->x + row * g.xs, (const T *)t->dt + row * g.dts, (const float *)t->A, (const T *)t->B + row * g.bs,
                               (const T *)t->C + row * g.cs, (const float *)t->D, t->z ? (const T *)t->z + row * g.zs : nullptr, (const float *)t->dt_bias,
                               t->slots ? (const int32_t *)t->slots + row : nullptr, (float *)t->state + own * d->C * d->N, (T *)t->y + row * g.ys);
        }
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
