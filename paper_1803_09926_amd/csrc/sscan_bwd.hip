// Selective state space scan, backward.  See sscan.hpp for the layout of the work, include/seqops.h for the contract.
//
// With g the gradient that arrives at h[t] (from y[t], and from h[t+1] times its decay), v = y before the gate and dv its gradient:
//   g += dv * C[t];  dC[t] = sum_c dv * h[t];  dB[t] = sum_c g * delta * x;  dx = D * dv + delta * sum_n g * B[t]
//   r = g * decay * h[t-1];  ddelta = x * sum_n g * B[t] + sum_n r * A;  dA += r * delta;  then g *= decay for the token before
// A tile is the 16 tokens between two states that the forward pass kept: a lane computes its 16 decays and states again, keeps them in registers (decay *
// h[t-1] is exact that way; the difference h[t] - delta x B would cancel), and walks back through them.  The sums over channels (dB, dC) go through the
// lanes of a wavefront by row swaps and moves, two instructions for the first two halvings, then through LDS over the block's wavefronts, then over the
// blocks in a second kernel.  Bound by its vector instructions: for a state and token 6 to come to the states again, 8 to walk back, 5 for the sums over
// channels, 2 for those over states and 4 for what is elementwise.  8192 tokens of 1536 channels of 16 states take 184 us, 45 more for the first pass, 12 for
// the sums; forward 44 and 62.  Vector instructions, 24 a state and token, are active in 79 % of the kernel's cycles.
//
// Where the tokens are split, a first pass finds the gradient that each part hands to the state before it, as the forward pass does with the states.
#include "sscan.hpp"

namespace dwc {

namespace {

template <int LPC> struct BackTile {
    static constexpr int CHANNELS = 256 / LPC, TOKENS = KEPT_EVERY, EACH = TOKENS / LPC, STATES = 4 * LPC, LANES = 256 / TOKENS;
    static constexpr int SHARED = (TOKENS * STATES + 255) / 256;
};

// f(k) for the slots that state n has beside slot n, of `states` of them.
template <typename F> __device__ __forceinline__ void each_copy(const Scan &g, int states, int n, F f)
{
    for (int k = n + g.N; k < g.N * g.copies; k += g.N) f(k);
    if (n < g.twice)
        for (int k = n + g.N * g.copies; k < states; k += g.twice) f(k);
}

struct BackIn {
    const void *x, *dt, *B, *C, *z, *dy;
    const float *A, *D, *dt_bias, *init, *kept;
};
struct BackOut {
    void *dx, *ddt, *dz;
    float *ends, *sums, *dA, *shared;    // as BwdSpace has them
};

// The first pass over the parts: from the last token of a part back to its first, the gradient that leaves the part, from zero, and the sum of step sizes.
template <typename T, int LPC, bool WHOLE>
__global__ __launch_bounds__(256) void k_sscan_bwd_carry(Scan g, BackIn in, BackOut out)
{
    typedef BackTile<LPC> S;
    constexpr int CHANNELS = S::CHANNELS, TOKENS = S::TOKENS, EACH = S::EACH, STATES = S::STATES, LANES = S::LANES, SHARED = S::SHARED;
    __shared__ __attribute__((aligned(16))) float steps[TOKENS][CHANNELS], dvs[TOKENS][CHANNELS];
    __shared__ float4 Cs[TOKENS][LPC];
    const ScanBlock at = scan_block(g);
    const int part = at.part + 1;                                    // (nothing comes before part 0)
    const int lane = threadIdx.x & 63, q = lane % LPC, wv = threadIdx.x >> 6;
    const int mine = wv * (64 / LPC) + lane / LPC, in_group = at.block * CHANNELS + mine, chan = at.group * g.per_group + in_group;
    const bool valid = in_group < g.per_group;
    constexpr int STEP = WHOLE ? 1 : LANES;                         // between a lane's channels: alone they are loads of their own, next to other lanes'
    const int row = threadIdx.x / LANES, col = threadIdx.x % LANES * (WHOLE ? EACH : 1);
    const int first_chan = at.group * g.per_group + at.block * CHANNELS + col, n = g.per_group - at.block * CHANNELS - col;
    const int t0 = (int)((long long)part * g.part);
    int t1 = g.seq.T - t0 < g.part ? g.seq.T : t0 + g.part;
    // only the sequence that the part before ends in hands anything back
    const int s0 = g.seq.of_one(t0), behind = g.seq.start(s0 + 1);
    if (t1 <= t0 || g.seq.start(s0) == t0) return;
    if (behind > t0 && behind < t1) t1 = behind;

    float a2[4], gr[4] = {0.f, 0.f, 0.f, 0.f}, bias[EACH];
#pragma unroll
    for (int i = 0; i < 4; ++i) a2[i] = valid ? in.A[(long long)chan * g.N + state_of(g, 4 * q + i)] * LOG2E : 0.f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) bias[i] = in.dt_bias && i * STEP < n ? in.dt_bias[first_chan + i * STEP] : 0.f;

    // offsets in bytes from a tile's first row: at most 16 rows of SEQOPS_MAX_STRIDE
    constexpr uint32_t W = sizeof(T);
    const uint32_t odt = ((uint32_t)row * (uint32_t)g.dts + first_chan) * W, oz = ((uint32_t)row * (uint32_t)g.zs + first_chan) * W;
    const uint32_t oy = ((uint32_t)row * (uint32_t)g.ys + first_chan) * W;
    const int last = t0 + (t1 - t0 - 1) / TOKENS * TOKENS;             // the tile that comes first
    Ahead<T, EACH, WHOLE, STEP> rdt, rz, rdy;
    Ahead<T, 1, true> rc[SHARED];
    // the rows of the tile that is loaded next
    const T *pdt = (const T *)in.dt + (long long)last * g.dts, *pdy = (const T *)in.dy + (long long)last * g.ys;
    const T *pz = in.z ? (const T *)in.z + (long long)last * g.zs : pdy, *pc = (const T *)in.C + (long long)last * g.cs + (long long)at.group * g.N;
    uint32_t oc[SHARED];
    float share[SHARED];                                             // of C that a slot has
#pragma unroll
    for (int i = 0; i < SHARED; ++i) {
        const int e = threadIdx.x + 256 * i, r = e / STATES, k = state_of(g, e % STATES);
        oc[i] = ((uint32_t)r * (uint32_t)g.cs + k) * W;
        share[i] = share_of(g, k);
    }
    auto load = [&](int tile) {
        const int left = t1 - tile, m = row < left ? n : 0;
        rdt.load(BufView(pdt, VIEW_BYTES), odt, m);
        rdy.load(BufView(pdy, VIEW_BYTES), oy, m);
        rz.load(BufView(pz, VIEW_BYTES), oz, in.z ? m : 0);
        const BufView c(pc, VIEW_BYTES);
#pragma unroll
        for (int i = 0; i < SHARED; ++i) rc[i].load(c, oc[i], (int)(threadIdx.x + 256 * i) / STATES < (left < TOKENS ? left : TOKENS));   // (a lane without a value: a row behind the tile)
        pdt -= TOKENS * g.dts;
        pdy -= TOKENS * g.ys;
        pz -= TOKENS * g.zs;
        pc -= TOKENS * g.cs;
    };
    // the sequence of the tile's first token, looked for again where a tile lies before it
    int s = g.seq.of_one(t1 - 1), head = g.seq.start(s), behind_it = g.seq.start(s + 1);
    float total = 0.f;
    load(last);
    for (int tile = last; tile >= t0; tile -= TOKENS) {
        float d[EACH], dv[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            d[i] = rdt.at(i) + bias[i];
            dv[i] = rdy.at(i);
        }
        step_sizes(g, d);
        if (in.z) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) { const float zv = rz.at(i); dv[i] *= zv * sigmoid(zv); }
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) { steps[row][col + i * STEP] = d[i]; dvs[row][col + i * STEP] = dv[i]; }
#pragma unroll
        for (int i = 0; i < SHARED; ++i) {
            const int e = threadIdx.x + 256 * i;
            if (e < TOKENS * STATES) reinterpret_cast<float *>(Cs)[e] = rc[i].at(0) * share[i];
        }
        if (tile < head) { s = g.seq.of_one(tile); head = g.seq.start(s); behind_it = g.seq.start(s + 1); }
        const bool any = head >= tile || behind_it < tile + TOKENS;
        int of = 0;
        const uint32_t firsts = any ? first_tokens(g.seq, tile, TOKENS, t1, of) : 0u;
        if (tile > t0) load(tile - TOKENS);
        __syncthreads();
        auto walk = [&](auto special) {
#pragma unroll 4
            for (int t = TOKENS - 1; t >= 0; --t) {
                if constexpr (decltype(special)::value) {
                    if (tile + t >= t1) continue;
                }
                const float d = steps[t][mine], dv = dvs[t][mine];
                const float4 c = Cs[t][q];
                const float cv[4] = {c.x, c.y, c.z, c.w};
                total += d;
#pragma unroll
                for (int i = 0; i < 4; ++i) gr[i] = fmaf(dv, cv[i], gr[i]) * exp2_fast(d * a2[i]);
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

template <typename T, int LPC, bool WHOLE>
__global__ __launch_bounds__(256, 2) void k_sscan_bwd(Scan g, BackIn in, BackOut out)
{
    typedef BackTile<LPC> S;
    // step sizes, these times x, dv, and sum C h; sum g B and sum r A take the places of the first two
    __shared__ __attribute__((aligned(16))) float steps[S::TOKENS][S::CHANNELS], gains[S::TOKENS][S::CHANNELS], dvs[S::TOKENS][S::CHANNELS],
        ys[S::TOKENS][S::CHANNELS];
    // B, C, and zeros that lanes without a channel have in their place: an infinity there would be NaN in the sums over channels
    __shared__ float4 shared_rows[4][S::TOKENS][LPC];
    __shared__ uint32_t states[LPC];                                 // offsets of a lane's four states, 8 bits each: worked out where init is read, 32 times a walk, it is code
    __shared__ float red[5][S::TOKENS][2 * S::STATES];               // dB and dC of each wavefront's channels; what lanes without a sum write
    const ScanBlock at = scan_block(g);
    const int lane = threadIdx.x & 63, q = lane % LPC, wv = threadIdx.x >> 6;
    const int mine = wv * (64 / LPC) + lane / LPC, in_group = at.block * S::CHANNELS + mine, chan = at.group * g.per_group + in_group;
    const bool valid = in_group < g.per_group;
    constexpr int STEP = WHOLE ? 1 : S::LANES;                         // between a lane's channels: alone they are loads of their own, next to other lanes'
    const int row = threadIdx.x / S::LANES, col = threadIdx.x % S::LANES * (WHOLE ? S::EACH : 1);
    // Rows that take more than 4 registers each are read twice, before and behind the walk: held meanwhile, they spill.
    constexpr bool AGAIN = Ahead<T, S::EACH, WHOLE, STEP>::WORDS > 4;
    // Of the tile's last tokens the decays stay in registers for the way back, as many as 256 registers hold: of none, 6 and 12 tokens 206, 197, 192 us (8192 x
    // 1536 x 16 in bf16).  What spills is slower: 12 in fp32 331 us both ways for 10's 330; 12 of 32 states 304 for 11's 302 (bf16), 318 for 10's 308 (fp32); 10
    // where channels are read one by one 364 for 6's 346 (1533 of them).
    constexpr int HELD = LPC == 4 ? (!WHOLE ? 6 : sizeof(T) == 4 ? 10 : 12) : LPC == 8 ? (WHOLE && sizeof(T) == 2 ? 11 : 10) : 0;
    const int first_chan = at.group * g.per_group + at.block * S::CHANNELS + col, n = g.per_group - at.block * S::CHANNELS - col;
    const int t0 = (int)((long long)at.part * g.part), t1 = g.seq.T - t0 < g.part ? g.seq.T : t0 + g.part;
    if (t1 <= t0) return;

    float a2[4], gr[4] = {0.f, 0.f, 0.f, 0.f}, dA[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) a2[i] = valid ? in.A[(long long)chan * g.N + state_of(g, 4 * q + i)] * LOG2E : 0.f;
    float bias[S::EACH], skip[S::EACH], dskip[S::EACH], dbias[S::EACH];
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) {
        bias[i] = in.dt_bias && i * STEP < n ? in.dt_bias[first_chan + i * STEP] : 0.f;
        skip[i] = in.D && i * STEP < n ? in.D[first_chan + i * STEP] : 0.f;
        dskip[i] = dbias[i] = 0.f;
    }

    // the sequence of the tile's first token, looked for again where a tile lies before it
    int s = g.seq.of_one(t1 - 1), head = g.seq.start(s), behind_it = g.seq.start(s + 1);
    if (out.ends && t1 < g.seq.T) {                                  // what the parts behind hand back to the sequence that goes on there
        // (parts whose first token that sequence still has)
        const long long reach = ((long long)(behind_it < g.seq.T ? behind_it : g.seq.T) - 1) / g.part - at.part;
        const int most = g.parts - 1 - at.part;
        gather_parts<LPC>(gr, a2, out.ends, out.sums, g.C, chan, q, valid, at.part + 1, 1, reach < most ? (int)reach : most);
    }

    // Where a lane's sum of dB or dC goes: state 4 q and the next for even and odd rows, two further for the upper eight lanes of a row.  A lane that is left
    // without one writes where nothing reads: no branch, across which the compiler would move work and hold more in registers.
    float *const sum_to = LPC == 16 || (lane & 7) < LPC
                              ? &red[wv][0][(lane >> 5) * S::STATES + 4 * q + (lane >> 4 & 1) + (LPC < 16 && lane & 8 ? 2 : 0)]
                              : &red[4][0][lane % (2 * S::STATES)];

    auto init_of = [&](int s, float (&h)[4]) {
        int own = threadIdx.x;                                       // rare: its addresses are not to be held in registers meanwhile
        asm volatile("" : "+v"(own));
        const BufView rows(in.init + ((long long)s * g.C + at.group * g.per_group + at.block * S::CHANNELS) * g.N, VIEW_BYTES);
        const uint32_t four = states[own % LPC], off = in.init && valid ? (uint32_t)(own / LPC * g.N) * 4 : BufView::OUTSIDE;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __uint_as_float(rows.b32(off + (four >> 8 * i & 0xff), 0));
    };

    // offsets in bytes from a tile's first row: at most 16 rows of SEQOPS_MAX_STRIDE
    constexpr uint32_t W = sizeof(T);
    const uint32_t ox = ((uint32_t)row * (uint32_t)g.xs + first_chan) * W, odt = ((uint32_t)row * (uint32_t)g.dts + first_chan) * W;
    const uint32_t oz = ((uint32_t)row * (uint32_t)g.zs + first_chan) * W, oy = ((uint32_t)row * (uint32_t)g.ys + first_chan) * W;
    const uint32_t oh = (uint32_t)(mine * S::STATES + 4 * q) * 4;    // from the block's first channel
    const int last = t0 + (t1 - t0 - 1) / S::TOKENS * S::TOKENS;       // the tile that comes first
    Ahead<T, S::EACH, WHOLE, STEP> rx, rdt, rz, rdy;
    Ahead<T, 1, true> rb[S::SHARED], rc[S::SHARED];
    Ahead<float, 4, true> rh;
    // the rows of the tile that is loaded next, and of the one that is written next
    const T *px = (const T *)in.x + (long long)last * g.xs, *pdt = (const T *)in.dt + (long long)last * g.dts, *pdy = (const T *)in.dy + (long long)last * g.ys;
    const T *pz = in.z ? (const T *)in.z + (long long)last * g.zs : px;
    const T *pb = (const T *)in.B + (long long)last * g.bs + (long long)at.group * g.N, *pc = (const T *)in.C + (long long)last * g.cs + (long long)at.group * g.N;
    const float *ph = in.kept + ((long long)(last / KEPT_EVERY) * g.C + chan - mine) * S::STATES;
    T *pdx = (T *)out.dx + (long long)last * g.xs, *pddt = (T *)out.ddt + (long long)last * g.dts, *pdz = in.z ? (T *)out.dz + (long long)last * g.zs : pdx;
    float *pshared = out.shared + ((long long)(at.group * g.blocks_of_group + at.block) * g.seq.T + last) * (2 * S::STATES);
    uint32_t ob[S::SHARED], oc[S::SHARED];
    float share[S::SHARED];                                          // of C that a slot has
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
        rdy.load(BufView(pdy, VIEW_BYTES), oy, m);
        rz.load(BufView(pz, VIEW_BYTES), oz, in.z ? m : 0);
        const BufView b(pb, VIEW_BYTES), c(pc, VIEW_BYTES);
#pragma unroll
        for (int i = 0; i < S::SHARED; ++i) {
            const int there = (int)(threadIdx.x + 256 * i) / S::STATES < (left < S::TOKENS ? left : S::TOKENS);     // (a lane without a value: a row behind the tile)
            rb[i].load(b, ob[i], there);
            rc[i].load(c, oc[i], there);
        }
        rh.load(BufView(ph, VIEW_BYTES), oh, valid);
        px -= S::TOKENS * g.xs;
        pdt -= S::TOKENS * g.dts;
        pdy -= S::TOKENS * g.ys;
        pz -= S::TOKENS * g.zs;
        pb -= S::TOKENS * g.bs;
        pc -= S::TOKENS * g.cs;
        ph -= (long long)g.C * S::STATES;
    };
    if (threadIdx.x < LPC) {
        uint32_t four = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) four |= (uint32_t)state_of(g, 4 * threadIdx.x + i) * 4 << 8 * i;
        states[threadIdx.x] = four;
    }
    for (int e = threadIdx.x; e < 2 * S::TOKENS * LPC; e += 256) shared_rows[2][0][e] = make_float4(0.f, 0.f, 0.f, 0.f);
    const float4 *const own_rows = &shared_rows[valid ? 0 : 2][0][q];
    load(last);
    for (int tile = last; tile >= t0; tile -= S::TOKENS) {
        Ahead<T, S::EACH, WHOLE, STEP> kx = rx, kdt = rdt, kz = rz, kdy = rdy;
        const T *const hx = px + S::TOKENS * g.xs, *const hdt = pdt + S::TOKENS * g.dts, *const hdy = pdy + S::TOKENS * g.ys;   // this tile's rows
        const T *const hz = pz + S::TOKENS * g.zs;
        const float hin[4] = {rh.at(0), rh.at(1), rh.at(2), rh.at(3)};
        const int m = tile + row < t1 ? n : 0;
        float delta[S::EACH];
        {
            float dv[S::EACH];
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) {
                delta[i] = kdt.at(i) + bias[i];
                dv[i] = kdy.at(i);
            }
            step_sizes(g, delta);
            if (in.z) {
#pragma unroll
                for (int i = 0; i < S::EACH; ++i) { const float zv = kz.at(i); dv[i] *= zv * sigmoid(zv); }
            }
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) {
                steps[row][col + i * STEP] = delta[i];
                gains[row][col + i * STEP] = delta[i] * kx.at(i);
                dvs[row][col + i * STEP] = dv[i];
            }
        }
#pragma unroll
        for (int i = 0; i < S::SHARED; ++i) {
            const int e = threadIdx.x + 256 * i;
            if (e < S::TOKENS * S::STATES) {
                reinterpret_cast<float *>(shared_rows[0])[e] = rb[i].at(0);
                reinterpret_cast<float *>(shared_rows[1])[e] = rc[i].at(0) * share[i];
            }
        }
        if (tile < head) { s = g.seq.of_one(tile); head = g.seq.start(s); behind_it = g.seq.start(s + 1); }
        const bool any = head >= tile || behind_it < tile + S::TOKENS;
        int of = 0;
        const uint32_t firsts = any ? first_tokens(g.seq, tile, S::TOKENS, t1, of) : 0u;
        if (tile > t0) load(tile - S::TOKENS);
        __syncthreads();

        auto walk = [&](auto special) {
            constexpr bool SPECIAL = decltype(special)::value;
            float h[S::TOKENS][4], decays[HELD > 0 ? HELD : 1][4], sums[LPC], more[LPC];
#pragma unroll
            for (int t = 0; t < S::TOKENS; ++t) {
                const float d = steps[t][mine], gain = gains[t][mine];
                const float4 b = own_rows[t * LPC], c = own_rows[(S::TOKENS + t) * LPC];
                const float bv[4] = {b.x, b.y, b.z, b.w}, cv[4] = {c.x, c.y, c.z, c.w};
                float before[4], sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) before[i] = t ? h[t ? t - 1 : 0][i] : hin[i];
                if constexpr (SPECIAL) {
                    if (firsts >> t & 1) init_of(sequence_of(of, t), before);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float decay = exp2_fast(d * a2[i]);
                    if (t >= S::TOKENS - HELD) decays[t >= S::TOKENS - HELD ? t - (S::TOKENS - HELD) : 0][i] = decay;
                    h[t][i] = fmaf(decay, before[i], gain * bv[i]);
                    sum = fmaf(cv[i], h[t][i], sum);
                }
                sums[t % LPC] = sum;
                if (t % LPC == LPC - 1) ys[t - (LPC - 1) + q][mine] = transpose_sum<LPC>(sums, q);
            }
            // Read LDS again on the way back: without these the compiler keeps what it read on the way there, 11 values a token, in registers, and spills.
            int mine2 = mine, skipped = 0;
            asm volatile("" : "+v"(mine2), "+v"(skipped));
            const float4 *const again = own_rows + skipped;
#pragma unroll
            for (int t = S::TOKENS - 1; t >= 0; --t) {
                if (SPECIAL && tile + t >= t1) {                     // behind the last token
                    sums[t % LPC] = more[t % LPC] = 0.f;
                } else {
                    const float d = steps[t][mine2], gain = gains[t][mine2], dv = dvs[t][mine2];
                    const float4 b = again[t * LPC], c = again[(S::TOKENS + t) * LPC];
                    const float bv[4] = {b.x, b.y, b.z, b.w}, cv[4] = {c.x, c.y, c.z, c.w};
                    float before[4], db[4], dc[4], sg = 0.f, sa = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) before[i] = t ? h[t ? t - 1 : 0][i] : hin[i];
                    if constexpr (SPECIAL) {
                        if (firsts >> t & 1) init_of(sequence_of(of, t), before);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        gr[i] = fmaf(dv, cv[i], gr[i]);
                        db[i] = gr[i] * gain;
                        dc[i] = dv * h[t][i];
                        sg = fmaf(gr[i], bv[i], sg);
                        gr[i] *= t >= S::TOKENS - HELD ? decays[t >= S::TOKENS - HELD ? t - (S::TOKENS - HELD) : 0][i] : exp2_fast(d * a2[i]);
                        const float r = gr[i] * before[i];
                        sa = fmaf(r, a2[i], sa);
                        dA[i] = fmaf(r, d, dA[i]);
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
                    float *const to = sum_to + t * 2 * S::STATES;
                    if constexpr (LPC == 16) {
                        to[0] = w0;
                        to[2] = w1;
                    } else {
                        const float u0 = w0 + lane_move<DPP_ROR8>(w0), u1 = w1 + lane_move<DPP_ROR8>(w1);   // (every lane moves: no branch here)
                        float w = lane & 8 ? u1 : u0;
                        if constexpr (LPC <= 4) w += lane_move<0x104>(w);        // four lanes further up; used in the lower four of eight
                        if constexpr (LPC == 2) w += lane_move<DPP_XOR2>(w);
                        *to = w;
                    }
                }
                if (t % LPC == 0) {
                    const float a = transpose_sum<LPC>(sums, q), b2 = transpose_sum<LPC>(more, q);
                    steps[t + q][mine] = a;
                    gains[t + q][mine] = b2 * LN2;
                }
            }
        };
        if (firsts || tile + S::TOKENS > t1) walk(std::true_type());
        else walk(std::false_type());
        if constexpr (AGAIN) {
            kx.load(BufView(hx, VIEW_BYTES), ox, m);
            kdt.load(BufView(hdt, VIEW_BYTES), odt, m);
            kdy.load(BufView(hdy, VIEW_BYTES), oy, m);
            kz.load(BufView(hz, VIEW_BYTES), oz, in.z ? m : 0);
        }
        __syncthreads();

        {
            // (a branch for all of a lane's channels, not one for each)
            float dv[S::EACH], dx[S::EACH], dd[S::EACH], dz[S::EACH] = {};
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) dv[i] = kdy.at(i);
            if (in.z) {
                float y[S::EACH];
#pragma unroll
                for (int i = 0; i < S::EACH; ++i) y[i] = ys[row][col + i * STEP];
                if (in.D) {
                    asm volatile("");                                // (a branch, not a choice for each)
#pragma unroll
                    for (int i = 0; i < S::EACH; ++i) y[i] = fmaf(skip[i], kx.at(i), y[i]);
                }
#pragma unroll
                for (int i = 0; i < S::EACH; ++i) {
                    const float zv = kz.at(i), sz = sigmoid(zv);
                    dz[i] = dv[i] * y[i] * (sz + zv * sz * (1.f - sz));
                    dv[i] *= zv * sz;
                }
            }
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) {
                const float gb = steps[row][col + i * STEP];
                dx[i] = delta[i] * gb;
                dd[i] = fmaf(kx.at(i), gb, gains[row][col + i * STEP]);
            }
            if (in.D) {
                asm volatile("");
#pragma unroll
                for (int i = 0; i < S::EACH; ++i) dx[i] = fmaf(skip[i], dv[i], dx[i]);
            }
            if (g.softplus) {
#pragma unroll
                for (int i = 0; i < S::EACH; ++i) dd[i] *= sigmoid(kdt.at(i) + bias[i]);
            }
            const bool counts = m > 0;
#pragma unroll
            for (int i = 0; i < S::EACH; ++i) {
                dskip[i] += counts ? dv[i] * kx.at(i) : 0.f;
                dbias[i] += counts ? dd[i] : 0.f;
            }
            store_late<T, S::EACH, WHOLE, STEP>(BufView(pdx, VIEW_BYTES), ox, m, dx);
            store_late<T, S::EACH, WHOLE, STEP>(BufView(pddt, VIEW_BYTES), odt, m, dd);
            store_late<T, S::EACH, WHOLE, STEP>(BufView(pdz, VIEW_BYTES), oz, in.z ? m : 0, dz);
            const BufView to(pshared, VIEW_BYTES);
            const int there = (t1 - tile) * 2 * S::STATES;
#pragma unroll
            for (int e = threadIdx.x, i = 0; i < (S::TOKENS * 2 * S::STATES + 255) / 256; ++i, e += 256) {
                const int t = e / (2 * S::STATES), k = e % (2 * S::STATES);
                if constexpr (S::TOKENS * 2 * S::STATES % 256 != 0) { if (e >= S::TOKENS * 2 * S::STATES) break; }
                const float sum[1] = {(red[0][t][k] + red[1][t][k]) + (red[2][t][k] + red[3][t][k])};
                store_late<float, 1, true>(to, (uint32_t)e * 4, e < there, sum);
            }
            pdx -= S::TOKENS * g.xs;
            pddt -= S::TOKENS * g.dts;
            pdz -= S::TOKENS * g.zs;
            pshared -= S::TOKENS * 2 * S::STATES;
        }
    }

    // the part's sums over tokens: [C,N] of A, then [C] of D and [C] of dt_bias
    float *const to = out.dA + (long long)at.part * ((long long)g.C * g.N + 2ll * g.C);
    float *const slots = &red[0][0][0];
    static_assert(S::CHANNELS * S::STATES <= (int)(sizeof red / sizeof(float)), "room for a value of each slot");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) slots[mine * S::STATES + 4 * q + i] = dA[i];
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) { steps[row][col + i * STEP] = dskip[i]; gains[row][col + i * STEP] = dbias[i]; }
    __syncthreads();
    if (valid) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = 4 * q + i;
            if (k >= g.N) continue;
            each_copy(g, S::STATES, k, [&](int copy) { dA[i] += slots[mine * S::STATES + copy]; });     // (which have their shares of it)
            to[(long long)chan * g.N + k] = dA[i];
        }
    }
    for (int c = threadIdx.x; c < S::CHANNELS; c += 256) {
        const int k = at.block * S::CHANNELS + c;
        if (k >= g.per_group) continue;
        float a = 0.f, b = 0.f;
        for (int r = 0; r < S::TOKENS; ++r) { a += steps[r][c]; b += gains[r][c]; }
        to[(long long)g.C * g.N + at.group * g.per_group + k] = a;
        to[(long long)g.C * g.N + g.C + at.group * g.per_group + k] = b;
    }
}

// dB and dC: the sum over a group's channel blocks, a lane a value, neighbours at neighbouring states; from value `first` on.
template <typename T>
__global__ __launch_bounds__(256) void k_sscan_bwd_shared(Scan g, int states, long long first, const float *__restrict__ shared, T *__restrict__ dB,
                                                          T *__restrict__ dC)
{
    const long long id = first + (long long)blockIdx.x * 256 + threadIdx.x;
    const int k = (int)(id % (2 * g.N)), n = k % g.N, is_c = k / g.N;
    const long long rest = id / (2 * g.N), t = rest / g.groups;
    const int group = (int)(rest % g.groups);
    if (t >= g.seq.T) return;
    const long long step = (long long)g.seq.T * 2 * states;
    const float *p = shared + (long long)group * g.blocks_of_group * step + t * 2 * states + is_c * states + n;
    float sum = 0.f;
    auto add = [&](int k) {
#pragma unroll 4
        for (int b = 0; b < g.blocks_of_group; ++b) sum += p[b * step + k - n];
    };
    add(n);
    if (!is_c) each_copy(g, states, n, add);                         // (dC is the same in all of them)
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
        const long long blocks = (long long)p.channel_blocks * p.parts, sums = ((long long)d->T * d->groups * 2 * d->N + 255) / 256;
        if (!launchable(blocks, 256)) return hipErrorInvalidValue;
        const hipError_t e = with_state_lanes(p.lanes, [&](auto lanes) {
            constexpr int LPC = decltype(lanes)::value;
            auto both = [&](auto whole) {
                constexpr bool WHOLE = decltype(whole)::value;
                if (p.carry) hipLaunchKernelGGL((k_sscan_bwd_carry<T, LPC, WHOLE>), dim3((unsigned)(blocks - p.channel_blocks)), dim3(256), 0, stream, g, in, out);
                hipLaunchKernelGGL((k_sscan_bwd<T, LPC, WHOLE>), dim3((unsigned)blocks), dim3(256), 0, stream, g, in, out);
            };
            const bool whole = whole_vectors<T>(BackTile<LPC>::EACH, g.per_group, {t->x, t->dt, t->z, t->dy, t->dx, t->ddt, t->dz}, {g.xs, g.dts, g.zs, g.ys});
            if (whole) both(std::true_type());
            else both(std::false_type());
            for (long long b = 0; b < sums; b += most_blocks(256)) {
                const long long n = sums - b < most_blocks(256) ? sums - b : most_blocks(256);
                hipLaunchKernelGGL(k_sscan_bwd_shared<T>, dim3((unsigned)n), dim3(256), 0, stream, g, 4 * LPC, b * 256, workspace + space.shared, (T *)t->dB,
                                   (T *)t->dC);
            }
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
