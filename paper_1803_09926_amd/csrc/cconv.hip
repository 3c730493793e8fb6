// Causal depthwise convolution over packed tokens, forward, backward and one token at a time.  The contract stands in include/seqops.h.
//
// A lane owns V neighbouring channels and walks down a strip of tokens with the last K - 1 rows in registers, so that each row is read once a strip (and
// K - 1 rows more at its head).  All three passes are bound by memory: forward 8191 x 1536 in bf16 takes 13 us, 3.9 TB/s, where a copy of these rows takes
// 10.5 (strips are 12 tokens there, and three rows of each come twice); backward 16384 x 1024 in fp32 47 us, 4.3 TB/s, and 4.7 for the sum of the partials,
// where an addition of tensors of that size takes 35.  At a sequence's first token the rows in registers are replaced by the sequence's
// rows of init, or zeros: what an earlier sequence holds, infinities and NaN among it, is never multiplied by anything of a later one.
//
// Backward: with dp = dy * dy/dp at token t, dx[t-(K-1)+k] += w[k] dp.  The walk holds the K - 1 sums that are not complete yet and goes K - 1 tokens
// past its strip; the pre-activation is computed again from x, which is read anyway for the filter's gradient.  That gradient's sums stay in
// registers over the strip, a block adds its strips in LDS in a fixed order, and the blocks' partials meet in seq_sum.hip.
#include "seq_common.hpp"
#include "tune.hpp"
#include <stdlib.h>

namespace dwc {

namespace {

struct Conv {
    int C, silu, per_block, strip;   // channel vectors of a block (a power of two up to 64); tokens of a strip
    unsigned across;                 // blocks that share a strip: a block's number is that of its strips times this, plus that of its channels
    long long x_stride, y_stride;
    Sequences seq;
};

// A lane's V channels of a row.  WHOLE: all there, at an address of theirs (one load, no branch, so that nothing waits for it before it is used); otherwise the
// first n of them are.
template <typename T, int V, bool WHOLE> __device__ __forceinline__ void load_row(Some<T, V> &v, const T *p, int n)
{
    if constexpr (WHOLE) v.load(p, V);
    else v.load(p, n);
}

// The rows before token t in registers: those of its own sequence, whose first token is `first` (clamped to 0 .. t by the caller), else init's, else zeros.
template <typename T, int K, int V, bool WHOLE>
__device__ __forceinline__ void window_at(float (&win)[K - 1][V], const Conv &g, const T *x, const T *init, int s, int first, int t, int c, int n)
{
    Some<T, V> rows[K - 1];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const int pos = t - (K - 1) + j, back = pos - first;    // back < 0: that many rows before the first token
        const T *const own = x + (long long)(back >= 0 ? pos : t) * g.x_stride + c;
        const T *const given = init + ((long long)s * (K - 1) + (K - 1) + (back >= 0 ? -1 : back)) * g.C + c;
        load_row<T, V, WHOLE>(rows[j], back >= 0 || !init ? own : given, n);
        if (back < 0 && !init) rows[j].zero();
    }
#pragma unroll
    for (int j = 0; j < K - 1; ++j) rows[j].get(win[j]);
}

template <typename T, int K, int V, bool WHOLE>
__global__ __launch_bounds__(256) void k_cconv_fwd(Conv g, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ b,
                                                   const T *__restrict__ init, T *__restrict__ y, T *__restrict__ final)
{
    constexpr int AHEAD = 4;                    // rows asked for at a time, before those in hand are used
    const int c = ((int)(blockIdx.x % g.across) * g.per_block + threadIdx.x % g.per_block) * V, n = g.C - c;
    const long long strip = (long long)(blockIdx.x / g.across) * (256 / g.per_block) + threadIdx.x / g.per_block;
    const int T_ = g.seq.T;
    if (n <= 0 || (strip > 0 && strip * g.strip >= T_)) return;
    const int t0 = (int)(strip * g.strip), t1 = T_ - t0 < g.strip ? T_ : t0 + g.strip;

    auto finish = [&](int s, const float (&rows)[K - 1][V]) {      // (as stored: what is rounded here was stored before)
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            Some<T, V> v;
            v.set(rows[j]);
            v.store(final + ((long long)s * (K - 1) + j) * g.C + c, n);
        }
    };
    auto finish_empty = [&](int s) {            // an empty sequence hands on what it was given
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            Some<T, V> v;
            v.zero();
            if (init) v.load(init + ((long long)s * (K - 1) + j) * g.C + c, n);
            v.store(final + ((long long)s * (K - 1) + j) * g.C + c, n);
        }
    };

    // the rows and the filter first: looking the sequence up takes several loads, one after the other
    Some<T, V> ahead[AHEAD], taps[K], biases;
    float win[K - 1][V], bias[V], tap[K][V];
    auto load = [&](int t) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load_row<T, V, WHOLE>(ahead[u], x + (long long)(t + u < t1 ? t + u : t1 - 1) * g.x_stride + c, n);
    };
    if (t1 > t0) load(t0);
#pragma unroll
    for (int k = 0; k < K; ++k) load_row<T, V, WHOLE>(taps[k], w + (long long)k * g.C + c, n);
    biases.zero();
    if (b) load_row<T, V, WHOLE>(biases, b + c, n);

    int s = T_ > 0 ? g.seq.of(t0) : g.seq.n;
    if (t0 == 0 && final)
        for (int e = 0; e < s; ++e) finish_empty(e);
    if (t1 <= t0) return;
    int next = g.seq.start(s + 1);
    {
        const int first = g.seq.start(s);
        window_at<T, K, V, WHOLE>(win, g, x, init, s, first < 0 ? 0 : first < t0 ? first : t0, t0, c, n);
    }

#pragma unroll
    for (int k = 0; k < K; ++k) taps[k].get(tap[k]);
    biases.get(bias);
    for (int t = t0; t < t1; t += AHEAD) {
        Some<T, V> rows[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) rows[u] = ahead[u];
        if (t + AHEAD < t1) load(t + AHEAD);
        auto token = [&](int u) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float p = bias[i];
#pragma unroll
                for (int k = 0; k < K - 1; ++k) p += tap[k][i] * win[k][i];
                p += tap[K - 1][i] * rows[u].at(i);
                o[i] = g.silu ? p * sigmoid(p) : p;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int k = 0; k + 1 < K - 1; ++k) win[k][i] = win[k + 1][i];
                win[K - 2][i] = rows[u].at(i);
            }
            Some<T, V> out;
            out.set(o);
            out.store(y + (long long)(t + u) * g.y_stride + c, WHOLE ? V : n);
        };
        if (t + AHEAD <= t1 && next > t + AHEAD && t + AHEAD < T_) {     // inside a sequence, and not to its end
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) token(u);
            continue;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (t + u >= t1) break;
            if (t + u == next) {                // a new sequence
                s = g.seq.of(t + u);
                next = g.seq.start(s + 1);
                window_at<T, K, V, WHOLE>(win, g, x, init, s, t + u, t + u, c, n);
            }
            token(u);
            if (final && (t + u + 1 == next || t + u + 1 == T_)) {
                finish(s, win);
                for (int e = s + 1; e < g.seq.n && g.seq.start(e + 1) <= t + u + 1; ++e) finish_empty(e);
            }
        }
    }
}

template <typename T, int K, int V, bool WHOLE>
__global__ __launch_bounds__(256, K <= 4 ? 3 : 2) void k_cconv_bwd(Conv g, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ b,
                                                   const T *__restrict__ init, const T *__restrict__ dy, T *__restrict__ dx, float *__restrict__ partials)
{
    constexpr int AHEAD = 2;
    extern __shared__ float lds[];              // [strips of the block][per_block][K + 1][V]
    const int strips = 256 / g.per_block, which = threadIdx.x / g.per_block, col = threadIdx.x % g.per_block;
    const int c = ((int)(blockIdx.x % g.across) * g.per_block + col) * V, n = g.C - c;
    const long long strip = (long long)(blockIdx.x / g.across) * strips + which;
    const int T_ = g.seq.T;
    float gw[K + 1][V];                         // the filter's gradient, and the bias's
#pragma unroll
    for (int k = 0; k <= K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) gw[k][i] = 0.f;

    if (n > 0 && strip * g.strip < T_) {
        const int t0 = (int)(strip * g.strip), t1 = T_ - t0 < g.strip ? T_ : t0 + g.strip;
        const int end = T_ - t1 < K - 1 ? T_ : t1 + K - 1;      // the last tokens only add to the strip's dx
        Some<T, V> rows_ahead[AHEAD], grads_ahead[AHEAD], taps[K], biases;
        float win[K - 1][V], bias[V], tap[K][V];
        auto load = [&](int t) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const long long at = t + u < end ? t + u : end - 1;
                load_row<T, V, WHOLE>(rows_ahead[u], x + at * g.x_stride + c, n);
                load_row<T, V, WHOLE>(grads_ahead[u], dy + at * g.y_stride + c, n);
            }
        };
        load(t0);
#pragma unroll
        for (int k = 0; k < K; ++k) load_row<T, V, WHOLE>(taps[k], w + (long long)k * g.C + c, n);
        biases.zero();
        if (b) load_row<T, V, WHOLE>(biases, b + c, n);
        int s = g.seq.of(t0), first = g.seq.start(s), next = g.seq.start(s + 1);
        first = first < 0 ? 0 : first < t0 ? first : t0;
        window_at<T, K, V, WHOLE>(win, g, x, init, s, first, t0, c, n);
        float open[K - 1][V];                   // dx of the K - 1 tokens before t, as far as it goes
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) open[k][i] = 0.f;

#pragma unroll
        for (int k = 0; k < K; ++k) taps[k].get(tap[k]);
        biases.get(bias);
        for (int t = t0; t < t1 + K - 1; t += AHEAD) {
            Some<T, V> rows[AHEAD], grads[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) { rows[u] = rows_ahead[u]; grads[u] = grads_ahead[u]; }
            if (t + AHEAD < end) load(t + AHEAD);
            // the gradient at the pre-activation of token t + u, whose rows move on
            auto gradient = [&](int u, bool mine, float (&dp)[V]) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float p = bias[i];
#pragma unroll
                    for (int k = 0; k < K - 1; ++k) p += tap[k][i] * win[k][i];
                    p += tap[K - 1][i] * rows[u].at(i);
                    float d = grads[u].at(i);
                    if (g.silu) { const float q = sigmoid(p); d *= q + p * q * (1.f - q); }
                    dp[i] = d;
                }
                if (mine) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
#pragma unroll
                        for (int k = 0; k < K - 1; ++k) gw[k][i] += dp[i] * win[k][i];
                        gw[K - 1][i] += dp[i] * rows[u].at(i);
                        gw[K][i] += dp[i];
                    }
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
#pragma unroll
                    for (int k = 0; k + 1 < K - 1; ++k) win[k][i] = win[k + 1][i];
                    win[K - 2][i] = rows[u].at(i);
                }
            };
            // what it adds to the tokens before it, `reach` of them at most; the one that is complete with it is written
            auto add = [&](int at, int reach, const float (&dp)[V]) {
                float done[V];
                auto adds = [&](int k, int i) { return reach >= K - 1 - k ? tap[k][i] * dp[i] : 0.f; };
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    done[i] = open[0][i] + adds(0, i);
#pragma unroll
                    for (int k = 0; k + 1 < K - 1; ++k) open[k][i] = open[k + 1][i] + adds(k + 1, i);
                    open[K - 2][i] = adds(K - 1, i);
                }
                if (at - (K - 1) >= t0) {
                    Some<T, V> out;
                    out.set(done);
                    out.store(dx + (long long)(at - (K - 1)) * g.x_stride + c, WHOLE ? V : n);
                }
            };
            if (t + AHEAD <= t1 && next >= t + AHEAD && t - first >= K - 1 && t - (K - 1) >= t0) {     // far inside a sequence and the strip
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    float dp[V];
                    gradient(u, true, dp);
                    float done[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        done[i] = open[0][i] + tap[0][i] * dp[i];
#pragma unroll
                        for (int k = 0; k + 1 < K - 1; ++k) open[k][i] = open[k + 1][i] + tap[k + 1][i] * dp[i];
                        open[K - 2][i] = tap[K - 1][i] * dp[i];
                    }
                    Some<T, V> out;
                    out.set(done);
                    out.store(dx + (long long)(t + u - (K - 1)) * g.x_stride + c, WHOLE ? V : n);
                }
                continue;
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int at = t + u;
                if (at >= t1 + K - 1) break;
                float dp[V];
#pragma unroll
                for (int i = 0; i < V; ++i) dp[i] = 0.f;
                if (at < end) {
                    if (at == next) {
                        s = g.seq.of(at);
                        first = at;
                        next = g.seq.start(s + 1);
                        window_at<T, K, V, WHOLE>(win, g, x, init, s, at, at, c, n);
                    }
                    gradient(u, at < t1, dp);
                }
                add(at, at < end ? at - first : -1, dp);        // (in its own sequence only)
            }
        }
    }

    // [K + 1][C] a block: its strips one after the other
    const int width = g.per_block * (K + 1) * V;
#pragma unroll
    for (int k = 0; k <= K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i)
            lds[which * width + (col * (K + 1) + k) * V + i] = gw[k][i];
    __syncthreads();
    float *out = partials + (long long)(blockIdx.x / g.across) * (K + 1) * g.C;
    for (int e = threadIdx.x; e < width; e += 256) {
        const int k = e / (g.per_block * V), ch = e % (g.per_block * V), from = (ch / V * (K + 1) + k) * V + ch % V;
        const int cc = (int)(blockIdx.x % g.across) * g.per_block * V + ch;
        if (cc >= g.C) continue;
        float sum = 0.f;
        for (int i = 0; i < strips; ++i) sum += lds[i * width + from];
        out[(long long)k * g.C + cc] = sum;
    }
}

// A block of 64 lanes takes neighbouring channels of one row, `across` of them the row: its slot is a scalar.
template <typename T, int K, int V>
__global__ __launch_bounds__(64) void k_cconv_step(Conv g, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ b,
                                                   const int32_t *__restrict__ slots, T *__restrict__ state, T *__restrict__ y)
{
    const int t = (int)(blockIdx.x / g.across), c = ((int)(blockIdx.x % g.across) * 64 + threadIdx.x) * V, n = g.C - c;
    if (n <= 0) return;
    const int slot = slots ? slots[t] : t;
    T *const yr = y + (long long)t * g.y_stride + c;
    Some<T, V> out;
    if (slot < 0 || slot >= g.seq.n) {
        out.zero();
        out.store(yr, n);
        return;
    }
    T *const st = state + (long long)slot * (K - 1) * g.C + c;
    Some<T, V> win[K], tap[K], bias;
#pragma unroll
    for (int k = 0; k < K - 1; ++k) win[k].load(st + (long long)k * g.C, n);
    win[K - 1].load(x + (long long)t * g.x_stride + c, n);
#pragma unroll
    for (int k = 0; k < K; ++k) tap[k].load(w + (long long)k * g.C + c, n);
    bias.zero();
    if (b) bias.load(b + c, n);
#pragma unroll
    for (int k = 0; k < K - 1; ++k) win[k + 1].store(st + (long long)k * g.C, n);
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float p = bias.at(i);
#pragma unroll
        for (int k = 0; k < K; ++k) p += tap[k].at(i) * win[k].at(i);
        o[i] = g.silu ? p * sigmoid(p) : p;
    }
    out.set(o);
    out.store(yr, n);
}

// ---- host ----------------------------------------------------------------------------------------

int validate(const cconv_desc *d)
{
    if (!d) return DWCONV_ERR_NULL;
    if (d->dtype != DWCONV_F32 && d->dtype != DWCONV_BF16) return DWCONV_ERR_BAD_ENUM;
    if (d->silu != 0 && d->silu != 1) return DWCONV_ERR_BAD_ENUM;
    if (d->T < 0 || d->C < 1 || d->K < 2 || d->sequences < 1) return DWCONV_ERR_BAD_DIM;
    if (d->T > 1 && (d->x_stride < d->C || d->y_stride < d->C)) return DWCONV_ERR_BAD_DIM;
    if (d->K > CCONV_MAX_K) return DWCONV_ERR_UNSUPPORTED;
    // tokens are counted in int, a strip beyond the last one included; offsets in 64 bits
    if (d->T > SEQOPS_MAX_T || d->sequences > SEQOPS_MAX_T || d->C > SEQOPS_MAX_C || d->x_stride > SEQOPS_MAX_STRIDE || d->y_stride > SEQOPS_MAX_STRIDE)
        return DWCONV_ERR_TOO_LARGE;
    return DWCONV_OK;
}

constexpr int CHANNELS = 4;                      // of a lane, in both types: 8 of bf16 are half the wavefronts, and 15.4 us for 8191 x 1536 instead of 12.3

int lanes_for(int vectors)                       // channel vectors of a block: a power of two, at most a wavefront's
{
    int p = 1;
    while (p < vectors && p < 64) p *= 2;
    return p;
}

struct Launch { int vectors, per_block, strip; long long down; unsigned across; };   // blocks along the tokens, and along the channels
// The head's K - 1 rows of a strip are read again, so strips are as long as leave each compute unit `lanes` lanes, from `least` tokens to `most`.
Launch plan_launch(const cconv_desc *d, int lanes, int least, int most)
{
    Launch l;
    l.vectors = cdiv(d->C, CHANNELS);
    l.per_block = lanes_for(l.vectors);
    l.across = (unsigned)cdiv(l.vectors, l.per_block);
    const long long tokens = (long long)d->T * l.across * l.per_block / (256 * lanes) / 4 * 4;
    const char *const forced = tune_env("DWCONV_TUNE_CCONV_STRIP");
    l.strip = forced && atoi(forced) > 0 ? atoi(forced) : (int)(tokens < least ? least : tokens > most ? most : tokens);
    const long long per = (long long)l.strip * (256 / l.per_block);
    l.down = d->T > 0 ? (d->T + per - 1) / per : 1;
    return l;
}
// Strips of 8, 12, 16, 20, 32, 64 tokens, forward, 8191 x 1536 in bf16 (12 by this rule): 15.4, 13.7, 13.9, 15.2, 16.1, 19.8 us.  Backward, 16384 x 1024 in
// fp32 (32 by this rule), 8, 16, 24, 32, 48, 64: 62, 59.5, 50.3, 50.5, 59.4, 60.3 us (a block's partials are K + 1 rows for strip * 256 / per_block
// tokens).  Few tokens: the walk down a strip is a chain, so it is short: strips of 4, 8, 16 tokens, backward, 200 x 768 in either type 12.0, 13.2, 16.1 us, 4000 x
// 768 in fp32 19.6, 20.3, 21.4, but 1000 x 2048 15.6, 13.8, 18.0 (bf16).
Launch plan_fwd(const cconv_desc *d) { return plan_launch(d, 768, 4, 64); }
Launch plan_bwd(const cconv_desc *d) { return plan_launch(d, 512, 4, 128); }

Conv geometry(const cconv_desc *d, const Launch &l, const void *starts)
{
    Conv g;
    g.C = d->C; g.silu = d->silu; g.per_block = l.per_block; g.strip = l.strip; g.across = l.across;
    g.x_stride = d->x_stride; g.y_stride = d->y_stride;
    g.seq = {(const int32_t *)starts, d->sequences, d->T / d->sequences, d->T};
    return g;
}

template <typename F> hipError_t with_taps(int K, F f)
{
    switch (K) {
    case 2: f(std::integral_constant<int, 2>()); break;
    case 3: f(std::integral_constant<int, 3>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 5: f(std::integral_constant<int, 5>()); break;
    case 6: f(std::integral_constant<int, 6>()); break;
    case 7: f(std::integral_constant<int, 7>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <typename T> hipError_t launch_fwd(const cconv_desc *d, const cconv_tensors *t, hipStream_t stream)
{
    const Launch l = plan_fwd(d);
    if (!launchable(l.down * l.across, 256)) return hipErrorInvalidValue;
    return with_taps(d->K, [&](auto k) {
        constexpr int K = decltype(k)::value, V = CHANNELS;
        auto run = [&](auto whole) {
            hipLaunchKernelGGL((k_cconv_fwd<T, K, V, decltype(whole)::value>), dim3((unsigned)(l.down * l.across)), dim3(256), 0, stream,
                               geometry(d, l, t->starts), (const T *)t->x, (const T *)t->w, (const T *)t->b, (const T *)t->init, (T *)t->y, (T *)t->final);
        };
        if (d->C % V == 0) run(std::true_type());
        else run(std::false_type());
    });
}

template <typename T> hipError_t launch_bwd(const cconv_desc *d, const cconv_tensors *t, float *partials, hipStream_t stream)
{
    const Launch l = plan_bwd(d);
    if (!launchable(l.down * l.across, 256)) return hipErrorInvalidValue;
    return with_taps(d->K, [&](auto k) {
        constexpr int K = decltype(k)::value, V = CHANNELS;
        auto run = [&](auto whole) {
            hipLaunchKernelGGL((k_cconv_bwd<T, K, V, decltype(whole)::value>), dim3((unsigned)(l.down * l.across)), dim3(256),
                               256 * (K + 1) * V * sizeof(float), stream, geometry(d, l, t->starts), (const T *)t->x, (const T *)t->w, (const T *)t->b,
                               (const T *)t->init, (const T *)t->dy, (T *)t->dx, partials);
        };
        if (d->C % V == 0) run(std::true_type());
        else run(std::false_type());
    });
}

template <typename T> hipError_t launch_step(const cconv_desc *d, const cconv_tensors *t, hipStream_t stream)
{
    const int vectors = cdiv(d->C, CHANNELS);
    const Launch l = {vectors, 64, 1, d->T, (unsigned)cdiv(vectors, 64)};
    const long long most = most_blocks(64) / l.across;                // rows of one launch
    return with_taps(d->K, [&](auto k) {
        constexpr int K = decltype(k)::value;
        for (long long row = 0; row < d->T; row += most) {
            const long long rows = d->T - row < most ? d->T - row : most, own = t->slots ? 0 : row;     // the first slot, where rows have their own number
            Conv g = geometry(d, l, nullptr);
            g.seq.n -= (int)own;
            hipLaunchKernelGGL((k_cconv_step<T, K, CHANNELS>), dim3((unsigned)(rows * l.across)), dim3(64), 0, stream, g, (const T *)t->x + row * d->x_stride,
                               (const T *)t->w, (const T *)t->b, t->slots ? (const int32_t *)t->slots + row : nullptr,
                               (T *)t->state + own * (K - 1) * d->C, (T *)t->y + row * d->y_stride);
        }
    });
}

int status(hipError_t e) { return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH; }

}  // namespace

}  // namespace dwc

using namespace dwc;

extern "C" {

int cconv_fwd(const cconv_desc *desc, const cconv_tensors *t, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || !t->w || (desc->T > 0 && (!t->x || !t->y))) return DWCONV_ERR_NULL;
    if (!t->starts && desc->T % desc->sequences) return DWCONV_ERR_BAD_DIM;
    for (const void *p : {t->x, t->w, t->b, t->init, (const void *)t->y, (const void *)t->final})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    if (unaligned4(t->starts)) return DWCONV_ERR_ALIGN;
    if (desc->T == 0 && !t->final) return DWCONV_OK;
    return status(desc->dtype == DWCONV_F32 ? launch_fwd<float>(desc, t, (hipStream_t)stream) : launch_fwd<bf16_t>(desc, t, (hipStream_t)stream));
}

size_t cconv_bwd_workspace_bytes(const cconv_desc *desc)
{
    if (validate(desc) != DWCONV_OK || desc->T == 0) return 0;
    return (size_t)plan_bwd(desc).down * (size_t)(desc->K + 1) * (size_t)desc->C * sizeof(float);
}

int cconv_bwd(const cconv_desc *desc, const cconv_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || !t->w || !t->dw || (desc->T > 0 && (!t->x || !t->dy || !t->dx))) return DWCONV_ERR_NULL;
    if (!t->starts && desc->T % desc->sequences) return DWCONV_ERR_BAD_DIM;
    for (const void *p : {t->x, t->w, t->b, t->init, t->dy, (const void *)t->dx})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    for (const void *p : {t->starts, (const void *)t->dw, (const void *)t->db})
        if (unaligned4(p)) return DWCONV_ERR_ALIGN;
    const size_t need = cconv_bwd_workspace_bytes(desc);
    if (need && (!workspace || workspace_bytes < need)) return DWCONV_ERR_WORKSPACE;
    if (need && unaligned16(workspace)) return DWCONV_ERR_ALIGN;
    const hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (desc->T > 0)
        e = desc->dtype == DWCONV_F32 ? launch_bwd<float>(desc, t, (float *)workspace, s) : launch_bwd<bf16_t>(desc, t, (float *)workspace, s);
    const long long kc = (long long)desc->K * desc->C;
    if (e == hipSuccess)
        e = launch_sum_partials((const float *)workspace, desc->T > 0 ? (int)plan_bwd(desc).down : 0, kc, kc + desc->C, kc + desc->C, (float *)t->dw,
                                (float *)t->db, nullptr, s);
    return status(e);
}

int cconv_step(const cconv_desc *desc, const cconv_tensors *t, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || (desc->T > 0 && (!t->x || !t->w || !t->y || !t->state))) return DWCONV_ERR_NULL;
    if (!t->slots && desc->T > desc->sequences) return DWCONV_ERR_BAD_DIM;
    for (const void *p : {t->x, t->w, t->b, (const void *)t->state, (const void *)t->y})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    if (unaligned4(t->slots)) return DWCONV_ERR_ALIGN;
    if (desc->T == 0) return DWCONV_OK;
    return status(desc->dtype == DWCONV_F32 ? launch_step<float>(desc, t, (hipStream_t)stream) : launch_step<bf16_t>(desc, t, (hipStream_t)stream));
}

}  // extern "C"
