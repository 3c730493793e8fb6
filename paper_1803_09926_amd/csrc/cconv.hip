// Causal depthwise convolution over packed tokens, forward, backward and one token at a time.  The contract stands in include/seqops.h.
//
// A lane owns V neighbouring channels and walks down a strip of tokens with the last K - 1 rows in registers, so that each row is read once a strip (and
// K - 1 rows more at its head).  All three passes are bound by memory.  At a sequence's first token the rows in registers are replaced by the sequence's
// rows of init, or zeros: what an earlier sequence holds, infinities and NaN among it, is never multiplied by anything of a later one.
//
// Backward: with dp = dy * dy/dp at token t, dx[t-(K-1)+k] += w[k] dp.  The walk holds the K - 1 sums that are not complete yet and goes K - 1 tokens
// past its strip; the pre-activation is computed again from x, which is read anyway for the filter's gradient.  That gradient's sums stay in
// registers over the strip, a block adds its strips in LDS in a fixed order, and the blocks' partials meet in seq_sum.hip.
#include "seq_common.hpp"

namespace dwc {

namespace {

struct Conv {
    int C, silu, per_block, strip;   // channel vectors of a block (a power of two up to 64); tokens of a strip
    unsigned across;                 // blocks that share a strip: a block's number is that of its strips times this, plus that of its channels
    long long x_stride, y_stride;
    Sequences seq;
};

// The rows before token t in registers: those of its own sequence, whose first token is `first` (clamped to 0 .. t by the caller), else init's, else zeros.
template <typename T, int K, int V>
__device__ __forceinline__ void window_at(Some<T, V> (&win)[K - 1], const Conv &g, const T *x, const T *init, int s, int first, int t, int c, int n)
{
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const int pos = t - (K - 1) + j, back = pos - first;    // back < 0: that many rows before the first token
        if (back >= 0) win[j].load(x + (long long)pos * g.x_stride + c, n);
        else if (init) win[j].load(init + ((long long)s * (K - 1) + (K - 1) + back) * g.C + c, n);
        else win[j].zero();
    }
}

template <typename T, int K, int V>
__global__ __launch_bounds__(256) void k_cconv_fwd(Conv g, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ b,
                                                   const T *__restrict__ init, T *__restrict__ y, T *__restrict__ final)
{
    constexpr int AHEAD = 8;                    // rows asked for at a time
    const int c = ((int)(blockIdx.x % g.across) * g.per_block + threadIdx.x % g.per_block) * V, n = g.C - c;
    const long long strip = (long long)(blockIdx.x / g.across) * (256 / g.per_block) + threadIdx.x / g.per_block;
    const int T_ = g.seq.T;
    if (n <= 0 || (strip > 0 && strip * g.strip >= T_)) return;
    const int t0 = (int)(strip * g.strip), t1 = T_ - t0 < g.strip ? T_ : t0 + g.strip;

    auto finish = [&](int s, const Some<T, V> (&rows)[K - 1]) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j) rows[j].store(final + ((long long)s * (K - 1) + j) * g.C + c, n);
    };
    auto finish_empty = [&](int s) {            // an empty sequence hands on what it was given
        Some<T, V> rows[K - 1];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            if (init) rows[j].load(init + ((long long)s * (K - 1) + j) * g.C + c, n);
            else rows[j].zero();
        }
        finish(s, rows);
    };

    int s = T_ > 0 ? g.seq.of(t0) : g.seq.n;
    if (t0 == 0 && final)
        for (int e = 0; e < s; ++e) finish_empty(e);
    if (t1 <= t0) return;
    int next = g.seq.start(s + 1);
    Some<T, V> win[K - 1], bias, tap[K];
    {
        const int first = g.seq.start(s);
        window_at<T, K, V>(win, g, x, init, s, first < 0 ? 0 : first < t0 ? first : t0, t0, c, n);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) tap[k].load(w + (long long)k * g.C + c, n);
    bias.zero();
    if (b) bias.load(b + c, n);

    for (int t = t0; t < t1; t += AHEAD) {
        Some<T, V> rows[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (t + u < t1) rows[u].load(x + (long long)(t + u) * g.x_stride + c, n);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (t + u >= t1) break;
            if (t + u == next) {                // a new sequence
                s = g.seq.of(t + u);
                next = g.seq.start(s + 1);
                window_at<T, K, V>(win, g, x, init, s, t + u, t + u, c, n);
            }
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float p = bias.at(i);
#pragma unroll
                for (int k = 0; k < K - 1; ++k) p += tap[k].at(i) * win[k].at(i);
                p += tap[K - 1].at(i) * rows[u].at(i);
                o[i] = g.silu ? p * sigmoid(p) : p;
            }
#pragma unroll
            for (int k = 0; k + 1 < K - 1; ++k) win[k] = win[k + 1];
            win[K - 2] = rows[u];
            Some<T, V> out;
            out.set(o);
            out.store(y + (long long)(t + u) * g.y_stride + c, n);
            if (final && (t + u + 1 == next || t + u + 1 == T_)) {
                finish(s, win);
                for (int e = s + 1; e < g.seq.n && g.seq.start(e + 1) <= t + u + 1; ++e) finish_empty(e);
            }
        }
    }
}

template <typename T, int K, int V>
__global__ __launch_bounds__(256) void k_cconv_bwd(Conv g, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ b,
                                                   const T *__restrict__ init, const T *__restrict__ dy, T *__restrict__ dx, float *__restrict__ partials)
{
    constexpr int AHEAD = 4;
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
        int s = g.seq.of(t0), first = g.seq.start(s), next = g.seq.start(s + 1);
        first = first < 0 ? 0 : first < t0 ? first : t0;
        Some<T, V> win[K - 1], bias, tap[K];
        window_at<T, K, V>(win, g, x, init, s, first, t0, c, n);
#pragma unroll
        for (int k = 0; k < K; ++k) tap[k].load(w + (long long)k * g.C + c, n);
        bias.zero();
        if (b) bias.load(b + c, n);
        float open[K - 1][V];                   // dx of the K - 1 tokens before t, as far as it goes
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) open[k][i] = 0.f;

        for (int t = t0; t < t1 + K - 1; t += AHEAD) {
            Some<T, V> rows[AHEAD], grads[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (t + u < end) {
                    rows[u].load(x + (long long)(t + u) * g.x_stride + c, n);
                    grads[u].load(dy + (long long)(t + u) * g.y_stride + c, n);
                }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int at = t + u;
                if (at >= t1 + K - 1) break;
                float dp[V];
                if (at < end) {
                    if (at == next) {
                        s = g.seq.of(at);
                        first = at;
                        next = g.seq.start(s + 1);
                        window_at<T, K, V>(win, g, x, init, s, at, at, c, n);
                    }
                    const bool mine = at < t1;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float p = bias.at(i);
#pragma unroll
                        for (int k = 0; k < K - 1; ++k) p += tap[k].at(i) * win[k].at(i);
                        p += tap[K - 1].at(i) * rows[u].at(i);
                        float d = grads[u].at(i);
                        if (g.silu) { const float q = sigmoid(p); d *= q + p * q * (1.f - q); }
                        dp[i] = d;
                    }
                    if (mine) {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
#pragma unroll
                            for (int k = 0; k < K - 1; ++k) gw[k][i] += dp[i] * win[k].at(i);
                            gw[K - 1][i] += dp[i] * rows[u].at(i);
                            gw[K][i] += dp[i];
                        }
                    }
#pragma unroll
                    for (int k = 0; k + 1 < K - 1; ++k) win[k] = win[k + 1];
                    win[K - 2] = rows[u];
                }
                // what this token adds to those before it, in its own sequence only
                const int reach = at < end ? at - first : -1;
                float done[V];
                auto adds = [&](int k, int i) { return reach >= K - 1 - k ? tap[k].at(i) * dp[i] : 0.f; };
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
                    out.store(dx + (long long)(at - (K - 1)) * g.x_stride + c, n);
                }
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

template <typename T, int K, int V>
__global__ __launch_bounds__(256) void k_cconv_step(Conv g, int nv, const T *__restrict__ x, const T *__restrict__ w, const T *__restrict__ b,
                                                    const int32_t *__restrict__ slots, T *__restrict__ state, T *__restrict__ y)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int t = (int)(id / nv), c = (int)(id % nv) * V, n = g.C - c;
    if (t >= g.seq.T) return;
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

// Channels of a lane: 16 bytes, in the backward pass 4 channels (five registers a channel and tap).
template <typename T> constexpr int fwd_channels() { return 16 / (int)sizeof(T); }
constexpr int BWD_CHANNELS = 4;

int lanes_for(int vectors)                       // channel vectors of a block: a power of two, at most a wavefront's
{
    int p = 1;
    while (p < vectors && p < 64) p *= 2;
    return p;
}

// Tokens of a strip: the head's K - 1 rows are read again, so a strip is long where there are enough of them for the card (256 compute
// units of 16 wavefronts), and short where there are not.
int strip_for(const cconv_desc *d, int vectors, int least, int most)
{
    const int lanes = lanes_for(vectors);
    const long long lanes_a_token = (long long)cdiv(vectors, lanes) * lanes;
    const long long tokens = d->T * lanes_a_token / (256 * 1024);
    return (int)(tokens < least ? least : tokens > most ? most : tokens);
}

struct Launch { int vectors, per_block, strip; long long down; unsigned across; };   // blocks along the tokens, and along the channels
Launch plan_launch(const cconv_desc *d, int V, int least, int most)
{
    Launch l;
    l.vectors = cdiv(d->C, V);
    l.per_block = lanes_for(l.vectors);
    l.strip = strip_for(d, l.vectors, least, most);
    const long long per = (long long)l.strip * (256 / l.per_block);
    l.down = d->T > 0 ? (d->T + per - 1) / per : 1;
    l.across = (unsigned)cdiv(l.vectors, l.per_block);
    return l;
}
Launch plan_fwd(const cconv_desc *d) { return plan_launch(d, d->dtype == DWCONV_F32 ? 4 : 8, 8, 64); }
// (a block's partials are K + 1 rows for strip * 256 / per_block tokens)
Launch plan_bwd(const cconv_desc *d) { return plan_launch(d, BWD_CHANNELS, 16, 128); }

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
        hipLaunchKernelGGL((k_cconv_fwd<T, decltype(k)::value, fwd_channels<T>()>), dim3((unsigned)(l.down * l.across)),
                           dim3(256), 0, stream, geometry(d, l, t->starts), (const T *)t->x, (const T *)t->w, (const T *)t->b, (const T *)t->init, (T *)t->y,
                           (T *)t->final);
    });
}

template <typename T> hipError_t launch_bwd(const cconv_desc *d, const cconv_tensors *t, float *partials, hipStream_t stream)
{
    const Launch l = plan_bwd(d);
    if (!launchable(l.down * l.across, 256)) return hipErrorInvalidValue;
    return with_taps(d->K, [&](auto k) {
        constexpr int K = decltype(k)::value;
        hipLaunchKernelGGL((k_cconv_bwd<T, K, BWD_CHANNELS>), dim3((unsigned)(l.down * l.across)), dim3(256),
                           256 * (K + 1) * BWD_CHANNELS * sizeof(float), stream, geometry(d, l, t->starts), (const T *)t->x, (const T *)t->w,
                           (const T *)t->b, (const T *)t->init, (const T *)t->dy, (T *)t->dx, partials);
    });
}

template <typename T> hipError_t launch_step(const cconv_desc *d, const cconv_tensors *t, hipStream_t stream)
{
    constexpr int V = fwd_channels<T>();
    const int nv = cdiv(d->C, V);
    const long long blocks = ((long long)d->T * nv + 255) / 256;
    if (!launchable(blocks, 256)) return hipErrorInvalidValue;
    const Launch l = {nv, 1, 1, 1, 1};
    return with_taps(d->K, [&](auto k) {
        hipLaunchKernelGGL((k_cconv_step<T, decltype(k)::value, V>), dim3((unsigned)blocks), dim3(256), 0, stream, geometry(d, l, nullptr), nv,
                           (const T *)t->x, (const T *)t->w, (const T *)t->b, (const int32_t *)t->slots, (T *)t->state, (T *)t->y);
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
