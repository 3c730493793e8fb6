// The gated delta rule token by token: single tokens of many rows.  The contract stands in include/deltaops.h.
//
// A block of 256 lanes holds 32 columns of one head's state in registers: eight lanes of four columns by 32 lanes of every 32nd row.  All that a token asks of the
// state is taken in one round: q^T S and k^T S of each column, and q.k, q.q, k.k, so that
//   u = beta (v - d rk k^T S),  y = scale rq (d q^T S + rk (q.k) u),  S = d S + rk k u^T        (d: the decay, rq and rk: one over the lengths)
// and the state is read once and written once.  Bound by its way through memory: 64 rows of 8 heads of 128 x 128 in bf16 15.7 us, 67 MB, 4.3 TB/s, in fp32 14.5 us, 4.6 TB/s, with three sets of
// states in turn (with one, which stays in the cache, 13.4 and 12.5); 128 rows of 16 heads of 64 x 64 16.8 and 16.4.  (Held to 64 registers a lane it spills.)
#include "gdelta.hpp"
#include "gdelta_launch.hpp"
#include <type_traits>

namespace dwc {

namespace {

constexpr int COLS = 8, ROWS = 32, WIDE = 4, THREADS = 256;   // lanes by columns, lanes by rows, columns a lane

// the sum over the eight rows of lanes of a wavefront
__device__ __forceinline__ float rows_sum(float v)
{
    v += lane_move<DPP_ROR8>(v);
    v = rows_join(v, v);
    return halves_join(v, v);
}

// How four columns of a row come from memory and go back.  AHEAD: by views without a branch, all of them on their way at once; WHOLE: as whole aligned vectors, else one by one.  Otherwise behind
// a branch, as vectors of any alignment where all four are there.  Measured with three sets of states in turn (64 rows of 8 heads of 128 x V, us): bf16 V 128 ahead 15.7, else 16.9; 100:
// 20.5, 24.5; 66: 20.5, 21.7; 130: 29.0, 31.0; but 33: 15.9, 13.5; 31: 8.5, 7.4.  fp32, which converts nothing: 128: 15.4, 14.2; 130: 29.4, 25.9; 33: 15.9, 12.3.
enum Way { BRANCH, AHEAD, AHEAD_WHOLE };
template <typename T, Way WAY> struct Four {
    static constexpr bool WHOLE = WAY == AHEAD_WHOLE;
    std::conditional_t<WAY == BRANCH, Some<T, WIDE>, Ahead<T, WIDE, WHOLE>> v;
    // elements from `at` on of the n that p has, uniform; those less than `there` are there
    __device__ __forceinline__ void load(const T *p, int n, int at, int there)
    {
        if constexpr (WAY == BRANCH) v.load(p + at, there);
        else v.load(BufView(p, (uint32_t)(n * (int)sizeof(T))), (uint32_t)(at * (int)sizeof(T)), there);
    }
    __device__ __forceinline__ float at(int i) const { return v.at(i); }
    static __device__ __forceinline__ void store(T *p, int n, int at, int there, const float (&x)[WIDE])
    {
        if constexpr (WAY == BRANCH) {
            Some<T, WIDE> w;
            w.set(x);
            w.store(p + at, there);
        } else store_late<T, WIDE, WHOLE>(BufView(p, (uint32_t)(n * (int)sizeof(T))), (uint32_t)(at * (int)sizeof(T)), there, x);
    }
};

// One round over all rows: what the state answers to q and k, and the products of q and k
struct Round { float qs[WIDE], ks[WIDE], qq, kk, qk; };

template <int NK, Way WAY> __device__ __forceinline__ void round_of(const Four<float, WAY> (&s)[NK], const float (&q)[NK], const float (&k)[NK], Round &r, float *lds)
{
    float v[2 * WIDE + 3];
#pragma unroll
    for (int i = 0; i < 2 * WIDE + 3; ++i) v[i] = 0.f;
#pragma unroll
    for (int j = 0; j < NK; ++j) {
#pragma unroll
        for (int i = 0; i < WIDE; ++i) {
            v[i] = fmaf(q[j], s[j].at(i), v[i]);
            v[WIDE + i] = fmaf(k[j], s[j].at(i), v[WIDE + i]);
        }
        v[2 * WIDE] = fmaf(q[j], q[j], v[2 * WIDE]);
        v[2 * WIDE + 1] = fmaf(k[j], k[j], v[2 * WIDE + 1]);
        v[2 * WIDE + 2] = fmaf(q[j], k[j], v[2 * WIDE + 2]);
    }
    const int wv = threadIdx.x / 64, col = threadIdx.x % COLS;
#pragma unroll
    for (int i = 0; i < 2 * WIDE + 3; ++i) v[i] = rows_sum(v[i]);
    if (threadIdx.x % 64 < COLS) {
#pragma unroll
        for (int i = 0; i < 2 * WIDE + 3; ++i) lds[(wv * (2 * WIDE + 3) + i) * COLS + col] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2 * WIDE + 3; ++i) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) t += lds[(w * (2 * WIDE + 3) + i) * COLS + col];
        v[i] = t;
    }
#pragma unroll
    for (int i = 0; i < WIDE; ++i) { r.qs[i] = v[i]; r.ks[i] = v[WIDE + i]; }
    r.qq = v[2 * WIDE]; r.kk = v[2 * WIDE + 1]; r.qk = v[2 * WIDE + 2];
}

template <typename T, int NK, Way WAY>
__global__ __launch_bounds__(THREADS) void k_gdelta_step(GdArgs g, const int32_t *__restrict__ slots, float *__restrict__ state, T *__restrict__ y, int first)
{
    __shared__ float lds[THREADS / 64 * (2 * WIDE + 3) * COLS];
    const int h = blockIdx.y, kh = __builtin_amdgcn_readfirstlane(h / (g.H / g.key_heads)), col = threadIdx.x % COLS, row = threadIdx.x / COLS;
    const int blocks = cdiv(g.V, COLS * WIDE);
    const int t = __builtin_amdgcn_readfirstlane(first + (int)(blockIdx.x / blocks)), c = (int)(blockIdx.x % blocks) * COLS * WIDE + col * WIDE, there = g.V - c;
    const int slot = __builtin_amdgcn_readfirstlane(slots ? slots[t] : t);
    T *const out = y + t * g.y_stride + (long long)h * g.V;
    if (slot < 0 || slot >= g.sequences) {
        if (row == 0) {
            const float none[WIDE] = {};
            Four<T, WAY>::store(out, g.V, c, there, none);
        }
        return;
    }
    float *const sp = state + ((long long)slot * g.H + h) * g.K * g.V;
    const T *const qp = (const T *)g.q + t * g.q_stride + (long long)kh * g.K, *const kp = (const T *)g.k + t * g.k_stride + (long long)kh * g.K;
    const T *const vp = (const T *)g.v + t * g.v_stride + (long long)h * g.V;
    Four<float, WAY> s[NK];
    Four<T, WAY> v;
    float q[NK], k[NK];
    if constexpr (WAY == BRANCH) {
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const int r = row + j * ROWS;
            s[j].load(sp, g.K * g.V, r * g.V + c, r < g.K ? there : 0);
            q[j] = r < g.K ? ldf(qp + r) : 0.f;
            k[j] = r < g.K ? ldf(kp + r) : 0.f;
        }
        v.load(vp, g.V, c, there);
    }
    Ahead<T, 1, false> q_[WAY == BRANCH ? 1 : NK], k_[WAY == BRANCH ? 1 : NK];
    if constexpr (WAY != BRANCH) {
        const BufView qs(qp, (uint32_t)(g.K * (int)sizeof(T))), ks(kp, (uint32_t)(g.K * (int)sizeof(T)));
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const int r = row + j * ROWS;
            s[j].load(sp, g.K * g.V, r * g.V + c, r < g.K ? there : 0);
            q_[j].load(qs, (uint32_t)(r * (int)sizeof(T)), 1);
            k_[j].load(ks, (uint32_t)(r * (int)sizeof(T)), 1);
        }
        v.load(vp, g.V, c, there);
    }
    const float raw = gd_raw(g, ldf((const T *)g.a + t * g.a_stride + h), h), d = expf(gd_log_decay(g, raw, g.A ? g.A[h] : -1.f));
    const float beta = gd_rate(g, ldf((const T *)g.b + t * g.b_stride + h));
    if constexpr (WAY != BRANCH) {
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            q[j] = q_[j].at(0);
            k[j] = k_[j].at(0);
        }
    }
    Round r;
    round_of<NK>(s, q, k, r, lds);
    const float rq = g.norm ? 1.f / sqrtf(r.qq + g.eps) : 1.f, rk = g.norm ? 1.f / sqrtf(r.kk + g.eps) : 1.f;
    float u[WIDE], o[WIDE];
#pragma unroll
    for (int i = 0; i < WIDE; ++i) {
        u[i] = beta * (v.at(i) - d * rk * r.ks[i]);
        o[i] = g.scale * rq * (d * r.qs[i] + rk * r.qk * u[i]);
    }
    if (row == 0) Four<T, WAY>::store(out, g.V, c, there, o);
#pragma unroll
    for (int j = 0; j < NK; ++j) {
        const int at = row + j * ROWS;
        if (WAY == BRANCH && at >= g.K) continue;
        float n[WIDE];
#pragma unroll
        for (int i = 0; i < WIDE; ++i) n[i] = d * s[j].at(i) + rk * k[j] * u[i];
        Four<float, WAY>::store(sp, g.K * g.V, at * g.V + c, at < g.K ? there : 0, n);
    }
}

template <typename T> hipError_t launch(const GdArgs &g, const int32_t *slots, float *state, void *y, hipStream_t stream)
{
    const int blocks = cdiv(g.V, COLS * WIDE), nk = cdiv(g.K, ROWS);
    const uintptr_t vector = WIDE * sizeof(T) - 1;
    const bool whole = g.V % WIDE == 0 && !unaligned16(state) && !((reinterpret_cast<uintptr_t>(g.v) | reinterpret_cast<uintptr_t>(y)) & vector) &&
                       (g.T < 2 || (g.v_stride % WIDE == 0 && g.y_stride % WIDE == 0));
    const long long most = most_blocks(THREADS) / ((long long)blocks * g.H);      // tokens of one launch
    for (long long first = 0; first < g.T; first += most) {
        const dim3 grid((unsigned)((g.T - first < most ? g.T - first : most) * blocks), (unsigned)g.H);
        auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(THREADS), 0, stream, g, slots, state, (T *)y, (int)first); };
        auto of = [&](auto n) {
            constexpr int NK = decltype(n)::value;
            if constexpr (sizeof(T) == 4) run(k_gdelta_step<T, NK, BRANCH>);
            else if (whole) run(k_gdelta_step<T, NK, AHEAD_WHOLE>);
            else if (g.V % 2 == 0) run(k_gdelta_step<T, NK, AHEAD>);
            else run(k_gdelta_step<T, NK, BRANCH>);
        };
        if (nk <= 1) of(std::integral_constant<int, 1>());
        else if (nk <= 2) of(std::integral_constant<int, 2>());
        else if (nk <= 4) of(std::integral_constant<int, 4>());
        else of(std::integral_constant<int, 8>());
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gdelta_step(int dtype, const GdArgs &g, const int32_t *slots, float *state, void *y, hipStream_t stream)
{
    return dtype == DWCONV_F32 ? launch<float>(g, slots, state, y, stream) : launch<bf16_t>(g, slots, state, y, stream);
}

}  // namespace dwc
