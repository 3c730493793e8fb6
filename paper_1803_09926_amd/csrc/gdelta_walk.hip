// The gated delta rule token by token: single tokens of many rows.  The contract stands in include/deltaops.h.
//
// A block of 256 lanes holds 32 columns of one head's state in registers: eight lanes of four columns by 32 lanes of every 32nd row.  All that a token asks of the
// state is taken in one round: q^T S and k^T S of each column, and q.k, q.q, k.k, so that
//   u = beta (v - d rk k^T S),  y = scale rq (d q^T S + rk (q.k) u),  S = d S + rk k u^T        (d: the decay, rq and rk: one over the lengths)
// and the state is read once and written once.  Bound by its way through memory: 64 rows of 8 heads of 128 x 128
// in bf16 13.1 us, 67 MB, 5.1 TB/s.  (With loads behind branches, each converted in its own, 15.2; in fp32, which converts nothing, that was 1 us less.  64 registers a lane spill: 16.)
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

// One round over all rows: what the state answers to q and k, and the products of q and k
struct Round { float qs[WIDE], ks[WIDE], qq, kk, qk; };

template <int NK, bool WHOLE> __device__ __forceinline__ void round_of(const Ahead<float, WIDE, WHOLE> (&s)[NK], const float (&q)[NK], const float (&k)[NK], Round &r, float *lds)
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

// WHOLE: four columns are whole aligned vectors, in all rows
template <typename T, int NK, bool WHOLE>
__global__ __launch_bounds__(THREADS) void k_gdelta_step(GdArgs g, const int32_t *__restrict__ slots, float *__restrict__ state, T *__restrict__ y, int first)
{
    __shared__ float lds[THREADS / 64 * (2 * WIDE + 3) * COLS];
    const int h = blockIdx.y, kh = __builtin_amdgcn_readfirstlane(h / (g.H / g.key_heads)), col = threadIdx.x % COLS, row = threadIdx.x / COLS;
    const int blocks = cdiv(g.V, COLS * WIDE);
    const int t = __builtin_amdgcn_readfirstlane(first + (int)(blockIdx.x / blocks)), c = (int)(blockIdx.x % blocks) * COLS * WIDE + col * WIDE, there = g.V - c;
    const int slot = __builtin_amdgcn_readfirstlane(slots ? slots[t] : t);
    const BufView out(y + t * g.y_stride + (long long)h * g.V, (uint32_t)(g.V * (int)sizeof(T)));
    const uint32_t place = (uint32_t)(c * (int)sizeof(T));
    if (slot < 0 || slot >= g.sequences) {
        if (row == 0) {
            const float none[WIDE] = {};
            store_late<T, WIDE, WHOLE>(out, place, there, none);
        }
        return;
    }
    // no branch between the loads: all of them are on their way at once
    const BufView sp(state + ((long long)slot * g.H + h) * g.K * g.V, (uint32_t)(g.K * g.V) * 4u);
    const BufView qp((const T *)g.q + t * g.q_stride + (long long)kh * g.K, (uint32_t)(g.K * (int)sizeof(T)));
    const BufView kp((const T *)g.k + t * g.k_stride + (long long)kh * g.K, (uint32_t)(g.K * (int)sizeof(T)));
    Ahead<float, WIDE, WHOLE> s[NK];
    Ahead<T, 1, false> q_[NK], k_[NK];
    Ahead<T, WIDE, WHOLE> v;
#pragma unroll
    for (int j = 0; j < NK; ++j) {
        const int r = row + j * ROWS;
        s[j].load(sp, (uint32_t)(r * g.V + c) * 4u, r < g.K ? there : 0);
        q_[j].load(qp, (uint32_t)(r * (int)sizeof(T)), 1);
        k_[j].load(kp, (uint32_t)(r * (int)sizeof(T)), 1);
    }
    v.load(BufView((const T *)g.v + t * g.v_stride + (long long)h * g.V, (uint32_t)(g.V * (int)sizeof(T))), place, there);
    const float raw = gd_raw(g, ldf((const T *)g.a + t * g.a_stride + h), h), d = expf(gd_log_decay(g, raw, g.A ? g.A[h] : -1.f));
    const float beta = gd_rate(g, ldf((const T *)g.b + t * g.b_stride + h));
    float q[NK], k[NK];
#pragma unroll
    for (int j = 0; j < NK; ++j) {
        q[j] = q_[j].at(0);
        k[j] = k_[j].at(0);
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
    if (row == 0) store_late<T, WIDE, WHOLE>(out, place, there, o);
#pragma unroll
    for (int j = 0; j < NK; ++j) {
        const int at = row + j * ROWS;
        float n[WIDE];
#pragma unroll
        for (int i = 0; i < WIDE; ++i) n[i] = d * s[j].at(i) + rk * k[j] * u[i];
        store_late<float, WIDE, WHOLE>(sp, (uint32_t)(at * g.V + c) * 4u, at < g.K ? there : 0, n);
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
            if (whole) run(k_gdelta_step<T, NK, true>);
            else run(k_gdelta_step<T, NK, false>);
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
