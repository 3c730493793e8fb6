// The gated delta rule, first pass: what a chunk's keys, queries and gates give without its state, for all chunks of 64 tokens at once.
//
// With G the sum of the decays' logarithms from the chunk's start, and S the state before the chunk, what its tokens write is U with
//   U = T (beta * (V - exp(G) * K S)),  T = (I + L)^-1,  L[i,j] = beta[i] exp(G[i] - G[j]) k[i].k[j] below the diagonal
// and what they answer is exp(G) * Q S + P U with P[i,j] = scale exp(G[i] - G[j]) q[i].k[j] on and below it.  T and P are made here.
//
// One block of four wavefronts a chunk and key head; the products of q and k are taken once and serve all value heads.  T by blocks of 16: the four on the
// diagonal by substitution, and each column of blocks below by products with the fp32 matrix instruction, a wavefront each.  Bound by vector instructions, then by what it writes:
// 16384 tokens of 16 heads of 128 wide keys in bf16 54 us (160 MB written), 16383 tokens of 16 heads with keys of their own of 64 58 us.
#include "gdelta_tile.hpp"
#include "gdelta_launch.hpp"

namespace dwc {

namespace {

constexpr int THREADS = 256, LDF = 68;            // floats of a row of an fp32 matrix in LDS

template <typename T, int KP> struct Prep {
    static constexpr int RAW = PartsOf<T>::RAW, LD = KP;
    static constexpr size_t TILE = (size_t)RAW * CHUNK * LD * 2, F32S = (size_t)CHUNK * LDF * 4;
    static constexpr size_t FIRST = TILE > F32S ? TILE : F32S;    // the keys, and when their products are taken the inverse
    static constexpr size_t LDS = FIRST + F32S + 64 * 8 + 5 * 64 * 4;
};

// the sum over N neighbouring lanes, 4 to 32, in every one of them
template <int N> __device__ __forceinline__ float group_sum(float v)
{
    v += lane_move<DPP_XOR1>(v);
    v += lane_move<DPP_XOR2>(v);
    if constexpr (N >= 8) v += lane_move<DPP_HALF_MIRROR>(v);
    if constexpr (N >= 16) v += lane_move<DPP_MIRROR>(v);
    if constexpr (N >= 32) v = rows_join(v, v);
    return v;
}
// the sum of a number over the lanes up to one's own, in 64 bits
template <int CTRL, int ROWS> __device__ __forceinline__ double lane_move64(double v)
{
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double sum_up_to(float x)
{
    double v = x;
    v += lane_move64<0x111, 0xf>(v);              // from 1, 2, 4 and 8 lanes to the left in a row of 16,
    v += lane_move64<0x112, 0xf>(v);
    v += lane_move64<0x114, 0xf>(v);
    v += lane_move64<0x118, 0xf>(v);
    v += lane_move64<0x142, 0xa>(v);              // the row before's last lane to the second and fourth row,
    return v + lane_move64<0x143, 0xc>(v);        // the second row's to the upper half
}

// Where decays grow: the first token at which neighbouring ones' logarithms, up to its own, add up to so much that the exponential passes fp32, alone or times the inverse of a
// key's or query's length (`inverse`; the largest counts).  It counts as not finite: an infinity in the chunk's matrices would reach the tokens before it.
__device__ __forceinline__ int grown_from(double G, float inverse)
{
    asm volatile("");                                    // (hardly ever taken: it stays a branch)
    const int lane = threadIdx.x & 63;
    double least = __shfl_up(G, 1, 64);                  // of the sums before the token
    if (lane == 0) least = 0.0;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        least = fmin(least, __shfl_up(least, off, 64));  // (below `off` lanes one's own)
        inverse = fmaxf(inverse, __shfl_xor(inverse, off, 64));
    }
    const uint64_t grown = __ballot(G - least > 88.0 - (double)logf(fmaxf(inverse, 1.f)));
    return grown ? __ffsll((unsigned long long)grown) - 1 : 64;
}

// the parts of an fp32 matrix in LDS, into memory: a lane a piece of 16 bytes, four numbers and the four 16 columns on
__device__ __forceinline__ void put_matrix(const float *f, char *to)
{
#pragma unroll
    for (int i = 0; i < (MATRIX_PIECES + THREADS - 1) / THREADS; ++i) {
        const int n = threadIdx.x + i * THREADS;
        if (n >= MATRIX_PIECES) break;
        const int row = n < 128 ? n / 4 : n / 8 + 16, piece = n < 128 ? n % 4 : n % 8;
        const float *const x = f + row * LDF + (piece / 4 * 32 + piece % 4 * 4);
        Frag w[INNER];
        split_tiles<INNER>(*reinterpret_cast<const v4f_t *>(x), *reinterpret_cast<const v4f_t *>(x + 16), w);
#pragma unroll
        for (int j = 0; j < INNER; ++j) reinterpret_cast<u4t_t *>(to)[j * MATRIX_PIECES + n] = w[j].w;
    }
}

template <typename T, int KP, bool WHOLE>
__global__ __launch_bounds__(THREADS) void k_gdelta_prep(GdArgs g, char *__restrict__ t_out, char *__restrict__ p_out, char *__restrict__ vec_out, long long matrix,
                                                         long long vectors, unsigned first)
{
    typedef Prep<T, KP> C;
    constexpr int RAW = C::RAW, LD = C::LD, PLANE = CHUNK * LD;
    extern __shared__ __align__(16) char lds[];
    bf16_t *const kt = reinterpret_cast<bf16_t *>(lds);
    float *const X = reinterpret_cast<float *>(lds), *const L = reinterpret_cast<float *>(lds + C::FIRST);      // the inverse; L, then P
    double *const Gs = reinterpret_cast<double *>(L + CHUNK * LDF);
    float *const betas = reinterpret_cast<float *>(Gs + 64), *const rks = betas + 64, *const rqs = rks + 64;
    int *const bads = reinterpret_cast<int *>(rqs + 64);          // [64] tokens whose key is not finite
    const unsigned id = first + blockIdx.x;
    const ChunkAt at = gd_chunk(g, (int)id, CHUNK);
    if (at.len == 0) return;
    const int kh = blockIdx.y, share = g.H / g.key_heads, lane = threadIdx.x & 63, wv = wave_number(), m = lane & 15, q4 = lane >> 4;

    // all that comes from memory is asked for at once: keys, queries (each wavefront its 16 rows, in the order of the operands), the first head's gates
    constexpr int PER_ROW = KP / 8, NROWS = CHUNK * PER_ROW / THREADS;
    Rows<T, KP, THREADS, WHOLE> rows;
    rows.load((const T *)g.k + at.first * g.k_stride + (long long)kh * g.K, g.k_stride, at.len, g.K);
    Ahead<T, 4, WHOLE> qs[KP / 32][2];
    {
        const BufView view = rows_view((const T *)g.q + at.first * g.q_stride + (long long)kh * g.K, g.q_stride, at.len, g.K);
#pragma unroll
        for (int c = 0; c < KP / 32; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int col = c * 32 + i * 16 + q4 * 4;
                qs[c][i].load(view, (uint32_t)((wv * 16 + m) * (int)g.q_stride + col) * (uint32_t)sizeof(T), g.K - col);
            }
    }
    const bool here = lane < at.len;
    Ahead<T, 1, false> gate_a, gate_b;
    float A, bias;
    auto ask_gates = [&](int h) {
        gate_a.load(rows_view((const T *)g.a + at.first * g.a_stride + h, g.a_stride, at.len, 1), (uint32_t)(lane * (int)g.a_stride) * (uint32_t)sizeof(T), 1);
        gate_b.load(rows_view((const T *)g.b + at.first * g.b_stride + h, g.b_stride, at.len, 1), (uint32_t)(lane * (int)g.b_stride) * (uint32_t)sizeof(T), 1);
        A = g.A ? g.A[h] : -1.f;
        bias = g.a_bias ? g.a_bias[h] : 0.f;
    };
    ask_gates(kh * share);
    // keys into LDS, and their lengths; a key that is not finite counts as none, and its token is remembered
#pragma unroll
    for (int i = 0; i < NROWS; ++i) {
        const int n = threadIdx.x + i * THREADS, row = n / PER_ROW, col = n % PER_ROW * 8;
        float x[8], s = 0.f, probe = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = rows.v[i].at(j);
            s += x[j] * x[j];
            probe = fmaf(x[j], 0.f, probe);
        }
        s = group_sum<PER_ROW>(s);
        const bool bad = !(group_sum<PER_ROW>(probe) == 0.f);
        const float rk = row >= at.len || bad ? 0.f : g.norm ? 1.f / sqrtf(s + g.eps) : 1.f;
        if (n % PER_ROW == 0) {
            bads[row] = bad || !finite(rk);              // (or a key of length zero without eps)
            rks[row] = finite(rk) ? rk : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = bad ? 0.f : x[j];
        put8<RAW, LD>(kt, PLANE, row, col, x);
    }
    Frag qa[KP / 32][RAW];
    {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < KP / 32; ++c) {
            uint32_t w[4][RAW];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) s += qs[c][i].at(j) * qs[c][i].at(j);
                split2<RAW>(qs[c][i].at(0), qs[c][i].at(1), w[2 * i]);
                split2<RAW>(qs[c][i].at(2), qs[c][i].at(3), w[2 * i + 1]);
            }
#pragma unroll
            for (int i = 0; i < RAW; ++i) qa[c][i].w = u4t_t{w[0][i], w[1][i], w[2][i], w[3][i]};
        }
        s = rows_join(s, s);
        s = halves_join(s, s);
        const int row = wv * 16 + m;
        if (q4 == 0) rqs[row] = row >= at.len ? 0.f : g.norm ? 1.f / sqrtf(s + g.eps) : 1.f;
    }
    __syncthreads();
    v4f_t kk[4], qk[4];                                  // rows 16 wv.., columns 16 n..
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        kk[n] = qk[n] = v4f_t{0.f, 0.f, 0.f, 0.f};
        if (n > wv) continue;
#pragma unroll
        for (int c = 0; c < KP / 32; ++c) {
            Frag a[RAW], b[RAW];
            frags_rows<RAW, LD>(a, kt, PLANE, wv * 16, c * 32);
            frags_rows<RAW, LD>(b, kt, PLANE, n * 16, c * 32);
            mma<RAW, RAW>(kk[n], a, b);
            mma<RAW, RAW>(qk[n], qa[c], b);
        }
    }
    settled();

    for (int hh = 0; hh < share; ++hh) {
        const int h = kh * share + hh;
        const long long where = (long long)id * g.H + h;
        float *const vec = reinterpret_cast<float *>(vec_out + where * vectors);
        // What one wavefront does alone another one does for the next chunk and head: each compute unit's four vector units have the same work.
        const int turn = ((int)id + hh) & 3;
        // gates: a lane a token
        if (wv == turn) {
            const int lane = lane_anew();                // (masks of lanes over all of the loop spill)
            float d = 0.f, beta = 0.f;
            if (lane < at.len) {
                d = gd_log_decay(g, gate_a.at(0) + bias, A);
                beta = gd_rate(g, gate_b.at(0));
            }
            const uint64_t bad = __ballot(!finite(d) || !finite(beta) || bads[lane] != 0);
            int bad_from = bad ? __ffsll((unsigned long long)bad) - 1 : 64;
            if (lane >= bad_from) d = beta = 0.f;
            double G = sum_up_to(d);
            if (__any(d > 0.f)) {
                const float ask = fabsf(g.scale) * rqs[lane];        // (infinite where a query has no length: then its own answer alone is not finite)
                bad_from = min(bad_from, grown_from(G, fmaxf(rks[lane], finite(ask) ? ask : 0.f)));
                if (lane >= bad_from) d = beta = 0.f;
                G = sum_up_to(d);
            }
            Gs[lane] = G;                                // (who reads the head before's is behind two barriers)
            betas[lane] = beta;
            reinterpret_cast<double *>(vec + VEC_G * 64)[lane] = G;
            if (lane == 63) {
                vec[VEC_ONE * 64] = expf((float)G);
                reinterpret_cast<int *>(vec + VEC_ONE * 64)[1] = bad_from;
            }
        }
        if (hh + 1 < share) ask_gates(h + 1);
        __syncthreads();
        // the vectors, by the others
        if (wv != turn) {
            const int lane = lane_anew(), which = (wv - turn) & 3;
            const double G = Gs[lane];
            if (which == 1) {
                const float rk = rks[lane];
                vec[VEC_READ * 64 + lane] = expf((float)G) * rk;
                vec[VEC_RK * 64 + lane] = rk;
            } else if (which == 2) {
                vec[VEC_WRITE * 64 + lane] = expf((float)(Gs[63] - G)) * rks[lane];
                vec[VEC_BETA * 64 + lane] = betas[lane];
            } else {
                const float rq = rqs[lane];
                vec[VEC_ASK * 64 + lane] = g.scale * expf((float)G) * rq;
                vec[VEC_RQ * 64 + lane] = rq;
            }
        }
        v4f_t pv[4];
        {
            const int lane = lane_anew(), m = lane & 15, q4 = lane >> 4;
            double gi[4];
            float bi[4], ki[4], qi[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = wv * 16 + 4 * q4 + r;
                gi[r] = Gs[i]; bi[r] = betas[i]; ki[r] = rks[i]; qi[r] = g.scale * rqs[i];
            }
            auto block = [&](int n, bool diagonal) {
                const int j = n * 16 + m;
                const double gj = Gs[j];
                const float kj = rks[j];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = wv * 16 + 4 * q4 + r;
                    // (first what the lengths make of the products: of short keys and queries they are small)
                    const float e = exp2_fast((float)(gi[r] - gj) * LOG2E) * kj, p = qi[r] * qk[n][r] * e, x = bi[r] * ki[r] * kk[n][r] * e;
                    pv[n][r] = diagonal && i < j ? 0.f : p;
                    L[i * LDF + j] = diagonal && i <= j ? 0.f : x;
                }
            };
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                pv[n] = v4f_t{0.f, 0.f, 0.f, 0.f};
                if (n < wv) block(n, false);
                else if (n == wv) block(n, true);
            }
        }
        __syncthreads();
        // the inverses of the four blocks on the diagonal: 16 lanes have one, a column each
        if (wv == ((turn + 2) & 3)) {
            const int lane = lane_anew(), m = lane & 15, q4 = lane >> 4;
            const float *const D = L + q4 * 16 * (LDF + 1);
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = i == m ? 1.f : 0.f;
#pragma unroll
                for (int j = 0; j < i; ++j) x[i] = fmaf(-D[i * LDF + j], x[j], x[i]);
                X[(q4 * 16 + i) * LDF + q4 * 16 + m] = x[i];
            }
        }
        __syncthreads();
        // the blocks of column wv below the diagonal, and zeros above it
        {
            const int lane = lane_anew(), m = lane & 15, q4 = lane >> 4;
            v4f_t col[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) col[0][r] = X[(wv * 16 + 4 * q4 + r) * LDF + wv * 16 + m];
#pragma unroll
            for (int n = 1; n < 4; ++n) {
                const int i = wv + n;                    // block row
                if (i > 3) break;
                v4f_t sums[3];                           // (each on its own: what the last block of the column has no part in is not behind it)
#pragma unroll
                for (int k = 0; k < n; ++k) {
                    const v4f_t a = *reinterpret_cast<const v4f_t *>(L + (i * 16 + m) * LDF + (wv + k) * 16 + 4 * q4);
                    sums[k] = v4f_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int r = 0; r < 4; ++r) sums[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], col[k][r], sums[k], 0, 0, 0);
                }
                const v4f_t s = n == 1 ? sums[0] : n == 2 ? sums[0] + sums[1] : sums[0] + sums[1] + sums[2];
                const float4 a = *reinterpret_cast<const float4 *>(X + (i * 16 + m) * LDF + i * 16 + 4 * q4);
                v4f_t c = {0.f, 0.f, 0.f, 0.f};
                c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x, -s[0], c, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.y, -s[1], c, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.z, -s[2], c, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.w, -s[3], c, 0, 0, 0);
                col[n] = c;
                settled();                               // (a factor of the next block's, and behind the loop's end)
            }
            // (the diagonal blocks that others read are not written here)
#pragma unroll
            for (int n = 1; n < 4; ++n) {
                if (wv + n < 4) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) X[((wv + n) * 16 + 4 * q4 + r) * LDF + wv * 16 + m] = col[n][r];
                }
                if (n <= wv) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) X[((wv - n) * 16 + 4 * q4 + r) * LDF + wv * 16 + m] = 0.f;
                }
            }
        }
        __syncthreads();
        put_matrix(X, t_out + where * matrix);
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) L[(wv * 16 + 4 * q4 + r) * LDF + n * 16 + m] = pv[n][r];
        __syncthreads();
        put_matrix(L, p_out + where * matrix);
    }
}

template <typename T, int KP> hipError_t launch(const GdArgs &g, const GdLayout &l, const GdSpace &s, hipStream_t stream)
{
    const auto kernel = whole_keys<T>(g) ? k_gdelta_prep<T, KP, true> : k_gdelta_prep<T, KP, false>;
    constexpr size_t lds = Prep<T, KP>::LDS;
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    const hipError_t e = gd_lds(kernel, lds);
    if (e != hipSuccess) return e;
    return gd_launches(l.chunks, THREADS, [&](long long first, unsigned now) {
        hipLaunchKernelGGL(kernel, dim3(now, (unsigned)g.key_heads), dim3(THREADS), lds, stream, g, s.T, s.P, s.vec, l.matrix, l.vectors,
                           (unsigned)first);
    });
}

template <typename T> hipError_t launch_of(const GdArgs &g, const GdLayout &l, const GdSpace &s, hipStream_t stream)
{
    switch (l.KP) {
    case 32: return launch<T, 32>(g, l, s, stream);
    case 64: return launch<T, 64>(g, l, s, stream);
    case 128: return launch<T, 128>(g, l, s, stream);
    default: return launch<T, 256>(g, l, s, stream);
    }
}

}  // namespace

hipError_t launch_gdelta_prep(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, hipStream_t stream)
{
    return dtype == DWCONV_F32 ? launch_of<float>(g, l, s, stream) : launch_of<bf16_t>(g, l, s, stream);
}

}  // namespace dwc
