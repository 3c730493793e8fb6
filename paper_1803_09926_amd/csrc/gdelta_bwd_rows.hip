// The gated delta rule backward: the gradients of queries, keys and gates, for all chunks of 64 tokens at once.
//
// With S the state before the chunk and dS its gradient behind it, U what the tokens write, X = T^T dU (gdelta_bwd.hip), E[i,j] = exp(G[i] - G[j]),
//   F = scale E * (dY U^T) on and below the diagonal,  M = -beta E * (X U^T) below it (rows and columns times the lengths' inverses)
//   dq = scale exp(G) * dY S^T + F K
//   dk = F^T Q + (M + M^T) K - beta exp(G) * X S^T + exp(G_end - G) * U dS^T
//   dbeta[i] = X[i].V[i] - exp(G[i]) k[i].(S X[i]) - sum_j E (X U^T)[i,j] k[i].k[j]
//   the gradient of the logarithm of token t's decay: the sum of what has passed it, exp(G_end) dS.S, all that tokens i >= t read of S, all that tokens j < t write for
//           the chunk's end, and F * QK^T + M * KK^T over i >= t > j.  No term is in it that does not carry the decay: none cancel, however small it is.
// One block a chunk and key head: the value heads that share it are added up in registers, in turn.  A wavefront has 16 tokens, of keys wider than 32 half of the columns.  What is contracted over V
// is read in blocks of 32 columns, keys and queries behind it, asked for in its last block.  8192 tokens of 8 heads of 128 x 128 in bf16: 131 us (with products of keys and queries
// before it, and one tile for both, 17 more; with blocks of columns in one place 9 more).
#include "gdelta_tile.hpp"
#include "gdelta_launch.hpp"

namespace dwc {

namespace {

constexpr int VB = 32, LDV = VB;

template <typename T, int KP> struct Back {
    static constexpr int RAW = PartsOf<T>::RAW, LD = KP;
    static constexpr int HALVES = KP >= 64 ? 2 : 1, THREADS = 256 * HALVES, KW = KP / HALVES, TILES = KW / 16;
    static constexpr bool TURNS = RAW == 3 && KP > 128;           // S and dS one after the other in the same place
    static constexpr size_t STATE = (size_t)INNER * KP * LDV * 2, COLS = (size_t)INNER * CHUNK * LDV * 2, DY = (size_t)RAW * CHUNK * LDV * 2;
    static constexpr size_t FIRST = (TURNS ? 1 : 2) * STATE + 2 * COLS + DY;
    static constexpr size_t TILE = (size_t)RAW * CHUNK * LD * 2, MATRIX = (size_t)INNER * CHUNK * CHUNK * 2;
    static constexpr bool TWO = 2 * TILE + 2 * MATRIX <= 144 * 1024;    // keys and queries at once; else one after the other in the same place
    static constexpr size_t SECOND = (TWO ? 2 : 1) * TILE + 2 * MATRIX;
    // behind it: [64] row sums of M KK^T / beta, X.V; [8][64] what of F QK^T and M KK^T passes a token, by wavefront; [HALVES][64] three products of rows; 8 sums; the chunk's vectors
    static constexpr size_t FLOATS = 2 * 64 + 8 * 64 + 3 * 2 * 64 + 8 + VECS * 64;
    // Blocks of columns in two places in turn, where that costs no block of a compute unit: one barrier a block, and wavefronts write the next one while others still take products
    static constexpr bool DOUBLE = !TURNS && !(RAW == 1 && KP <= 32) && 2 * FIRST + FLOATS * 4 <= 160 * 1024;
    static constexpr size_t BLOCKS = (DOUBLE ? 2 : 1) * FIRST, REGION = BLOCKS > SECOND ? BLOCKS : SECOND, LDS = REGION + FLOATS * 4;
};

constexpr int DPP_SHR1 = 0x111, DPP_SHR2 = 0x112, DPP_SHR4 = 0x114, DPP_SHR8 = 0x118;      // from the lane so many to the left, zero at a row's start
// the sum over the 16 lanes of a row, in every one of them
__device__ __forceinline__ float row_sum(float v)
{
    v += lane_move<DPP_XOR1>(v);
    v += lane_move<DPP_XOR2>(v);
    v += lane_move<DPP_HALF_MIRROR>(v);
    return v + lane_move<DPP_MIRROR>(v);
}

// the sum over the lanes to the left in a row of 16
__device__ __forceinline__ float sum_before(float v)
{
    float s = lane_move<DPP_SHR1>(v);
    s += lane_move<DPP_SHR1>(s);
    s += lane_move<DPP_SHR2>(s);
    s += lane_move<DPP_SHR4>(s);
    return s + lane_move<DPP_SHR8>(s);
}
template <int CTRL, int ROWS> __device__ __forceinline__ float lane_move_rows(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}
// the sum over the lanes up to one's own, of 64
__device__ __forceinline__ float sum_up_to(float v)
{
    v += lane_move<DPP_SHR1>(v);
    v += lane_move<DPP_SHR2>(v);
    v += lane_move<DPP_SHR4>(v);
    v += lane_move<DPP_SHR8>(v);
    v += lane_move_rows<0x142, 0xa>(v);           // the row before's last lane to the second and fourth row,
    return v + lane_move_rows<0x143, 0xc>(v);     // the second row's to the upper half
}

// WHOLE: eight columns of keys, queries, values and answers are there or not, and aligned
template <typename T, int KP, bool WHOLE>
__global__ __launch_bounds__((Back<T, KP>::THREADS), (PartsOf<T>::RAW == 1 && KP <= 32 ? 2 : 1)) void k_gdelta_bwd_rows(GdArgs g, GdLayout l, GdSpace s, const T *__restrict__ dy, T *__restrict__ dq,
                                                                             T *__restrict__ dk, T *__restrict__ da, T *__restrict__ db, unsigned first)
{
    typedef Back<T, KP> C;
    constexpr int RAW = C::RAW, LD = C::LD, PLANE = CHUNK * LD, PLANE_M = CHUNK * CHUNK, PLANE_S = KP * LDV, PLANE_V = CHUNK * LDV;
    constexpr int TILES = C::TILES, THREADS = C::THREADS, HALVES = C::HALVES;
    extern __shared__ __align__(16) char lds[];
    bf16_t *const kt = reinterpret_cast<bf16_t *>(lds), *const qt = C::TWO ? kt + RAW * PLANE : kt, *const fm = qt + RAW * PLANE, *const mm = fm + INNER * PLANE_M;
    float *const row_m = reinterpret_cast<float *>(lds + C::REGION), *const xv = row_m + 64;
    float *const passing = xv + 64, *const dot_a = passing + 8 * 64, *const dot_b = dot_a + 2 * 64, *const dot_c = dot_b + 2 * 64;
    float *const wave_sums = dot_c + 2 * 64, *const vec = wave_sums + 8;

    const unsigned id = first + blockIdx.x;
    const int kh = blockIdx.y, share = g.H / g.key_heads;
    const int wv = wave_number(), mt = wv & 3, half = wv >> 2, col0 = half * C::KW;
    const bool does_f = HALVES == 1 || half == 0, does_m = HALVES == 1 || half == 1;
    const ChunkAt at = gd_chunk(g, (int)id, CHUNK);
    if (at.len == 0) {
        for (int i = threadIdx.x; i < 2 * share; i += THREADS) s.partials[(long long)id * 2 * g.H + i / share * g.H + kh * share + i % share] = 0.f;
        return;
    }
    const T *const kp = (const T *)g.k + at.first * g.k_stride + (long long)kh * g.K, *const qp = (const T *)g.q + at.first * g.q_stride + (long long)kh * g.K;
    Rows<T, KP, THREADS, WHOLE> rows, others;        // the tiles of keys and queries on their way (one after the other in `rows` where they have one place)
    auto ask_keys = [&] { rows.load(kp, g.k_stride, at.len, g.K); };
    auto ask_queries = [&] { (C::TWO ? others : rows).load(qp, g.q_stride, at.len, g.K); };
    constexpr int BOTH = HALVES == 1 ? 2 : 1, AT_M = BOTH - 1;       // places of what two wavefronts that share rows have one of each
    const float *sp, *dsp, *xp, *up;                 // of the head in hand
    const T *yp, *vp;
    constexpr int VECS_PER = (VECS * 64 + THREADS - 1) / THREADS;
    float vec_ahead[VECS_PER];
    auto point_to = [&](int h) {
        const long long where = (long long)id * g.H + h;
        sp = s.S + where * (l.state / 4);
        dsp = s.dS + where * (l.state / 4);
        xp = s.X + where * (l.rows / 4);
        up = s.U + where * (l.rows / 4);
        yp = dy + at.first * g.y_stride + (long long)h * g.V;
        vp = (const T *)g.v + at.first * g.v_stride + (long long)h * g.V;
        const BufView view(s.vec + where * l.vectors, VECS * 64 * 4);
#pragma unroll
        for (int i = 0; i < VECS_PER; ++i) vec_ahead[i] = __uint_as_float(view.b32((threadIdx.x + i * THREADS) * 4, 0));
    };
    // what the next 32 columns of V take, on its way: 8 numbers a lane of each
    constexpr int ALL = KP * VB / 8, PER = (ALL + THREADS - 1) / THREADS;
    const int vrow = threadIdx.x % 256 / (VB / 8), vcol = threadIdx.x % (VB / 8) * 8;
    const bool takes_x = HALVES == 1 || wv < 4, takes_u = HALVES == 1 || wv >= 4;
    u4t_t sa[PER][2], sb[PER][2], w8[BOTH][2];       // w8: X and U,
    Ahead<T, 8, WHOLE> t8[BOTH];                    // t8: V and dY, of both or one of each pair
    auto ask = [&](int v0) {
        const BufView view_s(sp, (uint32_t)l.state), view_d(dsp, (uint32_t)l.state);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int n = threadIdx.x + i * THREADS;
            const uint32_t off = n < ALL ? (uint32_t)(n / (VB / 8) * l.VP + v0 + n % (VB / 8) * 8) * 4u : BufView::OUTSIDE;
            sa[i][0] = view_s.b128(off, 0);
            sa[i][1] = view_s.b128(off + 16, 0);
            sb[i][0] = view_d.b128(off, 0);
            sb[i][1] = view_d.b128(off + 16, 0);
        }
        const uint32_t off = (uint32_t)(vrow * l.VP + v0 + vcol) * 4u;
        if (takes_x) {
            const BufView view(xp, (uint32_t)l.rows), rows_v = rows_view(vp, g.v_stride, at.len, g.V);
            w8[0][0] = view.b128(off, 0);
            w8[0][1] = view.b128(off + 16, 0);
            t8[0].load(rows_v, (uint32_t)(vrow * (int)g.v_stride + v0 + vcol) * (uint32_t)sizeof(T), g.V - v0 - vcol);
        }
        if (takes_u) {
            const BufView view(up, (uint32_t)l.rows), rows_y = rows_view(yp, g.y_stride, at.len, g.V);
            w8[AT_M][0] = view.b128(off, 0);
            w8[AT_M][1] = view.b128(off + 16, 0);
            t8[AT_M].load(rows_y, (uint32_t)(vrow * (int)g.y_stride + v0 + vcol) * (uint32_t)sizeof(T), g.V - v0 - vcol);
        }
    };
    auto eight = [](const u4t_t (&w)[2], float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i / 4][i % 4]);
    };
    point_to(kh * share);
    ask(0);
    v4f_t gq[TILES], gk[TILES];                          // the gradients of q and k, their lengths taken for constants
#pragma unroll
    for (int t = 0; t < TILES; ++t) gq[t] = gk[t] = v4f_t{0.f, 0.f, 0.f, 0.f};

    for (int hh = 0; hh < share; ++hh) {
        const int h = kh * share + hh;
        if (hh) {
            point_to(h);
            ask(0);
        }
        v4f_t ys[TILES], xs[TILES], us[TILES], yu[BOTH][4];      // yu: dY U^T and X U^T
#pragma unroll
        for (int t = 0; t < TILES; ++t) ys[t] = xs[t] = us[t] = v4f_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < 4; ++n) yu[0][n] = yu[AT_M][n] = v4f_t{0.f, 0.f, 0.f, 0.f};
        Ahead<T, 1, false> gate_a, gate_b;               // of the token that a lane of the first wavefront has in the end
        if (wv == 0) {
            const uint32_t lane = threadIdx.x;
            gate_a.load(rows_view((const T *)g.a + at.first * g.a_stride + h, g.a_stride, at.len, 1), lane * (uint32_t)g.a_stride * (uint32_t)sizeof(T), 1);
            gate_b.load(rows_view((const T *)g.b + at.first * g.b_stride + h, g.b_stride, at.len, 1), lane * (uint32_t)g.b_stride * (uint32_t)sizeof(T), 1);
        }
        float ss = 0.f, xv_part = 0.f;                   // dS.S and X.V, this lane's share

        for (int v0 = 0; v0 < l.VP; v0 += VB) {
            if (!C::DOUBLE || v0 == 0) __syncthreads();
            bf16_t *const st = reinterpret_cast<bf16_t *>(lds + (C::DOUBLE && (v0 / VB) % 2 ? C::FIRST : 0)), *const dst = C::TURNS ? st : st + INNER * PLANE_S;
            bf16_t *const xt = dst + INNER * PLANE_S, *const ut = xt + INNER * PLANE_V, *const yt = ut + INNER * PLANE_V;
            if (v0 == 0) {
#pragma unroll
                for (int i = 0; i < VECS_PER; ++i)
                    if (threadIdx.x + i * THREADS < VECS * 64) vec[threadIdx.x + i * THREADS] = vec_ahead[i];
            }
            float keep[C::TURNS ? PER : 1][8];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int n = threadIdx.x + i * THREADS, row = n / (VB / 8), col = n % (VB / 8) * 8;
                if (ALL % THREADS && n >= ALL) break;
                float a[8], b[8];
                eight(sa[i], a);
                eight(sb[i], b);
#pragma unroll
                for (int j = 0; j < 8; ++j) ss += a[j] * b[j];
                put8<INNER, LDV>(st, PLANE_S, row, col, a);
                if constexpr (C::TURNS) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) keep[i][j] = b[j];
                } else put8<INNER, LDV>(dst, PLANE_S, row, col, b);
            }
            if (takes_x) {
                float x[8];
                eight(w8[0], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) xv_part += x[j] * t8[0].at(j);
                put8<INNER, LDV>(xt, PLANE_V, vrow, vcol, x);
            }
            if (takes_u) {
                float x[8];
                eight(w8[AT_M], x);
                put8<INNER, LDV>(ut, PLANE_V, vrow, vcol, x);
                put8_ahead<T, LDV, WHOLE>(yt, PLANE_V, vrow, vcol, t8[AT_M]);
            }
            if (v0 + VB < l.VP) ask(v0 + VB);
            else {
                ask_keys();
                if constexpr (C::TWO) ask_queries();
            }
            __syncthreads();
            const int lane = lane_anew();
            Frag ya[RAW], xa[INNER], ua[INNER];
            frags_rows<RAW, LDV>(ya, yt, PLANE_V, mt * 16, 0, lane);
            frags_rows<INNER, LDV>(xa, xt, PLANE_V, mt * 16, 0, lane);
            frags_rows<INNER, LDV>(ua, ut, PLANE_V, mt * 16, 0, lane);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                if (n > mt) continue;
                Frag b[INNER];
                frags_rows<INNER, LDV>(b, ut, PLANE_V, n * 16, 0, lane);
                if (does_f) mma<RAW, INNER>(yu[0][n], ya, b);
                if (does_m) mma<INNER, INNER>(yu[AT_M][n], xa, b);
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                Frag b[INNER];
                frags_rows<INNER, LDV>(b, st, PLANE_S, col0 + t * 16, 0, lane);
                mma<RAW, INNER>(ys[t], ya, b);
                mma<INNER, INNER>(xs[t], xa, b);
            }
            if constexpr (C::TURNS) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int n = threadIdx.x + i * THREADS;
                    put8<INNER, LDV>(dst, PLANE_S, n / (VB / 8), n % (VB / 8) * 8, keep[i]);
                }
                __syncthreads();
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                Frag b[INNER];
                frags_rows<INNER, LDV>(b, dst, PLANE_S, col0 + t * 16, 0, lane);
                mma<INNER, INNER>(us[t], ua, b);
            }
        }
        settled();
        __syncthreads();                                 // the first region is free
        rows.template put<LD>(kt);
        if constexpr (C::TWO) others.template put<LD>(qt);
        else ask_queries();
        ss = lanes_sum(ss);
        if (threadIdx.x % 64 == 0) wave_sums[wv] = ss;
        xv_part += lane_move<DPP_XOR1>(xv_part);
        xv_part += lane_move<DPP_XOR2>(xv_part);
        if (threadIdx.x < 256 && threadIdx.x % 4 == 0) xv[threadIdx.x / 4] = xv_part;

        __syncthreads();
        // Products of queries with keys, and of keys with keys: rows 16 mt.., columns 16 n...  Where two wavefronts share the rows each has one of them.
        v4f_t qk[BOTH][4];
        {
            const int lane = lane_anew();
            Frag qa[C::TWO ? 1 : KP / 32][RAW];
            if constexpr (!C::TWO) {
                const int row = mt * 16 + (lane & 15);
#pragma unroll
                for (int c = 0; c < KP / 32; ++c) {
                    Some<T, 4> v[2];
                    uint32_t w[4][RAW];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int col = c * 32 + i * 16 + (lane >> 4) * 4;
                        v[i].load(qp + row * g.q_stride + col, row < at.len ? g.K - col : 0);
                        split2<RAW>(v[i].at(0), v[i].at(1), w[2 * i]);
                        split2<RAW>(v[i].at(2), v[i].at(3), w[2 * i + 1]);
                    }
#pragma unroll
                    for (int i = 0; i < RAW; ++i) qa[c][i].w = u4t_t{w[0][i], w[1][i], w[2][i], w[3][i]};
                }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                qk[0][n] = qk[AT_M][n] = v4f_t{0.f, 0.f, 0.f, 0.f};
                if (n > mt) continue;
#pragma unroll
                for (int c = 0; c < KP / 32; ++c) {
                    Frag a[RAW], b[RAW];
                    frags_rows<RAW, LD>(b, kt, PLANE, n * 16, c * 32, lane);
                    if (does_m) {
                        frags_rows<RAW, LD>(a, kt, PLANE, mt * 16, c * 32, lane);
                        mma<RAW, RAW>(qk[AT_M][n], a, b);
                    }
                    if (does_f) {
                        if constexpr (C::TWO) {
                            frags_rows<RAW, LD>(a, qt, PLANE, mt * 16, c * 32, lane);
                            mma<RAW, RAW>(qk[0][n], a, b);
                        } else mma<RAW, RAW>(qk[0][n], qa[c], b);
                    }
                }
            }
        }
        // F and M + M^T, and what of their products passes each token
        settled();
        {
            const int lane = lane_anew(), m = lane & 15, q4 = lane >> 4;
            const double *const G = reinterpret_cast<const double *>(vec + VEC_G * 64);
            float rm[4], left[4], behind = 0.f;          // left: of a row in the tiles left of the diagonal's, this lane's columns; behind: those tiles' sums
#pragma unroll
            for (int r = 0; r < 4; ++r) rm[r] = left[r] = 0.f;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int j = n * 16 + m;
                float pass = 0.f;
                if (n > mt) {                            // above the diagonal all is zero
                    if (does_f) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int k = 0; k < INNER; ++k) fm[k * PLANE_M + place<CHUNK>(mt * 16 + 4 * q4 + r, j)] = 0;
                    }
                } else {
                    const double gj = G[j];
                    const float kj = vec[VEC_RK * 64 + j];
                    float x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = mt * 16 + 4 * q4 + r;
                        const float e = i >= j ? exp2_fast((float)(G[i] - gj) * LOG2E) * kj : 0.f;
                        uint32_t p[INNER];
                        x[r] = 0.f;
                        if (does_f) {
                            const float f = g.scale * vec[VEC_RQ * 64 + i] * e * yu[0][n][r];
                            x[r] = f * qk[0][n][r];
                            split2<INNER>(f, 0.f, p);
#pragma unroll
                            for (int k = 0; k < INNER; ++k) fm[k * PLANE_M + place<CHUNK>(i, j)] = (bf16_t)p[k];
                        }
                        if (does_m) {
                            const float b = i > j ? -vec[VEC_RK * 64 + i] * e * yu[AT_M][n][r] : 0.f, f = vec[VEC_BETA * 64 + i] * b;
                            rm[r] += b * qk[AT_M][n][r];
                            x[r] += f * qk[AT_M][n][r];
                            split2<INNER>(f, 0.f, p);
                            if (i >= j) {
#pragma unroll
                                for (int k = 0; k < INNER; ++k) {
                                    mm[k * PLANE_M + place<CHUNK>(i, j)] = (bf16_t)p[k];
                                    mm[k * PLANE_M + place<CHUNK>(j, i)] = (bf16_t)p[k];
                                }
                            }
                        }
                    }
                    // the sum over the columns before j, of the rows from j on: of tiles left of the diagonal's all rows, of that tile those from j on
                    if (n < mt) {
                        float c = (x[0] + x[1]) + (x[2] + x[3]);
                        c = rows_join(c, c);
                        c = halves_join(c, c);
                        pass = sum_before(c) + behind;
                        behind += row_sum(c);
#pragma unroll
                        for (int r = 0; r < 4; ++r) left[r] += x[r];
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float to = sum_before(x[r]) + row_sum(left[r]);
                            pass += mt * 16 + 4 * q4 + r >= j ? to : 0.f;
                        }
                        pass = rows_join(pass, pass);
                        pass = halves_join(pass, pass);
                    }
                }
                if (q4 == 0) passing[wv * 64 + j] = pass;
                __builtin_amdgcn_sched_barrier(0);       // (one tile after the other: the numbers of four at once spill)
            }
            if (does_m) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    rm[r] = row_sum(rm[r]);
                    if (m == 0) row_m[mt * 16 + 4 * q4 + r] = rm[r];
                }
            }
        }
        __syncthreads();
        {
            const int lane = lane_anew(), m = lane & 15, q4 = lane >> 4;
            float db_[4], dc_[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) db_[r] = dc_[r] = 0.f;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const v4f_t k = tile_of<RAW, LD>(kt, PLANE, mt * 16, col0 + t * 16, lane);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = mt * 16 + 4 * q4 + r;
                    const float x = xs[t][r] * vec[VEC_READ * 64 + i], u = us[t][r] * vec[VEC_WRITE * 64 + i];
                    gk[t][r] += u - vec[VEC_BETA * 64 + i] * x;
                    db_[r] += x * k[r];
                    dc_[r] += u * k[r];
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                db_[r] = row_sum(db_[r]);
                dc_[r] = row_sum(dc_[r]);
                if (m == 0) {
                    dot_b[half * 64 + mt * 16 + 4 * q4 + r] = db_[r];
                    dot_c[half * 64 + mt * 16 + 4 * q4 + r] = dc_[r];
                }
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                Frag a[INNER], b2[INNER];
                frags_rows<INNER, CHUNK>(a, fm, PLANE_M, mt * 16, ks * 32, lane);
                frags_rows<INNER, CHUNK>(b2, mm, PLANE_M, mt * 16, ks * 32, lane);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    Frag b[RAW];
                    frags_cols<RAW, LD>(b, kt, PLANE, ks * 32, col0 + t * 16, lane);
                    // (F is zero above the diagonal: of those products nothing comes, but they go without a branch)
                    mma<INNER, RAW>(gq[t], a, b);
                    mma<INNER, RAW>(gk[t], b2, b);
                }
            }
        }
        if constexpr (!C::TWO) {
            __syncthreads();
            rows.template put<LD>(qt);
            if (hh + 1 == share) ask_keys();
            __syncthreads();
        }
        {
            const int lane = lane_anew(), m = lane & 15, q4 = lane >> 4;
            float dot[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) dot[r] = 0.f;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const v4f_t q = tile_of<RAW, LD>(qt, PLANE, mt * 16, col0 + t * 16, lane);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = ys[t][r] * vec[VEC_ASK * 64 + mt * 16 + 4 * q4 + r];
                    gq[t][r] += x;
                    dot[r] += x * q[r];
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) { dot[r] = row_sum(dot[r]); if (m == 0) dot_a[half * 64 + mt * 16 + 4 * q4 + r] = dot[r]; }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if (ks < mt / 2) continue;
                Frag a[INNER];
                frags_cols<INNER, CHUNK>(a, fm, PLANE_M, ks * 32, mt * 16, lane);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    Frag b[RAW];
                    frags_cols<RAW, LD>(b, qt, PLANE, ks * 32, col0 + t * 16, lane);
                    mma<INNER, RAW>(gk[t], a, b);
                }
            }
            settled();
        }
        __syncthreads();
        if (wv == 0) {                                   // gates: a lane a token
            const int lane = threadIdx.x;
            const float beta = vec[VEC_BETA * 64 + lane];
            float a = dot_a[lane], b = dot_b[lane], c = dot_c[lane];
            if constexpr (HALVES == 2) { a += dot_a[64 + lane]; b += dot_b[64 + lane]; c += dot_c[64 + lane]; }
            float pass = 0.f, sum = 0.f;
#pragma unroll
            for (int i = 0; i < THREADS / 64; ++i) {
                pass += passing[i * 64 + lane];
                sum += wave_sums[i];
            }
            // what is read from the token on (summed with the lanes the other way round), and what was written before it
            const float d = __shfl(sum_up_to(__shfl(a - beta * b, 63 - lane, 64)), 63 - lane, 64);
            float w = __shfl_up(sum_up_to(c), 1, 64);
            if (lane == 0) w = 0.f;
            const float dbeta = xv[lane] - b + row_m[lane];
            float dg = d + w + (pass + vec[VEC_ONE * 64] * sum), for_a = 0.f, for_A = 0.f;
            if (lane < at.len) {
                const float raw = gd_raw(g, gate_a.at(0), h), soft = gd_soft(g, raw), A = g.A ? g.A[h] : -1.f;
                if (A * soft < GD_LEAST) dg = 0.f;
                for_A = dg * soft;
                for_a = dg * A * (g.softplus ? 1.f / (1.f + expf(-raw)) : 1.f);
                const float rate = gd_rate(g, gate_b.at(0));
                stf(da + (at.first + lane) * g.a_stride + h, for_a);
                stf(db + (at.first + lane) * g.b_stride + h, g.sigmoid ? dbeta * rate * (1.f - rate) : dbeta);
            }
            for_A = lanes_sum(for_A);
            for_a = lanes_sum(for_a);
            if (lane == 0) {
                s.partials[(long long)id * 2 * g.H + h] = for_A;
                s.partials[(long long)id * 2 * g.H + g.H + h] = for_a;
            }
        }
    }

    // The lengths: of n = r x the gradient r (dn - n (n.dn)), where the factor r is in already.
    auto finish = [&](v4f_t (&grad)[TILES], const bf16_t *tile, int which, T *out, long long stride) {
        const int lane = lane_anew(), m = lane & 15, q4 = lane >> 4;
        if (g.norm) {
            float dot[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) dot[r] = 0.f;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const v4f_t n = tile_of<RAW, LD>(tile, PLANE, mt * 16, col0 + t * 16, lane);
#pragma unroll
                for (int r = 0; r < 4; ++r) dot[r] += grad[t][r] * n[r];
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) dot[r] = row_sum(dot[r]);
            if constexpr (HALVES == 2) {
                __syncthreads();
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (m == 0) dot_a[half * 64 + mt * 16 + 4 * q4 + r] = dot[r];
                __syncthreads();
#pragma unroll
                for (int r = 0; r < 4; ++r) dot[r] = dot_a[mt * 16 + 4 * q4 + r] + dot_a[64 + mt * 16 + 4 * q4 + r];
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float inv = vec[which * 64 + mt * 16 + 4 * q4 + r];
                dot[r] *= inv * inv;
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const v4f_t n = tile_of<RAW, LD>(tile, PLANE, mt * 16, col0 + t * 16, lane);
#pragma unroll
                for (int r = 0; r < 4; ++r) grad[t][r] -= dot[r] * n[r];
            }
        }
        const BufView view = rows_view(out, stride, at.len, g.K);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int col = col0 + t * 16 + m;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x[1] = {grad[t][r]};
                store_late<T, 1, false>(view, (uint32_t)((mt * 16 + 4 * q4 + r) * (int)stride + col) * (uint32_t)sizeof(T), g.K - col, x);
            }
        }
    };
    finish(gq, qt, VEC_RQ, dq + at.first * g.q_stride + (long long)kh * g.K, g.q_stride);
    if constexpr (!C::TWO) {
        __syncthreads();
        rows.template put<LD>(kt);
        __syncthreads();
    }
    finish(gk, kt, VEC_RK, dk + at.first * g.k_stride + (long long)kh * g.K, g.k_stride);
}

template <typename T, int KP>
hipError_t launch(const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dq, void *dk, void *da, void *db, hipStream_t stream)
{
    typedef Back<T, KP> C;
    static_assert(C::LDS <= 160 * 1024, "LDS of a compute unit");
    const int v = 16 / (int)sizeof(T);
    const bool values = g.V % 8 == 0 && !unaligned16(g.v) && !unaligned16(dy) && (g.T < 2 || (g.v_stride % v == 0 && g.y_stride % v == 0));
    const auto kernel = whole_keys<T>(g) && values ? k_gdelta_bwd_rows<T, KP, true> : k_gdelta_bwd_rows<T, KP, false>;
    const hipError_t e = gd_lds(kernel, C::LDS);
    if (e != hipSuccess) return e;
    return gd_launches(l.chunks, C::THREADS, [&](long long first, unsigned now) {
        hipLaunchKernelGGL(kernel, dim3(now, (unsigned)g.key_heads), dim3(C::THREADS), C::LDS, stream, g, l, s, (const T *)dy, (T *)dq, (T *)dk, (T *)da, (T *)db, (unsigned)first);
    });
}

template <typename T>
hipError_t launch_of(const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dq, void *dk, void *da, void *db, hipStream_t stream)
{
    switch (l.KP) {
    case 32: return launch<T, 32>(g, l, s, dy, dq, dk, da, db, stream);
    case 64: return launch<T, 64>(g, l, s, dy, dq, dk, da, db, stream);
    case 128: return launch<T, 128>(g, l, s, dy, dq, dk, da, db, stream);
    default: return launch<T, 256>(g, l, s, dy, dq, dk, da, db, stream);
    }
}

}  // namespace

hipError_t launch_gdelta_bwd_rows(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dq, void *dk, void *da, void *db,
                                  hipStream_t stream)
{
    return dtype == DWCONV_F32 ? launch_of<float>(g, l, s, dy, dq, dk, da, db, stream) : launch_of<bf16_t>(g, l, s, dy, dq, dk, da, db, stream);
}

}  // namespace dwc
