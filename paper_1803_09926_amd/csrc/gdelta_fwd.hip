// The gated delta rule, the walk over a sequence's chunks: what they answer, and the state behind them.
//
// A block of four wavefronts has 16 or 32 columns of a head's state a wavefront in registers, from the sequence's first chunk to its last; the columns are independent.
// Of each chunk, with the first pass's T and P and the state S before it,
//   U = T (beta * (V - exp(G) * K S)),  Y = scale exp(G) * Q S + P U,  S = exp(G_end) S + (exp(G_end - G) * K)^T U
// all as products on the matrix cores: S, V, U and Y never leave the registers, as a result tile is an operand as it lies; K, Q, T and P go through LDS, and the next ones
// are on their way from memory meanwhile.  Bound by the way through a chunk, K S, T, K^T U, each of whose results is split and handed on: 128 x 128 in bf16 6.2 us a chunk where a
// compute unit has one block, 4.6 where it has two; 8 x 1024 tokens of 8 heads 100 us.  (K S and Q S at once, behind one pair of barriers, took 12 % more.)
//
// MAP: the map of a piece of a sequence instead (gdelta_launch.hpp).  What it makes of zero (of the state that the sequence begins with, in the first piece) is the walk without
// answers, and its matrix is what the walk without values makes of the K unit vectors: K columns more.
#include "gdelta_states.hpp"

namespace dwc {

namespace {

// Whether the product of a stretch's decays is zero in fp32, and all of them are numbers of at most one (a product in another order than the tokens' says nothing where some are larger)
__device__ __forceinline__ bool a_decay_is_zero(const GdArgs &g, const GdLayout &l, const GdSpace &s, const Stretch &at, int h)
{
    float p = 1.f;
    bool grows = false;
    for (int c = at.from + (int)(threadIdx.x & 63); c < at.to; c += 64) {
        const float d = reinterpret_cast<const float *>(s.vec + (((long long)at.base + c) * g.H + h) * l.vectors)[VEC_ONE * 64];
        grows |= !(d <= 1.f);
        p *= d;
    }
#pragma unroll
    for (int off = 1; off < 64; off *= 2) p *= __shfl_xor(p, off, 64);
    return !__any(grows) && p == 0.f;
}

template <typename T, int KP, bool MAP> using WalkOf = Walk<T, KP, !MAP, (MAP ? 1 : 2) * INNER>;

template <typename T, int KP, int NT, bool WHOLE, bool MAP>
__global__ __launch_bounds__(THREADS, (NT == 1 && KP <= (WHOLE ? 128 : 64) && PartsOf<T>::RAW == 1 ? 2 : 1)) void k_gdelta_fwd(GdArgs g, GdLayout l, GdSpace s, const float *__restrict__ init, T *__restrict__ y,
                                                           float *__restrict__ final, long long first, int blocks)
{
    typedef WalkOf<T, KP, MAP> W;
    constexpr int RAW = W::RAW, N = INNER;
    constexpr bool SHARE = W::SHARE;
    extern __shared__ __align__(16) char lds[];
    bf16_t *const kt = reinterpret_cast<bf16_t *>(lds), *const qt = SHARE || MAP ? kt : kt + RAW * CHUNK * KP;
    bf16_t *const tm = qt + RAW * CHUNK * KP, *const pm = tm + N * MATRIX_PLANE;
    float *const vecs = reinterpret_cast<float *>(pm + (MAP ? 0 : N) * MATRIX_PLANE);     // two chunks' worth, in turn
    const int share = g.H / g.key_heads;
    const Shared which = gd_shared(first + blockIdx.x, (unsigned)(blocks * share));      // of a key head: its value heads' blocks of columns
    if (which.item >= (l.piece ? l.pieces : (long long)g.sequences) * g.key_heads) return;
    const int id = uniform((int)quotient(which.item, (unsigned)g.key_heads)), kh = uniform((int)(which.item - (long long)id * g.key_heads)), h = uniform(kh * share + which.block / blocks);
    const int block = which.block % blocks;
    const Stretch at_ = stretch_of(g, l, id);
    const int seq = at_.seq, start = at_.start, end = at_.end, base = at_.base, chunks = at_.to;
    // the last piece's map is not asked for, nor the first one's matrix
    const int values = cdiv(l.VP, WAVES * 16 * NT);
    const bool unit = MAP && block >= values;
    if (at_.place < 0 || (MAP && (at_.place == at_.pieces - 1 || (unit && at_.place == 0)))) return;
    const Columns<NT> cols(block - (unit ? values : 0));
    const T *const kp = (const T *)g.k + (long long)kh * g.K, *const qp = (const T *)g.q + (long long)kh * g.K, *const vp = (const T *)g.v + (long long)h * g.V;

    if (unit && g.norm && g.sigmoid && a_decay_is_zero(g, l, s, at_, h)) {
        // keys of length one and rates below one: no product of the piece's factors is larger than its decays, and those are zero
        v4f_t none[KP / 16][NT] = {};
        store_tiles<NT, KP / 16>(none, s.maps + ((long long)id * g.H + h) * (l.map / 4), KP, cols);
        return;
    }

    v4f_t S[KP / 16][NT];
    const long long state = ((long long)seq * g.H + h) * g.K * g.V;
    const bool begins = at_.place == 0;
    if (!MAP && !begins) load_state<NT, KP / 16>(S, s.ends + ((long long)id * g.H + h) * (l.state / 4), KP, l.VP, cols);
    else if (init && begins) load_state<NT, KP / 16>(S, init + state, g.K, g.V, cols);
    else {
#pragma unroll
        for (int ct = 0; ct < KP / 16; ++ct)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[ct][nt][r] = unit && row_of(ct, r) == cols.c + nt ? 1.f : 0.f;
    }
    Frag Sp[KP / 32][NT][N];
    auto split_state = [&] {
#pragma unroll
        for (int c = 0; c < KP / 32; ++c)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) split_tiles<N>(S[2 * c][nt], S[2 * c + 1][nt], Sp[c][nt]);
    };
    split_state();

    Rows<T, KP, THREADS, WHOLE> rows;
    Matrix<N, THREADS> matrix, answers;
    Ahead<T, NT, WHOLE> v[4][4];
    float vec_next, decay_next;
    int bad_next;
    auto load_next = [&](int c) {
        const int at = start + c * CHUNK, len = min(CHUNK, end - at);
        const long long where = ((long long)base + c) * g.H + h;
        rows.load(kp + at * g.k_stride, g.k_stride, len, g.K);
        matrix.load(s.T + where * l.matrix);
        const float *const vec = reinterpret_cast<const float *>(s.vec + where * l.vectors);
        vec_next = vec[threadIdx.x];
        decay_next = vec[VEC_ONE * 64];
        bad_next = reinterpret_cast<const int *>(vec + VEC_ONE * 64)[1];
    };
    auto load_values = [&](int c) {
        const int at = start + c * CHUNK, len = min(CHUNK, end - at);
        const auto places = cols.template places<T>((int)g.v_stride, unit ? 0 : g.V);
        const BufView view = rows_view(vp + at * g.v_stride, g.v_stride, len, g.V);
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r) cols.load(v[mt][r], view, places, mt, r);
    };
    if (at_.from < chunks) {
        load_next(at_.from);
        load_values(at_.from);
    }
    for (int c = at_.from; c < chunks; ++c) {
        const int at = start + c * CHUNK, len = min(CHUNK, end - at);
        const long long where = ((long long)base + c) * g.H + h;
        float *const vl = vecs + (c & 1) * 256;
        if ((SHARE || MAP) && c > at_.from) __syncthreads();
        rows.template put<KP>(kt);
        matrix.put(tm);
        vl[threadIdx.x] = vec_next;
        const float decay = decay_next;
        const int bad = bad_next;
        if constexpr (MAP) {
            if (c + 1 < chunks) load_next(c + 1);
        } else {
            rows.load(qp + at * g.q_stride, g.q_stride, len, g.K);
            answers.load(s.P + where * l.matrix);
        }
        __syncthreads();
        if (!MAP && s.S) store_tiles<NT, KP / 16>(S, s.S + where * (l.state / 4), l.VP, cols);
        v4f_t R[4][NT];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) R[mt][nt] = v4f_t{0.f, 0.f, 0.f, 0.f};
        times_state<RAW, N, KP>(R, kt, Sp);
        // (here, not behind the state's sums: their registers and those of T's products do not fit beside it.  All wavefronts have read the chunk before's.)
        if constexpr (!MAP) {
            answers.put(pm);
            if constexpr (!SHARE) rows.template put<KP>(qt);
        }
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
            const float4 read = four(vl + VEC_READ * 64, mt), beta = four(vl + VEC_BETA * 64, mt);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const v4f_t x = {v[mt][0].at(nt), v[mt][1].at(nt), v[mt][2].at(nt), v[mt][3].at(nt)};
                R[mt][nt] = times(x - times(R[mt][nt], read), beta);
            }
        }
        // The first key or gate that is not finite, or the first number here that is not (of a value, or of a state that has grown): from there on the column is, and before it
        // nothing is of it.
        int from[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) from[nt] = bad;
        const bool odd = __any(bad < CHUNK || not_finite(R));
        if (odd) {
            seldom();
            rows_before(R, from);
        }
        Frag f[2][NT][N];
        split_rows<N, NT>(R, f);
        v4f_t U[4][NT];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) U[mt][nt] = v4f_t{0.f, 0.f, 0.f, 0.f};
        times_triangle<N, false>(U, tm, f);
        bool over = odd;
        if constexpr (!MAP) {
            settled();
            if (s.U) store_tiles<NT, 4>(U, s.U + where * (l.rows / 4), l.VP, cols);
            if (__any(not_finite(U))) {
                seldom();
                over = true;
                rows_before(U, from);
            }
        }
        v4f_t w[4][NT];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
            const float4 write = four(vl + VEC_WRITE * 64, mt);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) w[mt][nt] = times(U[mt][nt], write);
        }
        split_rows<N, NT>(w, f);
#pragma unroll
        for (int ct = 0; ct < KP / 16; ++ct)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[ct][nt] *= decay;
        add_to_state<RAW, KP>(S, kt, f);
        v4f_t O[4][NT];
        if constexpr (MAP) {
            if (c + 1 < chunks) load_values(c + 1);
        } else {
            if constexpr (SHARE) {
                __syncthreads();
                rows.template put<KP>(qt);
            }
            if (c + 1 < chunks) {
                load_next(c + 1);
                load_values(c + 1);
            }
            __syncthreads();
            Frag u[2][NT][N];
            split_rows<N, NT>(U, u);
#pragma unroll
            for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[mt][nt] = v4f_t{0.f, 0.f, 0.f, 0.f};
            times_state<RAW, N, KP>(O, qt, Sp);
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                const float4 ask = four(vl + VEC_ASK * 64, mt);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[mt][nt] = times(O[mt][nt], ask);
            }
            times_triangle<N, false>(O, pm, u);
        }
        settled();                                       // (the answers; of a map the state)
        if (over) {
            seldom();
            const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!MAP && row_of(mt, r) >= from[nt]) O[mt][nt][r] = nan;
#pragma unroll
                for (int ct = 0; ct < KP / 16; ++ct)
                    if (from[nt] < CHUNK) S[ct][nt] = v4f_t{nan, nan, nan, nan};
            }
        }
        if constexpr (!MAP) {
            const auto places = cols.template places<T>((int)g.y_stride, g.V);
            const BufView out = rows_view(y + at * g.y_stride + (long long)h * g.V, g.y_stride, len, g.V);
#pragma unroll
            for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float x[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) x[nt] = O[mt][nt][r];
                    cols.template store<T, WHOLE>(out, places, mt, r, x);
                }
        }
        split_state();
    }
    if constexpr (MAP) {
        const long long where = (long long)id * g.H + h;
        if (unit) store_tiles<NT, KP / 16>(S, s.maps + where * (l.map / 4), KP, cols);
        else store_tiles<NT, KP / 16>(S, s.ends + where * (l.state / 4), l.VP, cols);
    } else if (final && at_.place == at_.pieces - 1) store_state<NT, KP / 16>(S, final + state, g.K, g.V, cols);
}

template <typename T, int KP, int NT, bool MAP>
hipError_t launch(const GdArgs &g, const GdLayout &l, const GdSpace &s, const float *init, void *y, float *final, hipStream_t stream)
{
    constexpr size_t lds = WalkOf<T, KP, MAP>::LDS;
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    const bool whole = whole_keys<T>(g) && (NT == 1 || pair_values<T>(g, g.v, y, g.v_stride, g.y_stride));
    const auto kernel = whole ? k_gdelta_fwd<T, KP, NT, true, MAP> : k_gdelta_fwd<T, KP, NT, false, MAP>;
    const hipError_t e = gd_lds(kernel, lds);
    if (e != hipSuccess) return e;
    const int blocks = cdiv(l.VP, WAVES * 16 * NT) + (MAP ? cdiv(KP, WAVES * 16 * NT) : 0);
    const long long items = (l.piece ? l.pieces : (long long)g.sequences) * g.key_heads;
    return gd_launches(gd_shared_blocks(items, blocks * (g.H / g.key_heads)), THREADS, [&](long long first, unsigned now) {
        hipLaunchKernelGGL(kernel, dim3(now), dim3(THREADS), lds, stream, g, l, s, init, (T *)y, final, first, blocks);
    });
}

// The walk; where sequences go in pieces their maps first, and the states that they begin with
template <typename T, int KP>
hipError_t walk(const GdArgs &g, const GdLayout &l, const GdSpace &s, const float *init, void *y, float *final, hipStream_t stream)
{
    if (l.piece) {
        hipError_t e = launch<T, KP, 1, true>(g, l, s, init, y, final, stream);
        if (e == hipSuccess) e = launch_gdelta_join(g, l, s, false, stream);
        if (e != hipSuccess) return e;
    }
    if constexpr (may_have_two_tiles<T, KP>) {
        if (two_tiles(g, l)) return launch<T, KP, 2, false>(g, l, s, init, y, final, stream);
    }
    return launch<T, KP, 1, false>(g, l, s, init, y, final, stream);
}

template <typename T> hipError_t walk_of(const GdArgs &g, const GdLayout &l, const GdSpace &s, const float *init, void *y, float *final, hipStream_t stream)
{
    switch (l.KP) {
    case 32: return walk<T, 32>(g, l, s, init, y, final, stream);
    case 64: return walk<T, 64>(g, l, s, init, y, final, stream);
    case 128: return walk<T, 128>(g, l, s, init, y, final, stream);
    default: return walk<T, 256>(g, l, s, init, y, final, stream);
    }
}

}  // namespace

hipError_t launch_gdelta_fwd(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, const float *init, void *y, float *final, hipStream_t stream)
{
    return dtype == DWCONV_F32 ? walk_of<float>(g, l, s, init, y, final, stream) : walk_of<bf16_t>(g, l, s, init, y, final, stream);
}

}  // namespace dwc
