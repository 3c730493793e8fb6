// The gated delta rule backward, the walk back over a sequence's chunks: the gradient of the state, and of what the tokens write to it.
//
// As the walk forward (gdelta_fwd.hip), with dS the gradient of the state behind a chunk:
//   dU = P^T dY + (exp(G_end - G) * K) dS,  X = T^T dU,  dV = beta * X
//   dS = exp(G_end) dS + (scale exp(G) * Q)^T dY - (exp(G) * K)^T dV
// MAP: what a piece of a sequence makes of a gradient of zero (gdelta_launch.hpp); the map's matrix is the forward one's, transposed.
// X and the dS behind the chunk are what the gradients of keys, queries and gates take (gdelta_bwd_rows.hip), for all chunks at once.
// Bound as the walk forward is: 8 x 1024 tokens of 8 heads of 128 x 128 in bf16 96 us.
#include "gdelta_states.hpp"

namespace dwc {

namespace {

template <typename T, int KP, int NT, bool WHOLE, bool MAP>
__global__ __launch_bounds__(THREADS, (NT == 1 && KP <= (WHOLE ? 128 : 64) && PartsOf<T>::RAW == 1 ? 2 : 1)) void k_gdelta_bwd_states(GdArgs g, GdLayout l, GdSpace s, const T *__restrict__ dy, T *__restrict__ dv, long long first,
                                                                  int blocks)
{
    typedef Walk<T, KP, true, 2 * INNER> W;
    constexpr int RAW = W::RAW;
    constexpr bool SHARE = W::SHARE;
    extern __shared__ __align__(16) char lds[];
    bf16_t *const kt = reinterpret_cast<bf16_t *>(lds), *const qt = SHARE ? kt : kt + RAW * CHUNK * KP;
    bf16_t *const tm = qt + RAW * CHUNK * KP, *const pm = tm + INNER * MATRIX_PLANE;
    float *const vecs = reinterpret_cast<float *>(pm + INNER * MATRIX_PLANE);       // two chunks' worth, in turn
    const int share = g.H / g.key_heads;
    const Shared which = gd_shared(first + blockIdx.x, (unsigned)(blocks * share));      // of a key head: its value heads' blocks of columns
    if (which.item >= (l.piece ? l.pieces : (long long)g.sequences) * g.key_heads) return;
    const int id = uniform((int)quotient(which.item, (unsigned)g.key_heads)), kh = uniform((int)(which.item - (long long)id * g.key_heads)), h = uniform(kh * share + which.block / blocks);
    const Stretch at_ = stretch_of(g, l, id);
    const int start = at_.start, end = at_.end, base = at_.base, from = at_.from, last = at_.to - 1;
    if (at_.place < 0 || (MAP && at_.place == 0)) return;       // (nothing comes before the first piece)
    const Columns<NT> cols(which.block % blocks);
    const T *const kp = (const T *)g.k + (long long)kh * g.K, *const qp = (const T *)g.q + (long long)kh * g.K, *const yp = dy + (long long)h * g.V;

    v4f_t S[KP / 16][NT];
    const long long piece = (long long)id * g.H + h;
    if (!MAP && at_.place < at_.pieces - 1) load_state<NT, KP / 16>(S, s.ends + piece * (l.state / 4), KP, l.VP, cols);
    else {
#pragma unroll
        for (int ct = 0; ct < KP / 16; ++ct)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[ct][nt] = v4f_t{0.f, 0.f, 0.f, 0.f};
    }

    Rows<T, KP, THREADS, WHOLE> rows;
    Matrix<INNER, THREADS> matrix, second;
    Ahead<T, NT, WHOLE> o[4][4];
    float vec_next, decay_next;
    auto load_keys = [&](int c) {
        const int at = start + c * CHUNK, len = min(CHUNK, end - at);
        const long long where = ((long long)base + c) * g.H + h;
        rows.load(kp + at * g.k_stride, g.k_stride, len, g.K);
        matrix.load(s.T + where * l.matrix);
        second.load(s.P + where * l.matrix);
        const auto places = cols.template places<T>((int)g.y_stride, g.V);
        const BufView view = rows_view(yp + at * g.y_stride, g.y_stride, len, g.V);
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r) cols.load(o[mt][r], view, places, mt, r);
        const float *const vec = reinterpret_cast<const float *>(s.vec + where * l.vectors);
        vec_next = vec[threadIdx.x];
        decay_next = vec[VEC_ONE * 64];
    };
    if (from <= last) load_keys(last);
    for (int c = last; c >= from; --c) {
        const int at = start + c * CHUNK, len = min(CHUNK, end - at);
        const long long where = ((long long)base + c) * g.H + h;
        float *const vl = vecs + (c & 1) * 256;
        if (SHARE && c < last) __syncthreads();
        rows.template put<KP>(kt);
        matrix.put(tm);
        second.put(pm);
        vl[threadIdx.x] = vec_next;
        const float decay = decay_next;
        rows.load(qp + at * g.q_stride, g.q_stride, len, g.K);
        if (!MAP) store_tiles<NT, KP / 16>(S, s.dS + where * (l.state / 4), l.VP, cols);
        __syncthreads();
        // dU
        v4f_t U[4][NT];
        Frag f[2][NT][INNER];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) U[mt][nt] = v4f_t{0.f, 0.f, 0.f, 0.f};
        {
            Frag p[KP / 32][NT][INNER];
#pragma unroll
            for (int c0 = 0; c0 < KP / 32; ++c0)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) split_tiles<INNER>(S[2 * c0][nt], S[2 * c0 + 1][nt], p[c0][nt]);
            times_state<RAW, INNER, KP>(U, kt, p);
        }
        {
            v4f_t d[4][NT];
            Frag b[2][NT][RAW];
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                const float4 write = four(vl + VEC_WRITE * 64, mt);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    d[mt][nt] = v4f_t{o[mt][0].at(nt), o[mt][1].at(nt), o[mt][2].at(nt), o[mt][3].at(nt)};
                    U[mt][nt] = times(U[mt][nt], write);
                }
            }
            split_rows<RAW, NT>(d, b);
            times_triangle<INNER, true>(U, pm, b);
        }
        // X
        split_rows<INNER, NT>(U, f);
        v4f_t X[4][NT];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) X[mt][nt] = v4f_t{0.f, 0.f, 0.f, 0.f};
        times_triangle<INNER, true>(X, tm, f);
        if (!MAP) store_tiles<NT, 4>(X, s.X + where * (l.rows / 4), l.VP, cols);
        const auto places = cols.template places<T>((int)g.v_stride, g.V);
        const BufView out = rows_view(dv + at * g.v_stride + (long long)h * g.V, g.v_stride, len, g.V);
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
            const float4 beta = four(vl + VEC_BETA * 64, mt), read = four(vl + VEC_READ * 64, mt);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) X[mt][nt] = times(X[mt][nt], beta);
#pragma unroll
            for (int r = 0; r < (MAP ? 0 : 4); ++r) {
                float x[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) x[nt] = X[mt][nt][r];
                cols.template store<T, WHOLE>(out, places, mt, r, x);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) X[mt][nt] = -times(X[mt][nt], read);
        }
        // dS
        split_rows<INNER, NT>(X, f);
#pragma unroll
        for (int ct = 0; ct < KP / 16; ++ct)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[ct][nt] *= decay;
        add_to_state<RAW, KP>(S, kt, f);
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
            const float4 ask = four(vl + VEC_ASK * 64, mt);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) X[mt][nt] = times(v4f_t{o[mt][0].at(nt), o[mt][1].at(nt), o[mt][2].at(nt), o[mt][3].at(nt)}, ask);
        }
        split_rows<INNER, NT>(X, f);
        if constexpr (SHARE) __syncthreads();
        rows.template put<KP>(qt);
        if (c > from) load_keys(c - 1);
        __syncthreads();
        add_to_state<RAW, KP>(S, qt, f);
        settled();
    }
    if constexpr (MAP) store_tiles<NT, KP / 16>(S, s.ends + piece * (l.state / 4), l.VP, cols);
}

template <typename T, int KP, int NT, bool MAP>
hipError_t launch(const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dv, hipStream_t stream)
{
    constexpr size_t lds = Walk<T, KP, true, 2 * INNER>::LDS;
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    const bool whole = whole_keys<T>(g) && (NT == 1 || pair_values<T>(g, dy, dv, g.y_stride, g.v_stride));
    const auto kernel = whole ? k_gdelta_bwd_states<T, KP, NT, true, MAP> : k_gdelta_bwd_states<T, KP, NT, false, MAP>;
    const hipError_t e = gd_lds(kernel, lds);
    if (e != hipSuccess) return e;
    const int blocks = cdiv(l.VP, WAVES * 16 * NT);
    const long long items = (l.piece ? l.pieces : (long long)g.sequences) * g.key_heads;
    return gd_launches(gd_shared_blocks(items, blocks * (g.H / g.key_heads)), THREADS, [&](long long first, unsigned now) {
        hipLaunchKernelGGL(kernel, dim3(now), dim3(THREADS), lds, stream, g, l, s, (const T *)dy, (T *)dv, first, blocks);
    });
}

// As the walk forward: where sequences go in pieces what they make of zero first, and the gradients that they begin with
template <typename T, int KP> hipError_t walk(const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dv, hipStream_t stream)
{
    if (l.piece) {
        hipError_t e = launch<T, KP, 1, true>(g, l, s, dy, dv, stream);
        if (e == hipSuccess) e = launch_gdelta_join(g, l, s, true, stream);
        if (e != hipSuccess) return e;
    }
    if constexpr (may_have_two_tiles<T, KP>) {
        if (two_tiles(g, l)) return launch<T, KP, 2, false>(g, l, s, dy, dv, stream);
    }
    return launch<T, KP, 1, false>(g, l, s, dy, dv, stream);
}

template <typename T> hipError_t walk_of(const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dv, hipStream_t stream)
{
    switch (l.KP) {
    case 32: return walk<T, 32>(g, l, s, dy, dv, stream);
    case 64: return walk<T, 64>(g, l, s, dy, dv, stream);
    case 128: return walk<T, 128>(g, l, s, dy, dv, stream);
    default: return walk<T, 256>(g, l, s, dy, dv, stream);
    }
}

}  // namespace

hipError_t launch_gdelta_bwd_states(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dv, hipStream_t stream)
{
    return dtype == DWCONV_F32 ? walk_of<float>(g, l, s, dy, dv, stream) : walk_of<bf16_t>(g, l, s, dy, dv, stream);
}

}  // namespace dwc
