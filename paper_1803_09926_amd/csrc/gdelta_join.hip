// The gated delta rule, long sequences in pieces: the states that the pieces begin with (forward), or the gradients of those that they end with (backward).
//
// A piece makes M S + N of the state S before it; N lies in `ends`, M in `maps`.  A block has 64 columns of a sequence's head, 16 a wavefront, and goes from piece to
// piece: S <- M S + N, each S put in the place of the N that it is added to.  Backward S <- M^T S + N from the last piece to the first.  The matrix goes through LDS by
// 64 rows (backward 64 columns of them), the next ones on their way meanwhile.
#include "gdelta_states.hpp"

namespace dwc {

namespace {

template <int KP, int N, bool BACK>
__global__ __launch_bounds__(THREADS, 1) void k_gdelta_join(GdArgs g, GdLayout l, GdSpace s, unsigned first, int blocks)
{
    constexpr int ROWS = KP < 64 ? KP : 64;              // of the matrix, at a time
    constexpr int PLANE = ROWS * KP, PER = ROWS * KP / 8 / THREADS > 0 ? ROWS * KP / 8 / THREADS : 1;
    extern __shared__ __align__(16) char lds[];
    bf16_t *const tile = reinterpret_cast<bf16_t *>(lds);
    const unsigned bid = first + blockIdx.x;
    const int seq = (int)(bid / (unsigned)blocks), h = blockIdx.y;
    const Columns<1> cols((int)(bid % (unsigned)blocks));
    const int unit = l.piece * CHUNK, start = gd_start(g, seq), end = gd_start(g, seq + 1), base = gd_base(g, seq, unit);
    const long long chunks = min((long long)(end > start ? cdiv(end - start, CHUNK) : 0), l.chunks - gd_base(g, seq, CHUNK));
    const int pieces = (int)min((long long)(chunks > 0 ? cdiv((int)chunks, l.piece) : 0), l.pieces - base);
    if (pieces < 2) return;
    auto ends = [&](int p) { return s.ends + (((long long)base + p) * g.H + h) * (l.state / 4); };
    auto maps = [&](int p) { return s.maps + (((long long)base + p) * g.H + h) * (l.map / 4); };
    // forward: the state behind piece p, p = 0 .. pieces - 2, is what piece p + 1 begins with; backward: the gradient before piece p, p = pieces - 1 .. 1, piece p - 1's
    v4f_t S[KP / 16][1], next[KP / 16][1];
    const int begin = BACK ? pieces - 1 : 0, stop = BACK ? 1 : pieces - 2, step = BACK ? -1 : 1;
    load_state<1, KP / 16>(S, ends(begin), KP, l.VP, cols);
    u4t_t ahead[PER][2];
    // (the rows of M are contracted forward, its columns backward: rows of it in LDS either way)
    auto ask = [&](int p, int r0) {
        const BufView view(maps(p), (uint32_t)l.map);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int n = threadIdx.x + i * THREADS;
            const uint32_t off = n < ROWS * KP / 8 ? (uint32_t)((r0 + n / (KP / 8)) * KP + n % (KP / 8) * 8) * 4u : BufView::OUTSIDE;
            ahead[i][0] = view.b128(off, 0);
            ahead[i][1] = view.b128(off + 16, 0);
        }
    };
    if (begin != stop) {
        ask(begin + step, 0);
        load_state<1, KP / 16>(next, ends(begin + step), KP, l.VP, cols);
    }
    for (int p = begin; p != stop; p += step) {
        const int to = p + step;
        store_tiles<1, KP / 16>(S, ends(to), l.VP, cols);
        Frag f[KP / 32][N];
#pragma unroll
        for (int c = 0; c < KP / 32; ++c) split_tiles<N>(S[2 * c][0], S[2 * c + 1][0], f[c]);
#pragma unroll
        for (int r0 = 0; r0 < KP; r0 += ROWS) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int n = threadIdx.x + i * THREADS;
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(ahead[i][j / 4][j % 4]);
                if (n < ROWS * KP / 8) put8<N, KP>(tile, PLANE, n / (KP / 8), n % (KP / 8) * 8, x);
            }
            if (r0 + ROWS < KP) ask(to, r0 + ROWS);
            else if (to != stop) ask(to + step, 0);
            __syncthreads();
            if constexpr (!BACK) {
#pragma unroll
                for (int c = 0; c < KP / 32; ++c)
#pragma unroll
                    for (int t = 0; t < ROWS / 16; ++t) {
                        Frag a[N];
                        frags_rows<N, KP>(a, tile, PLANE, t * 16, c * 32);
                        mma<N, N>(next[r0 / 16 + t][0], a, f[c]);
                    }
            } else {
#pragma unroll
                for (int c = 0; c < ROWS / 32; ++c)
#pragma unroll
                    for (int t = 0; t < KP / 16; ++t) {
                        Frag a[N];
                        frags_cols<N, KP>(a, tile, PLANE, c * 32, t * 16);
                        mma<N, N>(next[t][0], a, f[r0 / 32 + c]);
                    }
            }
        }
#pragma unroll
        for (int t = 0; t < KP / 16; ++t) S[t][0] = next[t][0];
        if (to != stop) load_state<1, KP / 16>(next, ends(to + step), KP, l.VP, cols);
    }
    store_tiles<1, KP / 16>(S, ends(stop + step), l.VP, cols);
}

template <int KP, int N, bool BACK> hipError_t launch(const GdArgs &g, const GdLayout &l, const GdSpace &s, hipStream_t stream)
{
    constexpr size_t lds = (size_t)N * (KP < 64 ? KP : 64) * KP * 2;
    const auto kernel = k_gdelta_join<KP, N, BACK>;
    const hipError_t e = gd_lds(kernel, lds);
    if (e != hipSuccess) return e;
    const int blocks = cdiv(l.VP, WAVES * 16);
    return gd_launches((long long)g.sequences * blocks, THREADS, [&](unsigned first, unsigned now) {
        hipLaunchKernelGGL(kernel, dim3(now, (unsigned)g.H), dim3(THREADS), lds, stream, g, l, s, first, blocks);
    });
}
template <int KP> hipError_t launch_of(const GdArgs &g, const GdLayout &l, const GdSpace &s, bool backward, hipStream_t stream)
{
    if (l.inner == 2) return backward ? launch<KP, 2, true>(g, l, s, stream) : launch<KP, 2, false>(g, l, s, stream);
    return backward ? launch<KP, 3, true>(g, l, s, stream) : launch<KP, 3, false>(g, l, s, stream);
}

}  // namespace

hipError_t launch_gdelta_join(const GdArgs &g, const GdLayout &l, const GdSpace &s, bool backward, hipStream_t stream)
{
    switch (l.KP) {
    case 32: return launch_of<32>(g, l, s, backward, stream);
    case 64: return launch_of<64>(g, l, s, backward, stream);
    case 128: return launch_of<128>(g, l, s, backward, stream);
    default: return launch_of<256>(g, l, s, backward, stream);
    }
}

}  // namespace dwc
