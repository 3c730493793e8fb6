// The gated delta rule, long sequences in pieces: the states that the pieces begin with (forward), or the gradients of those that they end with (backward).
//
// A piece makes M S + N of the state S before it; N lies in `ends`, M in `maps`.  A block has 16 columns of a sequence's head and goes from piece to piece:
// S <- M S + N, each S put in the place of the N that it is added to; backward S <- M^T S + N from the last piece to the first.  A wavefront has 32 rows: of the matrix
// it reads its own straight into operands, the next piece's on their way meanwhile, and its rows of S it hands to the others through LDS as operands, which they are as they
// lie.  Bound by the way round: 15 pieces of 128 x 128 in 16 heads 45 us, where blocks of 64 columns that staged the matrix in LDS took
// 54.  (Two pieces' matrices on their way instead of one: 54.)
#include "gdelta_tile.hpp"
#include "gdelta_launch.hpp"

namespace dwc {

namespace {

template <int KP, bool BACK>
__global__ __launch_bounds__(2 * KP, 1) void k_gdelta_join(GdArgs g, GdLayout l, GdSpace s, long long first, int blocks)
{
    constexpr int GROUPS = KP / 32, N = INNER;           // of 32 rows: one a wavefront
    __shared__ u4t_t handed[2][GROUPS][N][64];
    const Shared which = gd_shared(first + blockIdx.x, (unsigned)blocks);
    if (which.item >= (long long)g.sequences * g.H) return;
    const int seq = uniform((int)quotient(which.item, (unsigned)g.H)), h = uniform((int)(which.item - (long long)seq * g.H)), w = wave_number(), lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
    const int col = which.block * 16 + m;
    const int unit = l.piece * CHUNK, start = gd_start(g, seq), end = gd_start(g, seq + 1), base = gd_base(g, seq, unit);
    const long long chunks = min((long long)(end > start ? cdiv(end - start, CHUNK) : 0), l.chunks - gd_base(g, seq, CHUNK));
    const int pieces = (int)min((long long)(chunks > 0 ? cdiv((int)chunks, l.piece) : 0), l.pieces - base);
    if (pieces < 2) return;
    auto ends = [&](int p) { return BufView(s.ends + (((long long)base + p) * g.H + h) * (l.state / 4), (uint32_t)l.state); };
    v4f_t S[2], next[2];
    auto load = [&](v4f_t (&x)[2], int p) {
        const BufView view = ends(p);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) x[t][r] = __uint_as_float(view.b32((uint32_t)((w * 32 + t * 16 + 4 * q + r) * l.VP + col) * 4u, 0));
    };
    auto store = [&](const v4f_t (&x)[2], int p) {
        const BufView view = ends(p);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) view.st32<false>(__float_as_uint(x[t][r]), (uint32_t)((w * 32 + t * 16 + 4 * q + r) * l.VP + col) * 4u, 0);
    };
    // the wavefront's 32 rows of the matrix (backward: of its transpose), eight numbers of a row for each operand
    v4f_t M[2][GROUPS][2];
    auto ask = [&](int p) {
        const BufView view(s.maps + (((long long)base + p) * g.H + h) * (l.map / 4), (uint32_t)l.map);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < GROUPS; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int row = w * 32 + t * 16 + m, k = c * 32 + i * 16 + 4 * q;
                    if constexpr (!BACK) M[t][c][i] = __builtin_bit_cast(v4f_t, view.b128((uint32_t)(row * KP + k) * 4u, 0));
                    else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) M[t][c][i][r] = __uint_as_float(view.b32((uint32_t)((k + r) * KP + row) * 4u, 0));
                    }
                }
    };
    // forward: the state behind piece p, p = 0 .. pieces - 2, is what piece p + 1 begins with; backward: the gradient before piece p, p = pieces - 1 .. 1, piece p - 1's
    const int begin = BACK ? pieces - 1 : 0, stop = BACK ? 1 : pieces - 2, step = BACK ? -1 : 1;
    load(S, begin);
    if (begin != stop) {
        ask(begin + step);
        load(next, begin + step);
    }
    int turn = 0;
    for (int p = begin; p != stop; p += step, turn ^= 1) {
        const int to = p + step;
        store(S, to);
        Frag f[GROUPS][N];
        split_tiles<N>(S[0], S[1], f[0]);
#pragma unroll
        for (int i = 0; i < N; ++i) handed[turn][w][i][lane] = f[0][i].w;
        __syncthreads();                                 // (who writes to the other half next has read this one two barriers before)
#pragma unroll
        for (int c = 0; c < GROUPS; ++c)
#pragma unroll
            for (int i = 0; i < N; ++i) f[c][i].w = handed[turn][c][i][lane];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            S[t] = next[t];
#pragma unroll
            for (int c = 0; c < GROUPS; ++c) {
                Frag a[N];
                split_tiles<N>(M[t][c][0], M[t][c][1], a);
                mma<N, N>(S[t], a, f[c]);
            }
        }
        if (to != stop) {
            ask(to + step);
            load(next, to + step);
        }
        settled();
    }
    store(S, stop + step);
}

template <int KP> hipError_t launch(const GdArgs &g, const GdLayout &l, const GdSpace &s, bool backward, hipStream_t stream)
{
    const int blocks = l.VP / 16;
    return gd_launches(gd_shared_blocks((long long)g.sequences * g.H, blocks), 2 * KP, [&](long long first, unsigned now) {
        if (backward) hipLaunchKernelGGL((k_gdelta_join<KP, true>), dim3(now), dim3(2 * KP), 0, stream, g, l, s, first, blocks);
        else hipLaunchKernelGGL((k_gdelta_join<KP, false>), dim3(now), dim3(2 * KP), 0, stream, g, l, s, first, blocks);
    });
}

}  // namespace

hipError_t launch_gdelta_join(const GdArgs &g, const GdLayout &l, const GdSpace &s, bool backward, hipStream_t stream)
{
    switch (l.KP) {
    case 32: return launch<32>(g, l, s, backward, stream);
    case 64: return launch<64>(g, l, s, backward, stream);
    case 128: return launch<128>(g, l, s, backward, stream);
    default: return launch<256>(g, l, s, backward, stream);
    }
}

}  // namespace dwc
