// What the two walks over a sequence's chunks share: columns of the state in registers.
#pragma once
#include "gdelta_tile.hpp"
#include "gdelta_launch.hpp"

namespace dwc {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

// A uniform number that the compiler takes for a new one each time: what is formed with it is formed where it is used, and does not occupy registers over the whole walk
__device__ __forceinline__ int fresh(int v)
{
    asm volatile("" : "+s"(v));
    return v;
}
// In a branch that is hardly ever taken: it stays one, instead of selections that are always made
__device__ __forceinline__ void seldom() { asm volatile(""); }

// The columns of a lane: NT neighbours, one in each of its NT result tiles, so that its numbers of a row lie beside each other.  PAIRS: they are read and written
// at once, aligned.  What is not there is asked for, and stored, outside the view: no branch.
template <int NT> struct Columns {
    int c;                                        // the first
    __device__ __forceinline__ Columns(int block) : c((block * WAVES + wave_number()) * 16 * NT + (int)(threadIdx.x & 15) * NT) {}
    __device__ __forceinline__ uint32_t at(int row, int stride, int size) const { return (uint32_t)(row * stride + c) * (uint32_t)size; }
    // Rows 16 mt + 4 q + r, `stride` apart, of `width` columns: the part of their places that differs between lanes (outside the view where the columns are outside
    // the row), and that which does not
    template <typename T> struct Places {
        uint32_t lane;
        int row, there;
        __device__ __forceinline__ uint32_t at(int mt, int r) const { return lane + (uint32_t)((16 * mt + r) * row); }
    };
    template <typename T> __device__ __forceinline__ Places<T> places(int stride, int width) const
    {
        stride = fresh(stride);
        const uint32_t off = (uint32_t)(4 * (int)((threadIdx.x & 63) >> 4) * stride + c) * (uint32_t)sizeof(T);
        return {c < width ? off : BufView::OUTSIDE, stride * (int)sizeof(T), width - c};
    }
    template <typename T, bool PAIRS> __device__ __forceinline__ void load(Ahead<T, NT, PAIRS> &x, const BufView &view, const Places<T> &p, int mt, int r) const
    {
        x.load(view, p.at(mt, r), PAIRS || NT == 1 ? 1 : p.there);
    }
    template <typename T, bool PAIRS> __device__ __forceinline__ void store(const BufView &view, const Places<T> &p, int mt, int r, const float (&x)[NT]) const
    {
        store_late<T, NT, PAIRS>(view, p.at(mt, r), PAIRS || NT == 1 ? 1 : p.there, x);
    }
};

// rows 16 mt + 4 q + r of a tile of tokens
__device__ __forceinline__ int row_of(int mt, int r) { return mt * 16 + 4 * (int)((threadIdx.x & 63) >> 4) + r; }
__device__ __forceinline__ float4 four(const float *v, int mt) { return *reinterpret_cast<const float4 *>(v + row_of(mt, 0)); }
__device__ __forceinline__ v4f_t times(const v4f_t &a, const float4 &b) { return v4f_t{a[0] * b.x, a[1] * b.y, a[2] * b.z, a[3] * b.w}; }

// the state of a sequence and head, [K][V], at a walk's ends
template <int NT, int CT> __device__ __forceinline__ void load_state(v4f_t (&S)[CT][NT], const float *p, int K, int V, const Columns<NT> &cols)
{
    const BufView view(p, (uint32_t)(K * V) * 4u);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            Ahead<float, NT, false> x;
            x.load(view, cols.at(row_of(ct, r), V, 4), row_of(ct, r) < K ? V - cols.c : 0);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[ct][nt][r] = x.at(nt);
        }
}
template <int NT, int CT> __device__ __forceinline__ void store_state(const v4f_t (&S)[CT][NT], float *p, int K, int V, const Columns<NT> &cols)
{
    const BufView view(p, (uint32_t)(K * V) * 4u);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float x[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) x[nt] = S[ct][nt][r];
            store_late<float, NT, false>(view, cols.at(row_of(ct, r), V, 4), row_of(ct, r) < K ? V - cols.c : 0, x);
        }
}
// what the passes hand to each other, [rows][VP]
template <int NT, int MT> __device__ __forceinline__ void store_tiles(const v4f_t (&x)[MT][NT], float *p, int VP, const Columns<NT> &cols)
{
    const BufView view(p, (uint32_t)(MT * 16 * VP) * 4u);
    const auto places = cols.template places<float>(VP, VP);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float y[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) y[nt] = x[mt][nt][r];
            cols.template store<float, true>(view, places, mt, r, y);
        }
}

// result tiles of 64 rows as operands that are contracted over them
template <int N, int NT> __device__ __forceinline__ void split_rows(const v4f_t (&x)[4][NT], Frag (&f)[2][NT][N])
{
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) split_tiles<N>(x[2 * ks][nt], x[2 * ks + 1][nt], f[ks][nt]);
}

// Whether some of a lane's numbers are not finite
template <int NT> __device__ __forceinline__ bool not_finite(const v4f_t (&x)[4][NT])
{
    float probe = 0.f;
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) probe = fmaf(x[mt][nt][r], 0.f, probe);
    return !(probe == 0.f);
}
// Zeros from a column's first row on that is not finite, or from `from` on where that comes before; `from` becomes the one of the two
template <int NT> __device__ __forceinline__ void rows_before(v4f_t (&x)[4][NT], int (&from)[NT])
{
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!finite(x[mt][nt][r])) from[nt] = min(from[nt], row_of(mt, r));
        const int up = __shfl_xor(from[nt], 16, 64);
        from[nt] = min(from[nt], up);
        const int far = __shfl_xor(from[nt], 32, 64);
        from[nt] = min(from[nt], far);
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (row_of(mt, r) >= from[nt]) x[mt][nt][r] = 0.f;
    }
}

// Products with operands out of LDS.  (Operands read by eight and sixteen ahead of their use were no faster than what the compiler orders: the walks are bound by the reads
// themselves and by vector instructions.)
// c += A B: A the 64 rows of a tile of KP columns, B the state's operands
template <int RAW, int PB, int KP, int NT, int NB> __device__ __forceinline__ void times_state(v4f_t (&c)[4][NT], const bf16_t *tile, const Frag (&b)[KP / 32][NT][NB])
{
#pragma unroll
    for (int c0 = 0; c0 < KP / 32; ++c0)
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
            Frag a[RAW];
            frags_rows<RAW, KP>(a, tile, CHUNK * KP, mt * 16, c0 * 32);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma<RAW, PB>(c[mt][nt], a, b[c0][nt]);
        }
}
// S += A^T B: A as above, B the operands of 64 rows
template <int RAW, int KP, int NT, int NB> __device__ __forceinline__ void add_to_state(v4f_t (&S)[KP / 16][NT], const bf16_t *tile, const Frag (&b)[2][NT][NB])
{
#pragma unroll
    for (int ct = 0; ct < KP / 16; ++ct)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            Frag a[RAW];
            frags_cols<RAW, KP>(a, tile, CHUNK * KP, ks * 32, ct * 16);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma<RAW, NB>(S[ct][nt], a, b[ks][nt]);
        }
}
// c += A B: A one of the first pass's matrices, which are zero above the diagonal, or (BACK) its transpose
template <int N, bool BACK, int PB, int NT> __device__ __forceinline__ void times_triangle(v4f_t (&c)[4][NT], const bf16_t *tile, const Frag (&b)[2][NT][PB])
{
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
        for (int ks = BACK ? mt / 2 : 0; ks <= (BACK ? 1 : mt / 2); ++ks) {
            Frag a[N];
            if constexpr (BACK) matrix_cols(a, tile, ks * 32, mt * 16);
            else matrix_rows(a, tile, mt * 16, ks * 32);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma<N, PB>(c[mt][nt], a, b[ks][nt]);
        }
}

// What a walk has in LDS: the keys' tile and (OTHER) the queries', which shares its place where both do not fit; so many parts of T and of P; two chunks' vectors
template <typename T, int KP, bool OTHER, int PARTS> struct Walk {
    static constexpr int RAW = PartsOf<T>::RAW;
    static constexpr size_t TILE = (size_t)RAW * CHUNK * KP * 2, REST = (size_t)PARTS * MATRIX_PLANE * 2 + 2 * 256 * 4;
    static constexpr bool SHARE = OTHER && 2 * TILE + REST > 160 * 1024;
    static constexpr size_t LDS = (OTHER && !SHARE ? 2 : 1) * TILE + REST;
};

// Which chunks a block of a walk has: those of a sequence, or of one of its pieces
struct Stretch { int seq, start, end, base, from, to, place, pieces; };       // chunks from .. to - 1 of the sequence's; the piece's number, and how many there are
__device__ __forceinline__ Stretch stretch_of(const GdArgs &g, const GdLayout &l, int id)
{
    Stretch s;
    s.seq = id;
    s.place = 0;
    s.pieces = 1;
    if (l.piece) {
        const ChunkAt at = gd_chunk(g, id, l.piece * CHUNK);
        s.seq = at.seq;
        s.place = at.place;
        s.start = at.start;
        s.end = at.end;
    } else {
        s.start = uniform(gd_start(g, s.seq));
        s.end = uniform(gd_start(g, s.seq + 1));
    }
    s.base = uniform(g.starts ? s.start / CHUNK + s.seq : gd_base(g, s.seq, CHUNK));
    const long long chunks = min((long long)(s.end > s.start ? cdiv(s.end - s.start, CHUNK) : 0), l.chunks - s.base);
    s.from = 0;
    s.to = (int)chunks;
    if (l.piece) {
        s.pieces = chunks > 0 ? cdiv((int)chunks, l.piece) : 1;
        if (s.place < 0 || s.place >= s.pieces) s.place = s.pieces = -1;       // nothing here
        else {
            s.from = s.place * l.piece;
            s.to = min(s.to, s.from + l.piece);
        }
    }
    return s;
}

// Whether a wavefront has 32 columns instead of 16: twice the products of what is read from LDS.  In fp32 with keys of up to 64, where that still fills the card (8192 tokens of 32
// sequences, 16 heads of 64 x 128: 120 us, with 16 columns 136; forward and backward of half of them 266 and 285).  In bf16, whose tiles have a part instead of three, more
// blocks are worth as much or more (16384 tokens of 32 sequences, 16 heads of 128 x 128: 221 and 202; of 64 x 128 171 and 159), and so they are with keys of up to 32 (fp32 97 and 90);
// wider ones have no registers for it.
template <typename T, int KP> constexpr bool may_have_two_tiles = sizeof(T) == 4 && KP == 64;
inline bool two_tiles(const GdArgs &g, const GdLayout &l) { return l.VP > 64 && !l.piece && (long long)g.sequences * g.H * cdiv(l.VP, 128) >= 256; }

// Whether two columns of the values are whole and aligned
template <typename T> bool pair_values(const GdArgs &g, const void *p, const void *q, long long p_stride, long long q_stride)
{
    const uintptr_t pair = 2 * sizeof(T) - 1;
    return g.V % 2 == 0 && !((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & pair) && (g.T < 2 || (p_stride % 2 == 0 && q_stride % 2 == 0));
}

}  // namespace

}  // namespace dwc
