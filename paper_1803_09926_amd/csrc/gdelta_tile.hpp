// Tiles of the gated delta rule's matrix products.
//
// All products run on the bf16 matrix instruction of 16 x 16 x 32.  A number of 32 bits takes part as a sum of bf16 parts: what a bf16 tensor holds is one part; what
// the kernels compute themselves (states, inverses, what tokens write and answer) three parts, which hold all of its 24 bits, and so does all that an fp32 tensor holds.
// Of a product of parts those count whose order is below the larger number of parts (1 x 3: three instructions, 3 x 3: six).  All sums are fp32, and what a call is asked
// for does not change a bit of its other outputs.  (With two parts, 2^-17 of a number, the states behind bf16 sequences were 2e-6 to 5e-6 off, and are 2e-7 with three.)
//
// Lanes: m = lane % 16, q = lane / 16.  A result tile has rows 4 q + r (r = 0..3) of column m in a lane.  Two result tiles below each other are an operand as they are: the
// contraction runs over their 32 rows in the order 4 q + 0..3 of the first, 4 q + 0..3 of the second.  Tiles in LDS are stored so that 16 consecutive bytes of a row hold the
// same order (within every 32 columns), and columns are read through the transposing reads of LDS.  Which 16 bytes of its row a piece has depends on the row: the pieces
// that an instruction reads, one of each of 16 rows, or four of each of four, then lie in all 64 banks (with padded rows instead the transposing reads met four to a bank).
#pragma once
#include "gdelta.hpp"

namespace dwc {

namespace {

typedef float v4f_t __attribute__((ext_vector_type(4)));
typedef __bf16 v8b_t __attribute__((ext_vector_type(8)));
typedef short v4h_t __attribute__((ext_vector_type(4)));
typedef uint32_t u4t_t __attribute__((ext_vector_type(4)));
typedef uint32_t u2t_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.402823466e38f; }

// `blocks` workgroups in launches that each have fewer than 2^32 lanes: f(the first (64 bits), how many)
template <typename F> hipError_t gd_launches(long long blocks, int threads, F f)
{
    const long long most = most_blocks(threads);
    for (long long first = 0; first < blocks; first += most) f(first, (unsigned)(blocks - first < most ? blocks - first : most));
    return hipGetLastError();
}
// Blocks that read the same rows, `blocks` of each of `items`, lie on one of the eight XCDs, whose L2 they share, and run close in time: the dispatcher hands blocks to the
// XCDs in turn.  The number of a launch's blocks; the item and the number in it of one of them (item may be behind the last one).
inline long long gd_shared_blocks(long long items, int blocks) { return (items + 7) / 8 * 8 * blocks; }
// (quotients of what fits 32 bits are formed in 32: those of 64 take hundreds of instructions)
__device__ __forceinline__ unsigned long long quotient(unsigned long long n, unsigned d) { return n >> 32 ? n / d : (unsigned)n / d; }
struct Shared { long long item; int block; };
__device__ __forceinline__ Shared gd_shared(unsigned long long n, unsigned blocks)
{
    const unsigned long long group = quotient(n, 8 * blocks);
    return {(long long)(group * 8 + n % 8), (int)((n - group * (8 * blocks)) / 8)};
}
// What is the same in all lanes, where the compiler does not see it: addresses are then formed once instead of in every lane
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// more LDS than a launch has without being told
template <typename K> hipError_t gd_lds(K kernel, size_t bytes)
{
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

constexpr int CHUNK = 64;

constexpr int INNER = 3;                          // parts of what the kernels compute themselves
template <typename T> struct PartsOf;            // RAW: of what a tensor holds
template <> struct PartsOf<bf16_t> { static constexpr int RAW = 1; };
template <> struct PartsOf<float> { static constexpr int RAW = 3; };

// The number of a lane's wavefront, as a scalar.  What is done by some wavefronts only has to be behind a scalar branch where it holds matrix instructions: those do not
// look at which lanes are on.
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// A lane's number that the compiler takes for a new one each time: what is formed with it is formed where it is used, and does not occupy registers from one part of
// a kernel to the next
__device__ __forceinline__ int lane_anew()
{
    int v = threadIdx.x & 63;
    asm volatile("" : "+v"(v));
    return v;
}

struct Frag { u4t_t w; };

__device__ __forceinline__ v4f_t mfma(const Frag &a, const Frag &b, v4f_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b_t, a.w), __builtin_bit_cast(v8b_t, b.w), c, 0, 0, 0);
}
// c += a b, of the first PA and PB parts
template <int PA, int PB, int NA, int NB> __device__ __forceinline__ void mma(v4f_t &c, const Frag (&a)[NA], const Frag (&b)[NB])
{
    static_assert(PA <= NA && PB <= NB, "parts that are there");
    constexpr int ORDER = PA > PB ? PA : PB;
#pragma unroll
    for (int i = PA - 1; i >= 0; --i)             // the small ones first
#pragma unroll
        for (int j = PB - 1; j >= 0; --j)
            if (i + j < ORDER) c = mfma(a[i], b[j], c);
}

// The hardware does not hold back what reads a matrix instruction's result, or writes over it, before it is there: 8 steps behind one of bf16, 10 behind one of fp32.  The compiler keeps
// them within straight code, but has left some out where branches lay between (and tests/test_matrix_waits.py counts them in what it made).  So where a branch lies between such an
// instruction and the first use of its result, the steps are waited for here, by all that comes behind.
__device__ __forceinline__ void settled()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 9");
    __builtin_amdgcn_sched_barrier(0);
}

// two numbers as N parts, each a pair of bf16: what is left after a part is taken is exact.  (The dot product instruction takes
// a part out in one instruction instead of two, and no walk was faster for it.)
template <int N> __device__ __forceinline__ void split2(float x, float y, uint32_t (&p)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = pack2_bf16(x, y);
        if (i + 1 < N) {
            x -= __uint_as_float(p[i] << 16);
            y -= __uint_as_float(p[i] & 0xffff0000u);
        }
    }
}
// two result tiles, one below the other, as an operand
template <int N> __device__ __forceinline__ void split_tiles(const v4f_t &a, const v4f_t &b, Frag (&f)[N])
{
    uint32_t p[4][N];
    split2<N>(a[0], a[1], p[0]);
    split2<N>(a[2], a[3], p[1]);
    split2<N>(b[0], b[1], p[2]);
    split2<N>(b[2], b[3], p[3]);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i].w = u4t_t{p[0][i], p[1][i], p[2][i], p[3][i]};
}

// the piece of 16 bytes, of a row of LD columns in memory order, that holds the four columns from 4 * j4 on, and which half of it
__device__ __forceinline__ constexpr int piece_of(int j4) { return (j4 >> 3) * 4 + (j4 & 3); }
__device__ __forceinline__ constexpr int half_of(int j4) { return (j4 >> 2) & 1; }
// where in LDS a row's piece lies
template <int LD> __device__ __forceinline__ constexpr int turned(int row, int piece)
{
    return piece ^ (LD == 32 ? (row >> 2) & 3 : LD == 64 ? ((row >> 1) & 1) << 2 | ((row >> 2) & 3) : (row & 3) << 2 | ((row >> 2) & 3));
}
template <int LD> __device__ __forceinline__ constexpr int place4(int row, int j4) { return row * LD + turned<LD>(row, piece_of(j4)) * 8 + half_of(j4) * 4; }
template <int LD> __device__ __forceinline__ constexpr int place(int row, int col) { return place4<LD>(row, col >> 2) + (col & 3); }

// Operands out of LDS tiles of leading dimension LD.  rows: 16 of them from r0, contracted over the 32 columns from c0 on.  cols: 16 of them from c0, contracted over
// the 32 rows from r0 on.
template <int LD> __device__ __forceinline__ Frag frag_rows(const bf16_t *tile, int r0, int c0, int lane)
{
    // (r0 is a multiple of 16: the rows' turns are those of the lane)
    return {*reinterpret_cast<const u4t_t *>(tile + (r0 + (lane & 15)) * LD + turned<LD>(lane & 15, c0 / 8 + (lane >> 4)) * 8)};
}
typedef __attribute__((address_space(3))) v4h_t *lds_v4h_t;
template <int LD> __device__ __forceinline__ Frag frag_cols(const bf16_t *tile, int r0, int c0, int lane)
{
    const int m = lane & 15, q = lane >> 4;
    const bf16_t *const p = tile + r0 * LD + place4<LD>(4 * q + (m >> 2), (c0 >> 2) + (m & 3));
    const v4h_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4h_t)p);
    const v4h_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4h_t)(p + 16 * LD));
    const u2t_t x = __builtin_bit_cast(u2t_t, a), y = __builtin_bit_cast(u2t_t, b);
    return {u4t_t{x.x, x.y, y.x, y.y}};
}
// the numbers of a tile of N parts where a result tile has its own: rows r0 + 4 q + r of column c0 + m
template <int N, int LD> __device__ __forceinline__ v4f_t tile_of(const bf16_t *tile, int plane, int r0, int c0, int lane)
{
    const int m = lane & 15, q = lane >> 4;
    v4f_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        const bf16_t *const p = tile + i * plane + r0 * LD + place4<LD>(4 * q + (m >> 2), (c0 >> 2) + (m & 3));
        const u2t_t w = __builtin_bit_cast(u2t_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4h_t)p));
        v += v4f_t{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
    }
    return v;
}
template <int N, int LD> __device__ __forceinline__ void frags_rows(Frag (&f)[N], const bf16_t *tile, int plane, int r0, int c0, int lane = threadIdx.x & 63)
{
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = frag_rows<LD>(tile + i * plane, r0, c0, lane);
}
template <int N, int LD> __device__ __forceinline__ void frags_cols(Frag (&f)[N], const bf16_t *tile, int plane, int r0, int c0, int lane = threadIdx.x & 63)
{
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = frag_cols<LD>(tile + i * plane, r0, c0, lane);
}

// eight consecutive numbers from a column that is a multiple of 8 on, into a row of an LDS tile of N parts
template <int N, int LD> __device__ __forceinline__ void put8(bf16_t *tile, int plane, int row, int col, const float (&x)[8])
{
    uint32_t p[4][N];
#pragma unroll
    for (int i = 0; i < 4; ++i) split2<N>(x[2 * i], x[2 * i + 1], p[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        *reinterpret_cast<u2t_t *>(tile + i * plane + place4<LD>(row, col >> 2)) = u2t_t{p[0][i], p[1][i]};
        *reinterpret_cast<u2t_t *>(tile + i * plane + place4<LD>(row, (col >> 2) + 1)) = u2t_t{p[2][i], p[3][i]};
    }
}
// the same for eight numbers as they came
template <typename T, int LD, bool WHOLE> __device__ __forceinline__ void put8_ahead(bf16_t *tile, int plane, int row, int col, const Ahead<T, 8, WHOLE> &v)
{
    if constexpr (sizeof(T) == 2) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (WHOLE) w[i] = v.w[i];
            else w[i] = v.w[2 * i] | v.w[2 * i + 1] << 16;
        }
        *reinterpret_cast<u2t_t *>(tile + place4<LD>(row, col >> 2)) = u2t_t{w[0], w[1]};
        *reinterpret_cast<u2t_t *>(tile + place4<LD>(row, (col >> 2) + 1)) = u2t_t{w[2], w[3]};
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v.at(i);
        put8<PartsOf<T>::RAW, LD>(tile, plane, row, col, x);
    }
}

// Rows of a chunk in memory: what lies behind the last row's `width` numbers is outside the view, and so is every row behind it
template <typename T> __device__ __forceinline__ BufView rows_view(const T *p, long long stride, int len, int width)
{
    return BufView(p, (uint32_t)(((len - 1) * stride + width) * (long long)sizeof(T)));
}

// A tile of 64 rows of KP columns on its way from memory to LDS: held by THREADS lanes, of which each has every THREADS-th eight columns.  WHOLE: eight columns are
// there or not, and aligned.  No branch: the loads are asked for early and used late.
template <typename T, int KP, int THREADS, bool WHOLE> struct Rows {
    static constexpr int PER_ROW = KP / 8, N = CHUNK * PER_ROW / THREADS;
    static_assert(CHUNK * PER_ROW % THREADS == 0, "all lanes alike");
    Ahead<T, 8, WHOLE> v[N];
    // len rows of `width` columns are there
    __device__ __forceinline__ void load(const T *p, long long stride, int len, int width)
    {
        const BufView view = rows_view(p, stride, len, width);
        const int row = threadIdx.x / PER_ROW, col = threadIdx.x % PER_ROW * 8;
        const uint32_t step = (uint32_t)(THREADS / PER_ROW * stride) * (uint32_t)sizeof(T);
        uint32_t off = (uint32_t)(row * (int)stride + col) * (uint32_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < N; ++i, off += step) v[i].load(view, off, width - col);
    }
    template <int LD> __device__ __forceinline__ void put(bf16_t *tile) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = threadIdx.x + i * THREADS;
            put8_ahead<T, LD, WHOLE>(tile, CHUNK * LD, at / PER_ROW, at % PER_ROW * 8, v[i]);
        }
    }
};

// One of the first pass's matrices, of N parts: zero above the diagonal, and the 32 x 32 block there is neither stored nor read.  A part is 384 pieces of 16 bytes in the
// LDS tiles' order of columns (not turned): four of each of the first 32 rows, eight of each of the others.  So it is in LDS too: a tile of 32 columns, one of 64 behind it.
constexpr int MATRIX_PIECES = 384, MATRIX_PLANE = MATRIX_PIECES * 8;
// ... on its way to LDS.  A wavefront has 64 pieces at a time, all of them of one of the two tiles: in LDS too they are those 64, in the order of the tile's turns.
template <int N, int THREADS> struct Matrix {
    static constexpr int ALL = N * MATRIX_PIECES, PER = (ALL + THREADS - 1) / THREADS;
    static_assert(THREADS % 64 == 0 && MATRIX_PIECES == 6 * 64, "64 at a time: two times of the first tile, four of the second");
    u4t_t v[PER];
    __device__ __forceinline__ void load(const char *p)
    {
        // (beyond the matrix nothing is read; a view for each time: all have one offset)
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = BufView(p + i * THREADS * 16, (ALL - i * THREADS) * 16).b128(threadIdx.x * 16, 0);
    }
    __device__ __forceinline__ void put(bf16_t *tile) const
    {
        const int lane = threadIdx.x & 63, w = wave_number();
        const int first = lane / 4 * 4 + turned<32>(lane / 4, lane % 4), second = lane / 8 * 8 + turned<64>(lane / 8, lane % 8);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int n = i * (THREADS / 64) + w, at = n % 6;
            // (eight rows on, turned<64> has its second bit the other way round)
            if (ALL % THREADS == 0 || n < ALL / 64) *reinterpret_cast<u4t_t *>(tile + (n * 64 + (at < 2 ? first : at % 2 ? second ^ 2 : second)) * 8) = v[i];
        }
    }
};
// operands out of it, as frags_rows and frags_cols; r0 and c0 are known when compiled
template <int N> __device__ __forceinline__ void matrix_rows(Frag (&f)[N], const bf16_t *tile, int r0, int c0)
{
    if (r0 < 32) frags_rows<N, 32>(f, tile, MATRIX_PLANE, r0, c0);
    else frags_rows<N, 64>(f, tile + 1024, MATRIX_PLANE, r0 - 32, c0);
}
template <int N> __device__ __forceinline__ void matrix_cols(Frag (&f)[N], const bf16_t *tile, int r0, int c0)
{
    if (r0 < 32) frags_cols<N, 32>(f, tile, MATRIX_PLANE, r0, c0);
    else frags_cols<N, 64>(f, tile + 1024, MATRIX_PLANE, r0 - 32, c0);
}

// Vectors of a chunk and head that the first pass leaves, 64 floats each
enum { VEC_READ = 0,     // exp(G) rk: what a row of k^T S is multiplied by
       VEC_BETA = 1,
       VEC_WRITE = 2,    // exp(G_end - G) rk: what a token's write is multiplied by at the chunk's end
       VEC_ASK = 3,      // scale exp(G) rq
       VEC_RQ = 4, VEC_RK = 5,
       VEC_G = 6,        // the sum of the decays' logarithms from the chunk's start, 64 doubles
       VEC_ONE = 8,      // [0] exp(G_end); [1] as int: the first token whose k, a or b is not finite, 64 if there is none
       VECS = 9 };

// Whether eight columns of keys and queries are whole aligned vectors
template <typename T> bool whole_keys(const GdArgs &g)
{
    const int v = 16 / (int)sizeof(T);
    return g.K % 8 == 0 && !unaligned16(g.q) && !unaligned16(g.k) && (g.T < 2 || (g.q_stride % v == 0 && g.k_stride % v == 0));
}

// ---- chunks of packed sequences ----
// Sequence s has its chunks at floor(starts[s] / 64) + s and the places behind it: no two sequences share one, and none has to be counted.
struct ChunkAt { int first, len, seq, place, start, end; };   // the first token, how many (0: nothing here), the sequence, the chunk's number in it, its tokens
__device__ __forceinline__ int gd_start(const GdArgs &g, int s)
{
    if (!g.starts) return s * g.length;
    const int v = g.starts[s];
    return v < 0 ? 0 : v > g.T ? g.T : v;
}
// The same holds for pieces of several chunks: unit is 64, or the tokens of a piece
__device__ __forceinline__ int gd_base(const GdArgs &g, int s, int unit)
{
    return g.starts ? gd_start(g, s) / unit + s : s * cdiv(g.length > 0 ? g.length : 1, unit);
}
// (id is the same in a wavefront's 64 lanes, all of which are here: up to 63 sequences one load and no other after it, which counts where the memory is busy)
__device__ __forceinline__ ChunkAt gd_chunk(const GdArgs &g, int id, int unit)
{
    int lo = 0, hi = g.sequences, base, start, end;
    const int lane = threadIdx.x & 63;
    if (g.starts && hi < 64) {
        const int mine = gd_start(g, min(lane, hi));
        lo = max(__popcll(__ballot(lane < hi && mine / unit + lane <= id)) - 1, 0);
        start = __builtin_amdgcn_readlane(mine, lo);
        end = __builtin_amdgcn_readlane(mine, lo + 1);
        base = start / unit + lo;
    } else {
        if (!g.starts) lo = min(id / cdiv(g.length > 0 ? g.length : 1, unit), g.sequences - 1);
        else while (hi - lo > 1) {
            const int step = (hi - lo + 63) / 64;
            const long long at = lo + (long long)step * (lane + 1);
            lo += step * __popcll(__ballot(at < hi && gd_base(g, at < hi ? (int)at : lo, unit) <= id));
            hi = hi - lo > step ? lo + step : hi;
        }
        lo = uniform(lo);
        base = gd_base(g, lo, unit);
        start = gd_start(g, lo);
        end = gd_start(g, lo + 1);
    }
    lo = uniform(lo);
    base = uniform(base);
    start = uniform(start);
    end = uniform(end);
    const int place = id - base;
    const long long first = start + (long long)place * unit;
    if (place < 0 || first >= end) return {0, 0, lo, place, start, end};
    return {(int)first, (int)min((long long)unit, end - first), lo, place, start, end};
}

}  // namespace

}  // namespace dwc
