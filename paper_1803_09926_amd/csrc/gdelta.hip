// Entry points of the gated delta rule (include/deltaops.h): checks, sizes, and the order of its kernels.
#include "gdelta_launch.hpp"
#include "tune.hpp"
#include <initializer_list>
#include <math.h>
#include <stdlib.h>

namespace dwc {

namespace {

constexpr long long TOKENS = 64;                  // of a chunk

int validate(const gdelta_desc *d)
{
    if (!d) return DWCONV_ERR_NULL;
    if (d->dtype != DWCONV_F32 && d->dtype != DWCONV_BF16) return DWCONV_ERR_BAD_ENUM;
    if ((d->softplus | 1) != 1 || (d->sigmoid | 1) != 1 || (d->norm | 1) != 1) return DWCONV_ERR_BAD_ENUM;
    if (d->T < 0 || d->H < 1 || d->K < 1 || d->V < 1 || d->key_heads < 1 || d->sequences < 1 || d->H % d->key_heads) return DWCONV_ERR_BAD_DIM;
    if (!isfinite(d->scale) || !(d->eps >= 0.f) || !isfinite(d->eps)) return DWCONV_ERR_BAD_DIM;
    if (d->K > GDELTA_MAX_K || d->V > GDELTA_MAX_V) return DWCONV_ERR_UNSUPPORTED;
    const long long keys = (long long)d->key_heads * d->K, values = (long long)d->H * d->V;
    if (d->T > SEQOPS_MAX_T || d->sequences > SEQOPS_MAX_T || d->H > GDELTA_MAX_H) return DWCONV_ERR_TOO_LARGE;
    for (const int64_t s : {d->q_stride, d->k_stride, d->v_stride, d->a_stride, d->b_stride, d->y_stride})
        if (s > GDELTA_MAX_STRIDE) return DWCONV_ERR_TOO_LARGE;
    if (d->T > 1 && (d->q_stride < keys || d->k_stride < keys || d->v_stride < values || d->a_stride < d->H || d->b_stride < d->H || d->y_stride < values))
        return DWCONV_ERR_BAD_DIM;
    // chunks are counted in 32 bits, bytes of all states in 64
    const long long chunks = d->T / TOKENS + d->sequences;
    long long all;
    if (chunks > 0x7fffffffll || __builtin_mul_overflow(chunks * d->H, 1ll << 20, &all)) return DWCONV_ERR_TOO_LARGE;
    return DWCONV_OK;
}

constexpr size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }

GdArgs args_of(const gdelta_desc *d, const gdelta_tensors *t)
{
    GdArgs g = {d->T, d->H, d->K, d->V, d->key_heads, d->sequences, t->starts ? 0 : d->T / d->sequences, d->softplus, d->sigmoid, d->norm, d->scale, d->eps,
                d->q_stride, d->k_stride, d->v_stride, d->a_stride, d->b_stride, d->y_stride, t->q, t->k, t->v, t->a, t->b, (const float *)t->A,
                (const float *)t->a_bias, (const int32_t *)t->starts};
    if (d->T < 2) {                               // the stride of a row alone says nothing
        g.q_stride = g.k_stride = (long long)d->key_heads * d->K;
        g.v_stride = g.y_stride = (long long)d->H * d->V;
        g.a_stride = g.b_stride = d->H;
    }
    return g;
}

// bytes of what the forward pass writes for itself, and of what it keeps for the backward pass besides
size_t forward_bytes(const gdelta_desc *d, const GdLayout &l)
{
    return (size_t)l.chunks * d->H * (size_t)(2 * l.matrix + l.vectors) + (size_t)l.pieces * d->H * (size_t)(l.state + l.map);
}
void place_forward(const gdelta_desc *d, const GdLayout &l, char *p, GdSpace *s)
{
    s->T = p;
    s->P = s->T + l.chunks * d->H * l.matrix;
    s->vec = s->P + l.chunks * d->H * l.matrix;
    s->ends = (float *)(s->vec + l.chunks * d->H * l.vectors);
    s->maps = (float *)((char *)s->ends + l.pieces * d->H * l.state);
}
void place_kept(const gdelta_desc *d, const GdLayout &l, void *kept, GdSpace *s)
{
    place_forward(d, l, (char *)kept, s);
    char *const p = (char *)kept + forward_bytes(d, l);
    s->S = (float *)p;
    s->U = (float *)(p + l.chunks * d->H * l.state);
}

size_t kept_bytes(const gdelta_desc *d, const GdLayout &l) { return forward_bytes(d, l) + (size_t)l.chunks * d->H * (size_t)(l.state + l.rows); }
size_t backward_bytes(const gdelta_desc *d, const GdLayout &l)
{
    return (size_t)l.chunks * d->H * (size_t)(l.state + l.rows) + (size_t)l.pieces * d->H * (size_t)l.state + round16((size_t)l.chunks * d->H * 2 * sizeof(float));
}

// How many chunks a piece of a sequence has that is walked beside others, 0 where sequences are walked whole: the least of an estimated time.  The estimate's unit is such that a chunk of a
// walk of 128-wide keys in bf16 takes 3.8 (5.5 us measured), of a piece and its map 5.5 together, both where a compute unit has one block; each more takes 2 a chunk of each pass; the two passes
// begin with another chunk's time and 4; a piece in the join takes 2.7.  Narrower keys take less of it, by 64 the share of 0.78, wider ones and fp32 more (1.45; 1.75, of wide keys, which spill, 3).
// Lengths that are not known here are taken to be those that points cut at random out of T: the longest is 0.6 + ln n times their mean, and nothing is left idle at the end of a round
// of blocks.  Measured, us, whole and in pieces: 16384 tokens of 16 heads of 128 x 128 in one sequence 1400 and 375, of 4 heads 1275 and 200, 1000 tokens of 8 heads 92 and 58, in fp32 of 4 heads of
// 256 x 256 335 and 158; 24 prompts of 2 to 2000 tokens, 16 heads of 64 x 128, 253 and 250; forward and backward of 5 prompts in 1501 tokens, 6 heads of 40 x 56 in fp32, 189 and 133.  Whole, as it
// should be: 8 sequences of 1024 tokens, 8 heads, forward and backward 345 and 361; 64 prompts of 256 tokens at the mean 185 and 204.  Of 29 sizes of both types the choice took 5 % more than the
// best of 17 lengths in the geometric mean, and where it is furthest off, 900 tokens in 3 sequences of 6 heads of 64 x 64, 57 for 38.
int piece_of(const gdelta_desc *d, const GdLayout &l, bool packed)
{
    const char *const forced = tune_env("DWCONV_TUNE_GDELTA_PIECE");
    if (forced) return atoi(forced) > 0 ? (int)fmin(atoi(forced), 1 << 24) : 0;      // (a piece's tokens are counted in 32 bits)
    const bool ragged = packed && d->sequences > 1;
    const double n = d->sequences, chunks = ceil((double)d->T / (n * TOKENS)), longest = ragged ? chunks * (0.6 + log(n)) : chunks, units = 256;
    const double columns = (double)((l.VP + 63) / 64), all = columns + (double)((l.KP + 63) / 64), join = 0.3 + 2.4 * l.KP / 128.0;
    const double work = (0.55 + 0.45 * l.KP / 128.0) * (d->dtype != DWCONV_F32 ? 1 : l.KP > 128 ? 3 : 1.75);
    auto more = [&](double blocks, double each, double part) {       // chunks' times of a pass beyond those of a block alone
        return ragged ? 1.3 * fmax(0, blocks * each * part / units - each) : 2 * each * (ceil(blocks / units) - 1);
    };
    double best = 0.92 * work * (3.8 * longest + more(n * d->H * columns * chunks / longest, longest, 1));
    int piece = 0;
    for (long long p = 1; 2 * p <= longest; p = p < 16 ? p + 1 : p * 5 / 4) {
        const double mapped = ragged ? (1 + p / chunks) * exp(-p / chunks) : 1, blocks = n * (ragged ? chunks / p : ceil(chunks / p)) * d->H;
        const double us = work * (5.5 * (p + 1) + more(blocks * all, p + (ragged ? 1. : 0.), mapped) + more(blocks * columns, p + (ragged ? 1. : 0.), 1)) + join * ceil(longest / p) + 4;
        if (us < best) {
            best = us;
            piece = (int)p;
        }
    }
    return piece;
}

}  // namespace

GdLayout gdelta_layout(const gdelta_desc *d, bool packed)
{
    GdLayout l = {};
    const long long length = d->T / d->sequences;
    l.chunks = d->T == 0 ? 0 : packed ? d->T / TOKENS + d->sequences : d->sequences * ((length + TOKENS - 1) / TOKENS);
    l.KP = d->K <= 32 ? 32 : d->K <= 64 ? 64 : d->K <= 128 ? 128 : 256;
    l.VP = cdiv(d->V, 32) * 32;
    l.matrix = 3 * 384 * 16;                      // (INNER * MATRIX_PIECES)
    l.vectors = 9 * TOKENS * 4;
    l.state = (long long)l.KP * l.VP * 4;
    l.rows = TOKENS * l.VP * 4;
    l.piece = d->T == 0 ? 0 : piece_of(d, l, packed);
    l.map = (long long)l.KP * l.KP * 4;
    const long long unit = l.piece * TOKENS;
    l.pieces = !l.piece ? 0 : packed ? d->T / unit + d->sequences : d->sequences * ((length + unit - 1) / unit);
    return l;
}

}  // namespace dwc

using namespace dwc;

extern "C" {

// (the layouts of sequences of equal and of other lengths differ)
size_t gdelta_kept_bytes(const gdelta_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    const size_t a = kept_bytes(desc, gdelta_layout(desc, false)), b = kept_bytes(desc, gdelta_layout(desc, true));
    return a > b ? a : b;
}

size_t gdelta_fwd_workspace_bytes(const gdelta_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    const size_t a = forward_bytes(desc, gdelta_layout(desc, false)), b = forward_bytes(desc, gdelta_layout(desc, true));
    return a > b ? a : b;
}

size_t gdelta_bwd_workspace_bytes(const gdelta_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    const size_t a = backward_bytes(desc, gdelta_layout(desc, false)), b = backward_bytes(desc, gdelta_layout(desc, true));
    return a > b ? a : b;
}

static int check_tensors(const gdelta_desc *d, const gdelta_tensors *t, std::initializer_list<const void *> stored, std::initializer_list<const void *> others)
{
    if (!t) return DWCONV_ERR_NULL;
    if (d->T > 0)
        for (const void *p : stored)
            if (!p) return DWCONV_ERR_NULL;
    for (const void *p : stored)
        if (unaligned_to(p, d->dtype)) return DWCONV_ERR_ALIGN;
    for (const void *p : others)
        if (unaligned4(p)) return DWCONV_ERR_ALIGN;
    return DWCONV_OK;
}

int gdelta_fwd(const gdelta_desc *desc, const gdelta_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t) return DWCONV_ERR_NULL;
    rc = check_tensors(desc, t, {t->q, t->k, t->v, t->a, t->b, t->y}, {t->A, t->a_bias, t->starts, t->init, t->final});
    if (rc != DWCONV_OK) return rc;
    if (!t->starts && desc->T % desc->sequences) return DWCONV_ERR_BAD_DIM;
    const GdLayout l = gdelta_layout(desc, t->starts != nullptr);
    GdSpace s = {};
    if (t->kept) {
        if (unaligned16(t->kept)) return DWCONV_ERR_ALIGN;
        place_kept(desc, l, t->kept, &s);
    } else if (l.chunks) {
        if (!workspace || workspace_bytes < gdelta_fwd_workspace_bytes(desc)) return DWCONV_ERR_WORKSPACE;
        if (unaligned16(workspace)) return DWCONV_ERR_ALIGN;
        place_forward(desc, l, (char *)workspace, &s);
    }
    if (desc->T == 0 && !t->final) return DWCONV_OK;
    const GdArgs g = args_of(desc, t);
    hipError_t e = hipSuccess;
    if (desc->T > 0) e = launch_gdelta_prep(desc->dtype, g, l, s, (hipStream_t)stream);
    if (e == hipSuccess) e = launch_gdelta_fwd(desc->dtype, g, l, s, (const float *)t->init, t->y, (float *)t->final, (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

int gdelta_bwd(const gdelta_desc *desc, const gdelta_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t) return DWCONV_ERR_NULL;
    rc = check_tensors(desc, t, {t->q, t->k, t->v, t->a, t->b, t->dy, t->dq, t->dk, t->dv, t->da, t->db}, {t->A, t->a_bias, t->starts, t->dA, t->da_bias});
    if (rc != DWCONV_OK) return rc;
    if (desc->T > 0 && !t->kept) return DWCONV_ERR_NULL;
    if (!t->starts && desc->T % desc->sequences) return DWCONV_ERR_BAD_DIM;
    const GdLayout l = gdelta_layout(desc, t->starts != nullptr);
    if (l.chunks) {
        if (!workspace || workspace_bytes < gdelta_bwd_workspace_bytes(desc)) return DWCONV_ERR_WORKSPACE;
        if (unaligned16(workspace) || unaligned16(t->kept)) return DWCONV_ERR_ALIGN;
    }
    GdSpace s = {};
    place_kept(desc, l, t->kept, &s);
    s.dS = (float *)workspace;
    s.X = (float *)((char *)workspace + l.chunks * desc->H * l.state);
    s.ends = (float *)((char *)s.X + l.chunks * desc->H * l.rows);
    s.partials = (float *)((char *)s.ends + l.pieces * desc->H * l.state);
    const GdArgs g = args_of(desc, t);
    hipError_t e = hipSuccess;
    if (desc->T > 0) {
        e = launch_gdelta_bwd_states(desc->dtype, g, l, s, t->dy, t->dv, (hipStream_t)stream);
        if (e == hipSuccess) e = launch_gdelta_bwd_rows(desc->dtype, g, l, s, t->dy, t->dq, t->dk, t->da, t->db, (hipStream_t)stream);
    }
    if (e == hipSuccess && (t->dA || t->da_bias))
        e = launch_sum_partials(s.partials, (int)l.chunks, desc->H, 2ll * desc->H, 2ll * desc->H, (float *)t->dA, (float *)t->da_bias, nullptr, (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

int gdelta_step(const gdelta_desc *desc, const gdelta_tensors *t, void *stream)
{
    int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t) return DWCONV_ERR_NULL;
    rc = check_tensors(desc, t, {t->q, t->k, t->v, t->a, t->b, t->y}, {t->A, t->a_bias, t->slots, t->state});
    if (rc != DWCONV_OK) return rc;
    if (desc->T == 0) return DWCONV_OK;
    if (!t->state) return DWCONV_ERR_NULL;
    if (!t->slots && desc->T > desc->sequences) return DWCONV_ERR_BAD_DIM;
    GdArgs g = args_of(desc, t);
    g.starts = nullptr;
    const hipError_t e = launch_gdelta_step(desc->dtype, g, (const int32_t *)t->slots, (float *)t->state, t->y, (hipStream_t)stream);
    return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH;
}

}  // extern "C"
