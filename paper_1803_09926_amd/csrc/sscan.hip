// Entry points of the selective state space scan: checks of arguments, how a launch is split, workspaces.
#include "sscan.hpp"
#include "tune.hpp"
#include <stdlib.h>

namespace dwc {

namespace {

int validate(const sscan_desc *d)
{
    if (!d) return DWCONV_ERR_NULL;
    if (d->dtype != DWCONV_F32 && d->dtype != DWCONV_BF16) return DWCONV_ERR_BAD_ENUM;
    if ((d->softplus != 0 && d->softplus != 1) || d->reserved != 0) return DWCONV_ERR_BAD_ENUM;
    if (d->T < 0 || d->C < 1 || d->N < 1 || d->groups < 1 || d->sequences < 1 || d->C % d->groups) return DWCONV_ERR_BAD_DIM;
    if (d->N > SSCAN_MAX_N) return DWCONV_ERR_UNSUPPORTED;
    if (d->T > SEQOPS_MAX_T || d->sequences > SEQOPS_MAX_T || d->C > SEQOPS_MAX_C) return DWCONV_ERR_TOO_LARGE;
    const long long shared = (long long)d->groups * d->N;
    if (d->T > 1) {
        for (const int64_t s : {d->x_stride, d->dt_stride, d->z_stride, d->y_stride})
            if (s < d->C) return DWCONV_ERR_BAD_DIM;
        if (d->b_stride < shared || d->c_stride < shared) return DWCONV_ERR_BAD_DIM;
    }
    for (const int64_t s : {d->x_stride, d->dt_stride, d->z_stride, d->y_stride, d->b_stride, d->c_stride})
        if (s > SEQOPS_MAX_STRIDE) return DWCONV_ERR_TOO_LARGE;
    return DWCONV_OK;
}

// 16-byte multiples, so that what follows is aligned
size_t floats(size_t n) { return (n + 3) / 4 * 4; }

// A block of the last part reads the states of all before it, so the parts of a launch are capped: at most 24, 32, 48, 64, 80 of them take 212, 163, 141, 132, 131 us
// forward at 16384 x 1024, where never more than 80 are asked for.  With fewer channels the cap leaves compute units idle: 32768 tokens of 64, 256, 512 channels
// (16 states) in one sequence take 119, 138, 168 us forward with 80 parts and 82, 105, 147 with 160, both ways 318, 394, 540 and 210, 315, 473; in 64
// sequences 110, 131, 159 and, with 320 parts, 44, 74, 121.
constexpr int MOST_PARTS = 80;
// A part is a whole number of tiles, one at the least: parts of 16, 32, 64, 112 tokens take 15.9, 17.5, 24.2, 35.7 us forward at 301 x 1024; both ways at 1501 x 728
// those of 32 tokens, the least that the cap allows there, 64 and 128 take 73, 88, 134 us, and of 16 with a cap of 95 78.
constexpr int PART_UNIT = KEPT_EVERY;

// One at the least: launches are divided by these numbers.
int tuned(const char *name, int otherwise)
{
    const char *v = tune_env(name);
    const int n = v ? atoi(v) : otherwise;
    return n > 1 ? n : 1;
}

// `want` blocks fill the card: five on each of 256 compute units forward (512, 768, 1024, 1280 of them 162, 141, 132.5, 131.5 us at 16384 x 1024, and 512, 768, 1024,
// 1280, 2048 303, 256, 240, 228, 223 at 16383 x 2048), three turns of two backward (504, 960, 1536, 1920: 343, 337, 320, 325 us both ways at 8192 x 1536).
// Where whole sequences of equal lengths give at least half of them, a part is one or more of these, and nothing has to be carried from part to part; otherwise
// the tokens are split wherever it may be.
ScanPlan plan(const sscan_desc *d, bool packed, int want)
{
    ScanPlan p;
    p.lanes = state_lanes(d->N);
    p.channel_blocks = d->groups * cdiv(d->C / d->groups, 256 / p.lanes);
    p.part = d->T > 0 ? d->T : 1;
    p.parts = 1;
    p.carry = false;
    const int length = d->T / d->sequences;
    const long long all = (long long)p.channel_blocks * d->sequences;
    if (!packed && d->sequences > 1 && length > 0 && length % PART_UNIT == 0 && all >= want / 2) {
        const long long together = all / (2 * want) > 1 ? all / (2 * want) : 1;     // at most about twice what fills the card
        p.part = (int)(together * length < d->T ? together * length : d->T);
        p.parts = cdiv(d->T, p.part);
        return p;
    }
    int parts = cdiv(want, p.channel_blocks);
    const int most = tuned("DWCONV_TUNE_SSCAN_MOST_PARTS", MOST_PARTS);
    if (parts > most) parts = most;
    if (parts > 1) {
        p.part = cdiv(cdiv(d->T > 0 ? d->T : 1, parts), PART_UNIT) * PART_UNIT;
        p.parts = d->T > 0 ? cdiv(d->T, p.part) : 1;
        p.carry = p.parts > 1;
    }
    return p;
}

}  // namespace

ScanPlan plan_sscan_fwd(const sscan_desc *d, bool packed)
{
    return plan(d, packed, tuned("DWCONV_TUNE_SSCAN_FWD_BLOCKS", 1280));
}
ScanPlan plan_sscan_bwd(const sscan_desc *d, bool packed)
{
    return plan(d, packed, tuned("DWCONV_TUNE_SSCAN_BWD_BLOCKS", 1536));
}

Scan sscan_geometry(const sscan_desc *d, const ScanPlan &p, const void *starts)
{
    Scan g;
    g.C = d->C; g.N = d->N; g.groups = d->groups; g.per_group = d->C / d->groups;
    g.blocks_of_group = p.channel_blocks / d->groups;
    g.copies = 1;
    while (2 * g.copies * d->N <= 4 * p.lanes) g.copies *= 2;
    g.twice = 4 * p.lanes / g.copies - d->N;
    g.share = 1.f / (float)g.copies;
    g.by_n = cdiv(1 << 16, d->N);
    g.by_twice = g.twice ? cdiv(1 << 16, g.twice) : 0;
    g.softplus = d->softplus; g.part = p.part; g.parts = p.parts;
    g.xs = d->x_stride; g.dts = d->dt_stride; g.zs = d->z_stride; g.bs = d->b_stride; g.cs = d->c_stride; g.ys = d->y_stride;
    g.seq = {(const int32_t *)starts, d->sequences, d->T / d->sequences, d->T};
    return g;
}

FwdSpace sscan_fwd_space(const sscan_desc *d, const ScanPlan &p)
{
    FwdSpace s = {0, 0, 0};
    if (!p.carry) return s;
    s.sums = (size_t)p.parts * d->C * 4 * p.lanes;
    s.total = s.sums + floats((size_t)p.parts * d->C);
    return s;
}

BwdSpace sscan_bwd_space(const sscan_desc *d, const ScanPlan &p)
{
    BwdSpace s = {0, 0, 0, 0, 0};
    if (d->T == 0) return s;
    if (p.carry) {
        s.sums = (size_t)p.parts * d->C * 4 * p.lanes;
        s.dA = s.sums + floats((size_t)p.parts * d->C);
    }
    s.shared = s.dA + floats((size_t)p.parts * ((size_t)d->C * d->N + 2 * (size_t)d->C));
    s.total = s.shared + (size_t)p.channel_blocks * d->T * 8 * p.lanes;
    return s;
}

}  // namespace dwc

using namespace dwc;

namespace {

int check_space(const void *workspace, size_t have, size_t need)
{
    if (!need) return DWCONV_OK;
    if (!workspace || have < need) return DWCONV_ERR_WORKSPACE;
    return unaligned16(workspace) ? DWCONV_ERR_ALIGN : DWCONV_OK;
}

int status(hipError_t e) { return e == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH; }

}  // namespace

extern "C" {

size_t sscan_kept_bytes(const sscan_desc *desc)
{
    if (validate(desc) != DWCONV_OK || desc->T == 0) return 0;
    return (size_t)cdiv(desc->T, KEPT_EVERY) * desc->C * 4 * state_lanes(desc->N) * sizeof(float);
}

size_t sscan_fwd_workspace_bytes(const sscan_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    // (with and without `starts`)
    const size_t equal = sscan_fwd_space(desc, plan_sscan_fwd(desc, false)).total, packed = sscan_fwd_space(desc, plan_sscan_fwd(desc, true)).total;
    return (equal > packed ? equal : packed) * sizeof(float);
}

size_t sscan_bwd_workspace_bytes(const sscan_desc *desc)
{
    if (validate(desc) != DWCONV_OK) return 0;
    const size_t equal = sscan_bwd_space(desc, plan_sscan_bwd(desc, false)).total, packed = sscan_bwd_space(desc, plan_sscan_bwd(desc, true)).total;
    return (equal > packed ? equal : packed) * sizeof(float);
}

int sscan_fwd(const sscan_desc *desc, const sscan_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || !t->A || (desc->T > 0 && (!t->x || !t->dt || !t->B || !t->C || !t->y))) return DWCONV_ERR_NULL;
    if (!t->starts && desc->T % desc->sequences) return DWCONV_ERR_BAD_DIM;
    for (const void *p : {t->x, t->dt, t->B, t->C, t->z, (const void *)t->y})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    for (const void *p : {t->A, t->D, t->dt_bias, t->starts, t->init, (const void *)t->final})
        if (unaligned4(p)) return DWCONV_ERR_ALIGN;
    if (unaligned16(t->kept)) return DWCONV_ERR_ALIGN;
    rc = check_space(workspace, workspace_bytes, sscan_fwd_workspace_bytes(desc));
    if (rc != DWCONV_OK) return rc;
    if (desc->T == 0 && !t->final) return DWCONV_OK;
    return status(launch_sscan_fwd(desc, t, (float *)workspace, (hipStream_t)stream));
}

int sscan_bwd(const sscan_desc *desc, const sscan_tensors *t, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || !t->A || !t->dA || (t->D && !t->dD)) return DWCONV_ERR_NULL;
    if (desc->T > 0 && (!t->x || !t->dt || !t->B || !t->C || !t->kept || !t->dy || !t->dx || !t->ddt || !t->dB || !t->dC || (t->z && !t->dz)))
        return DWCONV_ERR_NULL;
    if (!t->starts && desc->T % desc->sequences) return DWCONV_ERR_BAD_DIM;
    for (const void *p : {t->x, t->dt, t->B, t->C, t->z, t->dy, (const void *)t->dx, (const void *)t->ddt, (const void *)t->dB, (const void *)t->dC,
                          (const void *)t->dz})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    for (const void *p : {t->A, t->D, t->dt_bias, t->starts, t->init, (const void *)t->dA, (const void *)t->dD, (const void *)t->ddt_bias})
        if (unaligned4(p)) return DWCONV_ERR_ALIGN;
    if (unaligned16(t->kept)) return DWCONV_ERR_ALIGN;
    rc = check_space(workspace, workspace_bytes, sscan_bwd_workspace_bytes(desc));
    if (rc != DWCONV_OK) return rc;
    return status(launch_sscan_bwd(desc, t, (float *)workspace, (hipStream_t)stream));
}

int sscan_step(const sscan_desc *desc, const sscan_tensors *t, void *stream)
{
    const int rc = validate(desc);
    if (rc != DWCONV_OK) return rc;
    if (!t || (desc->T > 0 && (!t->x || !t->dt || !t->A || !t->B || !t->C || !t->y || !t->state))) return DWCONV_ERR_NULL;
    if (!t->slots && desc->T > desc->sequences) return DWCONV_ERR_BAD_DIM;
    for (const void *p : {t->x, t->dt, t->B, t->C, t->z, (const void *)t->y})
        if (unaligned_to(p, desc->dtype)) return DWCONV_ERR_ALIGN;
    for (const void *p : {t->A, t->D, t->dt_bias, t->slots, (const void *)t->state})
        if (unaligned4(p)) return DWCONV_ERR_ALIGN;
    if (desc->T == 0) return DWCONV_OK;
    return status(launch_sscan_step(desc, t, (hipStream_t)stream));
}

}  // extern "C"
