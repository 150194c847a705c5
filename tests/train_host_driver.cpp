// The host side of the cross entropy (csrc/dlf_ce.cpp, with the cuts of csrc/dlf_ffn.cpp) and of the optimizer (csrc/dlf_opt.cpp) with stand-ins for the
// launchers: random calls on addresses that nobody reads, each launch checked against what its kernels assume.  Usage: train_host_driver <seed>
// <calls>; prints what it saw, or the first fault.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <string>
#include <vector>

#include "../include/dlf_debug.h"
#include "../paper_2011_05630_amd/csrc/dlf_ce.h"
#include "../paper_2011_05630_amd/csrc/dlf_opt.h"

extern "C" hipError_t hipGetDevice(int* d)
{
    *d = 0;
    return hipSuccess;
}
static char g_error[512];
dlf_status dlf_set_error(dlf_status s, const char* msg)
{
    snprintf(g_error, sizeof g_error, "%s", msg);
    return s;
}

struct Region {
    uintptr_t lo, hi;
};
static struct Call {
    char text[512];
    uintptr_t ws = 0, ws_end = 0;
    std::map<std::string, Region> used;
    int launches = 0;
    int64_t rows_done = 0, dx_rows = 0, sums_out = 0, w_out = 0, packed = 0;
    const dlf_ce_desc* d = nullptr;
    const void *x, *w, *dx, *dw;
    const float *lse, *loss, *db, *dloss;
    const int64_t* target;
    bool kept = false, lse_given = false;
    std::vector<double> chunks;                              // of an optimizer's call: elements seen of each tensor
    int64_t parts = 0;
} g;
static std::map<std::string, long> g_seen;

#define NEED(C)                                                          \
    do {                                                                 \
        if (!(C)) {                                                      \
            printf("FAULT %s: %s (line %d)\n", g.text, #C, __LINE__);    \
            exit(1);                                                     \
        }                                                                \
    } while (0)

// A part of the workspace by what it is for: inside, and apart from the others.
static void use(const char* name, const void* p, double bytes)
{
    const uintptr_t lo = (uintptr_t)p;
    NEED(lo >= g.ws && lo <= g.ws_end && bytes <= (double)(g.ws_end - lo));
    Region r = {lo, lo + (uintptr_t)bytes};
    const auto have = g.used.find(name);
    if (have != g.used.end()) r = {std::min(r.lo, have->second.lo), std::max(r.hi, have->second.hi)};
    g.used[name] = r;
    for (const auto& o : g.used)
        if (o.first != name) NEED(r.hi <= o.second.lo || o.second.hi <= r.lo);
}
static bool in_ws(const void* p) { return (uintptr_t)p >= g.ws && (uintptr_t)p < g.ws_end; }
static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// An operand in whole lines: k of them exist in a row, or the row is filled up with zeros.
static bool lines(const void* p, int64_t ld, int64_t row, bool filled)
{
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && (filled || row % 8 == 0) && ld * 256 * 2 < ((int64_t)1 << 31);
}
static bool filled(const void* p) { return in_ws(p); }

static int64_t tiles(const DlfFfArgs& a, int shape, bool pt, bool qt)
{
    NEED(shape >= 0 && shape < DLF_FF_NUM_SHAPES && shape != DLF_FF_SHAPE_ANY64G);
    const DlfFfShape& s = DLF_FF_SHAPES[shape];
    NEED(a.nr > 0 && a.nc > 0 && a.nk >= 0 && a.problems == 1 && (a.segments == 1 || a.segments == 2) && a.splits >= 1);
    NEED(a.tiles_r == up(a.nr, s.br) && a.tiles_c == up(a.nc, s.bc));
    NEED(a.splits == 1 || up(a.nk, 64) * a.segments >= a.splits);
    for (int i = 0; i < a.segments; ++i) {
        NEED(a.nk == 0 || (a.p[i] && a.q[i]));
        if (shape == DLF_FF_SHAPE_256 || shape == DLF_FF_SHAPE_128 || shape == DLF_FF_SHAPE_128_DEEP)
            NEED(a.nk == 0 || (lines(a.p[i], a.ldp, pt ? a.nc : a.nk, filled(a.p[i])) && lines(a.q[i], a.ldq, qt ? a.nr : a.nk, filled(a.q[i]))));
        else
            NEED(a.ldp <= 1 << 24 && a.ldq <= 1 << 24);
    }
    const int64_t n = up((int64_t)a.tiles_r * a.tiles_c * a.splits, 8) * 8;
    NEED(n * 256 < (int64_t)1 << 32);
    if (a.splits > 1) {
        NEED(up((int64_t)a.nr * up(a.nc, 8), 256) * 256 < (int64_t)1 << 32);
        ++g_seen["split"];
    }
    return n;
}
static void given(const DlfCeGiven& v)
{
    NEED(v.one >= 0);
    if (v.one > 0) NEED(!v.dlse && (!v.dloss || v.dloss_stride == 0) && !v.unit);
    if (v.unit) {
        NEED(g.d->dtype == DLF_F16);
        use("unit", v.unit, 8);
    }
    if (g.d->dtype == DLF_F16) NEED(v.one > 0 || v.unit);
}
static void logits(const DlfCeArgs& a)
{
    const dlf_ce_desc& d = *g.d;
    const DlfFfArgs& t = a.t;
    NEED(t.nc == d.classes && t.nk == d.in_features && t.nr >= 1 && t.nr <= 65536 && a.ignore == d.ignore && a.ldz == up(d.classes, 8) * 8);
    const int64_t first = a.target - g.target;
    NEED(first >= 0 && first + t.nr <= d.rows);
    const int64_t xs = d.x_stride ? d.x_stride : d.in_features, wsd = d.w_stride ? d.w_stride : d.in_features;
    if (in_ws(t.q[0])) use("x", t.q[0], (double)t.nr * t.ldq * 2);
    else NEED(t.q[0] == (const char*)g.x + first * xs * 2 && t.ldq == xs);
    if (in_ws(t.p[0])) use("w", t.p[0], (double)t.nc * t.ldp * 2);
    else NEED(t.p[0] == g.w && t.ldp == wsd);
}
static void rest_low(const float* rest, const void* low, int64_t nr, int64_t ldz)
{
    use("rest", rest, (double)nr * 4);
    NEED((low != nullptr) == (g.d->rows <= DLF_FF_FEW_ROWS));
    if (low) use("low", low, (double)nr * ldz * 2);
}

extern "C" {
// (the feed-forward operators' own launchers are not reached)
int dlf_ff_kernels_init(void) { abort(); }
int dlf_ff_start_tile(const DlfFfArgs*, int, int, int, void*) { abort(); }
int dlf_ff_start_back(const DlfFfBackArgs*, int, int, void*) { abort(); }
int dlf_ff_start_few(const DlfFfArgs*, const DlfFfFew*, int, int, void*) { abort(); }
int dlf_ff_start_dz(const DlfFfDzArgs*, int, int, void*) { abort(); }

int dlf_ce_kernels_init(void) { return 0; }
int dlf_ce_start_pack(const DlfCePackArgs* a, void*)
{
    ++g.launches;
    ++g_seen["pack"];
    NEED(a->k == g.d->in_features && a->parts == up(a->k, 8) && a->m[0].rows + a->m[1].rows > 0);
    NEED(up((a->m[0].rows + a->m[1].rows) * a->parts, 256) * 256 < (int64_t)1 << 32);
    for (int i = 0; i < 2; ++i) {
        if (a->m[i].rows == 0) continue;
        use(i ? "w" : "x", a->m[i].to, (double)a->m[i].rows * a->parts * 16);
        NEED(!in_ws(a->m[i].from) && a->m[i].stride >= a->k);
        NEED(i == 0 || (a->m[i].rows == g.d->classes && a->m[i].from == g.w));
        if (i) ++g.packed;
    }
    return 0;
}
int dlf_ce_start_tile(const DlfCeArgs* a, int shape, int, int mode, void*)
{
    ++g.launches;
    ++g_seen["mode" + std::to_string(mode) + " shape" + std::to_string(shape)];
    logits(*a);
    NEED(a->t.splits == 1 && a->t.segments == 1);
    tiles(a->t, shape, false, false);
    const double nr = a->t.nr;
    if (mode == DLF_CE_DZ) {
        given(a->given);
        if (in_ws(a->lse)) {
            use("lse", a->lse, nr * 4);
            use("inverse", a->inverse, nr * 4);
        } else {
            NEED(a->lse - g.lse == a->target - g.target && !a->inverse);
        }
        rest_low(a->rest, a->low, a->t.nr, a->ldz);
        if (a->sums) use("sums", a->sums, 2.0 * a->t.tiles_r * a->t.nc * 4);
        NEED((a->sums != nullptr) == (g.db != nullptr));
        if (a->given.one > 0) use("unit", a->back, 4);
        use("dz", a->dz, nr * a->ldz * 2);
        g.rows_done += a->t.nr;
    } else {
        use("part", a->part, (double)up(a->t.nc, dlf_ce_width(shape)) * nr * 8);
        use("at", a->at, nr * 4);
        if (mode == DLF_CE_KEEP) use("dz", a->dz, nr * a->ldz * 2);
        if (mode == DLF_CE_LOGITS) use("z", a->z, nr * a->ldz * 4);
        NEED((mode == DLF_CE_LOGITS) == (a->z != nullptr));
        g.kept = mode == DLF_CE_KEEP || mode == DLF_CE_LOGITS;
        g.parts = up(a->t.nc, dlf_ce_width(shape));
    }
    return 0;
}
int dlf_ce_start_few(const DlfCeArgs* a, const DlfFfFew* c, int, void*)
{
    ++g.launches;
    ++g_seen[c->rows ? "few lines" : "few"];
    logits(*a);
    NEED(a->t.nr <= DLF_FF_FEW_ROWS);
    NEED((c->nf == 1 || (c->nf == 2 && c->mr == 2)) && (c->mr == 1 || c->mr == 2));
    NEED(c->waves == 1 || c->waves == 2 || c->waves == 4 || c->waves == 8);
    if (c->rows) NEED(lines(a->t.p[0], a->t.ldp, a->t.nk, false) && lines(a->t.q[0], a->t.ldq, a->t.nk, false));
    NEED(DLF_FF_ROWS_LDS(c->waves, c->nf, c->mr, 0) <= 160 * 1024);
    use("part", a->part, (double)up(a->t.nc, 16) * a->t.nr * 8);
    use("at", a->at, (double)a->t.nr * 4);
    if (a->z) use("z", a->z, (double)a->t.nr * a->ldz * 4);
    g.kept = a->z != nullptr;
    g.parts = up(a->t.nc, 16);
    return 0;
}
int dlf_ce_start_dz_sums(const DlfCeDzArgs* a, int, void*)
{
    ++g.launches;
    const bool few = !a->sums || !in_ws(a->sums);            // (a forced kernel: few rows on tiles)
    ++g_seen[few ? "dz few" : "dz sums"];
    NEED(g.kept && a->nr >= 1 && a->nr <= 65536 && a->target - g.target + a->nr <= g.d->rows && a->nc == g.d->classes && a->ldz == up(a->nc, 8) * 8);
    NEED(up(a->ldz, 256) * up(a->nr, DLF_CE_DZ_ROWS) * 512 < (int64_t)1 << 32);
    given(a->given);
    use("z", a->z, (double)a->nr * a->ldz * 4);
    use("dz", a->dz, (double)a->nr * a->ldz * 2);
    if (!a->lse) {
        ++g_seen[few ? "dz few with lse" : "dz sums with lse"];
        NEED(!g.lse_given && !a->inverse && a->parts == g.parts && a->loss - g.loss == a->target - g.target);
        use("part", a->part, (double)a->parts * a->nr * 8);
        use("at", a->at, (double)a->nr * 4);
    } else if (in_ws(a->lse)) {
        use("lse", a->lse, (double)a->nr * 4);
        use("inverse", a->inverse, (double)a->nr * 4);
    } else {
        NEED(a->lse == g.lse && !a->inverse);
    }
    rest_low(a->rest, a->low, a->nr, a->ldz);
    if (few) {
        NEED(a->low && a->nr == g.d->rows && a->sums == g.db);
        if (a->sums) ++g.sums_out;
    } else {
        NEED(g.db && !g.lse_given);
        use("sums", a->sums, (double)up(a->nr, DLF_CE_DZ_ROWS) * a->nc * 4);
    }
    if (a->given.one > 0) use("unit", a->back, 4);
    g.rows_done += a->nr;
    g.kept = false;
    return 0;
}
int dlf_ce_start_join(const DlfCeJoinArgs* a, void*)
{
    ++g.launches;
    ++g_seen["join"];
    NEED(a->parts == g.parts && a->nc == g.d->classes && a->nr >= 1);
    use("part", a->part, (double)a->parts * a->nr * 8);
    use("at", a->at, (double)a->nr * 4);
    if (a->lse && in_ws(a->lse)) use("lse", a->lse, (double)a->nr * 4);
    if (a->inverse) use("inverse", a->inverse, (double)a->nr * 4);
    NEED(!a->inverse || in_ws(a->lse));
    NEED(a->loss - g.loss == a->target - g.target);
    return 0;
}
int dlf_ce_start_dz(const DlfCeDzArgs* a, int, void*)
{
    ++g.launches;
    ++g_seen[a->z ? "dz of logits" : a->lse ? "dz" : "dz with lse"];
    if (a->z) {
        NEED(!a->lse && g.d->rows <= DLF_FF_FEW_ROWS);
        use("z", a->z, (double)a->nr * a->ldz * 4);
    }
    NEED(g.kept && a->parts == g.parts && a->parts == up(a->nc, a->width) && (a->width & (a->width - 1)) == 0 && a->nc == g.d->classes);
    NEED(a->slices == up(a->ldz, DLF_CE_DZ_COLS) && (int64_t)a->nr * a->slices * 256 < (int64_t)1 << 32);
    given(a->given);
    use("part", a->part, (double)a->parts * a->nr * 8);
    use("at", a->at, (double)a->nr * 4);
    use("dz", a->dz, (double)a->nr * a->ldz * 2);
    if (a->lse) use("lse", a->lse, (double)a->nr * 4);
    NEED(a->loss - g.loss == a->target - g.target);
    rest_low(a->rest, a->low, a->nr, a->ldz);
    if (a->given.one > 0) use("unit", a->back, 4);
    g.rows_done += a->nr;
    g.kept = false;
    return 0;
}
int dlf_ce_start_unit(const DlfCeUnitArgs* a, void*)
{
    ++g.launches;
    ++g_seen["unit"];
    NEED(g.d->dtype == DLF_F16 && a->rows == g.d->rows && !a->given.unit);
    use("unit", a->unit, 8);
    return 0;
}
int dlf_ce_start_back(const DlfCeBackArgs* e, int shape, int, void*)
{
    ++g.launches;
    ++g_seen["back shape" + std::to_string(shape)];
    const DlfFfBackArgs& b = e->b;
    const int64_t ldz = up(g.d->classes, 8) * 8, k = g.d->in_features;
    int64_t n = b.sum.blocks;
    double joined = 0;
    if (b.w.problems > 0) {
        n += tiles(b.w, shape, true, true);
        NEED(b.w.nr == g.d->classes && b.w.nc == k && b.w.ldq == ldz && b.w.out[0] == g.dw && b.w.ldo == k);
        if (b.w.nk > 0) use("dz", b.w.q[0], (double)b.w.nk * ldz * 2);
        if (b.w.segments == 2) use("low", b.w.q[1], (double)b.w.nk * ldz * 2);
        if (e->sum) use("sum", e->sum, (double)b.w.nr * k * 4);
        NEED((e->add || e->keep) == (e->sum != nullptr));
        if (!e->keep) ++g.w_out;
        if (b.w.splits > 1) {
            use("join", b.w.part, (double)b.w.splits * b.w.nr * b.w.nc * 4);
            joined += std::ceil((double)b.w.nr * up(b.w.nc, 8) / 256) * 256;
        }
    }
    if (b.x.problems > 0) {
        n += tiles(b.x, shape, true, false);
        NEED(b.x.nc == k && b.x.nk == g.d->classes && b.x.ldq == ldz && b.x.ldo == k);
        NEED(b.x.out[0] == (const char*)g.dx + g.dx_rows * k * 2);
        use("dz", b.x.q[0], (double)b.x.nr * ldz * 2);
        use("rest", e->rest, (double)b.x.nr * 4);
        NEED(e->target - g.target == g.dx_rows);
        g.dx_rows += b.x.nr;
        if (b.x.splits > 1) {
            use(b.w.problems > 0 && b.w.splits > 1 ? "join x" : "join", b.x.part, (double)b.x.splits * b.x.nr * b.x.nc * 4);
            joined += std::ceil((double)b.x.nr * up(b.x.nc, 8) / 256) * 256;
        }
    }
    g.used.erase("join");                                    // (written and read within the call, by each piece anew)
    g.used.erase("join x");
    NEED(n > 0 && n * 256 < (int64_t)1 << 32 && joined < (double)((int64_t)1 << 32));
    if (b.sum.blocks > 0) {
        NEED(b.sum.n == g.d->classes && b.sum.blocks == up(b.sum.n, 64) && b.sum.part[0]);
        if (b.sum.chunks > 0) use("sums", b.sum.part[0], (double)b.sum.chunks * b.sum.n * 4);
        if (b.sum.out[0] == g.db) ++g.sums_out;
        else use("sums", b.sum.out[0], (double)b.sum.n * 4);
    }
    if (e->back) use("unit", e->back, 4);
    else NEED(g.d->rows == 0 || (g.d->dtype == DLF_BF16 && g.dloss));
    return 0;
}

int dlf_opt_start_norm(const DlfNormArgs* a, int groups, void*)
{
    ++g.launches;
    ++g_seen["norm"];
    NEED(a->tensors >= 1 && a->tensors <= DLF_OPT_NORM_TENSORS && a->chunks >= 1 && groups >= 1 && groups <= DLF_OPT_GROUPS && groups <= a->chunks);
    int64_t at = 0;
    for (int i = 0; i < a->tensors; ++i) {
        NEED(a->g[i] && a->n[i] > 0 && a->first[i] == at && a->type[i] <= 2);
        at += up(a->n[i], DLF_OPT_CHUNK);
        g.chunks.push_back((double)a->n[i]);
    }
    NEED(at == a->chunks);
    use(("part" + std::to_string(g.launches)).c_str(), a->part, 8.0 * groups);
    g.parts += groups;
    return 0;
}
int dlf_opt_start_norm_join(const DlfNormJoinArgs* a, void*)
{
    ++g.launches;
    NEED(a->parts == g.parts);
    if (a->parts > 0) NEED((uintptr_t)a->part == g.ws && a->parts * 8.0 <= (double)(g.ws_end - g.ws));
    return 0;
}
static std::vector<DlfOptChunk> g_table;                     // what dlf_adamw_table has filled, at the table's address
static uintptr_t g_table_at;
int dlf_opt_start_step(const DlfStepArgs* a, int small, int groups, void*)
{
    ++g.launches;
    ++g_seen[small ? "step small" : "step"];
    NEED(a->chunks >= 0 && groups >= 1 && groups <= DLF_OPT_GROUPS && (groups <= a->chunks || groups == 1));
    const int64_t first = (int64_t)((uintptr_t)a->table - g_table_at) / (int64_t)sizeof(DlfOptChunk);
    NEED(first >= 0 && first + a->chunks <= (int64_t)g_table.size());
    for (int64_t i = first; i < first + a->chunks; ++i) {
        const DlfOptChunk& c = g_table[i];
        const int t = c.tensor - a->first_tensor;
        NEED(t >= 0 && t < DLF_OPT_STEP_TENSORS && c.n >= 1 && c.n <= DLF_OPT_CHUNK && c.at % DLF_OPT_CHUNK == 0 && c.state % DLF_ADAMW_BLOCK == 0);
        NEED(a->g[t] == nullptr || (uintptr_t)a->g[t] == ((uintptr_t)1 << 45) + (uintptr_t)c.tensor * 4096);
        NEED(a->type[t] <= 2);
        g.chunks[c.tensor] += c.n;
    }
    NEED((small != 0) == (a->m_scale != nullptr));
    g.parts += a->last;
    return 0;
}
}

static std::mt19937_64 rng;
static int64_t pick(int64_t lo, int64_t hi)
{
    std::uniform_real_distribution<double> u(std::log((double)lo), std::log((double)hi + 0.49));
    const int64_t v = std::min(hi, std::max(lo, (int64_t)std::llround(std::exp(u(rng)))));
    const int64_t unit = rng() % 2 ? 1 : rng() % 2 ? 8 : 64;
    return std::max(lo, v / unit * unit);
}
static int64_t stride(int64_t row)
{
    switch (rng() % 8) {
    case 0: return row + (int64_t)(rng() % 9);
    case 1: return std::max(row, (int64_t)(rng() % ((1 << 24) + 3)));
    case 2: return row + 8 * (int64_t)(rng() % 9);
    case 3: return std::max<int64_t>(row, (1 << 22) - 8 + 8 * (int64_t)(rng() % 3));
    default: return rng() % 2 ? 0 : row;
    }
}
static void* place(int64_t i, int align) { return (void*)(((uintptr_t)1 << 40) + (uintptr_t)i * ((uintptr_t)1 << 46) / 16 + (rng() % 3 ? 0 : rng() % 32 * align)); }

static dlf_status entropy(int c)
{
    dlf_ce_desc d;
    memset(&d, 0, sizeof d);
    const int what = (int)(rng() % 3);
    d.dtype = (int)(rng() % 2);
    d.rows = rng() % 40 == 0 ? 0 : pick(1, rng() % 3 ? 8192 : 1 << 20);
    d.in_features = (int)pick(1, rng() % 4 ? 12000 : 1 << 20);
    d.classes = (int)pick(1, rng() % 4 ? 140000 : 1 << 20);
    d.dbias = (int)(rng() % 2);
    d.ignore = -100;
    d.x_stride = stride(d.in_features);
    d.w_stride = stride(d.in_features);
    d.piece_bytes = rng() % 2 ? 0 : pick(1, (int64_t)1 << 32);
    const bool forced = rng() % 3 == 0;
    dlf_debug_ff_kernel(forced ? (int)(rng() % (2 + DLF_FF_NUM_SHAPES)) : 0, forced && rng() % 2 ? 1 + (int)(rng() % 16) : 0);
    g = Call();
    snprintf(g.text, sizeof g.text, "call %d what %d dtype %d rows %lld in %d classes %d strides %lld %lld piece %lld", c, what, d.dtype, (long long)d.rows,
             d.in_features, d.classes, (long long)d.x_stride, (long long)d.w_stride, (long long)d.piece_bytes);
    const size_t need = what == 0 ? dlf_cross_entropy_workspace_bytes(&d) : what == 1 ? dlf_cross_entropy_backward_workspace_bytes(&d)
                                                                                      : dlf_cross_entropy_gradients_workspace_bytes(&d);
    const bool refused = need == SIZE_MAX;
    const int some = (int)(rng() % 64);
    void *x = place(0, 2), *w = place(1, 2), *dx = place(2, 2), *dw = place(3, 2), *ws = (void*)((uintptr_t)1 << 47);
    float *bias = (float*)place(4, 4), *lse = (float*)place(5, 4), *loss = (float*)place(6, 4), *db = (float*)place(7, 4), *dloss = (float*)place(8, 4),
          *dlse = (float*)place(9, 4);
    int64_t* target = (int64_t*)place(10, 8);
    g.ws = (uintptr_t)ws;
    g.ws_end = g.ws + (refused ? 0 : need);
    g.d = &d;
    g.x = x; g.w = w; g.lse = lse; g.loss = loss; g.target = target;
    g.dx = some & 1 ? dx : nullptr;
    g.dw = some & 2 ? dw : nullptr;
    g.db = some & 4 && (what == 1 || d.dbias) ? db : nullptr;
    g.lse_given = what == 1;
    g.dloss = some & 8 ? dloss : nullptr;
    const int64_t ls = some & 16 ? 1 : 0;
    const float* const b = some & 32 ? bias : nullptr;
    g_error[0] = 0;
    auto call = [&](size_t have) {
        return what == 0   ? dlf_cross_entropy(&d, x, w, b, target, loss, some & 1 ? lse : nullptr, ws, have, nullptr)
               : what == 1 ? dlf_cross_entropy_backward(&d, x, w, b, target, lse, g.dloss, ls, 1.0f, some & 4 ? dlse : nullptr, ls, (void*)g.dx, (void*)g.dw,
                                                        (float*)g.db, ws, have, nullptr)
                           : dlf_cross_entropy_gradients(&d, x, w, b, target, g.dloss, ls, 1.0f, loss, (void*)g.dx, (void*)g.dw, (float*)g.db, ws, have, nullptr);
    };
    if (what == 1 && (some & 4)) g.dloss = dloss;            // (for the check of what scales the products)
    const dlf_status s = call(refused ? 0 : need);
    NEED((s != DLF_OK) == refused && (s == DLF_OK) == (g_error[0] == 0));
    NEED(s == DLF_OK || g.launches == 0);
    if (s == DLF_OK) {
        if (what > 0) {
            const bool any = g.dx || g.dw || g.db;
            NEED(g.rows_done == (any ? d.rows : 0) && g.dx_rows == (g.dx ? d.rows : 0));
            NEED(g.w_out == (g.dw ? 1 : 0) && g.sums_out == (g.db ? 1 : 0));
        }
        NEED(g.packed <= 1);
        if (need > 0 && g.launches > 0) {
            g.launches = 0;
            NEED(call(need - 1) == DLF_ERR_OOM && g.launches == 0);
        }
    }
    return s;
}

static dlf_status optimizer(int c)
{
    g = Call();
    const int n = (int)pick(1, 1200);
    std::vector<int64_t> counts;
    std::vector<const void*> grads;
    std::vector<int32_t> types;
    std::vector<dlf_adamw_tensor> tensors;
    for (int i = 0; i < n; ++i) {
        counts.push_back(rng() % 10 == 0 ? 0 : pick(1, 200000));
        grads.push_back((const void*)(((uintptr_t)1 << 45) + (uintptr_t)i * 4096));
        types.push_back((int)(rng() % 3));
        tensors.push_back({(void*)(((uintptr_t)1 << 44) + (uintptr_t)i * (1 << 22)), nullptr, counts[i], types[i], 0, 0.0f, 0});
    }
    snprintf(g.text, sizeof g.text, "call %d optimizer %d tensors", c, n);
    if (rng() % 2) {
        const size_t need = dlf_gradient_norm_workspace_bytes(counts.data(), n);
        NEED(need != SIZE_MAX);
        g.ws = (uintptr_t)1 << 47;
        g.ws_end = g.ws + need;
        float out[2];
        const dlf_status s = dlf_gradient_norm(grads.data(), counts.data(), types.data(), n, 1.0f, 1.0f, out, out + 1, (void*)g.ws, need, nullptr);
        size_t k = 0;
        for (int i = 0; i < n; ++i)
            if (counts[i] > 0) NEED(k < g.chunks.size() && g.chunks[k++] == (double)counts[i]);
        NEED(k == g.chunks.size());
        return s;
    }
    const size_t bytes = dlf_adamw_table_bytes(tensors.data(), n);
    g_table.assign(bytes / sizeof(DlfOptChunk), DlfOptChunk());
    NEED(bytes == g_table.size() * sizeof(DlfOptChunk) && dlf_adamw_table(tensors.data(), n, g_table.data(), bytes) == DLF_OK);
    g_table_at = (uintptr_t)1 << 46;
    for (int i = 0; i < n; ++i)
        if (rng() % 20 == 0) grads[i] = nullptr;
    g.chunks.assign((size_t)n, 0.0);
    const bool small = rng() % 2;
    const dlf_adamw_desc d = {0.9, 0.95, 1e-8f, 1, small ? DLF_ADAMW_8BIT : DLF_ADAMW_FP32, 0};
    float* const f = (float*)((uintptr_t)1 << 43);
    const dlf_status s = dlf_adamw_step(&d, tensors.data(), n, (const void*)g_table_at, grads.data(), types.data(), f, f, small ? f : nullptr, small ? f : nullptr,
                                        (double*)f, 0.1f, nullptr, nullptr, nullptr);
    for (int i = 0; i < n; ++i) NEED(g.chunks[i] == (double)counts[i]);
    NEED(g.parts == 1);                                      // one launch counts the step
    return s;
}

int main(int argc, char** argv)
{
    rng.seed(argc > 1 ? strtoull(argv[1], nullptr, 10) : 1);
    const int calls = argc > 2 ? atoi(argv[2]) : 1000;
    int status[16] = {0};
    for (int c = 0; c < calls; ++c) ++status[rng() % 20 == 0 ? optimizer(c) : entropy(c)];
    printf("calls %d ok %d invalid %d unsupported %d seen", calls, status[DLF_OK], status[DLF_ERR_INVALID_ARG], status[DLF_ERR_UNSUPPORTED]);
    for (const auto& s : g_seen) printf(" [%s] %ld", s.first.c_str(), s.second);
    printf("\n");
    return 0;
}
