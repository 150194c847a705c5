// The host side of the feed-forward operators (csrc/dlf_ffn.cpp) with stand-ins for the launchers: random calls on addresses that nobody
// reads, each launch checked against what its kernels assume.  Usage: ff_host_driver <seed> <calls> | devices;
// prints what it saw, or the first fault.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "../include/dlf_debug.h"
#include "../paper_2011_05630_amd/csrc/dlf_ffn.h"

// The devices of a machine with eight; the library's kernels are set up once on each that it runs on.
static int g_device = 0, g_setups[8], g_broken = -1;
extern "C" hipError_t hipGetDevice(int* d)
{
    *d = g_device;
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
    Region used[8];
    int uses = 0;
    const float* db[2] = {nullptr, nullptr};
    int launches = 0;
} g;
static int g_seen[DLF_FF_NUM_SHAPES + 3], g_split;

#define NEED(C)                                                          \
    do {                                                                 \
        if (!(C)) {                                                      \
            printf("FAULT %s: %s (line %d)\n", g.text, #C, __LINE__);    \
            exit(1);                                                     \
        }                                                                \
    } while (0)

// A part of the workspace that one launch of this call writes and a later one reads: inside, and apart from the others.
static void use(const void* p, double bytes)
{
    const uintptr_t lo = (uintptr_t)p;
    NEED(lo >= g.ws && bytes <= (double)(g.ws_end - lo) && lo <= g.ws_end);
    const Region r = {lo, lo + (uintptr_t)bytes};
    for (int i = 0; i < g.uses; ++i) NEED(r.hi <= g.used[i].lo || g.used[i].hi <= r.lo);
    NEED(g.uses < 8);
    g.used[g.uses++] = r;
}
static bool lines(const void* p, int64_t ld, int64_t row) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && row % 8 == 0 && ld * 256 * 2 < ((int64_t)1 << 31); }
static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// -> workgroups.  pt, qt: k across the rows
static int64_t tiles(const DlfFfArgs& a, int shape, bool gated, bool pt, bool qt)
{
    NEED(shape >= 0 && shape < DLF_FF_NUM_SHAPES);
    NEED(shape == DLF_FF_SHAPE_ANY64 ? !gated : shape == DLF_FF_SHAPE_ANY64G ? gated : true);
    const DlfFfShape& s = DLF_FF_SHAPES[shape];
    NEED(a.nr > 0 && a.nc > 0 && a.nk >= 0 && a.problems >= 1 && a.problems <= 2 && a.segments >= 1 && a.segments <= 2 && a.splits >= 1);
    NEED(a.tiles_r == up(a.nr, s.br) && a.tiles_c == up(a.nc, s.bc / (gated ? 2 : 1)));
    NEED(a.splits == 1 || up(a.nk, 64) * a.segments >= a.splits);
    const int operands = gated ? 2 : std::max(a.segments, a.problems);
    for (int i = 0; i < operands; ++i) {
        const void *p = a.p[i], *q = a.q[gated ? 0 : i];
        NEED(a.nk == 0 || (p && q));
        if (shape == DLF_FF_SHAPE_256 || shape == DLF_FF_SHAPE_128 || shape == DLF_FF_SHAPE_128_DEEP)
            NEED(lines(p, a.ldp, pt ? a.nc : a.nk) && lines(q, a.ldq, qt ? a.nr : a.nk));
        else
            NEED(a.ldp <= 1 << 24 && a.ldq <= 1 << 24);      // 32-bit offsets of 128 rows
        NEED(gated || i >= a.problems || a.out[i]);
    }
    NEED(!gated || a.out[0]);
    const int64_t n = up((int64_t)a.tiles_r * a.tiles_c * a.problems * a.splits, 8) * 8;
    NEED(n * 256 < (int64_t)1 << 32);
    ++g_seen[shape];
    if (a.splits > 1) {
        ++g_split;
        use(a.part, (double)a.splits * (gated ? 2 : a.problems) * a.nr * a.nc * 4);
        NEED(up((int64_t)a.nr * a.problems * up(a.nc, 8), 256) * 256 < (int64_t)1 << 32);
    }
    return n;
}

extern "C" {
int dlf_ff_kernels_init(void)
{
    ++g_setups[g_device];
    return g_device == g_broken ? hipErrorInvalidValue : 0;
}
int dlf_ff_start_tile(const DlfFfArgs* a, int shape, int, int gated, void*)
{
    ++g.launches;
    tiles(*a, shape, gated, false, false);
    return 0;
}
int dlf_ff_start_back(const DlfFfBackArgs* a, int shape, int, void*)
{
    ++g.launches;
    int64_t n = a->sum.blocks;
    NEED(shape != DLF_FF_SHAPE_ANY64G);
    const int uses = g.uses;
    if (a->w.problems > 0) n += tiles(a->w, shape, false, true, true);
    if (a->x.problems > 0) n += tiles(a->x, shape, false, true, false);
    NEED(n > 0 && n * 256 < (int64_t)1 << 32);
    double joined = 0;
    for (const DlfFfArgs* p : {&a->w, &a->x})
        if (p->problems > 0 && p->splits > 1) joined += std::ceil((double)p->nr * p->problems * up(p->nc, 8) / 256) * 256;
    NEED(joined < (double)((int64_t)1 << 32));
    if (a->sum.blocks > 0) NEED(a->sum.chunks > 1 && a->sum.n > 0 && a->sum.blocks % up(a->sum.n, 64) == 0);
    g.uses = uses;                                           // the partial sums are read within the call
    return 0;
}
int dlf_ff_start_few(const DlfFfArgs* a, const DlfFfFew* c, int, int gated, void*)
{
    ++g.launches;
    ++g_seen[DLF_FF_NUM_SHAPES + (c->rows ? 1 : 0)];
    NEED(a->nr >= 1 && a->nr <= DLF_FF_FEW_ROWS && a->splits <= 1 && a->out[0] && a->p[0] && a->q[0] && (!gated || a->p[1]));
    NEED((c->nf == 1 || (c->nf == 2 && c->mr == 2 && !gated)) && (c->mr == 1 || c->mr == 2));
    NEED(c->waves == 1 || c->waves == 2 || c->waves == 4 || c->waves == 8);
    if (c->rows) NEED(lines(a->p[0], a->ldp, a->nk) && lines(a->q[0], a->ldq, a->nk) && (!gated || lines(a->p[1], a->ldp, a->nk)));
    NEED(DLF_FF_ROWS_LDS(c->waves, c->nf, c->mr, gated) <= 160 * 1024);
    // the waves' sums meet in the ring
    NEED(DLF_FF_ROWS_LDS(c->waves, c->nf, c->mr, gated) >= c->waves * (gated ? 2 : c->nf) * c->mr * 1024);
    return 0;
}
int dlf_ff_start_dz(const DlfFfDzArgs* a, int, int gated, void*)
{
    ++g.launches;
    ++g_seen[DLF_FF_NUM_SHAPES + 2];
    const int nz = gated ? 2 : 1;
    NEED(a->dy || a->rows == 0);
    NEED(a->chunk >= 1 && a->n >= 1);
    const int64_t chunks = a->rows > 0 ? up(a->rows, a->chunk) : 1;
    NEED(chunks <= DLF_FF_MAX_CHUNKS && a->chunk % DLF_FF_CHUNK_ROWS == 0);
    for (int i = 0; i < nz; ++i) {
        if (a->saved) {
            NEED(a->lddz >= a->n && a->lddz % 8 == 0);
            use(a->dz[i], (double)a->rows * a->lddz * 2);
        }
        if (a->sums[i] && chunks > 1) use(a->sums[i], (double)chunks * a->n * 4);
        else NEED(a->sums[i] == g.db[i]);
    }
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
    case 3: return (1 << 22) - 8 + 8 * (int64_t)(rng() % 3);
    default: return rng() % 2 ? 0 : row;
    }
}
static uintptr_t g_next;
static void* place(double bytes)
{
    const uintptr_t p = g_next + (rng() % 3 ? 0 : rng() % 32 * 2);
    g_next = (g_next + (uintptr_t)bytes + 4096) / 4096 * 4096 + 4096;
    return (void*)p;
}

static int devices()
{
    dlf_ff_desc d;
    memset(&d, 0, sizeof d);
    d.rows = 3;
    d.in_features = d.out_features = 16;
    void *x = (void*)0x100000, *w = (void*)0x200000, *y = (void*)0x300000;
    g_broken = 5;
    for (int turn = 0; turn < 3; ++turn)
        for (g_device = 0; g_device < 8; ++g_device)
            if ((dlf_linear(&d, x, w, nullptr, nullptr, y, nullptr, nullptr, 0, nullptr) == DLF_OK) != (g_device != g_broken)) return 1;
    printf("setups");
    for (int n : g_setups) printf(" %d", n);
    printf("\n");
    return 0;
}

int main(int argc, char** argv)
{
    if (argc > 1 && strcmp(argv[1], "devices") == 0) return devices();
    rng.seed(argc > 1 ? strtoull(argv[1], nullptr, 10) : 1);
    const int calls = argc > 2 ? atoi(argv[2]) : 1000;
    int status[16] = {0}, most = 0;
    for (int c = 0; c < calls; ++c) {
        const bool gated = rng() % 2, back = rng() % 2, forced = rng() % 3 == 0;
        const int kernel = forced ? (int)(rng() % (2 + DLF_FF_NUM_SHAPES)) : 0, splits = forced && rng() % 2 ? 1 + (int)(rng() % 16) : 0;
        dlf_debug_ff_kernel(kernel, splits);
        dlf_ff_desc d;
        memset(&d, 0, sizeof d);
        d.dtype = (int)(rng() % 2);
        d.act = (int)(rng() % 7);
        d.rows = rng() % 40 == 0 ? 0 : pick(1, rng() % 3 ? 8192 : (int64_t)1 << 30);
        d.in_features = (int)pick(1, rng() % 4 ? 12000 : 1 << 20);
        d.out_features = (int)pick(1, rng() % 4 ? 12000 : 1 << 20);
        if (rng() % 50 == 0) {                               // about as many tiles as a launch holds, or a few too many
            d.in_features = (int)pick(1, 512);
            d.out_features = (int)pick(1, 512);
            const int64_t i = up(d.in_features, 64), o = up(d.out_features, 64);
            const int64_t m = std::min(((int64_t)1 << 24) / (2 * o), ((int64_t)1 << 24) / i - 2 * o - 2 * (o + i - 1) / i);
            d.rows = std::min((int64_t)1 << 30, 64 * (m - (int64_t)(rng() % 20)) - (int64_t)(rng() % 64));
        }
        d.x_stride = stride(d.in_features);
        d.w_stride = stride(d.in_features);
        d.y_stride = stride(d.out_features);
        d.res_stride = stride(d.out_features);
        d.dy_stride = stride(d.out_features);
        g = Call();
        snprintf(g.text, sizeof g.text, "call %d %s%s dtype %d act %d rows %lld in %d out %d strides %lld %lld %lld %lld %lld kernel %d splits %d", c,
                 gated ? "gated" : "linear", back ? " backward" : "", d.dtype, d.act, (long long)d.rows, d.in_features, d.out_features, (long long)d.x_stride,
                 (long long)d.w_stride, (long long)d.y_stride, (long long)d.res_stride, (long long)d.dy_stride, kernel, splits);
        const size_t need = back ? (gated ? dlf_gated_backward_workspace_bytes(&d) : dlf_linear_backward_workspace_bytes(&d))
                                 : (gated ? dlf_gated_workspace_bytes(&d) : dlf_linear_workspace_bytes(&d));
        g_next = (uintptr_t)1 << 40;
        const double row = 2.0 * (1 << 24);
        void *x = place(row * d.rows), *w0 = place(row * d.out_features), *w1 = place(row * d.out_features), *y = place(row * d.rows), *dy = place(row * d.rows),
             *dx = place(row * d.rows), *dw0 = place(row * d.out_features), *dw1 = place(row * d.out_features);
        auto floats = [&](double n) { return (float*)((uintptr_t)place(4 * n) & ~(uintptr_t)3); };
        float *b0 = floats(d.out_features), *b1 = floats(d.out_features), *saved = floats(2.0 * d.rows * d.out_features);
        const int some = (int)(rng() % 32);
        void* const ws = (void*)((uintptr_t)1 << 46);
        const bool refused = need == SIZE_MAX;
        g.ws = (uintptr_t)ws;
        g.ws_end = g.ws + (refused ? 0 : need);
        g_error[0] = 0;
        dlf_status s;
        if (!back) {
            s = gated ? dlf_gated(&d, x, w0, w1, some & 1 ? b0 : nullptr, some & 2 ? b1 : nullptr, y, some & 4 ? saved : nullptr, ws, refused ? 0 : need, nullptr)
                      : dlf_linear(&d, x, w0, some & 1 ? b0 : nullptr, some & 2 ? dy : nullptr, y, some & 4 ? saved : nullptr, ws, refused ? 0 : need, nullptr);
        } else {
            g.db[0] = some & 8 ? b0 : nullptr;
            g.db[1] = some & 16 && gated ? b1 : nullptr;
            s = gated ? dlf_gated_backward(&d, dy, x, w0, w1, saved, some & 1 ? dx : nullptr, some & 2 ? dw0 : nullptr, some & 4 ? dw1 : nullptr,
                                           (float*)g.db[0], (float*)g.db[1], ws, refused ? 0 : need, nullptr)
                      : dlf_linear_backward(&d, dy, x, w0, saved, some & 1 ? dx : nullptr, some & 2 ? dw0 : nullptr, (float*)g.db[0], ws, refused ? 0 : need,
                                            nullptr);
        }
        NEED((s != DLF_OK) == refused && (s == DLF_OK) == (g_error[0] == 0));
        NEED(s == DLF_OK || g.launches == 0);
        if (s == DLF_OK && need > 0 && g.launches > 0) {     // a byte less is refused before anything is launched
            g.launches = 0;
            s = back ? (gated ? dlf_gated_backward(&d, dy, x, w0, w1, saved, dx, dw0, dw1, b0, b1, ws, need - 1, nullptr)
                              : dlf_linear_backward(&d, dy, x, w0, saved, dx, dw0, b0, ws, need - 1, nullptr))
                     : (gated ? dlf_gated(&d, x, w0, w1, b0, b1, y, saved, ws, need - 1, nullptr) : dlf_linear(&d, x, w0, b0, dy, y, saved, ws, need - 1, nullptr));
            NEED(s == DLF_ERR_OOM && g.launches == 0);
            s = DLF_OK;
        }
        ++status[s];
        most = std::max(most, g.launches);
    }
    printf("calls %d ok %d invalid %d unsupported %d split %d seen", calls, status[DLF_OK], status[DLF_ERR_INVALID_ARG], status[DLF_ERR_UNSUPPORTED], g_split);
    for (int n : g_seen) printf(" %d", n);
    printf("\n");
    return 0;
}
