// Host side of the feed-forward operators: checks of the arguments, workspace layout, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "../../include/dlf_debug.h"
#include "dlf_ffn.h"

namespace {

dlf_status fail(dlf_status s, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return dlf_set_error(s, buf);
}

// A description with its strides filled in.
struct Ff {
    dlf_ff_desc d;
    bool gated;
    const char* call;
};

dlf_status check_desc(const dlf_ff_desc* d, bool gated, const char* call, Ff& f)
{
    if (!d) return fail(DLF_ERR_INVALID_ARG, "%s: null description", call);
    f.d = *d;
    f.gated = gated;
    f.call = call;
    if (d->dtype != DLF_F16 && d->dtype != DLF_BF16) return fail(DLF_ERR_INVALID_ARG, "%s: dtype %d", call, d->dtype);
    if (d->act < DLF_ACT_NONE || d->act > DLF_ACT_SIGMOID) return fail(DLF_ERR_INVALID_ARG, "%s: act %d", call, d->act);
    if (d->rows < 0 || d->rows > (int64_t)1 << 30) return fail(DLF_ERR_INVALID_ARG, "%s: %lld rows", call, (long long)d->rows);
    if (d->in_features < 1 || d->in_features > 1 << 20 || d->out_features < 1 || d->out_features > 1 << 20)
        return fail(DLF_ERR_INVALID_ARG, "%s: %d -> %d features", call, d->in_features, d->out_features);
    struct { int64_t* s; int64_t row; const char* name; } strides[] = {
        {&f.d.x_stride, d->in_features, "x"}, {&f.d.w_stride, d->in_features, "weight"}, {&f.d.y_stride, d->out_features, "y"},
        {&f.d.res_stride, d->out_features, "residual"}, {&f.d.dy_stride, d->out_features, "dy"}};
    for (auto& q : strides) {
        if (*q.s == 0) *q.s = q.row;
        if (*q.s < q.row || *q.s >= (int64_t)1 << 24)
            return fail(DLF_ERR_INVALID_ARG, "%s: %s has rows of %lld elements, %lld apart", call, q.name, (long long)q.row, (long long)*q.s);
    }
    // the products of the forward pass and of the gradients by the tiles of their grids
    const int64_t t = 64, m = (d->rows + t - 1) / t, i = (d->in_features + t - 1) / t, o = (d->out_features + t - 1) / t;
    if (std::max({m * o * 2, m * i, 2 * i * o}) >= (int64_t)1 << 24)
        return fail(DLF_ERR_UNSUPPORTED, "%s: %lld rows, %d -> %d features are more tiles than a launch holds", call, (long long)d->rows,
                    d->in_features, d->out_features);
    return DLF_OK;
}

dlf_status check_ptr(const Ff& f, const void* p, const char* name, bool wanted, uintptr_t align)
{
    if (!p && wanted) return fail(DLF_ERR_INVALID_ARG, "%s: null %s", f.call, name);
    if (((uintptr_t)p & (align - 1)) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: %s is not aligned to %d bytes", f.call, name, (int)align);
    return DLF_OK;
}

dlf_status check_ws(const Ff& f, const void* ws, size_t have, size_t need)
{
    if (need == 0) return DLF_OK;
    if (have < need) return fail(DLF_ERR_OOM, "%s: workspace too small: %zu < %zu", f.call, have, need);
    if (!ws || ((uintptr_t)ws & 255) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: workspace must be a 256-byte aligned device pointer", f.call);
    return DLF_OK;
}

#define TRY(X)                             \
    do {                                   \
        const dlf_status try_s = (X);      \
        if (try_s != DLF_OK) return try_s; \
    } while (0)

dlf_status launched(const Ff& f, int e)
{
    if (e != 0) return fail(DLF_ERR_HIP, "%s: launch failed: %s", f.call, hipGetErrorString((hipError_t)e));
    return DLF_OK;
}

// Testing hook: 0 = by rule, 1 = k_ff_few wherever a few-rows kernel applies, 2 + shape = a tile kernel wherever it applies.
int g_force = 0;

std::once_flag g_once;
int g_once_rc = 0;

dlf_status kernels_ready()
{
    std::call_once(g_once, [] { g_once_rc = dlf_ff_kernels_init(); });
    if (g_once_rc != 0) return fail(DLF_ERR_HIP, "kernel setup failed: %s", hipGetErrorString((hipError_t)g_once_rc));
    return DLF_OK;
}

// Whether the tile kernel takes an operand: rows in whole 16-byte lines, offsets inside a tile that fit 31 bits.
bool lines(const void* p, int64_t ld, int64_t row)
{
    return ((uintptr_t)p & 15) == 0 && (ld & 7) == 0 && (row & 7) == 0 && ld < (int64_t)1 << 22;
}



// The forward product of few rows, straight from memory.
dlf_status few_rows(const Ff& f, DlfFfArgs& a, bool gated, void* stream)
{
    DlfFfFew c;
    c.rows = g_force != 1 && lines(a.p[0], a.ldp, a.nk) && (!gated || lines(a.p[1], a.ldp, a.nk)) && lines(a.q[0], a.ldq, a.nk);
    // Rows per workgroup: 32 rather than 64 of them even where 64 exist (gated 64 x 2048 -> 2 x 5632: 16.6 against 18.4 us), there with
    // 32 features for the reads of x (64 x 4096 -> 4096: 12.1 against 14.8 us; fewer workgroups lose below 33 rows).
    c.mr = a.nr <= 16 ? 1 : 2;
    c.nf = gated || a.nr <= 32 ? 1 : 2;
    // Waves that share k: eight while every workgroup has a compute unit to itself, else four (2001 of them: 24.3 against 24.7 us, 680
    // gated: 31.8 against 35.9), and no more than there are stages of 64 k.
    const int64_t groups = (int64_t)((a.nc + 16 * c.nf - 1) / (16 * c.nf)) * ((a.nr + 16 * c.mr - 1) / (16 * c.mr));
    c.waves = groups <= 256 ? 8 : 4;
    while (c.waves > 1 && c.waves * 64 >= 2 * a.nk) c.waves >>= 1;
    return launched(f, dlf_ff_start_few(&a, &c, f.d.dtype, gated, stream));
}

// How a product of these sizes is cut: a tile shape and the workgroups that share a tile's k.
struct Cut {
    int shape = DLF_FF_SHAPE_128, splits = 1, tiles_r = 0, tiles_c = 0;
    size_t part_bytes = 0;
};
int g_force_splits = 0;

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

Cut cut_as(int shape, int splits, int64_t nr, int64_t nc, int problems, bool gated)
{
    Cut c;
    c.shape = shape;
    c.splits = splits;
    c.tiles_r = ceil_div(nr, DLF_FF_SHAPES[shape].br);
    c.tiles_c = ceil_div(nc, DLF_FF_SHAPES[shape].bc / (gated ? 2 : 1));
    if (splits > 1) c.part_bytes = (size_t)splits * (gated ? 2 : problems) * nr * nc * 4;
    return c;
}

// Modelled time of a cut in ns, from measurements at 4096^3 and around: a stage of 64 k takes a 256 x 256 tile 1450 ns; two 128 x 128
// tiles that share a compute unit 900 ns, one that has it to itself waits for memory, 900 ns a stage, unless four stages are on their way: 500;
// through registers 1250 and 950; the first loads and the epilogue of a tile 7, 4 and 5 us; joining, a launch and the partial sums' bytes twice.
double cut_ns(const Cut& c, int64_t nr, int64_t nc, int64_t nk, int segments, int problems, bool gated)
{
    const int64_t wgs = (int64_t)c.tiles_r * c.tiles_c * problems * c.splits;
    const double stages = (double)ceil_div(nk, 64) * segments / c.splits;
    double t;
    if (c.shape == DLF_FF_SHAPE_256) {
        t = (double)ceil_div(wgs, 256) * (stages * 1450 + 7000);
    } else if (c.shape == DLF_FF_SHAPE_ANY64) {
        t = (double)(wgs / 768) * (stages * 760 + 4000);
        if (wgs % 768 > 0) t += stages * (wgs % 768 > 512 ? 760 : wgs % 768 > 256 ? 620 : 530) + 4000;
    } else if (c.shape == DLF_FF_SHAPE_ANY) {
        t = (double)(wgs / 512) * (stages * 1250 + 5000);
        if (wgs % 512 > 256) t += stages * 1250 + 5000;
        else if (wgs % 512 > 0) t += stages * 950 + 5000;
    } else if (c.shape == DLF_FF_SHAPE_128_DEEP) {
        t = (double)ceil_div(wgs, 256) * (stages * 500 + 5000);
    } else {
        t = (double)(wgs / 512) * (stages * 900 + 4000);
        if (wgs % 512 > 256) t += stages * 900 + 4000;
        else if (wgs % 512 > 0) t += stages * 900 + 4000;
    }
    if (c.splits > 1) t += 3500 + (double)c.part_bytes * 2 / 4000;
    return t;
}

// any: the operands' rows start anywhere.
Cut least_cut(int64_t nr, int64_t nc, int64_t nk, int segments, int problems, bool gated, bool any)
{
    Cut best;
    double least = 0;
    const int64_t stages = (int64_t)ceil_div(nk, 64) * segments;
    auto takes = [&](int shape) {
        if (shape == DLF_FF_SHAPE_ANY64) return !gated;
        return shape == DLF_FF_SHAPE_ANY ? any || g_force == 2 + shape : !any;
    };
    for (int shape = 0; shape < DLF_FF_NUM_SHAPES; ++shape) {
        if (!takes(shape) || (g_force >= 2 && takes(g_force - 2) && shape != g_force - 2)) continue;
        for (int splits = 1; splits <= 16; ++splits) {
            if (splits > 1 && stages / splits < 4) break;
            if (g_force_splits > 0 && splits != std::min<int64_t>(g_force_splits, std::max<int64_t>(1, stages / 4))) continue;
            const Cut c = cut_as(shape, splits, nr, nc, problems, gated);
            const double t = cut_ns(c, nr, nc, nk, segments, problems, gated);
            if (least == 0 || t < least) { least = t; best = c; }
        }
    }
    return best;
}

// A call asks for its products' cuts several times (sizes of workspaces, launches), a program for the same ones again and again: the last
// ones are kept by their sizes.
Cut choose(int64_t nr, int64_t nc, int64_t nk, int segments, int problems, bool gated, bool any)
{
    struct Kept {
        int64_t key[6];
        Cut cut;
    };
    static thread_local Kept kept[64] = {};
    const int64_t key[6] = {nr, nc, nk, segments * 16 + problems * 4 + (gated ? 2 : 0) + (any ? 1 : 0), g_force, g_force_splits};
    uint64_t h = 0;
    for (int64_t k : key) h = (h ^ (uint64_t)k) * 0x9e3779b97f4a7c15ull;
    Kept& e = kept[h >> 58];
    if (memcmp(e.key, key, sizeof key) != 0) {
        e.cut = least_cut(nr, nc, nk, segments, problems, gated, any);
        memcpy(e.key, key, sizeof key);
    }
    return e.cut;
}

// Workspace of a product: what its addresses are is not known yet.
size_t part_bytes(int64_t nr, int64_t nc, int64_t nk, int segments, int problems, bool gated)
{
    return std::max(choose(nr, nc, nk, segments, problems, gated, false).part_bytes, choose(nr, nc, nk, segments, problems, gated, true).part_bytes);
}

bool is_few(int64_t rows) { return rows <= DLF_FF_FEW_ROWS && (g_force == 0 || g_force == 1); }
size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

// One product of the operators; part: the workspace of its cut.
dlf_status product(const Ff& f, DlfFfArgs& a, int layout, bool gated, char* part, void* stream)
{
    TRY(kernels_ready());
    if (layout == DLF_FF_NN && is_few(a.nr)) return few_rows(f, a, gated, stream);
    bool whole = true;
    const int n = gated ? 2 : std::max(a.segments, a.problems);
    for (int i = 0; i < n; ++i) {
        whole = whole && lines(a.p[i], a.ldp, layout == DLF_FF_NN ? a.nk : a.nc);
        if (!gated) whole = whole && lines(a.q[i], a.ldq, layout == DLF_FF_TT ? a.nr : a.nk);
    }
    if (gated) whole = whole && lines(a.q[0], a.ldq, a.nk);
    const Cut c = choose(a.nr, a.nc, a.nk, a.segments, a.problems, gated, !whole);
    a.tiles_r = c.tiles_r;
    a.tiles_c = c.tiles_c;
    a.splits = c.splits;
    a.part = (float*)part;
    return launched(f, dlf_ff_start_tile(&a, c.shape, f.d.dtype, layout, gated, stream));
}

// The workspace of a backward call.
struct BackLayout {
    size_t lddz = 0, part = 0, join = 0, bytes = 0;   // elements per row of dz; offsets of the column sums and of the products' partial sums
    int chunk = 0, chunks = 0;
};
bool needs_dz(const Ff& f) { return f.gated || f.d.act != DLF_ACT_NONE; }
BackLayout back_layout(const Ff& f)
{
    BackLayout l;
    const size_t nz = f.gated ? 2 : 1;
    l.lddz = ((size_t)f.d.out_features + 7) / 8 * 8;
    l.chunk = f.d.rows <= DLF_FF_SUM_ROWS ? DLF_FF_SUM_ROWS : (f.d.rows + DLF_FF_MAX_CHUNKS - 1) / DLF_FF_MAX_CHUNKS;
    l.chunks = f.d.rows > 0 ? (int)((f.d.rows + l.chunk - 1) / l.chunk) : 1;
    if (needs_dz(f)) l.bytes = nz * align256((size_t)f.d.rows * l.lddz * 2);
    l.part = l.bytes;
    if (l.chunks > 1) l.bytes += align256(nz * l.chunks * (size_t)f.d.out_features * 4);
    l.join = l.bytes;
    const int problems = f.gated ? 2 : 1;
    l.bytes += align256(std::max(part_bytes(std::max<int64_t>(1, f.d.rows), f.d.in_features, f.d.out_features, problems, 1, false),
                                 part_bytes(f.d.out_features, f.d.in_features, f.d.rows, 1, problems, false)));
    return l;
}

size_t forward_ws(const Ff& f)
{
    if (f.d.rows == 0 || is_few(f.d.rows)) return 0;
    return align256(part_bytes(f.d.rows, f.d.out_features, f.d.in_features, 1, 1, f.gated));
}

dlf_status forward(const Ff& f, const void* x, const void* const w[2], const float* const bias[2], const void* res, void* y, float* saved,
                   char* ws, void* stream)
{
    if (f.d.rows == 0) return DLF_OK;
    DlfFfArgs a;
    memset(&a, 0, sizeof a);
    a.p[0] = w[0]; a.p[1] = w[1];
    a.q[0] = x;
    a.ldp = f.d.w_stride; a.ldq = f.d.x_stride;
    a.nr = (int)f.d.rows; a.nc = f.d.out_features; a.nk = f.d.in_features;
    a.segments = a.problems = 1;
    a.bias[0] = bias[0]; a.bias[1] = bias[1];
    a.res = res; a.ldres = f.d.res_stride;
    a.out[0] = y; a.ldo = f.d.y_stride;
    a.saved = saved; a.act = f.d.act;
    return product(f, a, DLF_FF_NN, f.gated, ws, stream);
}

dlf_status backward(const Ff& f, const void* dy, const void* x, const void* const w[2], const float* saved, void* dx, void* const dw[2],
                    float* const db[2], char* ws, void* stream)
{
    const BackLayout l = back_layout(f);
    const int nz = f.gated ? 2 : 1;
    const bool sums = db[0] || db[1], products = dx || dw[0] || dw[1];
    const void* dz[2] = {dy, nullptr};
    int64_t lddz = f.d.dy_stride;
    if (sums || (products && needs_dz(f))) {
        DlfFfDzArgs z;
        memset(&z, 0, sizeof z);
        z.dy = dy; z.lddy = f.d.dy_stride;
        z.rows = (int)f.d.rows; z.n = f.d.out_features; z.act = f.d.act; z.chunk = l.chunk;
        float* const part = (float*)(ws + l.part);
        for (int i = 0; i < nz; ++i)
            if (db[i]) z.sums[i] = l.chunks > 1 ? part + (size_t)i * l.chunks * f.d.out_features : db[i];
        if (needs_dz(f)) {
            z.saved = saved;
            z.lddz = lddz = (int64_t)l.lddz;
            for (int i = 0; i < nz; ++i) dz[i] = z.dz[i] = ws + i * align256((size_t)f.d.rows * l.lddz * 2);
        }
        TRY(launched(f, dlf_ff_start_dz(&z, f.d.dtype, f.gated, stream)));
        if (sums && l.chunks > 1) {
            DlfFfSumArgs s = {part, {db[0], db[1]}, z.n, l.chunks};
            TRY(launched(f, dlf_ff_start_sum(&s, f.gated, stream)));
        }
    }
    DlfFfArgs a;
    if (dx && f.d.rows > 0) {
        memset(&a, 0, sizeof a);
        for (int i = 0; i < nz; ++i) { a.p[i] = w[i]; a.q[i] = dz[i]; }
        a.ldp = f.d.w_stride; a.ldq = lddz;
        a.nr = (int)f.d.rows; a.nc = f.d.in_features; a.nk = f.d.out_features;
        a.segments = nz; a.problems = 1;
        a.out[0] = dx; a.ldo = f.d.in_features;
        TRY(product(f, a, DLF_FF_TN, false, ws + l.join, stream));
    }
    memset(&a, 0, sizeof a);
    a.segments = 1;
    for (int i = 0; i < nz; ++i)
        if (dw[i]) {
            a.p[a.problems] = x; a.q[a.problems] = dz[i]; a.out[a.problems] = dw[i];
            ++a.problems;
        }
    if (a.problems > 0) {
        a.ldp = f.d.x_stride; a.ldq = lddz;
        a.nr = f.d.out_features; a.nc = f.d.in_features; a.nk = (int)f.d.rows;
        a.ldo = f.d.in_features;
        TRY(product(f, a, DLF_FF_TT, false, ws + l.join, stream));
    }
    return DLF_OK;
}

size_t forward_bytes(const dlf_ff_desc* d, bool gated, const char* call)
{
    Ff f;
    return check_desc(d, gated, call, f) == DLF_OK ? forward_ws(f) : SIZE_MAX;
}
size_t backward_bytes(const dlf_ff_desc* d, bool gated, const char* call)
{
    Ff f;
    return check_desc(d, gated, call, f) == DLF_OK ? back_layout(f).bytes : SIZE_MAX;
}

}  // namespace

extern "C" {

void dlf_debug_ff_kernel(int32_t kernel, int32_t splits)
{
    g_force = kernel >= 0 && kernel < 2 + DLF_FF_NUM_SHAPES ? kernel : 0;
    g_force_splits = splits > 0 ? splits : 0;
}

size_t dlf_linear_workspace_bytes(const dlf_ff_desc* d) { return forward_bytes(d, false, "dlf_linear_workspace_bytes"); }
size_t dlf_gated_workspace_bytes(const dlf_ff_desc* d) { return forward_bytes(d, true, "dlf_gated_workspace_bytes"); }
size_t dlf_linear_backward_workspace_bytes(const dlf_ff_desc* d) { return backward_bytes(d, false, "dlf_linear_backward_workspace_bytes"); }
size_t dlf_gated_backward_workspace_bytes(const dlf_ff_desc* d) { return backward_bytes(d, true, "dlf_gated_backward_workspace_bytes"); }

dlf_status dlf_linear(const dlf_ff_desc* d, const void* x, const void* weight, const float* bias, const void* residual, void* y,
                      float* saved, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    Ff f;
    TRY(check_desc(d, false, "dlf_linear", f));
    const bool some = f.d.rows > 0;
    TRY(check_ptr(f, x, "x", some, 2));
    TRY(check_ptr(f, weight, "weight", some, 2));
    TRY(check_ptr(f, bias, "bias", false, 4));
    TRY(check_ptr(f, residual, "residual", false, 2));
    TRY(check_ptr(f, y, "y", some, 2));
    TRY(check_ptr(f, saved, "saved", false, 4));
    TRY(check_ws(f, workspace, workspace_bytes, forward_ws(f)));
    const void* w[2] = {weight, nullptr};
    const float* b[2] = {bias, nullptr};
    return forward(f, x, w, b, residual, y, saved, (char*)workspace, hip_stream);
}

dlf_status dlf_gated(const dlf_ff_desc* d, const void* x, const void* w_gate, const void* w_up, const float* b_gate, const float* b_up,
                     void* h, float* saved, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    Ff f;
    TRY(check_desc(d, true, "dlf_gated", f));
    const bool some = f.d.rows > 0;
    TRY(check_ptr(f, x, "x", some, 2));
    TRY(check_ptr(f, w_gate, "w_gate", some, 2));
    TRY(check_ptr(f, w_up, "w_up", some, 2));
    TRY(check_ptr(f, b_gate, "b_gate", false, 4));
    TRY(check_ptr(f, b_up, "b_up", false, 4));
    TRY(check_ptr(f, h, "h", some, 2));
    TRY(check_ptr(f, saved, "saved", false, 4));
    TRY(check_ws(f, workspace, workspace_bytes, forward_ws(f)));
    const void* w[2] = {w_gate, w_up};
    const float* b[2] = {b_gate, b_up};
    return forward(f, x, w, b, nullptr, h, saved, (char*)workspace, hip_stream);
}

dlf_status dlf_linear_backward(const dlf_ff_desc* d, const void* dy, const void* x, const void* weight, const float* saved, void* dx,
                               void* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    Ff f;
    TRY(check_desc(d, false, "dlf_linear_backward", f));
    const bool some = f.d.rows > 0;
    TRY(check_ptr(f, dy, "dy", some, 2));
    TRY(check_ptr(f, x, "x", some && dweight, 2));
    TRY(check_ptr(f, weight, "weight", some && dx, 2));
    TRY(check_ptr(f, saved, "saved", some && needs_dz(f), 4));
    TRY(check_ptr(f, dx, "dx", false, 2));
    TRY(check_ptr(f, dweight, "dweight", false, 2));
    TRY(check_ptr(f, dbias, "dbias", false, 4));
    TRY(check_ws(f, workspace, workspace_bytes, back_layout(f).bytes));
    const void* w[2] = {weight, nullptr};
    void* dw[2] = {dweight, nullptr};
    float* db[2] = {dbias, nullptr};
    return backward(f, dy, x, w, saved, dx, dw, db, (char*)workspace, hip_stream);
}

dlf_status dlf_gated_backward(const dlf_ff_desc* d, const void* dh, const void* x, const void* w_gate, const void* w_up, const float* saved,
                              void* dx, void* dw_gate, void* dw_up, float* db_gate, float* db_up, void* workspace, size_t workspace_bytes,
                              void* hip_stream)
{
    Ff f;
    TRY(check_desc(d, true, "dlf_gated_backward", f));
    const bool some = f.d.rows > 0;
    TRY(check_ptr(f, dh, "dh", some, 2));
    TRY(check_ptr(f, x, "x", some && (dw_gate || dw_up), 2));
    TRY(check_ptr(f, w_gate, "w_gate", some && dx, 2));
    TRY(check_ptr(f, w_up, "w_up", some && dx, 2));
    TRY(check_ptr(f, saved, "saved", some, 4));
    TRY(check_ptr(f, dx, "dx", false, 2));
    TRY(check_ptr(f, dw_gate, "dw_gate", false, 2));
    TRY(check_ptr(f, dw_up, "dw_up", false, 2));
    TRY(check_ptr(f, db_gate, "db_gate", false, 4));
    TRY(check_ptr(f, db_up, "db_up", false, 4));
    TRY(check_ws(f, workspace, workspace_bytes, back_layout(f).bytes));
    const void* w[2] = {w_gate, w_up};
    void* dw[2] = {dw_gate, dw_up};
    float* db[2] = {db_gate, db_up};
    return backward(f, dh, x, w, saved, dx, dw, db, (char*)workspace, hip_stream);
}

}  // extern "C"
