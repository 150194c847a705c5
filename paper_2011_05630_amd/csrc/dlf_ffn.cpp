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

// A launch holds fewer than 2^32 threads, 256 to a workgroup.
constexpr int64_t MOST_WORKGROUPS = (int64_t)1 << 24;

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
    // the products of the forward pass and of the gradients, with the column sums, by the workgroups of their launches, each product's a
    // multiple of eight
    const int64_t t = 64, m = (d->rows + t - 1) / t, i = (d->in_features + t - 1) / t, o = (d->out_features + t - 1) / t;
    if (std::max(m * o * 2, m * i + 2 * i * o + 2 * o) >= MOST_WORKGROUPS - 16)
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

// Rows in memory, in bytes.
struct Span {
    uintptr_t p;
    int64_t rows, row, stride;
    Span(const void* at, int64_t rows_, int64_t row_, int64_t stride_) : p((uintptr_t)at), rows(rows_), row(row_), stride(rows_ > 1 ? stride_ : row_) {}
    uintptr_t end() const { return p + (uintptr_t)((rows - 1) * stride + row); }
    // whether a byte of [lo, hi), which meets [p, end()), lies in a row: the last row that starts in front of hi has the farthest end
    bool meets(uintptr_t lo, uintptr_t hi) const
    {
        const int64_t last = std::min<int64_t>(rows - 1, (int64_t)((hi - 1 - p) / (uintptr_t)stride));
        return p + (uintptr_t)(last * stride + row) > lo;
    }
};
// Whether two sets of rows share a byte.  Columns of one matrix lie between each other's rows and share none.  (Rows at two different
// distances, neither of them the row itself, are taken as apart.)
bool share(const Span& a, const Span& b)
{
    if (a.rows <= 0 || b.rows <= 0 || a.end() <= b.p || b.end() <= a.p) return false;
    if (a.stride == a.row) return b.meets(a.p, a.end());
    if (b.stride == b.row) return a.meets(b.p, b.end());
    if (a.stride != b.stride) return false;
    const Span &lo = a.p <= b.p ? a : b, &hi = a.p <= b.p ? b : a;
    const int64_t gap = (int64_t)(hi.p - lo.p), at = gap % lo.stride;        // hi's rows start here in lo's
    return at < lo.row || (at + hi.row > lo.stride && gap / lo.stride + 1 < lo.rows);
}
// y is written while other workgroups read the operands: it may lie on the residual alone, element on element.
dlf_status check_output(const Ff& f, const void* y, const void* x, const void* const w[2], const float* const bias[2], const void* res,
                        const char* const (&names)[2][2])
{
    const int64_t in = (int64_t)f.d.in_features * 2, out = (int64_t)f.d.out_features * 2;
    const char* const name = f.gated ? "h" : "y";
    const Span s(y, f.d.rows, out, f.d.y_stride * 2);
    if (share(s, Span(x, f.d.rows, in, f.d.x_stride * 2))) return fail(DLF_ERR_INVALID_ARG, "%s: %s overlaps x", f.call, name);
    for (int i = 0; i < (f.gated ? 2 : 1); ++i) {
        if (share(s, Span(w[i], f.d.out_features, in, f.d.w_stride * 2))) return fail(DLF_ERR_INVALID_ARG, "%s: %s overlaps %s", f.call, name, names[0][i]);
        if (bias[i] && share(s, Span(bias[i], 1, out * 2, out * 2))) return fail(DLF_ERR_INVALID_ARG, "%s: %s overlaps %s", f.call, name, names[1][i]);
    }
    if (res && !(res == y && (f.d.rows == 1 || f.d.res_stride == f.d.y_stride)) && share(s, Span(res, f.d.rows, out, f.d.res_stride * 2)))
        return fail(DLF_ERR_INVALID_ARG, "%s: %s overlaps the residual and is not the residual", f.call, name);
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

// A kernel's attributes belong to the device that it is set up on: once for each that calls run on.
constexpr int MOST_DEVICES = 64;
std::once_flag g_once[MOST_DEVICES];
int g_once_rc[MOST_DEVICES];

dlf_status kernels_ready()
{
    int device = 0;
    const hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return fail(DLF_ERR_HIP, "no device: %s", hipGetErrorString(e));
    if (device < 0 || device >= MOST_DEVICES) return fail(DLF_ERR_UNSUPPORTED, "device %d", device);
    std::call_once(g_once[device], [device] { g_once_rc[device] = dlf_ff_kernels_init(); });
    if (g_once_rc[device] != 0) return fail(DLF_ERR_HIP, "kernel setup failed: %s", hipGetErrorString((hipError_t)g_once_rc[device]));
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
    // Rows per workgroup: 32 rather than 16 (the kernel, 64 rows 2048 -> 2 x 5632: 13.0 against 15.7 us, 4096 -> 4096 11.8 against 14.0), above 32
    // rows with 32 features for the reads of x (64 x 4096 -> 4096 10.9 against 11.8, 48 x 2048 -> 32001 38 against 45; 32 x 4096 -> 4096 would
    // lose, 10.5 against 8.4: fewer workgroups).
    c.mr = a.nr <= 16 ? 1 : 2;
    c.nf = gated || a.nr <= 32 ? 1 : 2;
    // Waves that share k: eight while every workgroup has a compute unit to itself (128 of them: 7.6 us, with four 9.2), else four (2001: 24.7,
    // with eight 25.6; 680 gated: 32.1, with eight 36.6), and no more than there are stages of 64 k.
    const int64_t groups = (int64_t)((a.nc + 16 * c.nf - 1) / (16 * c.nf)) * ((a.nr + 16 * c.mr - 1) / (16 * c.mr));
    c.waves = groups <= 256 ? 8 : 4;
    while (c.waves > 1 && c.waves * 64 >= 2 * a.nk) c.waves >>= 1;
    return launched(f, dlf_ff_start_few(&a, &c, f.d.dtype, gated, stream));
}

// How a product of these sizes is cut: a tile shape and the workgroups that share a tile's k.
struct Cut {
    int shape = DLF_FF_SHAPE_128, splits = 1, tiles_r = 0, tiles_c = 0;
    size_t part_bytes = 0;
    int64_t tiles() const { return (int64_t)tiles_r * tiles_c; }
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

// Modelled times in ns, from measurements at 4096^3 and around.  A stage of 64 k takes a 256 x 256 tile 1450; two 128 x 128 tiles that share
// a compute unit 900, and one that has it to itself waits for memory as long, unless four stages are on their way: 500.  Through registers
// tiles share a compute unit by two (128 x 128) or three.  The first loads and the epilogue of a tile come on top.
struct Rate {
    int share;              // workgroups of a compute unit
    double stage[3], rest;  // by how many share it
};
const Rate& rate(int shape)
{
    static const Rate rates[DLF_FF_NUM_SHAPES] = {{1, {1450}, 7000}, {2, {900, 900}, 4000}, {2, {750, 1130}, 5000}, {1, {500}, 5000},
                                                  {3, {380, 490, 640}, 4000}, {2, {550, 730}, 4000}};
    return rates[shape];
}
// Tiles of two lengths, the first kind's started first, as they fill the compute units.
double fill_ns(int shape, int64_t n0, double stages0, int64_t n1, double stages1)
{
    const Rate& r = rate(shape);
    const int level = (int)std::min<int64_t>(r.share, std::max<int64_t>(1, ceil_div(n0 + n1, 256))) - 1;
    const int64_t slots = 256 * (level + 1);
    const double t0 = stages0 * r.stage[level] + r.rest, t1 = stages1 * r.stage[level] + r.rest, a = (double)(n0 / slots) * t0;
    const int64_t late = n0 % slots;                          // slots that are free t0 later than the others
    double end = late > 0 ? a + t0 : a;
    if (n1 > 0) {
        double last = 0;
        for (int64_t k = std::max<int64_t>(0, n1 / slots - (int64_t)(t0 / t1) - 2);; ++k) {     // rounds of the slots that are free first
            const double at = a + (double)(k + 1) * t1, second = late > 0 ? std::max(0.0, at - a - t0) / t1 : 0;
            last = at;
            if ((slots - late) * (k + 1) + late * (int64_t)(second + 1e-9) >= n1) break;
            if (late > 0) {                                   // the late ones' round that ends before the next
                const int64_t q = (int64_t)(second + 1e-9) + 1;
                const double at2 = a + t0 + (double)q * t1;
                last = at2;
                if (at2 < at + t1 && (slots - late) * (k + 1) + late * q >= n1) break;
            }
        }
        end = std::max(end, last);
    }
    return end;
}
double join_ns(size_t part_bytes) { return part_bytes > 0 ? 3500 + (double)part_bytes * 2 / 4000 : 0; }

// The splits that a product of nr x nc outputs in so many tiles may have: at least four stages each, and workgroups that the launches have room
// for: `spare` of them beside its tiles, half for either of two products, and half of the launch that joins the sums, by eights of outputs.
template <typename F> void each_split(int64_t stages, int64_t nr, int64_t nc, int64_t tiles, int64_t spare, F&& f)
{
    const bool joins = nr * ((nc + 7) / 8) / 256 < MOST_WORKGROUPS / 2 - 1;
    const int64_t most = joins ? std::max<int64_t>(1, std::min<int64_t>({16, stages / 4, 1 + spare / (2 * tiles)})) : 1;
    for (int splits = 1; splits <= most; ++splits) {
        if (g_force_splits > 0 && splits != std::min<int64_t>(g_force_splits, most)) continue;
        f(splits);
    }
}
// any: the operands' rows start anywhere.  (Tiles through registers take all operands; the larger ones lose where direct loads apply.)
bool takes(int shape, bool gated, bool any)
{
    if (shape == DLF_FF_SHAPE_ANY64) return !gated;
    if (shape == DLF_FF_SHAPE_ANY64G) return gated;
    return shape == DLF_FF_SHAPE_ANY ? any || g_force == 2 + shape : !any;
}
template <typename F> void each_shape(bool gated, bool any, F&& f)
{
    const bool forced = g_force >= 2 && takes(g_force - 2, gated, any);
    for (int shape = 0; shape < DLF_FF_NUM_SHAPES; ++shape)
        if (takes(shape, gated, any) && (!forced || shape == g_force - 2)) f(shape);
}

Cut least_forward(int64_t nr, int64_t nc, int64_t nk, bool gated, bool any)
{
    Cut best;
    double least = 0;
    each_shape(gated, any, [&](int shape) {
        const int64_t tiles = cut_as(shape, 1, nr, nc, 1, gated).tiles();
        each_split(ceil_div(nk, 64), nr, nc, tiles, MOST_WORKGROUPS - 16 - tiles, [&](int splits) {
            const Cut c = cut_as(shape, splits, nr, nc, 1, gated);
            const double t = fill_ns(shape, c.tiles() * splits, (double)ceil_div(nk, 64) / splits, 0, 0) + join_ns(c.part_bytes);
            if (least == 0 || t < least) { least = t; best = c; }
        });
    });
    return best;
}

// The two products of a backward pass in one launch: both in tiles of one shape.
struct BackCut {
    Cut w, x;
    bool x_first = false;
};
// rows, in, out as of the layer; problems: 2 for the gated pair
BackCut least_back(int64_t rows, int64_t in, int64_t out, int problems, bool any, bool want_w, bool want_x)
{
    BackCut best;
    double least = 0;
    const int64_t stages_w = ceil_div(rows, 64), stages_x = (int64_t)ceil_div(out, 64) * problems;
    each_shape(false, any, [&](int shape) {
        const int64_t tiles_w = cut_as(shape, 1, out, in, 1, false).tiles() * problems, tiles_x = cut_as(shape, 1, rows, in, 1, false).tiles();
        const int64_t spare = MOST_WORKGROUPS - 16 - 2 * (int64_t)ceil_div(out, 64) - tiles_w - tiles_x;
        each_split(want_w ? stages_w : 1, out * problems, in, tiles_w, spare, [&](int sw) {
            const Cut w = cut_as(shape, sw, out, in, problems, false);
            each_split(want_x ? stages_x : 1, rows, in, tiles_x, spare, [&](int sx) {
                const Cut x = cut_as(shape, sx, rows, in, 1, false);
                const int64_t nw = want_w ? w.tiles() * problems * sw : 0, nx = want_x ? x.tiles() * sx : 0;
                const double lw = (double)stages_w / sw, lx = (double)stages_x / sx;
                const bool x_first = lx > lw;
                const double t = (x_first ? fill_ns(shape, nx, lx, nw, lw) : fill_ns(shape, nw, lw, nx, lx)) +
                                 join_ns((want_w ? w.part_bytes : 0) + (want_x ? x.part_bytes : 0));
                if (least == 0 || t < least) { least = t; best = {w, x, x_first}; }
            });
        });
    });
    if (!want_w) best.w.part_bytes = 0;
    if (!want_x) best.x.part_bytes = 0;
    return best;
}

// A call asks for its cuts several times (sizes of workspaces, launches), a program for the same ones again and again: the last ones are
// kept by their sizes.
template <typename C, typename F> C kept_cut(const int64_t (&sizes)[4], F&& make)
{
    struct Kept {
        int64_t key[6];
        C cut;
    };
    static thread_local Kept kept[64] = {};
    const int64_t key[6] = {sizes[0], sizes[1], sizes[2], sizes[3], g_force, g_force_splits};
    uint64_t h = 0;
    for (int64_t k : key) h = (h ^ (uint64_t)k) * 0x9e3779b97f4a7c15ull;
    Kept& e = kept[h >> 58];
    if (memcmp(e.key, key, sizeof key) != 0) {
        e.cut = make();
        memcpy(e.key, key, sizeof key);
    }
    return e.cut;
}
Cut choose(int64_t nr, int64_t nc, int64_t nk, bool gated, bool any)
{
    return kept_cut<Cut>({nr, nc, nk, (gated ? 2 : 0) + (any ? 1 : 0)}, [&] { return least_forward(nr, nc, nk, gated, any); });
}
BackCut choose_back(int64_t rows, int64_t in, int64_t out, int problems, bool any, bool want_w, bool want_x)
{
    return kept_cut<BackCut>({rows, in, out, problems * 8 + (any ? 4 : 0) + (want_w ? 2 : 0) + (want_x ? 1 : 0)},
                             [&] { return least_back(rows, in, out, problems, any, want_w, want_x); });
}

bool is_few(int64_t rows) { return rows <= DLF_FF_FEW_ROWS && (g_force == 0 || g_force == 1); }
size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

// The workspace of a backward call: dz, partial column sums, partial sums of the products.  What the addresses are, and which gradients are
// wanted, is not known where its size is asked for.
struct BackLayout {
    size_t lddz = 0, part = 0, join = 0, bytes = 0;   // elements per row of dz; offsets
    int chunk = 0, chunks = 0;
};
bool needs_dz(const Ff& f) { return f.gated || f.d.act != DLF_ACT_NONE; }
BackLayout back_layout(const Ff& f)
{
    BackLayout l;
    const size_t nz = f.gated ? 2 : 1;
    l.lddz = ((size_t)f.d.out_features + 7) / 8 * 8;
    l.chunk = std::max(1, ceil_div(f.d.rows, (int64_t)DLF_FF_MAX_CHUNKS * DLF_FF_CHUNK_ROWS)) * DLF_FF_CHUNK_ROWS;
    l.chunks = std::max(1, ceil_div(f.d.rows, l.chunk));
    if (needs_dz(f)) l.bytes = nz * align256((size_t)f.d.rows * l.lddz * 2);
    l.part = l.bytes;
    if (l.chunks > 1) l.bytes += align256(nz * l.chunks * (size_t)f.d.out_features * 4);
    l.join = l.bytes;
    size_t most = 0;
    if (f.d.rows > 0)
        for (int k = 0; k < 8; ++k) {
            const bool want_w = k & 1, want_x = k & 2;
            if (!want_w && !want_x) continue;
            const BackCut c = choose_back(f.d.rows, f.d.in_features, f.d.out_features, (int)nz, k & 4, want_w, want_x);
            most = std::max(most, align256(c.w.part_bytes) + c.x.part_bytes);
        }
    l.bytes += align256(most);
    return l;
}

size_t forward_ws(const Ff& f)
{
    if (f.d.rows == 0 || is_few(f.d.rows)) return 0;
    const int64_t nr = f.d.rows, nc = f.d.out_features, nk = f.d.in_features;
    return align256(std::max(choose(nr, nc, nk, f.gated, false).part_bytes, choose(nr, nc, nk, f.gated, true).part_bytes));
}

void set_cut(DlfFfArgs& a, const Cut& c, char* part)
{
    a.tiles_r = c.tiles_r;
    a.tiles_c = c.tiles_c;
    a.splits = c.splits;
    a.part = (float*)part;
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
    TRY(kernels_ready());
    if (is_few(a.nr)) return few_rows(f, a, f.gated, stream);
    const bool whole = lines(a.p[0], a.ldp, a.nk) && (!f.gated || lines(a.p[1], a.ldp, a.nk)) && lines(a.q[0], a.ldq, a.nk);
    const Cut c = choose(a.nr, a.nc, a.nk, f.gated, !whole);
    set_cut(a, c, ws);
    return launched(f, dlf_ff_start_tile(&a, c.shape, f.d.dtype, f.gated, stream));
}

dlf_status backward(const Ff& f, const void* dy, const void* x, const void* const w[2], const float* saved, void* dx, void* const dw[2],
                    float* const db[2], char* ws, void* stream)
{
    const BackLayout l = back_layout(f);
    const int nz = f.gated ? 2 : 1;
    const bool sums = db[0] || db[1], want_w = dw[0] || dw[1], want_x = dx && f.d.rows > 0;
    const void* dz[2] = {dy, nullptr};
    int64_t lddz = f.d.dy_stride;
    TRY(kernels_ready());
    DlfFfBackArgs b;
    memset(&b, 0, sizeof b);
    b.w.splits = b.x.splits = 1;
    if (sums || ((want_w || want_x) && needs_dz(f))) {
        DlfFfDzArgs z;
        memset(&z, 0, sizeof z);
        z.dy = dy; z.lddy = f.d.dy_stride;
        z.rows = (int)f.d.rows; z.n = f.d.out_features; z.act = f.d.act; z.chunk = l.chunk;
        float* const part = (float*)(ws + l.part);
        for (int i = 0; i < nz; ++i) {
            if (!db[i]) continue;
            z.sums[i] = l.chunks > 1 ? part + (size_t)i * l.chunks * f.d.out_features : db[i];
            b.sum.part[i] = z.sums[i];
            b.sum.out[i] = db[i];
        }
        if (needs_dz(f)) {
            z.saved = saved;
            z.lddz = lddz = (int64_t)l.lddz;
            for (int i = 0; i < nz; ++i) dz[i] = z.dz[i] = ws + i * align256((size_t)f.d.rows * l.lddz * 2);
        }
        TRY(launched(f, dlf_ff_start_dz(&z, f.d.dtype, f.gated, stream)));
        if (sums && l.chunks > 1) {
            b.sum.n = z.n;
            b.sum.chunks = l.chunks;
            b.sum.blocks = nz * ceil_div(z.n, 64);
        }
    }
    bool whole_x = want_x, whole_w = want_w;
    if (want_x) {
        DlfFfArgs& a = b.x;
        for (int i = 0; i < nz; ++i) {
            a.p[i] = w[i]; a.q[i] = dz[i];
            whole_x = whole_x && lines(w[i], f.d.w_stride, f.d.in_features) && lines(dz[i], lddz, f.d.out_features);
        }
        a.ldp = f.d.w_stride; a.ldq = lddz;
        a.nr = (int)f.d.rows; a.nc = f.d.in_features; a.nk = f.d.out_features;
        a.segments = nz; a.problems = 1;
        a.out[0] = dx; a.ldo = f.d.in_features;
    }
    if (want_w) {
        DlfFfArgs& a = b.w;
        a.segments = 1;
        for (int i = 0; i < nz; ++i)
            if (dw[i]) {
                a.p[a.problems] = x; a.q[a.problems] = dz[i]; a.out[a.problems] = dw[i];
                ++a.problems;
                whole_w = whole_w && lines(x, f.d.x_stride, f.d.in_features) && lines(dz[i], lddz, f.d.out_features);
            }
        a.ldp = f.d.x_stride; a.ldq = lddz;
        a.nr = f.d.out_features; a.nc = f.d.in_features; a.nk = (int)f.d.rows;
        a.ldo = f.d.in_features;
    }
    if (!want_x && !want_w && b.sum.blocks == 0) return DLF_OK;
    // operands of different alignment: a launch each
    const bool apart = want_x && want_w && whole_x != whole_w;
    for (int part = 0; part < (apart ? 2 : 1); ++part) {
        DlfFfBackArgs c = b;
        const bool cw = want_w && !(apart && part == 1), cx = want_x && !(apart && part == 0), any = !(cw ? whole_w : whole_x);
        if (!cw) c.w.problems = 0;
        if (!cx) c.x.problems = 0;
        if (part == 1) c.sum.blocks = 0;
        const BackCut k = choose_back(std::max<int64_t>(1, f.d.rows), f.d.in_features, f.d.out_features, nz, cw || cx ? any : false, cw, cx);
        c.x_first = k.x_first;
        set_cut(c.w, k.w, ws + l.join);
        set_cut(c.x, k.x, ws + l.join + align256(k.w.part_bytes));
        TRY(launched(f, dlf_ff_start_back(&c, k.w.shape, f.d.dtype, stream)));
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
    const void* w[2] = {weight, nullptr};
    const float* b[2] = {bias, nullptr};
    TRY(check_output(f, y, x, w, b, residual, {{"weight", ""}, {"bias", ""}}));
    TRY(check_ws(f, workspace, workspace_bytes, forward_ws(f)));
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
    const void* w[2] = {w_gate, w_up};
    const float* b[2] = {b_gate, b_up};
    TRY(check_output(f, h, x, w, b, nullptr, {{"w_gate", "w_up"}, {"b_gate", "b_up"}}));
    TRY(check_ws(f, workspace, workspace_bytes, forward_ws(f)));
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
