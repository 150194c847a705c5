// Host side of the cross entropy of a linear layer: checks of the arguments, pieces of rows, workspace layout, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "dlf_ce.h"
#include "dlf_ff_plan.h"

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
#define TRY(X)                             \
    do {                                   \
        const dlf_status try_s = (X);      \
        if (try_s != DLF_OK) return try_s; \
    } while (0)

constexpr int64_t MOST_WORKGROUPS = (int64_t)1 << 24;       // a launch holds fewer than 2^32 threads, 256 to a workgroup
constexpr int64_t LEAST_PIECE = 256, MOST_PIECE = 1 << 16;  // rows
// Whether operands whose rows start anywhere are copied to rows of whole lines first: modelled in ns, a launch and the copy against what `products` products
// take longer on tiles through registers.  Bf16, us with the copy and without: loss of 1024 x 2051 over 32001 classes 178 and 205, of 768 rows 184 and 158;
// with gradients 2048 rows 942 and 1325, 512 339 and 363, 256 255 and 209; 1300 x 523 over 2999 classes, fp16, 56 and 71, 515 x 770 over 5003 55 and 56,
// 300 rows 48 and 45; with a bias 62 and 77, 61 and 62, 54 and 51.
constexpr int PRODUCTS_LOSS = 1, PRODUCTS_GRADIENTS = 3;
bool copy_pays(int64_t rows, int64_t in, int64_t classes, int products)
{
    return rows > DLF_FF_FEW_ROWS && products * 1.2e-6 * (double)rows * in * classes > 4400 + 4.0 * (double)(rows + classes) * in / 3800;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

// Where the workgroups of dz form their rows' lse themselves instead of reading what a launch of k_ce_join leaves.  Whole calls of gradients, replayed, 256
// features, bf16, us with that launch and without it.
//
// k_ce_dz_sums (a bias's gradient): while a thread has few parts to add up, and not many workgroups repeat it.  16 parts or fewer: 4096 rows over 2000
// classes 56.7 and 54.8, 2048 over 5000 (640 workgroups) 70.7 and 69.2, over 6000 (768) 72.5 and 72.0, 100 over 8000 31.7 and 31.2; 20 of 1024 over 10000
// 70.2 and 70.7; 32 of 60 over 4000 26.5 and 26.2, of 16 over 16000 30.8 and 30.1, of 4 over 64000 56.1 and 55.1, but of 100 over 16000 40.8 and 42.0;
// 47 to 118 of 60 over 6000 27.7 and 28.2, 16000 40.7 and 45.9, 16 over 24000 36.5 and 36.2, 60000 59.4 and 62.2.  More workgroups: 1000 of 55 to 62 parts
// (512 over 32000) 94.5 and 98.4; with 8 parts they would still gain (4096 over 4096, 1024 workgroups: 87.5 and 85.5), which is left.
constexpr int64_t MOST_PARTS_OF_A_THREAD = 32, MOST_FORMING = 768;
// k_ce_dz of few rows' logits, a workgroup of 2048 classes to a row, each reading all of the row's parts: by rows times parts.  1 x 103104 (6444) 75.1 and
// 72.6, 15 x 48000 (45000) 50.1 and 48.3, 15 x 64000 (60000) 59.2 and 58.8, 60 x 16000 (60000) 40.0 and 34.6, 33 x 32000 (66000) 49.3 and 48.0; 15 x 80000 (75000)
// 68.4 and 71.5, 33 x 48000 (99000) 61.7 and 64.3, 60 x 48000 (180000) 65.2 and 72.4, 60 x 103104 111 and 172.
constexpr int64_t MOST_PARTS_OF_FEW_ROWS = 66000;
// k_ce_dz of kept exponentials: up to as many workgroups as run at once.  2000 x 2000 (2000 workgroups) 41.2 and 39.7, 512 x 8000 (2048) 42.3 and 41.9, 128 x
// 32000 (2048) 46.3 and 47.8; 4096 x 2000 (4096) 51.5 and 51.4, 1024 x 8000 (4096) 48.8 and 51.7, 256 x 32000 (4096) 55.0 and 58.7, 4096 x 32000 405 and 486.
constexpr int64_t MOST_FORMING_KEPT = 2048;

// A description with its strides filled in, and the rows of a piece.
struct Ce {
    dlf_ce_desc d;
    const char* call;
    int64_t ldz, piece;     // elements of a row of dz; rows
    int64_t lines;          // 16-byte parts of a row of x or weight
    bool pack_x, pack_w;    // copied to rows of whole lines, or room for it
    int64_t pieces() const { return std::max<int64_t>(1, ceil_div(d.rows, piece)); }
    int64_t first(int64_t p) const { return p * piece; }
    int64_t rows(int64_t p) const { return std::min(piece, d.rows - p * piece); }
};

// Whether a piece of so many rows fits the launches: its tiles of 64 x 64, those of the gradients' products with the column sums, and k_ce_dz.
bool launches(int64_t rows, int64_t in, int64_t classes)
{
    const int64_t m = ceil_div(rows, 64), i = ceil_div(in, 64), o = ceil_div(classes, 64);
    return 2 * m * o < MOST_WORKGROUPS - 16 && m * i + 2 * i * o + 2 * o < MOST_WORKGROUPS - 16 &&
           rows * ceil_div(classes, DLF_CE_DZ_COLS) < MOST_WORKGROUPS - 16;
}

dlf_status check_desc(const dlf_ce_desc* d, bool gradients, const char* call, Ce& f)
{
    if (!d) return fail(DLF_ERR_INVALID_ARG, "%s: null description", call);
    f.d = *d;
    f.call = call;
    if (d->dtype != DLF_F16 && d->dtype != DLF_BF16) return fail(DLF_ERR_INVALID_ARG, "%s: dtype %d", call, d->dtype);
    if (d->dbias != 0 && d->dbias != 1) return fail(DLF_ERR_INVALID_ARG, "%s: dbias %d, 0 or 1 expected", call, d->dbias);
    if (d->rows < 0 || d->rows > (int64_t)1 << 30) return fail(DLF_ERR_INVALID_ARG, "%s: %lld rows", call, (long long)d->rows);
    if (d->in_features < 1 || d->in_features > 1 << 20 || d->classes < 1 || d->classes > 1 << 20)
        return fail(DLF_ERR_INVALID_ARG, "%s: %d features, %d classes", call, d->in_features, d->classes);
    struct { int64_t* s; const char* name; } strides[] = {{&f.d.x_stride, "x"}, {&f.d.w_stride, "weight"}};
    for (auto& q : strides) {
        if (*q.s == 0) *q.s = d->in_features;
        if (*q.s < d->in_features || *q.s >= (int64_t)1 << 24)
            return fail(DLF_ERR_INVALID_ARG, "%s: %s has rows of %d elements, %lld apart", call, q.name, d->in_features, (long long)*q.s);
    }
    if (d->piece_bytes < 0 || d->piece_bytes > (int64_t)1 << 50) return fail(DLF_ERR_INVALID_ARG, "%s: piece_bytes %lld", call, (long long)d->piece_bytes);
    if (!launches(LEAST_PIECE, d->in_features, d->classes))
        return fail(DLF_ERR_UNSUPPORTED, "%s: %d features, %d classes are more tiles than a launch holds", call, d->in_features, d->classes);
    f.ldz = ceil_div(d->classes, 8) * 8;
    const int64_t most = (d->piece_bytes == 0 ? (int64_t)1 << 30 : d->piece_bytes) / (2 * f.ldz);
    f.piece = std::max(LEAST_PIECE, std::min(MOST_PIECE, most) / LEAST_PIECE * LEAST_PIECE);
    while (f.piece > LEAST_PIECE && !launches(f.piece, d->in_features, d->classes)) f.piece = std::max(LEAST_PIECE, f.piece / 2 / LEAST_PIECE * LEAST_PIECE);
    // pieces of about one size
    const int64_t n = std::max<int64_t>(1, ceil_div(d->rows, f.piece));
    f.piece = std::max(LEAST_PIECE, ceil_div(ceil_div(d->rows, n), LEAST_PIECE) * LEAST_PIECE);
    f.lines = ceil_div(d->in_features, 8);
    const bool pays = copy_pays(d->rows, d->in_features, d->classes, gradients ? PRODUCTS_GRADIENTS : PRODUCTS_LOSS) && (f.piece + d->classes) * f.lines / 256 < MOST_WORKGROUPS - 16;
    f.pack_x = pays && !dlf_ff_lines(nullptr, f.d.x_stride, d->in_features);
    f.pack_w = pays && !dlf_ff_lines(nullptr, f.d.w_stride, d->in_features);
    return DLF_OK;
}

dlf_status check_ptr(const Ce& f, const void* p, const char* name, bool wanted, uintptr_t align)
{
    if (!p && wanted) return fail(DLF_ERR_INVALID_ARG, "%s: null %s", f.call, name);
    if (((uintptr_t)p & (align - 1)) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: %s is not aligned to %d bytes", f.call, name, (int)align);
    return DLF_OK;
}
dlf_status check_ws(const Ce& f, const void* ws, size_t have, size_t need)
{
    if (need == 0) return DLF_OK;
    if (have < need) return fail(DLF_ERR_OOM, "%s: workspace too small: %zu < %zu", f.call, have, need);
    if (!ws || ((uintptr_t)ws & 255) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: workspace must be a 256-byte aligned device pointer", f.call);
    return DLF_OK;
}
dlf_status launched(const Ce& f, int e)
{
    if (e != 0) return fail(DLF_ERR_HIP, "%s: launch failed: %s", f.call, hipGetErrorString((hipError_t)e));
    return DLF_OK;
}

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
    std::call_once(g_once[device], [device] { g_once_rc[device] = dlf_ce_kernels_init(); });
    if (g_once_rc[device] != 0) return fail(DLF_ERR_HIP, "kernel setup failed: %s", hipGetErrorString((hipError_t)g_once_rc[device]));
    return DLF_OK;
}

// The tiles of a piece's logits.  any: the operands' rows start anywhere.
DlfFfCut cut_of(const Ce& f, int64_t rows, bool any) { return dlf_ff_whole_cut(rows, f.d.classes, f.d.in_features, any); }
int64_t parts_of(const Ce& f, const DlfFfCut& c) { return ceil_div(f.d.classes, dlf_ce_width(c.shape)); }

// Few rows: the weight's gradient, each row of which is the product of one or two elements of dz and their rows of x, would be off by those elements'
// roundings (0.0027 of its norm rather than 0.0017, bf16).  It is multiplied from dz and what its rounding took, as a sum of twice as many rows, which costs
// next to nothing beside the bytes of the result.
bool twice(const Ce& f) { return f.d.rows <= DLF_FF_FEW_ROWS; }

// What a call keeps in the workspace, for its largest piece (column sums: for all of them); addresses are not known where its size is asked for.
struct Layout {
    size_t x = 0, w = 0, z = 0, part = 0, at = 0, lse = 0, inverse = 0, unit = 0, rest = 0, dz = 0, low = 0, sums = 0, sum = 0, join = 0, bytes = 0;
    size_t take(size_t n)
    {
        const size_t here = bytes;
        bytes += align256(n);
        return here;
    }
};
// logits: their parts are needed; gradients: what the gradients need; kept: the logits in 32 bits
Layout layout_of(const Ce& f, bool logits, bool gradients, bool kept = false)
{
    Layout l;
    const int64_t most = std::min(f.piece, f.d.rows), nc = f.d.classes;
    if (most == 0) return l;
    int64_t parts = dlf_ff_is_few(most) ? ceil_div(nc, 16) : 0, chunks = 0;
    // the last piece may be cut otherwise than the others, and few rows are
    for (const int64_t rows : {most, f.rows(f.pieces() - 1)})
        for (const bool any : {false, true}) {
            const DlfFfCut c = cut_of(f, rows, any);
            parts = std::max(parts, ceil_div(parts_of(f, c) * rows, most));
            if (dlf_ff_is_few(rows)) parts = std::max(parts, ceil_div(ceil_div(nc, 16) * rows, most));
            chunks = std::max<int64_t>(chunks, (int64_t)c.tiles_r * 2);
        }
    if (f.pack_x) l.x = l.take((size_t)most * f.lines * 16);
    if (f.pack_w) l.w = l.take((size_t)nc * f.lines * 16);
    if (logits) {
        l.part = l.take((size_t)parts * most * 8);
        l.at = l.take((size_t)most * 4);
        l.lse = l.take((size_t)most * 4);
    }
    if (!gradients) return l;
    if (kept || dlf_ff_is_few(most)) l.z = l.take((size_t)most * f.ldz * 4);
    l.inverse = l.take((size_t)most * 4);
    l.unit = l.take(8);
    l.rest = l.take((size_t)most * 4);
    l.dz = l.take((size_t)most * f.ldz * 2);
    if (twice(f)) l.low = l.take((size_t)most * f.ldz * 2);
    chunks = std::max(chunks, ceil_div(most, DLF_CE_DZ_ROWS));
    l.sums = l.take((size_t)(1 + chunks) * nc * 4);         // the pieces' in front, the piece's chunks
    if (f.pieces() > 1) l.sum = l.take((size_t)nc * f.d.in_features * 4);
    size_t join = 0;
    for (const int64_t rows : {most, f.rows(f.pieces() - 1)})
        for (int k = 0; k < 8; ++k) {
            if (!(k & 3)) continue;
            const DlfFfBackCut c = dlf_ff_back_cut(rows, f.d.in_features, nc, k & 4, k & 1, k & 2);
            join = std::max(join, align256(c.w.part_bytes) + align256(c.x.part_bytes));
        }
    l.join = l.take(join);
    return l;
}

// A call's operands.
struct In {
    const void *x, *w;
    const float* bias;
    const int64_t* target;
};
// ... those of a piece, as its products read them.
struct Piece {
    int64_t first, rows;
    const void *x, *w;
    int64_t ldx, ldw;
    bool whole;             // rows of whole lines
};
dlf_status piece_of(const Ce& f, const In& in, int64_t p, int products, const Layout& l, char* ws, Piece& q, void* stream)
{
    q.first = f.first(p);
    q.rows = f.rows(p);
    q.x = (const char*)in.x + q.first * f.d.x_stride * 2;
    q.w = in.w;
    q.ldx = f.d.x_stride;
    q.ldw = f.d.w_stride;
    const bool x = dlf_ff_lines(in.x, q.ldx, f.d.in_features), w = dlf_ff_lines(in.w, q.ldw, f.d.in_features);
    const bool pays = copy_pays(f.d.rows, f.d.in_features, f.d.classes, products);
    q.whole = (x || (f.pack_x && pays)) && (w || (f.pack_w && pays));
    if (!q.whole || (x && w) || q.rows == 0) return DLF_OK;
    DlfCePackArgs a;
    memset(&a, 0, sizeof a);
    a.k = f.d.in_features;
    a.parts = (int)f.lines;
    if (f.pack_x && !x) {
        a.m[0] = {q.x, ws + l.x, q.ldx, q.rows};
        q.x = ws + l.x;
        q.ldx = f.lines * 8;
    }
    if (f.pack_w && !w) {
        if (p == 0) a.m[1] = {q.w, ws + l.w, q.ldw, f.d.classes};
        q.w = ws + l.w;
        q.ldw = f.lines * 8;
    }
    return a.m[0].rows + a.m[1].rows > 0 ? launched(f, dlf_ce_start_pack(&a, stream)) : DLF_OK;
}
void product(const Ce& f, const In& in, const Piece& q, DlfCeArgs& a)
{
    memset(&a, 0, sizeof a);
    a.t.p[0] = q.w; a.t.q[0] = q.x;
    a.t.ldp = q.ldw; a.t.ldq = q.ldx;
    a.t.nr = (int)q.rows; a.t.nc = f.d.classes; a.t.nk = f.d.in_features;
    a.t.segments = a.t.problems = a.t.splits = 1;
    a.t.bias[0] = in.bias;
    a.target = in.target + q.first;
    a.ignore = f.d.ignore;
    a.ldz = f.ldz;
}
void set_cut(DlfFfArgs& a, const DlfFfCut& c)
{
    a.tiles_r = c.tiles_r;
    a.tiles_c = c.tiles_c;
}

// The parts of a piece's rows; keep: the exponentials too, in dz; z: the logits too, there.  tiles: by tiles also where the piece, a last one, has few
// rows: the kernels for few rows keep no exponentials.  -> the classes of a part
dlf_status logits(const Ce& f, const In& in, const Piece& q, bool tiles, bool keep, float* z, const Layout& l, char* ws, int& width, void* stream)
{
    DlfCeArgs a;
    product(f, in, q, a);
    a.part = (float*)(ws + l.part);
    a.at = (float*)(ws + l.at);
    a.z = z;
    if (!tiles && dlf_ff_is_few(q.rows)) {
        const DlfFfFew c = dlf_ff_few_cut(a.t);
        width = 16;
        return launched(f, dlf_ce_start_few(&a, &c, f.d.dtype, stream));
    }
    const DlfFfCut c = cut_of(f, q.rows, !q.whole);
    set_cut(a.t, c);
    if (keep) a.dz = ws + l.dz;
    width = dlf_ce_width(c.shape);
    return launched(f, dlf_ce_start_tile(&a, c.shape, f.d.dtype, keep ? DLF_CE_KEEP : z ? DLF_CE_LOGITS : DLF_CE_STAT, stream));
}
// ... and from them loss and lse, either of which may be null.
dlf_status join(const Ce& f, const In& in, const Piece& q, const Layout& l, char* ws, int width, float* loss, float* lse, float* inverse, void* stream)
{
    const DlfCeJoinArgs j = {(const float*)(ws + l.part), (const float*)(ws + l.at), in.target + q.first, f.d.ignore, (int)ceil_div(f.d.classes, width),
                             (int)q.rows, f.d.classes, loss, lse, inverse};
    return launched(f, dlf_ce_start_join(&j, stream));
}

struct Out {
    void *dx, *dw;
    float* db;
};
// The gradients of all rows: dz of a piece from the lse given, or with loss and lse computed on the way, then the products.
dlf_status gradients(const Ce& f, const In& in, const float* lse, DlfCeGiven given, float* loss, const Out& out, char* ws, void* stream)
{
    // Few rows: their logits are kept in 32 bits, which costs less than to form them again.
    const bool few = dlf_ff_is_few(f.d.rows);
    const Layout l = layout_of(f, lse == nullptr || few, true, lse == nullptr && f.d.dbias);
    const int64_t pieces = f.pieces(), nc = f.d.classes, k = f.d.in_features;
    const bool wanted = out.dx || out.dw || out.db;
    TRY(kernels_ready());
    if (!given.dlse && (!given.dloss || given.dloss_stride == 0)) {
        given.one = f.d.dtype == DLF_F16 ? 16384.0f : 1.0f;
    } else if (f.d.rows > 0 && f.d.dtype == DLF_F16 && wanted) {
        const DlfCeUnitArgs u = {given, in.target, f.d.ignore, f.d.rows, (float*)(ws + l.unit)};
        TRY(launched(f, dlf_ce_start_unit(&u, stream)));
        given.unit = u.unit;
    }
    float* const back = given.one > 0.0f && f.d.rows > 0 && wanted ? (float*)(ws + l.unit) : nullptr;
    // The exponentials are kept where they need not say what the bias's gradient is, which has 32 bits; where they do, the logits are.
    const bool keep = !lse && wanted && !out.db && !few, keep_logits = (few && wanted) || (!lse && out.db);
    for (int64_t p = 0; p < pieces; ++p) {
        int chunks = 0;
        Piece q;
        TRY(piece_of(f, in, p, PRODUCTS_GRADIENTS, l, ws, q, stream));
        DlfCeGiven g = given;
        if (g.dloss) g.dloss += q.first * g.dloss_stride;
        if (g.dlse) g.dlse += q.first * g.dlse_stride;
        if (q.rows > 0) {
            float* inverse = nullptr;
            const float* piece_lse = lse ? lse + q.first : nullptr;
            float* const piece_loss = loss ? loss + q.first : nullptr;
            int width = 0;
            if (!lse || keep_logits) TRY(logits(f, in, q, wanted && !few, keep, keep_logits ? (float*)(ws + l.z) : nullptr, l, ws, width, stream));
            const bool forms = few && wanted && !out.db && q.rows * ceil_div(nc, 16) <= MOST_PARTS_OF_FEW_ROWS;
            const int64_t chunk = std::min<int64_t>(q.rows, DLF_CE_DZ_ROWS);
            const bool sums_form = !lse && out.db && ceil_div(ceil_div(nc, width), dlf_ce_dz_groups((int)chunk)) <= MOST_PARTS_OF_A_THREAD &&
                                   ceil_div(f.ldz, 256) * ceil_div(q.rows, DLF_CE_DZ_ROWS) <= MOST_FORMING;
            if (!lse && !keep && !forms && !sums_form) {
                float* const to = (float*)(ws + l.lse);
                inverse = (float*)(ws + l.inverse);
                TRY(join(f, in, q, l, ws, width, piece_loss, to, inverse, stream));
                piece_lse = to;
            }
            if (!wanted) continue;
            DlfCeDzArgs z;
            memset(&z, 0, sizeof z);
            z.dz = ws + l.dz; z.ldz = f.ldz;
            z.part = (const float*)(ws + l.part); z.at = (const float*)(ws + l.at);
            z.nr = (int)q.rows; z.nc = (int)nc;
            z.slices = (int)ceil_div(f.ldz, DLF_CE_DZ_COLS);
            z.target = in.target + q.first; z.ignore = f.d.ignore;
            z.lse = piece_lse; z.inverse = inverse; z.loss = piece_loss;
            z.given = g; z.rest = (float*)(ws + l.rest); z.back = back;
            z.low = twice(f) ? ws + l.low : nullptr;
            if (width > 0) { z.width = width; z.parts = (int)ceil_div(nc, width); }
            if (keep_logits) {
                z.z = (const float*)(ws + l.z);
                if (out.db) z.sums = few ? out.db : (float*)(ws + l.sums) + nc;
                if (!few) chunks = (int)ceil_div(q.rows, DLF_CE_DZ_ROWS);
                TRY(launched(f, piece_lse || sums_form ? dlf_ce_start_dz_sums(&z, f.d.dtype, stream) : dlf_ce_start_dz(&z, f.d.dtype, stream)));
            } else if (keep) {
                if (q.rows * z.slices > MOST_FORMING_KEPT) {
                    float *const to = (float*)(ws + l.lse), *const of = (float*)(ws + l.inverse);
                    TRY(join(f, in, q, l, ws, width, piece_loss, to, of, stream));
                    z.lse = to;
                    z.inverse = of;
                }
                TRY(launched(f, dlf_ce_start_dz(&z, f.d.dtype, stream)));
            } else {
                DlfCeArgs a;
                product(f, in, q, a);
                const DlfFfCut c = cut_of(f, q.rows, !q.whole);
                set_cut(a.t, c);
                a.dz = ws + l.dz;
                a.lse = piece_lse;
                a.rest = (float*)(ws + l.rest);
                a.low = twice(f) ? ws + l.low : nullptr;
                a.given = g;
                a.back = back;
                if (out.db) a.sums = (float*)(ws + l.sums) + nc;
                chunks = c.tiles_r * 2;
                TRY(launched(f, dlf_ce_start_tile(&a, c.shape, f.d.dtype, DLF_CE_DZ, stream)));
            }
        }
        DlfCeBackArgs e;
        memset(&e, 0, sizeof e);
        DlfFfBackArgs& b = e.b;
        b.w.splits = b.x.splits = 1;
        const bool last = p == pieces - 1, want_x = out.dx && q.rows > 0, want_w = out.dw != nullptr;
        const char* const dz = q.rows > 0 ? ws + l.dz : nullptr;
        if (want_x) {
            DlfFfArgs& a = b.x;
            a.p[0] = q.w; a.q[0] = dz;
            a.ldp = q.ldw; a.ldq = f.ldz;
            a.nr = (int)q.rows; a.nc = (int)k; a.nk = (int)nc;
            a.segments = a.problems = 1;
            a.out[0] = (char*)out.dx + q.first * k * 2; a.ldo = k;
        }
        if (want_w) {
            DlfFfArgs& a = b.w;
            a.p[0] = q.x; a.q[0] = dz;
            a.ldp = q.ldx; a.ldq = f.ldz;
            a.nr = (int)nc; a.nc = (int)k; a.nk = (int)q.rows;
            a.segments = a.problems = 1;
            if (twice(f) && q.rows > 0) {
                a.segments = 2;
                a.p[1] = a.p[0]; a.q[1] = ws + l.low;
            }
            a.out[0] = out.dw; a.ldo = k;
        }
        if (out.db && !(few && q.rows > 0)) {
            // (of no rows nothing is read: zeros)
            float* const sums = chunks > 0 ? (float*)(ws + l.sums) : out.db;
            b.sum.part[0] = p > 0 ? sums : chunks > 0 ? sums + nc : sums;
            b.sum.out[0] = last ? out.db : sums;
            b.sum.n = (int)nc;
            b.sum.chunks = chunks + (p > 0 ? 1 : 0);
            b.sum.blocks = (int)ceil_div(nc, 64);
        }
        if (!want_x && !want_w && b.sum.blocks == 0) continue;
        // (dz has rows of whole lines, zeros behind the last class: only the other operands decide)
        const DlfFfBackCut c = dlf_ff_back_cut(std::max<int64_t>(1, q.rows), k, nc, (want_x || want_w) && !q.whole, want_w, want_x);
        b.x_first = c.x_first;
        set_cut(b.w, c.w);
        set_cut(b.x, c.x);
        b.w.splits = c.w.splits;
        b.x.splits = c.x.splits;
        b.w.part = (float*)(ws + l.join);
        b.x.part = (float*)(ws + l.join + align256(c.w.part_bytes));
        if (!want_w) { b.w.problems = 0; b.w.splits = 1; }
        if (!want_x) { b.x.problems = 0; b.x.splits = 1; }
        if (want_x) {
            e.rest = (const float*)(ws + l.rest);
            e.target = in.target + q.first;
        }
        e.back = back ? back : given.unit ? given.unit + 1 : nullptr;
        if (want_w && pieces > 1) {
            e.sum = (float*)(ws + l.sum);
            e.add = p > 0;
            e.keep = !last;
        }
        TRY(launched(f, dlf_ce_start_back(&e, c.w.shape, f.d.dtype, stream)));
    }
    return DLF_OK;
}

size_t bytes_of(const dlf_ce_desc* d, bool logits, bool gradients, bool kept, const char* call)
{
    Ce f;
    return check_desc(d, gradients, call, f) == DLF_OK ? layout_of(f, logits, gradients, kept && d->dbias).bytes : SIZE_MAX;
}
dlf_status check_in(const Ce& f, const In& in)
{
    const bool some = f.d.rows > 0;
    TRY(check_ptr(f, in.x, "x", some, 2));
    TRY(check_ptr(f, in.w, "weight", some, 2));
    TRY(check_ptr(f, in.bias, "bias", false, 4));
    return check_ptr(f, in.target, "target", some, 8);
}
dlf_status check_given(const Ce& f, const DlfCeGiven& g)
{
    TRY(check_ptr(f, g.dloss, "dloss", false, 4));
    TRY(check_ptr(f, g.dlse, "dlse", false, 4));
    if (g.dloss_stride < 0 || g.dlse_stride < 0 || g.dloss_stride > (int64_t)1 << 24 || g.dlse_stride > (int64_t)1 << 24)
        return fail(DLF_ERR_INVALID_ARG, "%s: dloss and dlse lie %lld and %lld apart", f.call, (long long)g.dloss_stride, (long long)g.dlse_stride);
    if (!g.dloss && !(std::fabs(g.dloss_value) <= 3e38f)) return fail(DLF_ERR_INVALID_ARG, "%s: dloss is not finite", f.call);
    return DLF_OK;
}
dlf_status check_out(const Ce& f, const Out& o)
{
    TRY(check_ptr(f, o.dx, "dx", false, 2));
    TRY(check_ptr(f, o.dw, "dweight", false, 2));
    return check_ptr(f, o.db, "dbias", false, 4);
}

}  // namespace

extern "C" {

size_t dlf_cross_entropy_workspace_bytes(const dlf_ce_desc* d) { return bytes_of(d, true, false, false, "dlf_cross_entropy_workspace_bytes"); }
size_t dlf_cross_entropy_backward_workspace_bytes(const dlf_ce_desc* d)
{
    return bytes_of(d, d && dlf_ff_is_few(d->rows), true, false, "dlf_cross_entropy_backward_workspace_bytes");
}
size_t dlf_cross_entropy_gradients_workspace_bytes(const dlf_ce_desc* d) { return bytes_of(d, true, true, true, "dlf_cross_entropy_gradients_workspace_bytes"); }

dlf_status dlf_cross_entropy(const dlf_ce_desc* d, const void* x, const void* weight, const float* bias, const int64_t* target, float* loss,
                             float* lse, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    Ce f;
    TRY(check_desc(d, false, "dlf_cross_entropy", f));
    const In in = {x, weight, bias, target};
    TRY(check_in(f, in));
    TRY(check_ptr(f, loss, "loss", f.d.rows > 0, 4));
    TRY(check_ptr(f, lse, "lse", false, 4));
    const Layout l = layout_of(f, true, false);
    TRY(check_ws(f, workspace, workspace_bytes, l.bytes));
    if (f.d.rows == 0) return DLF_OK;
    TRY(kernels_ready());
    for (int64_t p = 0; p < f.pieces(); ++p) {
        Piece q;
        int width;
        TRY(piece_of(f, in, p, PRODUCTS_LOSS, l, (char*)workspace, q, hip_stream));
        TRY(logits(f, in, q, false, false, nullptr, l, (char*)workspace, width, hip_stream));
        TRY(join(f, in, q, l, (char*)workspace, width, loss + q.first, lse ? lse + q.first : nullptr, nullptr, hip_stream));
    }
    return DLF_OK;
}

dlf_status dlf_cross_entropy_backward(const dlf_ce_desc* d, const void* x, const void* weight, const float* bias, const int64_t* target,
                                      const float* lse, const float* dloss, int64_t dloss_stride, float dloss_value, const float* dlse,
                                      int64_t dlse_stride, void* dx, void* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                                      void* hip_stream)
{
    Ce f;
    TRY(check_desc(d, true, "dlf_cross_entropy_backward", f));
    const In in = {x, weight, bias, target};
    const DlfCeGiven given = {dloss, dlse, dloss_stride, dlse_stride, dloss_value, nullptr, 0.0f};
    const Out out = {dx, dweight, dbias};
    TRY(check_in(f, in));
    TRY(check_ptr(f, lse, "lse", f.d.rows > 0, 4));
    TRY(check_given(f, given));
    TRY(check_out(f, out));
    TRY(check_ws(f, workspace, workspace_bytes, layout_of(f, dlf_ff_is_few(f.d.rows), true).bytes));
    static const float none = 0.0f;                         // (of no rows nothing is read)
    return gradients(f, in, lse ? lse : &none, given, nullptr, out, (char*)workspace, hip_stream);
}

dlf_status dlf_cross_entropy_gradients(const dlf_ce_desc* d, const void* x, const void* weight, const float* bias, const int64_t* target,
                                       const float* dloss, int64_t dloss_stride, float dloss_value, float* loss, void* dx, void* dweight,
                                       float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    Ce f;
    TRY(check_desc(d, true, "dlf_cross_entropy_gradients", f));
    const In in = {x, weight, bias, target};
    const DlfCeGiven given = {dloss, nullptr, dloss_stride, 0, dloss_value, nullptr, 0.0f};
    const Out out = {dx, dweight, dbias};
    TRY(check_in(f, in));
    TRY(check_given(f, given));
    TRY(check_ptr(f, loss, "loss", f.d.rows > 0, 4));
    TRY(check_out(f, out));
    if (dbias && !f.d.dbias) return fail(DLF_ERR_INVALID_ARG, "%s: dbias is not in the description", f.call);
    TRY(check_ws(f, workspace, workspace_bytes, layout_of(f, true, true, f.d.dbias).bytes));
    return gradients(f, in, nullptr, given, loss, out, (char*)workspace, hip_stream);
}

}  // extern "C"
