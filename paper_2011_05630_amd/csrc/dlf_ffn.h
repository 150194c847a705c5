// Shared between the host side of the feed-forward operators (dlf_ffn.cpp) and their kernels (dlf_ffn.hip).
//
// Every product of the operators is C[r][c] = sum over k of Q[r][k] * P[c][k], c running along the rows of C in memory:
//   forward            r = token, c = output feature, k = input feature:   Q = x,  P = weight   both with k along the row
//   gradient of x      r = token, c = input feature,  k = output feature:  Q = dz, P = weight   P with k across the rows ("T")
//   gradient of weight r = output feature, c = input feature, k = token:   Q = dz, P = x        both with k across the rows
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/dlf.h"

struct DlfFfArgs {
    const void* p[2];       // two of them: gate and up (gated), or the operands of the second segment / problem
    const void* q[2];
    int64_t ldp, ldq;       // elements between the rows of P and Q as they lie in memory
    int32_t nr, nc, nk;
    int32_t segments;       // 2: the sum runs over (p[0], q[0]) and then over (p[1], q[1])
    int32_t problems;       // 2: two products of one shape, (p[0], q[0]) -> out[0] and (p[1], q[1]) -> out[1]
    int32_t tiles_r, tiles_c;
    int32_t splits;         // > 1: as many workgroups share a tile's k and leave their sums in part, which a second launch adds up
    float* part;            // [splits][planes][nr][nc], planes: gate and up, or problems
    // epilogue
    const float* bias[2];
    const void* res;
    int64_t ldres;
    void* out[2];
    int64_t ldo;
    float* saved;           // pre-activations, [1 or 2][nr][nc], or null
    int32_t act;
};

// dz = dy * act'(z), gated: dg = dh * u * act'(g), du = dh * act(g); and the column sums of either in 32 bits.
struct DlfFfDzArgs {
    const void* dy;
    int64_t lddy;
    const float* saved;     // null: dz = dy, only the sums are wanted
    void* dz[2];            // rows of lddz elements, a multiple of eight, zeros behind column n
    int64_t lddz;
    int32_t rows, n, act;
    int32_t chunk;          // rows of one partial sum
    float* sums[2];         // [chunks][n], or null
};
// The partial sums of the columns added up.
struct DlfFfSumArgs {
    const float* part[2];   // [chunks][n]; null: none
    float* out[2];
    int32_t n, chunks, blocks;   // blocks: workgroups of 64 columns, over both
};
// What one launch of the backward pass does: tiles of the weights' gradients, of the input's, column sums; each may be none (no tiles).
struct DlfFfBackArgs {
    DlfFfArgs w, x;
    DlfFfSumArgs sum;
    int32_t blocks_w, blocks_x;  // workgroups of either; the sums' come last
    int32_t x_first;             // x's tiles are the longer ones and start first, else w's
};

// Partial column sums: of at most this many parts, of at least so many rows (those that a workgroup of k_ff_dz takes at a time).
#define DLF_FF_MAX_CHUNKS 64
#define DLF_FF_CHUNK_ROWS 8

// Shapes of the tile kernel: a workgroup's part of C (columns x rows; gated: half as many columns of both projections) and the stages of
// 64 k that LDS holds.  ANY: for rows that start anywhere.
struct DlfFfShape { int bc, br, stages; };
enum { DLF_FF_SHAPE_256 = 0, DLF_FF_SHAPE_128 = 1, DLF_FF_SHAPE_ANY = 2, DLF_FF_SHAPE_128_DEEP = 3, DLF_FF_SHAPE_ANY64 = 4, DLF_FF_SHAPE_ANY64G = 5,
       DLF_FF_NUM_SHAPES = 6 };      // ANY64G: gated products only, ANY64: all others
static constexpr DlfFfShape DLF_FF_SHAPES[DLF_FF_NUM_SHAPES] = {{256, 256, 2}, {128, 128, 2}, {128, 128, 2}, {128, 128, 4}, {64, 64, 2}, {64, 128, 2}};

// Forward products of few rows: on k_ff_rows (operands of whole lines) or k_ff_few, 16 nf features x 16 mr rows (each 1 or 2) per workgroup.
#define DLF_FF_FEW_ROWS 64
struct DlfFfFew { int rows, nf, mr, waves; };
// k_ff_rows: stages of 64 k that a wave holds in LDS (the kernel with 2, 3 and 4 of them: 16 x 5632 -> 2048 takes 7.2, 7.1 and 7.5 us, 1 x 4096 ->
// 2 x 10880 gated 32.1, 31.5 and 35.4, 16 x 2048 -> 2 x 5632 gated 10.1, 11.1 and 12.9: with more, fewer workgroups share a compute unit, and
// eight waves of 32 features and 32 rows would pass its LDS); LDS of a workgroup.
#define DLF_FF_ROWS_RING 2
#define DLF_FF_ROWS_LDS(WAVES, NF, MR, GATED) ((WAVES) * DLF_FF_ROWS_RING * (((GATED) ? 2 : (NF)) + (MR)) * 2048)

extern "C" {
int dlf_ff_kernels_init(void);
int dlf_ff_start_tile(const DlfFfArgs* a, int shape, int dtype, int gated, void* stream);
int dlf_ff_start_back(const DlfFfBackArgs* a, int shape, int dtype, void* stream);
int dlf_ff_start_few(const DlfFfArgs* a, const DlfFfFew* c, int dtype, int gated, void* stream);
int dlf_ff_start_dz(const DlfFfDzArgs* a, int dtype, int gated, void* stream);
}

// Sets the message of dlf_last_error and returns the status (dlf_host.cpp).
__attribute__((visibility("hidden"))) dlf_status dlf_set_error(dlf_status s, const char* msg);
