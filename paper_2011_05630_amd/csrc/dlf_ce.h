// Shared between the host side of the cross entropy of a linear layer (dlf_ce.cpp) and its kernels (dlf_ce.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "dlf_ffn.h"

// What a product's epilogue does with the logits of its tile.
enum { DLF_CE_STAT = 0,         // a maximum and a sum of exponentials of each row over a part of the classes, the target's logit
       DLF_CE_KEEP = 1,         // ... and the exponentials themselves, in 16 bits
       DLF_CE_DZ = 2,           // their gradient
       DLF_CE_LOGITS = 3 };     // STAT, and the logits themselves, in 32 bits
// A row's gradients of loss and lse as the caller gives them.
struct DlfCeGiven {
    const float *dloss, *dlse;  // null: dloss_value, none
    int64_t dloss_stride, dlse_stride;
    float dloss_value;
    const float* unit;          // {a power of two that dz is scaled by, its inverse}, or null
    float one;                  // > 0: dloss is the same for all rows and there is no dlse: dz is formed for a dloss of so much, see k_ce_back
};
// A matrix copied to rows of whole 16-byte lines, zeros behind column k.
struct DlfCePack {
    const void* from;
    void* to;
    int64_t stride, rows;       // no rows: nothing
};
struct DlfCePackArgs {
    DlfCePack m[2];
    int32_t k, parts;           // columns; lines of a row
};
struct DlfCeArgs {
    DlfFfArgs t;                // p: weight, q: x, bias
    const int64_t* target;
    int64_t ignore;
    float* part;                // [parts][nr] {maximum, sum of exp(z - maximum)}
    float* at;                  // [nr] the target's logit, of rows whose target is a class
    float* z;                   // few rows (where not null), LOGITS: [nr][ldz] the logits
    void* dz;                   // [nr][ldz], zeros behind column nc; KEEP: exp(z - its part's maximum) in 16 bits
    int64_t ldz;                // a multiple of eight
    const float *lse, *inverse; // DZ: p = exp(z - lse), lse as the caller gives it; inverse is null
    DlfCeGiven given;
    float* rest;                // [nr] what dz's rounding takes from a row's target, or null
    float* sums;                // [chunks][nc] column sums of dz, in 32 bits, or null
    float* back;                // what the products of dz are to be scaled by goes here, or null
    void* low;                  // what the rounding of dz takes from it, laid out as it, or null
};
struct DlfCeJoinArgs {
    const float* part;
    const float* at;
    const int64_t* target;
    int64_t ignore;
    int32_t parts, nr, nc;
    float *loss, *lse;          // either may be null
    float* inverse;             // null, or: the maximum goes to lse, 1 / the sum of exp(z - maximum) here
};
struct DlfCeDzArgs {
    void* dz;                   // KEEP's in, dz out
    const float* z;             // ... or the logits in, and nothing in dz
    int64_t ldz;
    const float* part;
    const float* at;
    int32_t parts, width;       // classes of a part
    int32_t nr, nc;
    int32_t slices;             // workgroups of a row, DLF_CE_DZ_COLS columns each
    const int64_t* target;
    int64_t ignore;
    const float* lse;           // or null: lse and loss are formed here, from the parts
    const float* inverse;       // p = exp(z - lse) * inverse (null: 1): a row's maximum is in lse then, 1 / its sum here; never null with exponentials kept
    float* loss;
    DlfCeGiven given;
    float *rest, *back;         // as in DlfCeArgs
    void* low;
    float* sums;                // of logits: [chunks of DLF_CE_DZ_ROWS][nc] column sums of dz, scaled back, or null
};
struct DlfCeUnitArgs {
    DlfCeGiven given;
    const int64_t* target;
    int64_t ignore, rows;
    float* unit;
};
struct DlfCeBackArgs {
    DlfFfBackArgs b;
    const float* back;          // the products are scaled by it; or null
    float* sum;                 // [classes][in] the weight's gradient over the pieces in front, or null
    int32_t add, keep;
    const float* rest;          // of dz, see DlfCeArgs; or null
    const int64_t* target;
};
// Classes of a part, by tile shape: what a wave's columns are.
static inline int dlf_ce_width(int shape) { return DLF_FF_SHAPES[shape].bc / 2; }
// Rows of a workgroup of k_ce_join, and up to how many rows a workgroup has one.
#define DLF_CE_JOIN_ROWS 16
#define DLF_CE_JOIN_FEW 256
// Columns of a workgroup of k_ce_dz.
#define DLF_CE_DZ_COLS 2048
// Rows of a workgroup of k_ce_dz_sums, which has 256 columns, and threads.
#define DLF_CE_DZ_ROWS 64
#define DLF_CE_DZ_THREADS 512
// How many of its threads share a row's parts where it forms their lse: those left when the next power of two of them take the rows.
__host__ __device__ static inline int dlf_ce_dz_groups(int rows)
{
    int n = DLF_CE_DZ_THREADS;
    for (int span = 1; span < rows; span *= 2) n /= 2;
    return n;
}

extern "C" {
int dlf_ce_kernels_init(void);
int dlf_ce_start_tile(const DlfCeArgs* a, int shape, int dtype, int mode, void* stream);
int dlf_ce_start_few(const DlfCeArgs* a, const DlfFfFew* c, int dtype, void* stream);
int dlf_ce_start_join(const DlfCeJoinArgs* a, void* stream);
int dlf_ce_start_dz(const DlfCeDzArgs* a, int dtype, void* stream);
int dlf_ce_start_dz_sums(const DlfCeDzArgs* a, int dtype, void* stream);
int dlf_ce_start_pack(const DlfCePackArgs* a, void* stream);
int dlf_ce_start_unit(const DlfCeUnitArgs* a, void* stream);
int dlf_ce_start_back(const DlfCeBackArgs* a, int shape, int dtype, void* stream);
}
