// How the products of the feed-forward operators are cut, for other operators that launch tiles of their own (dlf_ffn.cpp).
#pragma once
#include "dlf_ffn.h"

// How a product of these sizes is cut: a tile shape and the workgroups that share a tile's k.
struct DlfFfCut {
    int shape = DLF_FF_SHAPE_128, splits = 1, tiles_r = 0, tiles_c = 0;
    size_t part_bytes = 0;
    int64_t tiles() const { return (int64_t)tiles_r * tiles_c; }
};
// The two products of a backward pass in one launch: both in tiles of one shape.
struct DlfFfBackCut {
    DlfFfCut w, x;
    bool x_first = false;
};
// Whether the tile kernel takes an operand: rows in whole 16-byte lines, offsets inside a tile that fit 31 bits.
inline bool dlf_ff_lines(const void* p, int64_t ld, int64_t row)
{
    return ((uintptr_t)p & 15) == 0 && (ld & 7) == 0 && (row & 7) == 0 && ld < (int64_t)1 << 22;
}

#define DLF_HIDDEN __attribute__((visibility("hidden")))
// any: the operands' rows start anywhere.
DLF_HIDDEN bool dlf_ff_is_few(int64_t rows);
DLF_HIDDEN DlfFfFew dlf_ff_few_cut(const DlfFfArgs& a);
// A forward product whose tiles each have all of k.
DLF_HIDDEN DlfFfCut dlf_ff_whole_cut(int64_t nr, int64_t nc, int64_t nk, bool any);
DLF_HIDDEN DlfFfBackCut dlf_ff_back_cut(int64_t rows, int64_t in, int64_t out, bool any, bool want_w, bool want_x);
