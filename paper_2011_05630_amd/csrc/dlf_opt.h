// Shared between the host side of the optimizer's operators (dlf_opt.cpp) and their kernels (dlf_opt.hip).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/dlf.h"

// A workgroup takes this many consecutive elements of one tensor at a time: a whole number of the states' blocks, 16 of a thread.
#define DLF_OPT_CHUNK 4096
// Tensors of one launch, whose addresses travel in its arguments (below 4 KB).
#define DLF_OPT_NORM_TENSORS 160
#define DLF_OPT_STEP_TENSORS 384
// Workgroups of one launch: eight to a compute unit, which take chunks in turn.
#define DLF_OPT_GROUPS 2048

struct DlfNormArgs {
    const void* g[DLF_OPT_NORM_TENSORS];
    int64_t n[DLF_OPT_NORM_TENSORS];
    int32_t first[DLF_OPT_NORM_TENSORS];    // the tensor's first chunk in this launch
    uint8_t type[DLF_OPT_NORM_TENSORS];
    int32_t tensors, chunks;
    double* part;                           // one sum of each workgroup
};
struct DlfNormJoinArgs {
    const double* part;
    int32_t parts;
    float most, scale;
    float *norm, *factor;
};

// A chunk as the table on the device holds it.
struct DlfOptChunk {
    void *p, *c;            // the chunk's first parameter and its copy, or null
    int64_t state;          // ... its place in m and v
    int64_t at;             // ... in its tensor
    int32_t n, tensor;      // elements, tensor
    float decay;
    uint8_t p_type, c_type, pad[2];
};
struct DlfStepArgs {
    const void* g[DLF_OPT_STEP_TENSORS];    // null: the tensor is left as it is
    uint8_t type[DLF_OPT_STEP_TENSORS];
    const DlfOptChunk* table;
    int32_t chunks, first_tensor;
    void *m, *v;
    float *m_scale, *v_scale;
    double* counter;        // steps done, beta1 and beta2 to their power, workgroups that have ended (32 bits)
    const float *rate_at, *factor;
    float rate, b1, c1, b2, c2, eps;
    double beta1, beta2;
    uint32_t seed;
    int32_t last;           // the step's last launch: it counts the step
};

extern "C" {
int dlf_opt_start_norm(const DlfNormArgs* a, int groups, void* stream);
int dlf_opt_start_norm_join(const DlfNormJoinArgs* a, void* stream);
int dlf_opt_start_step(const DlfStepArgs* a, int small, int groups, void* stream);
}

__attribute__((visibility("hidden"))) dlf_status dlf_set_error(dlf_status s, const char* msg);
