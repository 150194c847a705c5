// Host side of the optimizer's operators: checks of the arguments, the table of chunks, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "dlf_opt.h"

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

constexpr int64_t MOST_OF_ONE = (int64_t)1 << 40, MOST_OF_ALL = (int64_t)1 << 42;

dlf_status launched(const char* call, int e)
{
    if (e != 0) return fail(DLF_ERR_HIP, "%s: launch failed: %s", call, hipGetErrorString((hipError_t)e));
    return DLF_OK;
}
int64_t chunks_of(int64_t count) { return (count + DLF_OPT_CHUNK - 1) / DLF_OPT_CHUNK; }
uintptr_t size_of(int dtype) { return dtype == DLF_F32 ? 4 : 2; }

dlf_status check_counts(const char* call, const int64_t* counts, int32_t n)
{
    if (n < 0 || (n > 0 && !counts)) return fail(DLF_ERR_INVALID_ARG, "%s: %d tensors", call, n);
    int64_t all = 0;
    for (int i = 0; i < n; ++i) {
        if (counts[i] < 0 || counts[i] > MOST_OF_ONE) return fail(DLF_ERR_INVALID_ARG, "%s: tensor %d has %lld elements", call, i, (long long)counts[i]);
        all += counts[i];
        if (all > MOST_OF_ALL) return fail(DLF_ERR_UNSUPPORTED, "%s: more than 2^42 elements", call);
    }
    return DLF_OK;
}
dlf_status check_gradient(const char* call, int i, const void* p, int32_t dtype, int64_t count, bool wanted)
{
    if (dtype != DLF_F16 && dtype != DLF_BF16 && dtype != DLF_F32) return fail(DLF_ERR_INVALID_ARG, "%s: gradient %d: dtype %d", call, i, dtype);
    if (!p && wanted && count > 0) return fail(DLF_ERR_INVALID_ARG, "%s: null gradient %d", call, i);
    if (((uintptr_t)p & (size_of(dtype) - 1)) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: gradient %d is not aligned to its elements", call, i);
    return DLF_OK;
}

// The launches of a norm: for each, f(first tensor, tensors, chunks, workgroups).  (A launch's chunks are counted in 32 bits.)
template <typename F> dlf_status each_norm(const int64_t* counts, int32_t n, F&& f)
{
    for (int i = 0; i < n;) {
        int64_t chunks = 0;
        int k = 0;
        for (; i + k < n && k < DLF_OPT_NORM_TENSORS && chunks + chunks_of(counts[i + k]) < (int64_t)1 << 31; ++k) chunks += chunks_of(counts[i + k]);
        if (chunks > 0) TRY(f(i, k, (int)chunks, (int)std::min<int64_t>(chunks, DLF_OPT_GROUPS)));
        i += k;
    }
    return DLF_OK;
}

dlf_status check_tensors(const char* call, const dlf_adamw_tensor* t, int32_t n)
{
    if (n < 0 || (n > 0 && !t)) return fail(DLF_ERR_INVALID_ARG, "%s: %d tensors", call, n);
    int64_t all = 0;
    for (int i = 0; i < n; ++i) {
        const dlf_adamw_tensor& q = t[i];
        if (q.count < 0 || q.count > MOST_OF_ONE) return fail(DLF_ERR_INVALID_ARG, "%s: tensor %d has %lld elements", call, i, (long long)q.count);
        all += q.count;
        if (all > MOST_OF_ALL) return fail(DLF_ERR_UNSUPPORTED, "%s: more than 2^42 elements", call);
        if (q.param_dtype != DLF_F16 && q.param_dtype != DLF_BF16 && q.param_dtype != DLF_F32)
            return fail(DLF_ERR_INVALID_ARG, "%s: parameter %d: dtype %d", call, i, q.param_dtype);
        if (q.reserved != 0) return fail(DLF_ERR_INVALID_ARG, "%s: tensor %d: reserved is not 0", call, i);
        if (!(std::fabs(q.decay) <= 3e38f)) return fail(DLF_ERR_INVALID_ARG, "%s: tensor %d: decay is not finite", call, i);
        if (!q.param && q.count > 0) return fail(DLF_ERR_INVALID_ARG, "%s: null parameter %d", call, i);
        if (((uintptr_t)q.param & (size_of(q.param_dtype) - 1)) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: parameter %d is not aligned to its elements", call, i);
        if (!q.copy) continue;
        if (q.param_dtype != DLF_F32 || (q.copy_dtype != DLF_F16 && q.copy_dtype != DLF_BF16))
            return fail(DLF_ERR_INVALID_ARG, "%s: copy %d: an fp16 or bf16 copy of an fp32 parameter expected", call, i);
        if (((uintptr_t)q.copy & 1) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: copy %d is not aligned to its elements", call, i);
    }
    return DLF_OK;
}
int64_t on_blocks(int64_t count) { return (count + DLF_ADAMW_BLOCK - 1) / DLF_ADAMW_BLOCK * DLF_ADAMW_BLOCK; }

}  // namespace

extern "C" {

size_t dlf_gradient_norm_workspace_bytes(const int64_t* counts, int32_t n)
{
    if (check_counts("dlf_gradient_norm_workspace_bytes", counts, n) != DLF_OK) return SIZE_MAX;
    size_t parts = 0;
    each_norm(counts, n, [&](int, int, int, int groups) { parts += (size_t)groups; return DLF_OK; });
    return (parts * 8 + 255) & ~(size_t)255;
}

dlf_status dlf_gradient_norm(const void* const* gradients, const int64_t* counts, const int32_t* dtypes, int32_t n, float most, float scale,
                             float* norm, float* factor, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const char* const call = "dlf_gradient_norm";
    TRY(check_counts(call, counts, n));
    if (n > 0 && (!gradients || !dtypes)) return fail(DLF_ERR_INVALID_ARG, "%s: null list", call);
    for (int i = 0; i < n; ++i) TRY(check_gradient(call, i, gradients[i], dtypes[i], counts[i], true));
    if (!(most >= 0)) return fail(DLF_ERR_INVALID_ARG, "%s: most is %g", call, (double)most);
    if (!(std::fabs(scale) <= 3e38f)) return fail(DLF_ERR_INVALID_ARG, "%s: scale is not finite", call);
    if (!norm || ((uintptr_t)norm & 3) != 0 || ((uintptr_t)factor & 3) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: norm and factor are one fp32 each", call);
    const size_t need = dlf_gradient_norm_workspace_bytes(counts, n);
    if (need > 0 && workspace_bytes < need) return fail(DLF_ERR_OOM, "%s: workspace too small: %zu < %zu", call, workspace_bytes, need);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) != 0))
        return fail(DLF_ERR_INVALID_ARG, "%s: workspace must be a 256-byte aligned device pointer", call);
    double* part = (double*)workspace;
    DlfNormJoinArgs j = {part, 0, most, scale, norm, factor};
    TRY(each_norm(counts, n, [&](int first, int tensors, int chunks, int groups) {
        DlfNormArgs a;
        memset(&a, 0, sizeof a);
        int at = 0;
        for (int i = 0; i < tensors; ++i) {
            if (counts[first + i] == 0) continue;           // (every tensor of a launch has a chunk, which a search can find)
            a.g[a.tensors] = gradients[first + i];
            a.n[a.tensors] = counts[first + i];
            a.type[a.tensors] = (uint8_t)dtypes[first + i];
            a.first[a.tensors++] = at;
            at += (int)chunks_of(counts[first + i]);
        }
        a.chunks = chunks;
        a.part = part + j.parts;
        j.parts += groups;
        return launched(call, dlf_opt_start_norm(&a, groups, hip_stream));
    }));
    return launched(call, dlf_opt_start_norm_join(&j, hip_stream));
}

size_t dlf_adamw_state_elements(const dlf_adamw_tensor* tensors, int32_t n)
{
    if (check_tensors("dlf_adamw_state_elements", tensors, n) != DLF_OK) return SIZE_MAX;
    int64_t all = 0;
    for (int i = 0; i < n; ++i) all += on_blocks(tensors[i].count);
    return (size_t)all;
}

size_t dlf_adamw_table_bytes(const dlf_adamw_tensor* tensors, int32_t n)
{
    if (check_tensors("dlf_adamw_table_bytes", tensors, n) != DLF_OK) return SIZE_MAX;
    int64_t all = 0;
    for (int i = 0; i < n; ++i) all += chunks_of(tensors[i].count);
    return (size_t)all * sizeof(DlfOptChunk);
}

dlf_status dlf_adamw_table(const dlf_adamw_tensor* tensors, int32_t n, void* host_table, size_t bytes)
{
    const char* const call = "dlf_adamw_table";
    TRY(check_tensors(call, tensors, n));
    const size_t need = dlf_adamw_table_bytes(tensors, n);
    if (bytes < need || (need > 0 && !host_table)) return fail(DLF_ERR_OOM, "%s: table too small: %zu < %zu", call, bytes, need);
    char* to = (char*)host_table;
    int64_t state = 0;
    for (int i = 0; i < n; ++i) {
        const dlf_adamw_tensor& t = tensors[i];
        for (int64_t at = 0; at < t.count; at += DLF_OPT_CHUNK, to += sizeof(DlfOptChunk)) {
            DlfOptChunk c;
            memset(&c, 0, sizeof c);
            c.p = (char*)t.param + at * (int64_t)size_of(t.param_dtype);
            c.c = t.copy ? (char*)t.copy + at * 2 : nullptr;
            c.state = state + at;
            c.at = at;
            c.n = (int32_t)std::min<int64_t>(DLF_OPT_CHUNK, t.count - at);
            c.tensor = i;
            c.decay = t.decay;
            c.p_type = (uint8_t)t.param_dtype;
            c.c_type = (uint8_t)(t.copy ? t.copy_dtype : 0);
            memcpy(to, &c, sizeof c);                       // (a buffer of any alignment)
        }
        state += on_blocks(t.count);
    }
    return DLF_OK;
}

dlf_status dlf_adamw_step(const dlf_adamw_desc* d, const dlf_adamw_tensor* tensors, int32_t n, const void* table, const void* const* gradients,
                          const int32_t* gradient_dtypes, void* m, void* v, float* m_scale, float* v_scale, double* counter, float rate,
                          const float* rate_at, const float* factor, void* hip_stream)
{
    const char* const call = "dlf_adamw_step";
    if (!d) return fail(DLF_ERR_INVALID_ARG, "%s: null description", call);
    if (!(d->beta1 >= 0 && d->beta1 < 1 && d->beta2 >= 0 && d->beta2 < 1)) return fail(DLF_ERR_INVALID_ARG, "%s: betas %g, %g", call, d->beta1, d->beta2);
    // (the reciprocal's instruction takes numbers from 2^-126 on, and gives none below)
    if (!(d->eps == 0 || (d->eps >= 0x1p-126f && d->eps <= 0x1p126f))) return fail(DLF_ERR_INVALID_ARG, "%s: eps %g", call, (double)d->eps);
    if (d->state != DLF_ADAMW_FP32 && d->state != DLF_ADAMW_8BIT) return fail(DLF_ERR_INVALID_ARG, "%s: state %d", call, d->state);
    if (d->reserved != 0) return fail(DLF_ERR_INVALID_ARG, "%s: reserved is not 0", call);
    TRY(check_tensors(call, tensors, n));
    if (n > 0 && (!gradients || !gradient_dtypes)) return fail(DLF_ERR_INVALID_ARG, "%s: null list", call);
    const bool small = d->state == DLF_ADAMW_8BIT;
    bool any = false;
    for (int i = 0; i < n; ++i) {
        if (gradients[i]) TRY(check_gradient(call, i, gradients[i], gradient_dtypes[i], tensors[i].count, false));
        any = any || tensors[i].count > 0;
    }
    if (any && (!table || !m || !v || ((uintptr_t)table & 15) != 0 || ((uintptr_t)m & 15) != 0 || ((uintptr_t)v & 15) != 0))
        return fail(DLF_ERR_INVALID_ARG, "%s: table, m and v are 16-byte aligned device pointers", call);
    if (any && small && (!m_scale || !v_scale || ((uintptr_t)m_scale & 15) != 0 || ((uintptr_t)v_scale & 15) != 0))
        return fail(DLF_ERR_INVALID_ARG, "%s: m_scale and v_scale are 16-byte aligned device pointers", call);
    if (!counter || ((uintptr_t)counter & 7) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: counter is an 8-byte aligned device pointer", call);
    if (((uintptr_t)rate_at & 3) != 0 || ((uintptr_t)factor & 3) != 0) return fail(DLF_ERR_INVALID_ARG, "%s: rate_at and factor are one fp32 each", call);
    if (!rate_at && !(std::fabs(rate) <= 3e38f)) return fail(DLF_ERR_INVALID_ARG, "%s: rate is not finite", call);
    DlfStepArgs a;
    memset(&a, 0, sizeof a);
    a.m = m; a.v = v; a.m_scale = m_scale; a.v_scale = v_scale; a.counter = counter;
    a.rate_at = rate_at; a.factor = factor; a.rate = rate;
    a.beta1 = d->beta1; a.beta2 = d->beta2;
    a.b1 = (float)d->beta1; a.c1 = (float)(1.0 - d->beta1);
    a.b2 = (float)d->beta2; a.c2 = (float)(1.0 - d->beta2);
    a.eps = d->eps; a.seed = d->seed;
    const DlfOptChunk* at = (const DlfOptChunk*)table;
    // (the last launch counts the step, also where it has no chunks, or no tensors)
    int i = 0;
    do {
        int64_t chunks = 0;
        int k = 0;
        for (; i + k < n && k < DLF_OPT_STEP_TENSORS && chunks + chunks_of(tensors[i + k].count) < (int64_t)1 << 31; ++k) {
            a.g[k] = gradients[i + k];
            a.type[k] = (uint8_t)(gradients[i + k] ? gradient_dtypes[i + k] : 0);
            chunks += chunks_of(tensors[i + k].count);
        }
        a.table = at;
        a.chunks = (int32_t)chunks;
        a.first_tensor = i;
        i += k;
        at += chunks;
        a.last = i >= n ? 1 : 0;
        if (chunks > 0 || a.last)
            TRY(launched(call, dlf_opt_start_step(&a, small ? 1 : 0, (int)std::max<int64_t>(1, std::min<int64_t>(chunks, DLF_OPT_GROUPS)), hip_stream)));
    } while (i < n);
    return DLF_OK;
}

}  // extern "C"
