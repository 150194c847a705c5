// gfx950 (CDNA4) kernels of the optimizer's operators: the norm of all gradients, and AdamW over many tensors.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "dlf_opt.h"

typedef float f2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float from_bf16(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// Eight consecutive elements of which n exist, in 32 bits, zeros behind them.  Tensors start where they like: a 16-byte access of any
// alignment is one instruction here.
__device__ __forceinline__ void load8(const void* base, int64_t at, int n, int type, float (&f)[8])
{
    if (type == DLF_F32) {
        const float* p = (const float*)base + at;
        if (n >= 8) {
            __builtin_memcpy(f, p, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.0f;
        }
        return;
    }
    uint16_t h[8];
    const uint16_t* p = (const uint16_t*)base + at;
    if (n >= 8) {
        __builtin_memcpy(h, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < n ? p[i] : (uint16_t)0;
    }
    if (type == DLF_BF16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = from_bf16(h[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)__builtin_bit_cast(_Float16, h[i]);
    }
}
__device__ __forceinline__ void store8(void* base, int64_t at, int n, int type, const float (&f)[8])
{
    if (type == DLF_F32) {
        float* p = (float*)base + at;
        if (n >= 8) {
            __builtin_memcpy(p, f, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[i] = f[i];
        }
        return;
    }
    uint16_t h[8];
    uint16_t* p = (uint16_t*)base + at;
    if (type == DLF_BF16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = __builtin_bit_cast(uint16_t, (__bf16)f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = __builtin_bit_cast(uint16_t, (_Float16)f[i]);
    }
    if (n >= 8) {
        __builtin_memcpy(p, h, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = h[i];
    }
}

// The sum over a workgroup of 256 or 1024 threads, in a fixed order, for thread 0.
__device__ __forceinline__ double sum_of_all(double s, double* waves)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_down(s, d, 64);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += waves[w];
    return s;
}

// ------------------------------------------------------------------------------------------------
// k_norm, k_norm_join: sum of the squares of all elements, each once from memory, and its root.  Squares and sums are held in 64 bits: no
// gradient is too large or too small for its square, and the order of a sum does not show.  A workgroup leaves one sum, and one
// workgroup adds them up in order.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_norm(const DlfNormArgs a)
{
    __shared__ double waves[4];
    double s = 0.0;
    for (int k = blockIdx.x; k < a.chunks; k += gridDim.x) {
        int lo = 0, hi = a.tensors - 1;                     // the last tensor that starts at or in front of the chunk
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.first[mid] <= k) lo = mid;
            else hi = mid - 1;
        }
        const int type = a.type[lo];
        const int64_t at = (int64_t)(k - a.first[lo]) * DLF_OPT_CHUNK, left = a.n[lo] - at;
        const int n = left < DLF_OPT_CHUNK ? (int)left : DLF_OPT_CHUNK;
        float f[DLF_OPT_CHUNK / 2048][8];
#pragma unroll
        for (int u = 0; u < DLF_OPT_CHUNK / 2048; ++u) {
            const int e = u * 2048 + (int)threadIdx.x * 8;
            load8(a.g[lo], at + e, n - e, type, f[u]);
        }
#pragma unroll
        for (int u = 0; u < DLF_OPT_CHUNK / 2048; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fma((double)f[u][i], (double)f[u][i], s);
    }
    s = sum_of_all(s, waves);
    if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void k_norm_join(const DlfNormJoinArgs a)
{
    __shared__ double waves[16];
    double s = 0.0;
    for (int k = threadIdx.x; k < a.parts; k += 1024) s += a.part[k];
    s = sum_of_all(s, waves);
    if (threadIdx.x != 0) return;
    const double norm = fabs((double)a.scale) * sqrt(s);
    const float root = (float)norm;
    *a.norm = root;
    if (a.factor != nullptr)
        *a.factor = !(root <= 3.402823466e38f) ? __builtin_nanf("") : norm > (double)a.most ? (float)((double)a.scale * ((double)a.most / norm)) : a.scale;
}

// ------------------------------------------------------------------------------------------------
// k_step: AdamW.  One pass over parameters, gradients and states, bound by memory.
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g g,  p' = p (1 - rate decay) - rate m' / (1 - b1^t) / (sqrt(v' / (1 - b2^t)) + eps)
// m' and v' are formed by single operations of 32 bits in this order, none fused, so that codes of 8 bits are the same wherever they are
// computed.  The powers of b1 and b2 are kept beside the count of steps, in 64 bits, and the last workgroup to end counts on.
// States in 8 bits (SMALL): m as e4m3, v as e5m2, 64 elements to a scale, which is a power of two: dividing by it rounds nothing.  A
// rounding to the nearest would hold v fast, which b2 = 0.999 moves by less than half a step: codes are rounded up as often as what is
// missing says, by a hash of the seed, the step and the element's place.  v keeps off zero while it is anything (its root divides m).
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t stir(uint32_t h)
{
    // two odd multipliers, the digits of the golden ratio and of the root of 2; each half reaches the other
    h = (h ^ h >> 16) * 0x9E3779B9u;
    h = (h ^ h >> 15) * 0x6A09E667u;
    return h ^ h >> 16;
}
// The largest of eight lanes' values, in all of them.
__device__ __forceinline__ uint32_t max_of_8(uint32_t x)
{
    uint32_t y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true);     // lane ^ 1
    x = x > y ? x : y;
    y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true);              // lane ^ 2
    x = x > y ? x : y;
    y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, true);             // 7 - lane
    return x > y ? x : y;
}
// The bits of a block's scale, a power of two by which the largest finite value comes to at most 1.75 * 2^TOP, from that value's bits.
template <int TOP> __device__ __forceinline__ uint32_t scale_of(uint32_t most)
{
    const int e = (int)((most + 0x1fffffu) >> 23) - TOP;
    return (uint32_t)(e < 17 ? 17 : e) << 23;
}
// The code of x times `inverse` in MANTISSA bits behind the point, least normal number 2^LOW (below it steps of its last place: an
// addition of 2^LOW lines them up).  noise: 16 bits.  KEPT: nothing but zero becomes zero.
template <int MANTISSA, int LOW, bool KEPT> __device__ __forceinline__ uint32_t code_of(float x, float inverse, uint32_t noise)
{
    constexpr int CUT = 23 - MANTISSA;
    constexpr uint32_t FIRST = (uint32_t)(127 + LOW) << MANTISSA;
    const float low = __builtin_bit_cast(float, (uint32_t)(127 + LOW) << 23), y = fabsf(x) * inverse;
    const bool small = y < low;
    const uint32_t b = __builtin_bit_cast(uint32_t, small ? y + low : y);
    uint32_t c = ((b + (noise << (CUT - 16)) + (1u << (CUT - 17))) >> CUT) - (small ? FIRST : FIRST - (1u << MANTISSA));
    if (KEPT) c = x > 0.0f && c == 0 ? 1u : c;             // (x: its quotient may be zero)
    const uint32_t bits = __builtin_bit_cast(uint32_t, x);
    return (bits & 0x7fffffffu) >= 0x7f800000u ? 0x7fu : c | (bits >> 31) << 7;
}
template <bool E5M2> __device__ __forceinline__ void decode8(const uint32_t (&w)[2], float scale, float (&f)[8])
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const f2v lo = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)w[k], false) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false);
        const f2v hi = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)w[k], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
        f[k * 4] = lo.x * scale;
        f[k * 4 + 1] = lo.y * scale;
        f[k * 4 + 2] = hi.x * scale;
        f[k * 4 + 3] = hi.y * scale;
    }
}
__device__ __forceinline__ uint32_t finite_bits(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// What a launch's threads share.
struct Step {
    float factor, by, root, rate;
    uint32_t key;
};
// Eight consecutive elements on their way: of a type that the compiler knows they are loaded first and converted when they are used; loads and
// conversions behind a branch on the type would wait for each other.
template <int TYPE> struct Raw {
    float f[8];
    __device__ __forceinline__ void load(const void* base, int64_t at)
    {
        __builtin_memcpy(f, (const char*)base + at * (TYPE == DLF_F32 ? 4 : 2), TYPE == DLF_F32 ? 32 : 16);
    }
    __device__ __forceinline__ void to(float (&out)[8]) const
    {
        uint16_t h[8];
        __builtin_memcpy(h, f, 16);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            out[i] = TYPE == DLF_F32 ? f[i] : TYPE == DLF_BF16 ? from_bf16(h[i]) : (float)__builtin_bit_cast(_Float16, h[i]);
    }
};
// The square root by its instruction, off by a unit of the last place; numbers near the end of the range are brought up for it.  (Its result is none near the
// end, nor is eps, so that the reciprocal's instruction takes their sum as it is.  Root and quotient correctly rounded: 2.5 times the instructions of the whole update.)
__device__ __forceinline__ float root_of(float x)
{
    const bool small = x < 0x1p-96f;
    const float r = __builtin_amdgcn_sqrtf(small ? x * 0x1p64f : x);
    return small ? r * 0x1p-32f : r;
}
// m', v' of eight elements, and p'.
__device__ __forceinline__ void update(const DlfStepArgs& a, const Step& w, float away, const float (&g)[8], float (&p)[8], float (&m)[8], float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma clang fp contract(off)
        const float q = a.factor != nullptr ? g[i] * w.factor : g[i];
        m[i] = a.b1 * m[i] + a.c1 * q;
        v[i] = a.b2 * v[i] + a.c2 * q * q;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)                             // (a factor 1 - rate decay would be rounded by a good part of what it takes off)
        p[i] -= __builtin_fmaf(p[i], away, w.by * m[i] * __builtin_amdgcn_rcpf(root_of(v[i] * w.root) + a.eps));
}
// The states of eight elements in 8 bits; the eight lanes of a block are here together.
__device__ __forceinline__ void store_small(const DlfStepArgs& a, const Step& w, int64_t st, const float (&m)[8], const float (&v)[8])
{
    uint32_t bm = 0, bv = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t qm = finite_bits(m[i]), qv = finite_bits(v[i]);
        bm = bm > qm ? bm : qm;
        bv = bv > qv ? bv : qv;
    }
    const uint32_t sm = scale_of<8>(max_of_8(bm)), sv = scale_of<15>(max_of_8(bv));
    const float im = __builtin_bit_cast(float, (254u << 23) - sm), iv = __builtin_bit_cast(float, (254u << 23) - sv);
    const uint32_t mine = w.key ^ stir((uint32_t)((uint64_t)st >> 32));
    uint32_t wm[2] = {0, 0}, wv[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t h = stir((uint32_t)(st + i) ^ mine);
        wm[i >> 2] |= code_of<3, -6, false>(m[i], im, h >> 16) << (i & 3) * 8;
        wv[i >> 2] |= code_of<2, -14, true>(v[i], iv, h & 0xffffu) << (i & 3) * 8;
    }
    __builtin_memcpy((char*)a.m + st, wm, 8);
    __builtin_memcpy((char*)a.v + st, wv, 8);
    if ((threadIdx.x & 7) == 0) {
        a.m_scale[st >> 6] = __builtin_bit_cast(float, sm);
        a.v_scale[st >> 6] = __builtin_bit_cast(float, sv);
    }
}
// A whole chunk, of known types.
template <bool SMALL, int G, int P, int C> __device__ __forceinline__ void whole_chunk(const DlfStepArgs& a, const Step& w, const DlfOptChunk& c, const void* g)
{
    // eight elements a thread at a time, or sixteen: with states in 8 bits more waves share a compute unit instead
    constexpr int UNITS = SMALL ? 1 : DLF_OPT_CHUNK / 2048;
    const float away = w.rate * c.decay;
#pragma unroll 1
    for (int from = (int)threadIdx.x * 8; from < DLF_OPT_CHUNK; from += UNITS * 2048) {
        Raw<G> rg[UNITS];
        Raw<P> rp[UNITS];
        float m[UNITS][8], v[UNITS][8], ms[UNITS], vs[UNITS];
        uint32_t m8[UNITS][2], v8[UNITS][2];
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int e = from + u * 2048;
            const int64_t st = c.state + e;
            rg[u].load(g, c.at + e);
            rp[u].load(c.p, e);
            if (SMALL) {
                __builtin_memcpy(m8[u], (const char*)a.m + st, 8);
                __builtin_memcpy(v8[u], (const char*)a.v + st, 8);
                ms[u] = a.m_scale[st >> 6];
                vs[u] = a.v_scale[st >> 6];
            } else {
                __builtin_memcpy(m[u], (const float*)a.m + st, 32);
                __builtin_memcpy(v[u], (const float*)a.v + st, 32);
            }
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int e = from + u * 2048;
            const int64_t st = c.state + e;
            float gf[8], pf[8];
            rg[u].to(gf);
            rp[u].to(pf);
            if (SMALL) {
                decode8<false>(m8[u], ms[u], m[u]);
                decode8<true>(v8[u], vs[u], v[u]);
            }
            update(a, w, away, gf, pf, m[u], v[u]);
            store8(c.p, e, 8, P, pf);
            if (C >= 0) store8(c.c, e, 8, C, pf);
            if (SMALL) {
                store_small(a, w, st, m[u], v[u]);
            } else {
                store8(a.m, st, 8, DLF_F32, m[u]);
                store8(a.v, st, 8, DLF_F32, v[u]);
            }
        }
    }
}
// A tensor's last chunk, of any types.
template <bool SMALL> __device__ __forceinline__ void last_chunk(const DlfStepArgs& a, const Step& w, const DlfOptChunk& c, const void* g, int g_type)
{
    const float away = w.rate * c.decay;
    for (int e = (int)threadIdx.x * 8; SMALL ? (e & ~63) < c.n : e < c.n; e += 2048) {   // (the eight lanes of a block of 64 stay together)
        const int n = c.n - e;
        const int64_t st = c.state + e;
        float gf[8], pf[8], m[8], v[8];
        load8(g, c.at + e, n, g_type, gf);
        load8(c.p, e, n, c.p_type, pf);
        if (SMALL) {
            uint32_t m8[2], v8[2];
            __builtin_memcpy(m8, (const char*)a.m + st, 8);
            __builtin_memcpy(v8, (const char*)a.v + st, 8);
            decode8<false>(m8, a.m_scale[st >> 6], m);
            decode8<true>(v8, a.v_scale[st >> 6], v);
        } else {
            load8(a.m, st, n, DLF_F32, m);
            load8(a.v, st, n, DLF_F32, v);
        }
        update(a, w, away, gf, pf, m, v);
        store8(c.p, e, n, c.p_type, pf);
        if (c.c != nullptr) store8(c.c, e, n, c.c_type, pf);
        if (SMALL) {
            store_small(a, w, st, m, v);
        } else {
            store8(a.m, st, n, DLF_F32, m);
            store8(a.v, st, n, DLF_F32, v);
        }
    }
}
template <bool SMALL, int G> __device__ __forceinline__ void whole_chunk_of(const DlfStepArgs& a, const Step& w, const DlfOptChunk& c, const void* g)
{
    if (c.p_type == DLF_F32) {
        if (c.c == nullptr) whole_chunk<SMALL, G, DLF_F32, -1>(a, w, c, g);
        else if (c.c_type == DLF_BF16) whole_chunk<SMALL, G, DLF_F32, DLF_BF16>(a, w, c, g);
        else whole_chunk<SMALL, G, DLF_F32, DLF_F16>(a, w, c, g);
    } else if (c.p_type == DLF_BF16) whole_chunk<SMALL, G, DLF_BF16, -1>(a, w, c, g);
    else whole_chunk<SMALL, G, DLF_F16, -1>(a, w, c, g);
}

template <bool SMALL>
__global__ __launch_bounds__(256) void k_step(const DlfStepArgs a)
{
    Step w;
    w.factor = a.factor != nullptr ? *a.factor : 1.0f;
    if (!(fabsf(w.factor) <= 3.402823466e38f)) return;      // a step that is to be left out
    const double t0 = a.counter[0], p1 = a.counter[1] * a.beta1, p2 = a.counter[2] * a.beta2;
    w.rate = a.rate_at != nullptr ? *a.rate_at : a.rate;
    w.by = (float)((double)w.rate / (1.0 - p1));
    w.root = (float)(1.0 / (1.0 - p2));
    w.key = SMALL ? stir(stir(a.seed) + (uint32_t)(int64_t)t0) : 0u;
    for (int k = blockIdx.x; k < a.chunks; k += gridDim.x) {
        const DlfOptChunk c = a.table[k];
        const int tensor = c.tensor - a.first_tensor;
        const void* const g = a.g[tensor];
        if (g == nullptr) continue;
        const int g_type = a.type[tensor];
        if (c.n < DLF_OPT_CHUNK) last_chunk<SMALL>(a, w, c, g, g_type);
        else if (g_type == DLF_F32) whole_chunk_of<SMALL, DLF_F32>(a, w, c, g);
        else if (g_type == DLF_BF16) whole_chunk_of<SMALL, DLF_BF16>(a, w, c, g);
        else whole_chunk_of<SMALL, DLF_F16>(a, w, c, g);
    }
    if (a.last == 0) return;
    // every workgroup has read the counter when the last of them arrives here
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t* const ended = (uint32_t*)(a.counter + 3);
        if (__hip_atomic_fetch_add(ended, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1) {
            __hip_atomic_store(ended, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            a.counter[0] = t0 + 1.0;
            a.counter[1] = p1;
            a.counter[2] = p2;
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------------
extern "C" int dlf_opt_start_norm(const DlfNormArgs* a, int groups, void* stream)
{
    hipLaunchKernelGGL(k_norm, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_opt_start_norm_join(const DlfNormJoinArgs* a, void* stream)
{
    hipLaunchKernelGGL(k_norm_join, dim3(1), dim3(1024), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_opt_start_step(const DlfStepArgs* a, int small, int groups, void* stream)
{
    if (small) hipLaunchKernelGGL(k_step<true>, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, *a);
    else hipLaunchKernelGGL(k_step<false>, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
