// gfx950 (CDNA4) kernels of the feed-forward operators: matrix products with bias, activation and residual in the
// epilogue, the gated pair of projections, and their gradients.  The forms of the products are in dlf_ffn.h.
//
// P is the MFMA "A" operand and Q the "B" operand: a lane then holds four consecutive c of one r, as a row-major C wants.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include "dlf_ffn.h"

typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef unsigned u4v __attribute__((ext_vector_type(4)));

// The two element types and their 32x32x16 matrix instruction.
struct F16 {
    typedef _Float16 e;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f16v mma(v8 a, v8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
struct BF16 {
    typedef __bf16 e;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f16v mma(v8 a, v8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// ------------------------------------------------------------------------------------------------
// Activations, in 32 bits.
// ------------------------------------------------------------------------------------------------

// 1 / (1 + exp(-x)).  exp(-x) = 2^t with t = -x * log2(e): the instruction gives 2^t to one unit in the last place, but a t of
// magnitude 100 has lost seven bits of the exponent's fraction, so what the product rounds off (its low part and that of log2(e))
// is put back as a factor 1 + d * ln(2).  The bounds keep infinities out of that correction and let NaN through.
__device__ __forceinline__ float sigmoid(float x)
{
    float n = -x;
    n = n > 126.0f ? 126.0f : n;
    n = n < -126.0f ? -126.0f : n;
    const float t = n * 1.44269502f;
    const float d = __builtin_fmaf(n, 1.92596299e-8f, __builtin_fmaf(n, 1.44269502f, -t));
    const float p = __builtin_amdgcn_exp2f(t);
    return __builtin_amdgcn_rcpf(1.0f + p * __builtin_fmaf(d, 0.693147182f, 1.0f));   // p may be infinite: the factor is not 0
}
#define GELU_2C 1.59576912f       // 2 sqrt(2 / pi): 0.5 (1 + tanh(y)) = 1 / (1 + exp(-2 y))
#define GELU_A 0.044715f
#define SQRT_HALF 0.707106769f
#define INV_SQRT_2PI 0.398942280f

template <int ACT> __device__ __forceinline__ float act_of(float z)
{
    if constexpr (ACT == DLF_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == DLF_ACT_RELU6) return z < 0.0f ? 0.0f : z > 6.0f ? 6.0f : z;
    if constexpr (ACT == DLF_ACT_GELU) return 0.5f * z * (1.0f + erff(z * SQRT_HALF));
    if constexpr (ACT == DLF_ACT_GELU_TANH) return z * sigmoid(GELU_2C * (z + GELU_A * z * z * z));
    if constexpr (ACT == DLF_ACT_SILU) return z * sigmoid(z);
    if constexpr (ACT == DLF_ACT_SIGMOID) return sigmoid(z);
    return z;
}
// act(z) and act'(z) (of the activations with a step: 0 on the step).
template <int ACT> __device__ __forceinline__ void act_grad_of(float z, float& a, float& d)
{
    if constexpr (ACT == DLF_ACT_NONE) { a = z; d = 1.0f; }
    if constexpr (ACT == DLF_ACT_RELU) { a = z < 0.0f ? 0.0f : z; d = z <= 0.0f ? 0.0f : z > 0.0f ? 1.0f : z; }
    if constexpr (ACT == DLF_ACT_RELU6) {
        a = z < 0.0f ? 0.0f : z > 6.0f ? 6.0f : z;
        d = z <= 0.0f || z >= 6.0f ? 0.0f : z == z ? 1.0f : z;
    }
    if constexpr (ACT == DLF_ACT_GELU) {
        const float c = 0.5f * (1.0f + erff(z * SQRT_HALF));
        a = z * c;
        d = __builtin_fmaf(z, INV_SQRT_2PI * expf(-0.5f * z * z), c);
    }
    if constexpr (ACT == DLF_ACT_GELU_TANH) {
        const float s = sigmoid(GELU_2C * (z + GELU_A * z * z * z));
        a = z * s;
        // s (1 - s) underflows to zero before the cubic's derivative overflows (|z| > 1e19: keep 0 * inf out)
        const float t = s * (1.0f - s);
        d = t == 0.0f ? s : __builtin_fmaf(z * t, GELU_2C * (1.0f + 3.0f * GELU_A * z * z), s);
    }
    if constexpr (ACT == DLF_ACT_SILU) { const float s = sigmoid(z); a = z * s; d = s * __builtin_fmaf(z, 1.0f - s, 1.0f); }
    if constexpr (ACT == DLF_ACT_SIGMOID) { const float s = sigmoid(z); a = s; d = s * (1.0f - s); }
}
// Calls f with the activation (uniform over the launch) as a constant.
template <typename F> __device__ __forceinline__ void with_act(int act, F&& f)
{
    switch (act) {
    case DLF_ACT_RELU: f(std::integral_constant<int, DLF_ACT_RELU>()); break;
    case DLF_ACT_RELU6: f(std::integral_constant<int, DLF_ACT_RELU6>()); break;
    case DLF_ACT_GELU: f(std::integral_constant<int, DLF_ACT_GELU>()); break;
    case DLF_ACT_GELU_TANH: f(std::integral_constant<int, DLF_ACT_GELU_TANH>()); break;
    case DLF_ACT_SILU: f(std::integral_constant<int, DLF_ACT_SILU>()); break;
    case DLF_ACT_SIGMOID: f(std::integral_constant<int, DLF_ACT_SIGMOID>()); break;
    default: f(std::integral_constant<int, DLF_ACT_NONE>()); break;
    }
}

// ------------------------------------------------------------------------------------------------
// Eight consecutive elements, of which n exist (n may be anything; nothing outside them is touched).
// Rows start where they like: a 16-byte access of any 2-byte alignment is one instruction here.
// ------------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ typename T::v8 load8(const void* base, int64_t at, int n)
{
    const typename T::e* p = (const typename T::e*)base + at;
    typename T::v8 v;
    if (n >= 8) {
        __builtin_memcpy(&v, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (typename T::e)0.0f;
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store8(void* base, int64_t at, int n, const float (&f)[8])
{
    typename T::e* p = (typename T::e*)base + at;
    typename T::v8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (typename T::e)f[i];
    if (n >= 8) {
        __builtin_memcpy(p, &v, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}
__device__ __forceinline__ void load8f(const float* p, int n, float (&f)[8])
{
    if (n >= 8) {
        __builtin_memcpy(f, p, 32);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void store8f(float* p, int n, const float (&f)[8])
{
    if (n >= 8) {
        __builtin_memcpy(p, f, 32);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = f[i];
    }
}

// The epilogue of eight outputs C[r][c .. c + n): bias, pre-activations kept, activation, product with the second projection,
// residual, one rounding.
template <typename T, bool GATED>
__device__ __forceinline__ void finish8(const DlfFfArgs& a, int prob, int r, int c, int n, float (&v)[8], float (&u)[8])
{
    if (a.bias[0] != nullptr) {
        float b[8];
        load8f(a.bias[0] + c, n, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += b[i];
    }
    if (GATED && a.bias[1] != nullptr) {
        float b[8];
        load8f(a.bias[1] + c, n, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] += b[i];
    }
    if (a.saved != nullptr) {
        store8f(a.saved + (int64_t)r * a.nc + c, n, v);
        if (GATED) store8f(a.saved + ((int64_t)a.nr + r) * a.nc + c, n, u);
    }
    if (a.act != DLF_ACT_NONE)
        with_act(a.act, [&](auto k) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = act_of<decltype(k)::value>(v[i]);
        });
    if (GATED) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= u[i];
    }
    if (a.res != nullptr) {
        const typename T::v8 q = load8<T>(a.res, (int64_t)r * a.ldres + c, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += (float)q[i];
    }
    store8<T>(a.out[prob], (int64_t)r * a.ldo + c, n, v);
}

// ------------------------------------------------------------------------------------------------
// k_ff_any: the product for operands of any alignment, stride and size.  A workgroup of four waves computes 64 x 64 of C (gated: of
// both projections); 32 k at a time pass through registers into LDS, where every operand lies with k along the row, the next 32 being
// on their way meanwhile.
// ------------------------------------------------------------------------------------------------
template <typename T, bool PT, bool QT, bool GATED>
__global__ __launch_bounds__(256) void k_ff_any(const DlfFfArgs a)
{
    typedef typename T::e e;
    typedef typename T::v8 v8;
    constexpr int TILE = DLF_FF_ANY_TILE, KS = 32, ROW = KS + 8, NP = GATED ? 2 : 1, CROW = TILE + 4;
    constexpr int OPS = (NP + 1) * TILE * ROW * 2, OUT = NP * TILE * CROW * 4;
    __shared__ __attribute__((aligned(16))) char mem[OPS > OUT ? OPS : OUT];
    e* const ls = (e*)mem;                     // P (, second P), Q: [64][ROW]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lhi = lane >> 5;
    int t = blockIdx.x;
    const int per = a.tiles_r * a.tiles_c;
    const int prob = t / per;
    t -= prob * per;
    const int r0 = t / a.tiles_c * TILE, c0 = t % a.tiles_c * TILE;
    const int steps = (a.nk + KS - 1) / KS, total = steps * a.segments;

    // 64 rows of 32 k, or 32 rows of 64: one chunk of eight per thread
    const int nrow = tid >> 2, nch = (tid & 3) * 8, trow = tid >> 3, tch = (tid & 7) * 8;
    auto chunk = [&](const void* base, int64_t ld, bool tr, int i0, int ni, int k0) __attribute__((always_inline)) -> v8 {
        const int row = tr ? k0 + trow : i0 + nrow, col = tr ? i0 + tch : k0 + nch;
        const int rows = tr ? a.nk : ni, cols = tr ? ni : a.nk;
        return load8<T>(base, (int64_t)row * ld + col, row < rows ? cols - col : 0);
    };
    auto put = [&](e* to, bool tr, v8 v) __attribute__((always_inline)) {
        if (!tr) {
            *(v8*)(to + nrow * ROW + nch) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[(tch + i) * ROW + trow] = v[i];
        }
    };
    v8 np[NP], nq;
    auto request = [&](int s) __attribute__((always_inline)) {
        const int seg = s >= steps ? 1 : 0, k0 = (s - seg * steps) * KS, w = a.problems == 2 ? prob : seg;
#pragma unroll
        for (int i = 0; i < NP; ++i) np[i] = chunk(a.p[GATED ? i : w], a.ldp, PT, c0, a.nc, k0);
        nq = chunk(a.q[GATED ? 0 : w], a.ldq, QT, r0, a.nr, k0);
    };
    f16v acc[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;
    const int wc = (wave & 1) * 32, wr = (wave >> 1) * 32;
    if (total > 0) request(0);
    for (int s = 0; s < total; ++s) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NP; ++i) put(ls + i * TILE * ROW, PT, np[i]);
        put(ls + NP * TILE * ROW, QT, nq);
        __syncthreads();
        if (s + 1 < total) request(s + 1);
#pragma unroll
        for (int k = 0; k < KS; k += 16) {
            const v8 q = *(const v8*)(ls + (NP * TILE + wr + l32) * ROW + k + lhi * 8);
#pragma unroll
            for (int i = 0; i < NP; ++i) acc[i] = T::mma(*(const v8*)(ls + (i * TILE + wc + l32) * ROW + k + lhi * 8), q, acc[i]);
        }
    }
    // through LDS, so that a thread finishes eight consecutive c and the activations are unrolled once
    __syncthreads();
    float* const lf = (float*)mem;             // [NP][64 r][CROW]
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(f4v*)(lf + (i * TILE + wr + l32) * CROW + wc + q * 8 + lhi * 4) =
                f4v{acc[i][q * 4], acc[i][q * 4 + 1], acc[i][q * 4 + 2], acc[i][q * 4 + 3]};
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < TILE * TILE / 8; i += 256) {
        const int r = i >> 3, c = (i & 7) * 8;
        if (r0 + r >= a.nr || c0 + c >= a.nc) continue;
        float v[8], u[8];
        load8f(lf + r * CROW + c, 8, v);
        if (GATED) load8f(lf + (TILE + r) * CROW + c, 8, u);
        finish8<T, GATED>(a, prob, r0 + r, c0 + c, a.nc - c0 - c, v, u);
    }
}

// ------------------------------------------------------------------------------------------------
// k_ff_dz: the gradient behind the activation, and partial column sums of it in 32 bits (before it is rounded).  A workgroup takes
// `chunk` rows of 256 columns: 32 threads by eight columns, 8 rows at a time; the sums of the 8 meet in LDS in a fixed order.
// ------------------------------------------------------------------------------------------------
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_ff_dz(const DlfFfDzArgs a)
{
    constexpr int NZ = GATED ? 2 : 1;
    __shared__ float sums[NZ][8][256];
    const int tc = threadIdx.x & 31, tr = threadIdx.x >> 5;
    const int c = (blockIdx.x * 32 + tc) * 8, n = a.n - c;
    const int r0 = blockIdx.y * a.chunk, r1 = min(a.rows, r0 + a.chunk);
    float sum[NZ][8];
#pragma unroll
    for (int z = 0; z < NZ; ++z)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[z][i] = 0.0f;
    if (n > 0) {
        for (int r = r0 + tr; r < r1; r += 8) {
            const typename T::v8 dy = load8<T>(a.dy, (int64_t)r * a.lddy + c, n);
            float d[NZ][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[0][i] = (float)dy[i];
            if (a.saved != nullptr) {
                float z[8], u[8];
                load8f(a.saved + (int64_t)r * a.n + c, n, z);
                if (GATED) load8f(a.saved + ((int64_t)a.rows + r) * a.n + c, n, u);
                with_act(a.act, [&](auto k) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float av, dv;
                        act_grad_of<decltype(k)::value>(z[i], av, dv);
                        if constexpr (GATED) {
                            d[NZ - 1][i] = d[0][i] * av;
                            d[0][i] *= u[i] * dv;
                        } else {
                            d[0][i] *= dv;
                        }
                    }
                });
                // rows of dz are whole eights: what lies behind column n is read as zeros by the products
#pragma unroll
                for (int z2 = 0; z2 < NZ; ++z2) {
                    if (n < 8) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[z2][i] = i < n ? d[z2][i] : 0.0f;
                    }
                    store8<T>(a.dz[z2], (int64_t)r * a.lddz + c, 8, d[z2]);
                }
            }
#pragma unroll
            for (int z2 = 0; z2 < NZ; ++z2)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[z2][i] += d[z2][i];
        }
    }
    if (a.part == nullptr) return;
#pragma unroll
    for (int z = 0; z < NZ; ++z)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[z][tr][tc * 8 + i] = sum[z][i];
    __syncthreads();
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col < a.n) {
#pragma unroll
        for (int z = 0; z < NZ; ++z) {
            float t = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t += sums[z][k][threadIdx.x];
            a.part[((int64_t)z * gridDim.y + blockIdx.y) * a.n + col] = t;
        }
    }
}
// The partial sums of a column added in order: the result does not depend on which workgroup came first.
__global__ __launch_bounds__(256) void k_ff_sum(const DlfFfSumArgs a)
{
    const int col = blockIdx.x * 256 + threadIdx.x, z = blockIdx.y;
    if (col >= a.n || a.out[z] == nullptr) return;
    float t = 0.0f;
    for (int k = 0; k < a.chunks; ++k) t += a.part[((int64_t)z * a.chunks + k) * a.n + col];
    a.out[z][col] = t;
}

// ------------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------------
template <typename T> static void (*any_kernel(int layout, int gated))(const DlfFfArgs)
{
    if (gated) return k_ff_any<T, false, false, true>;
    switch (layout) {
    case DLF_FF_NN: return k_ff_any<T, false, false, false>;
    case DLF_FF_TN: return k_ff_any<T, true, false, false>;
    default: return k_ff_any<T, true, true, false>;
    }
}
extern "C" int dlf_ff_start_any(const DlfFfArgs* a, int dtype, int layout, int gated, void* stream)
{
    hipLaunchKernelGGL(dtype == DLF_F16 ? any_kernel<F16>(layout, gated) : any_kernel<BF16>(layout, gated),
                       dim3((unsigned)(a->tiles_r * a->tiles_c * a->problems)), dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ff_start_dz(const DlfFfDzArgs* a, int dtype, int gated, void* stream)
{
    const dim3 grid((unsigned)((a->n + 255) / 256), (unsigned)(a->rows > 0 ? (a->rows + a->chunk - 1) / a->chunk : 1));
    hipLaunchKernelGGL(dtype == DLF_F16 ? (gated ? k_ff_dz<F16, true> : k_ff_dz<F16, false>) : (gated ? k_ff_dz<BF16, true> : k_ff_dz<BF16, false>),
                       grid, dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ff_start_sum(const DlfFfSumArgs* a, int gated, void* stream)
{
    hipLaunchKernelGGL(k_ff_sum, dim3((unsigned)((a->n + 255) / 256), gated ? 2 : 1), dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
