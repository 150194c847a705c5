// Device code of the matrix products on gfx950 (CDNA4), shared by the feed-forward operators (dlf_ffn.hip) and the cross entropy of a linear
// layer (dlf_ce.hip): tiles through LDS with their epilogues, few rows straight from memory.  The forms of the products are in dlf_ffn.h.
//
// P is the MFMA "A" operand and Q the "B" operand: a lane then holds four consecutive c of one r, as a row-major C wants.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include "dlf_ffn.h"

typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef unsigned u4v __attribute__((ext_vector_type(4)));

// The two element types and their matrix instructions, 32x32x16 and 16x16x32.
struct F16 {
    typedef _Float16 e;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f16v mma(v8 a, v8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f4v mma16(v8 a, v8 b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
struct BF16 {
    typedef __bf16 e;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f16v mma(v8 a, v8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f4v mma16(v8 a, v8 b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// ------------------------------------------------------------------------------------------------
// Activations, in 32 bits.
// ------------------------------------------------------------------------------------------------

// 1 / (1 + exp(-x)), exp(-x) = 2^t with t = -x log2(e).  t is rounded once, which costs the exponential |t| * 2^-24 of its value: below
// 1e-6 where the result is not within 1e-6 of 0 or 1 anyway.  (A matrix tile's epilogue is bound by vector instructions: what the
// product rounds off, put back as a factor, took twice as many.)
__device__ __forceinline__ float sigmoid(float x)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269502f));
}
// The normal distribution's density (without its factor 1 / sqrt(2 pi)) and distribution function: Phi(-|z|) = exp(-z^2 / 2) erfcx(a) / 2 with
// a = |z| / sqrt(2) and erfcx(a) = exp(a^2) erfc(a), which is t times a polynomial in t = 1 / (1 + 0.4 a) to 1.3e-7 of its value (a
// least-squares fit of degree 8 at Chebyshev nodes), so the far tail keeps its relative precision.  The library's erff costs a 4096 x 4096 tile
// product 25 us, this 9.
__device__ __forceinline__ float normal_cdf(float z, float& density)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(z), 0.282842712f, 1.0f));
    float p = 0.0501872883f;
    p = __builtin_fmaf(p, t, -0.182615347f);
    p = __builtin_fmaf(p, t, 0.168643858f);
    p = __builtin_fmaf(p, t, -0.00525540996f);
    p = __builtin_fmaf(p, t, 0.141277341f);
    p = __builtin_fmaf(p, t, 0.168578172f);
    p = __builtin_fmaf(p, t, 0.207838584f);
    p = __builtin_fmaf(p, t, 0.225669773f);
    p = __builtin_fmaf(p, t, 0.225675861f);
    density = __builtin_amdgcn_exp2f(z * z * -0.721347520f);
    const float tail = 0.5f * t * p * density;
    return z < 0.0f ? tail : 1.0f - tail;
}
#define GELU_2C 1.59576912f       // 2 sqrt(2 / pi): 0.5 (1 + tanh(y)) = 1 / (1 + exp(-2 y))
#define GELU_A 0.044715f
#define INV_SQRT_2PI 0.398942280f

template <int ACT> __device__ __forceinline__ float act_of(float z)
{
    if constexpr (ACT == DLF_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == DLF_ACT_RELU6) return z < 0.0f ? 0.0f : z > 6.0f ? 6.0f : z;
    if constexpr (ACT == DLF_ACT_GELU) { float density; return z * normal_cdf(z, density); }
    if constexpr (ACT == DLF_ACT_GELU_TANH) return z * sigmoid(z * __builtin_fmaf(z * z, GELU_2C * GELU_A, GELU_2C));
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
        float density;
        const float c = normal_cdf(z, density);
        a = z * c;
        d = __builtin_fmaf(z, INV_SQRT_2PI * density, c);
    }
    if constexpr (ACT == DLF_ACT_GELU_TANH) {
        const float s = sigmoid(z * __builtin_fmaf(z * z, GELU_2C * GELU_A, GELU_2C));
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
// V consecutive elements, of which n exist (n may be anything; nothing outside them is touched).
// Rows start where they like: a 16-byte access of any 2-byte alignment is one instruction here.
// ------------------------------------------------------------------------------------------------
template <typename T, int V> struct Some { typedef typename T::e v __attribute__((ext_vector_type(V))); };
template <typename T, int V> __device__ __forceinline__ typename Some<T, V>::v load_some(const void* base, int64_t at, int n)
{
    const typename T::e* p = (const typename T::e*)base + at;
    typename Some<T, V>::v v;
    if (n >= V) {
        __builtin_memcpy(&v, p, 2 * V);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < n ? p[i] : (typename T::e)0.0f;
    }
    return v;
}
template <typename T> __device__ __forceinline__ typename T::v8 load8(const void* base, int64_t at, int n)
{
    return __builtin_bit_cast(typename T::v8, load_some<T, 8>(base, at, n));
}
template <typename T, int V> __device__ __forceinline__ void store_some(void* base, int64_t at, int n, const float (&f)[V])
{
    typename T::e* p = (typename T::e*)base + at;
    typename Some<T, V>::v v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (typename T::e)f[i];
    if (n >= V) {
        __builtin_memcpy(p, &v, 2 * V);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = v[i];
    }
}
template <int V> __device__ __forceinline__ void load_floats(const float* p, int n, float (&f)[V])
{
    if (n >= V) {
        __builtin_memcpy(f, p, 4 * V);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < n ? p[i] : 0.0f;
    }
}
template <int V> __device__ __forceinline__ void store_floats(float* p, int n, const float (&f)[V])
{
    if (n >= V) {
        __builtin_memcpy(p, f, 4 * V);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = f[i];
    }
}

// What a kernel adds to the epilogue.  OWN: it has one of its own, see tile(); SUMS: correct() and take() change the outputs before they
// are stored, and the latter says whether they are.  ready(): what of it is used where the epilogue begins.
struct Plain {
    static constexpr bool OWN = false, SUMS = false;
    __device__ __forceinline__ const Plain& ready() const { return *this; }
};
// The epilogue of V outputs C[r][c .. c + n): bias, pre-activations kept, activation, product with the second projection,
// residual, one rounding.
template <typename T, bool GATED, int V, typename E>
__device__ __forceinline__ void finish(const DlfFfArgs& a, const E& extra, int prob, int r, int c, int n, float (&v)[V], float (&u)[V])
{
    if (a.bias[0] != nullptr) {
        float b[V];
        load_floats(a.bias[0] + c, n, b);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += b[i];
    }
    if (GATED && a.bias[1] != nullptr) {
        float b[V];
        load_floats(a.bias[1] + c, n, b);
#pragma unroll
        for (int i = 0; i < V; ++i) u[i] += b[i];
    }
    if (a.saved != nullptr) {
        store_floats(a.saved + (int64_t)r * a.nc + c, n, v);
        if (GATED) store_floats(a.saved + ((int64_t)a.nr + r) * a.nc + c, n, u);
    }
    if (a.act != DLF_ACT_NONE)
        with_act(a.act, [&](auto k) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = act_of<decltype(k)::value>(v[i]);
        });
    if (GATED) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] *= u[i];
    }
    if (a.res != nullptr) {
        const typename Some<T, V>::v q = load_some<T, V>(a.res, (int64_t)r * a.ldres + c, n);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += (float)q[i];
    }
    if constexpr (E::SUMS) {
        extra.template correct<T, 1, V>(a, r, 0, c, n, &v);
        if (!extra.take(a, r, c, n, v)) return;
    }
    store_some<T, V>(a.out[prob], (int64_t)r * a.ldo + c, n, v);
}

// ... of N units of eight outputs, `step` rows apart, of columns that all exist: their loads share a wait.
template <typename T, bool GATED, int N, typename E>
__device__ __forceinline__ void finish_many(const DlfFfArgs& a, const E& extra, int prob, int r, int step, int c, float (&v)[N][8], float (&u)[N][8])
{
    typename T::v8 q[N];
    if (a.res != nullptr) {
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = load8<T>(a.res, (int64_t)min(r + k * step, a.nr - 1) * a.ldres + c, 8);
    }
    if (a.bias[0] != nullptr) {
        float b[8];
        load_floats(a.bias[0] + c, 8, b);
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] += b[i];
    }
    if (GATED && a.bias[1] != nullptr) {
        float b[8];
        load_floats(a.bias[1] + c, 8, b);
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) u[k][i] += b[i];
    }
    if (a.saved != nullptr) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (r + k * step >= a.nr) continue;
            store_floats(a.saved + (int64_t)(r + k * step) * a.nc + c, 8, v[k]);
            if (GATED) store_floats(a.saved + ((int64_t)a.nr + r + k * step) * a.nc + c, 8, u[k]);
        }
    }
    if (a.act != DLF_ACT_NONE)
        with_act(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] = act_of<decltype(act)::value>(v[k][i]);
        });
    if constexpr (E::SUMS) extra.template correct<T, N, 8>(a, r, step, c, 8, v);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (GATED) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] *= u[k][i];
        }
        if (a.res != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] += (float)q[k][i];
        }
        if (r + k * step >= a.nr) continue;
        if constexpr (E::SUMS) {
            if (!extra.take(a, r + k * step, c, 8, v[k])) continue;
        }
        store_some<T, 8>(a.out[prob], (int64_t)(r + k * step) * a.ldo + c, 8, v[k]);
    }
}

// ------------------------------------------------------------------------------------------------
// tile (k_ff_tile, k_ff_back): a workgroup of WC x WR waves computes BC x BR of C (gated: BC / 2 features of both projections), a wave FC x FR
// blocks of 32 x 32; 64 k at a time ("stage") pass through LDS, two or four stages in turn.  DIRECT: for operands whose rows are whole
// 16-byte lines; otherwise through registers (Stager).  Bound by the matrix units and what they may draw: 8192^3 takes 790 us (1.39
// PFLOP/s at 1.9 GHz), 4096^3 112 to 117, of which 12 are the first loads, the epilogue and the launch; a stage takes 1.5 us, its
// multiplications alone 1.08 at that clock: the rest are the barrier and the waits around it, which a second wave per SIMD would cover,
// but the registers of 128 x 128 blocks leave no room for one, and smaller blocks read LDS half as often again.
//   Global -> LDS: 16-byte direct loads, 1 KiB per instruction, lane l's 16 bytes at 16 l.  Rows, columns and k that do not exist
//     are read from an offset behind the resource's end, which brings zeros and no traffic.
//   An operand with k along its rows lies in LDS as [row][64 k], 128 bytes a row, its 16-byte part c at position c ^ (row / 2) % 8: the 16
//     lanes that LDS serves at a time, 16 rows of one part, fall into 16 different 16-byte groups of the 256 bytes of banks.
//   An operand with k across its rows lies as [k][row] as it comes, and is turned on its way into registers: one transposing
//     read gives a lane four k of its row, the 16 lanes of a group reading 4 k x 16 rows.  The 64-byte part b of line k is kept at b ^ f(k),
//     f(k) = k % 4 + 4 * (k / 8 % 2) (modulo the parts of a line): the eight lines of a read fall into different banks.
//   The multiplications of 16 k run while the operands of the next 16 are read.  Behind the third of a stage's four steps a wave has all of the
//     stage in registers: there it waits for its part of the next stage and for the other waves, and requests the stage after that into
//     the LDS just read, half of it during the fourth step, half during the first of the next stage (over three steps the last requests
//     came late: 8192^3 2 % slower; all in one 6 %).  The addresses of a stage are formed ahead of the barrier, not behind it (2 %).
//     Stages of 32 k, four in LDS, wait less but read half lines: 4096^3 124 against 115 us.
//   Through registers, 4096 x 4099 -> 4101 takes 248 us (0.56 PFLOP/s), 4096 x 4099 -> 2 x 10881 gated 1071 (0.68), 128 x 128 tiles both: loads of
//     rows off their lines, a write to LDS and a barrier a stage.
//   The epilogue goes through LDS, 64 rows of a wave at a time, so that stores are whole lines and the code of the activations is there
//     once; a lane's loads for several rows go out together (one after the other they made the epilogue of 256 x 256 take 16 us).
// Workgroup b runs on XCD b % 8: each XCD takes a run of tiles, in bands of four rows of tiles, and its workgroups share operands
// in its L2.  XCDs start at different k, see below.
// ------------------------------------------------------------------------------------------------
#define OOB ((int)0x80000000)
typedef int i4v __attribute__((ext_vector_type(4)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));
extern __shared__ __attribute__((aligned(16))) char ff_lds[];
typedef __attribute__((address_space(3))) char lds_char;

__device__ __forceinline__ i4v resource(const void* p, int bytes = 0x7fffffff)
{
    const unsigned long long v = (unsigned long long)p;
    i4v r;
    r.x = __builtin_amdgcn_readfirstlane((int)(unsigned)v);
    r.y = __builtin_amdgcn_readfirstlane((int)((unsigned)(v >> 32) & 0xffffu));
    r.z = bytes;
    r.w = 0x00020000;
    return r;
}
// Lane l's 16 bytes at base + off into LDS at dst + 16 l.  Written as an instruction: the compiler would wait for such loads
// wherever it waits for an LDS read.
__device__ __forceinline__ void line_to_lds(const i4v& base, int off, unsigned dst)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(base), "s"(dst) : "memory", "m0");
}
#define WAIT_LDS 0xc07f          // s_waitcnt lgkmcnt(0)
// s_waitcnt vmcnt(N) lgkmcnt(0); known to the compiler, unlike an instruction in assembly
#define WAIT_LOADS_AND_LDS(N) (0x0070 | ((N) & 15) | ((N) >> 4) << 14)
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// What the 16-byte parts of row `row` are kept at: position c ^ swizzle.
__device__ __forceinline__ int swizzle(int row) { return row >> 1 & 7; }
// One operand's way from memory into LDS: a wave's N instructions of a stage.  ROWS of the operand per tile; TR: k across the rows.
template <int N, int ROWS, bool TR, int KB> struct Loader {
    static constexpr int CPL = TR ? ROWS / 8 : KB / 8;      // 16-byte parts of a line in LDS
    int off[N];
    // first: the wave's first instruction; avail: rows of the operand from the tile's first on; half: gated P, see below
    __device__ __forceinline__ static int line(int first, int i) { return (first + i) * (64 / CPL) + (threadIdx.x & 63) / CPL; }
    __device__ __forceinline__ static int part(int first, int i)
    {
        const int l = line(first, i), p = (threadIdx.x & 63) % CPL;
        if (!TR) return p ^ swizzle(l);
        return p ^ ((((l & 3) | ((l >> 3) & 1) << 2) & (ROWS / 32 - 1)) << 2);
    }
    template <bool GATED> __device__ __forceinline__ void setup(int first, int avail, int64_t ld)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int l = line(first, i), p = part(first, i);
            // a gated tile's lines: for every 32 features 32 lines of the gate projection and 32 of the other
            const int row = GATED ? (l >> 6) * 32 + (l & 31) : l;
            if (!TR) off[i] = row < avail ? (int)(row * ld + p * 8) * 2 : OOB;
            else off[i] = p * 8 < avail ? (int)(l * ld + p * 8) * 2 : OOB;
        }
    }
    // zeros for what lies behind the operand's last k_left k of a stage
    __device__ __forceinline__ void mask(int first, int k_left)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) off[i] = (TR ? line(first, i) : part(first, i) * 8) < k_left ? off[i] : OOB;
    }
    template <bool TAIL> __device__ __forceinline__ void issue(const i4v& base, int first, unsigned dst, int k_left) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            line_to_lds(base, !TAIL || (TR ? line(first, i) : part(first, i) * 8) < k_left ? off[i] : OOB, dst + (unsigned)(first + i) * 1024);
    }
};
// ... of rows that start anywhere: through registers, by a load and, a stage later, a write to LDS.  Rows and columns that do not exist
// are read as others and not stored.  A part of eight that ends behind the operand's last k (or column) is read as the last eight there
// are and shifted, zeros moving in: a 16-byte load never leaves the operand.  Only operands of less than eight are read one by one.
// Which parts those are is the same for every stage that is not whole, so a load is one instruction without a branch: with branches the compiler
// loses count of the loads on their way and waits for all of them.
template <typename T, int N, int ROWS, bool TR, int KB> struct Stager {
    typedef Loader<N, ROWS, TR, KB> Map;
    static constexpr int BIAS = 128;        // bytes: what a part may begin in front of the stage's first
    unsigned off[N], last[N];               // of a whole stage, of one that is not
    typename T::v8 v[N];
    int edge;               // across: columns of a tile that ends inside a part of eight, else 0
    int tail;               // k of the stage in v if they are not whole, else 0
    bool tiny;              // less than eight k (along) or columns (across) in all
    template <bool GATED> __device__ __forceinline__ void setup(int first, int avail, int64_t ld, int extent, int nk)
    {
        tiny = extent < 8;
        tail = 0;
        edge = TR && avail < ROWS && (avail & 7) != 0 ? avail : 0;
        const int left = nk % KB;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int l = Map::line(first, i), p = Map::part(first, i) * 8, row = GATED ? (l >> 6) * 32 + (l & 31) : l;
            const int at = !TR ? p : edge > 0 && !tiny ? min(p, avail - 8) : p < avail ? p : 0;
            off[i] = (unsigned)((!TR ? min(row, avail - 1) : l) * ld * 2 + at * 2 + BIAS);
            if (!TR) last[i] = off[i] - (unsigned)(max(0, 8 - (left - p)) * 2);
            else last[i] = off[i] - (unsigned)(max(0, l - (left - 1)) * ld * 2);
        }
    }
    // elements of part i that exist, in a stage of `left` k
    __device__ __forceinline__ int count(int first, int i, int left) const
    {
        const int p = Map::part(first, i) * 8;
        return !TR ? left - p : Map::line(first, i) >= left ? 0 : edge > 0 ? edge - p : 8;
    }
    __device__ __forceinline__ void load(const char* base, int k_left)
    {
        const bool whole = k_left >= KB;
        tail = whole ? 0 : k_left;
#pragma unroll
        for (int i = 0; i < N; ++i) __builtin_memcpy(&v[i], base - BIAS + (whole ? off[i] : last[i]), 16);
    }
    // ... of an operand of less than eight
    __device__ __forceinline__ void load_tiny(const char* base, int first, int k_left)
    {
        tail = k_left < KB ? k_left : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = load8<T>(base - BIAS + off[i], 0, count(first, i, k_left));
    }
    __device__ __forceinline__ void put(unsigned dst, int first)
    {
        if (!tiny && (tail > 0 || edge > 0)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int gone = 8 - min(8, max(0, count(first, i, tail > 0 ? tail : KB)));
                const unsigned __int128 x = __builtin_bit_cast(unsigned __int128, v[i]);
                v[i] = __builtin_bit_cast(typename T::v8, gone > 7 ? (unsigned __int128)0 : x >> (gone * 16));
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            *(__attribute__((address_space(3))) typename T::v8*)((lds_char*)ff_lds + (dst + (unsigned)(first + i) * 1024 + (threadIdx.x & 63) * 16)) = v[i];
    }
};
// ... and from LDS into registers: the fragment of 32 rows and 16 k as the matrix instruction takes it (lane l: row l % 32, k = 8 (l / 32) + 0 .. 7).
template <typename T, int ROWS, bool TR, int KB> struct Reader {
    unsigned at[4];         // byte offsets, by step of 16 k (k along the rows) or by block of 32 rows (across)
    __device__ __forceinline__ void setup(int row0)
    {
        const int lane = threadIdx.x & 63, l32 = lane & 31, lhi = lane >> 5;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!TR) at[i] = (row0 + l32) * (KB * 2) + (((2 * i + lhi) ^ swizzle(l32)) << 4);
            else {
                const int f = ((lane >> 2 & 3) | lhi << 2) & (ROWS / 32 - 1);
                at[i] = (lhi * 8 + (lane >> 2 & 3)) * (ROWS * 2) + (((row0 / 32 + i) ^ f) << 6) + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
            }
        }
    }
    __device__ __forceinline__ typename T::v8 get(unsigned stage, int step, int block) const
    {
        if constexpr (!TR) {
            return *(const __attribute__((address_space(3))) typename T::v8*)((const lds_char*)ff_lds + (stage + at[step] + block * (KB * 64)));
        } else {
            const unsigned a = stage + at[block] + step * (16 * ROWS * 2);
            const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)((lds_char*)ff_lds + a));
            const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)((lds_char*)ff_lds + (a + 4 * ROWS * 2)));
            return __builtin_bit_cast(typename T::v8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

template <int I, int N, typename F> __device__ __forceinline__ void static_for(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        static_for<I + 1, N>(f);
    }
}

template <typename T, int BC, int BR, int WC, int WR, int KB, int RING, bool DIRECT, bool PT, bool QT, bool GATED, typename E>
__device__ __forceinline__ void tile(const DlfFfArgs& a, const E& extra, int block)
{
    typedef typename T::v8 v8;
    constexpr int NW = WC * WR, FC = BC / WC / 32, FR = BR / WR / 32, KS = KB / 16;
    constexpr unsigned QOFF = BC * KB * 2, STAGE = (BC + BR) * KB * 2;
    constexpr int LP = BC * KB / 512 / NW, LQ = BR * KB / 512 / NW;
    static_assert(FC <= 4 && FR <= 4 && LP >= 1 && LQ >= 1 && KS == 4, "");
    constexpr int LINES = LP * 512 / KB;                    // a wave's lines of P: of both projections of a gated tile, or of one
    constexpr bool TWO = GATED && LINES == 64;
    static_assert(!GATED || ((TWO || LINES == 32 || LINES == 16) && FC % 2 == 0 && !PT), "");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, lhi = lane >> 5;
    const int wc = wave % WC, wr = wave / WC;
    // tile
    const int per = a.tiles_r * a.tiles_c, all = per * a.problems * a.splits, each = (all + 7) >> 3;
    int t = (block & 7) * each + (block >> 3);
    if ((block >> 3) >= each || t >= all) return;
    const int split = t / (per * a.problems);
    t -= split * (per * a.problems);
    const int prob = t / per;
    t -= prob * per;
    const int band = t / (4 * a.tiles_c), rows = min(4, a.tiles_r - band * 4), in = t - band * 4 * a.tiles_c;
    constexpr int CF = GATED ? BC / 2 : BC;            // columns of C per tile
    const int r0 = (band * 4 + in % rows) * BR, c0 = in / rows * CF;

    typename std::conditional<DIRECT, Loader<LP, BC, PT, KB>, Stager<T, LP, BC, PT, KB>>::type lp;
    typename std::conditional<DIRECT, Loader<LQ, BR, QT, KB>, Stager<T, LQ, BR, QT, KB>>::type lq;
    Reader<T, BC, PT, KB> rp;
    Reader<T, BR, QT, KB> rq;
    rp.setup(wc * FC * 32);
    rq.setup(wr * FR * 32);
    const int64_t p0 = PT ? (int64_t)c0 : (int64_t)c0 * a.ldp, q0 = QT ? (int64_t)r0 : (int64_t)r0 * a.ldq;
    const int64_t pstep = (PT ? a.ldp : 1) * (KB * 2), qstep = (QT ? a.ldq : 1) * (KB * 2);   // bytes
    const char *pb, *qb, *ub = nullptr;
    int k_left;
    auto offsets = [&]() __attribute__((always_inline)) {
        if constexpr (DIRECT) {
            lp.template setup<GATED>(wave * LP, a.nc - c0, a.ldp);
            lq.template setup<false>(wave * LQ, a.nr - r0, a.ldq);
        } else {
            lp.template setup<GATED>(wave * LP, a.nc - c0, a.ldp, PT ? a.nc : a.nk, a.nk);
            lq.template setup<false>(wave * LQ, a.nr - r0, a.ldq, QT ? a.nr : a.nk, a.nk);
        }
    };
    if constexpr (!DIRECT) offsets();
    // Requests go on with stage `at` of segment w (operand pair) at the next call of next().
    auto segment = [&](int w, int at) __attribute__((always_inline)) {
        pb = (const char*)a.p[GATED ? TWO ? 0 : wave * LINES / 32 & 1 : w] + p0 * 2 + (at - 1) * pstep;
        if (TWO) ub = (const char*)a.p[1] + p0 * 2 + (at - 1) * pstep;
        qb = (const char*)a.q[GATED ? 0 : w] + q0 * 2 + (at - 1) * qstep;
        k_left = a.nk - (at - 1) * KB;
        if constexpr (DIRECT) offsets();                    // (the last stage of a segment masks them)
    };
    // this workgroup's stages, of one segment or two
    const int per_seg = (a.nk + KB - 1) / KB, stages = per_seg * a.segments;
    const int first = (int)((int64_t)stages * split / a.splits), total = (int)((int64_t)stages * (split + 1) / a.splits) - first;
    // All of k: each XCD starts an eighth of it behind the last and comes round to where it started.  Workgroups of an XCD share operands in its L2
    // and stay together; if all XCDs read the same k at a time, 8192^3 takes 3 % longer, 4096 x 16384 -> 4096 10 %.
    const int start = a.splits > 1 ? first : (int)((int64_t)total * (block & 7) >> 3);
    int seg = start >= per_seg && total > 0 ? 1 : 0, requests = total;   // segment; stages to request
    if (total > 0) segment(a.problems == 2 ? prob : seg, start - seg * per_seg);
    const unsigned lds0 = (unsigned)(size_t)(lds_char*)ff_lds;
    // The next stage's requests: first where they start, then one after the other, load 0 .. LP + LQ - 1.  Behind this workgroup's last stage direct
    // loads go on with resources of no bytes (zeros into LDS that nobody reads), so that the loop below has one form.
    i4v pres, qres, ures;
    int limit = 0x7fffffff;
    int plain = 0;                                          // further stages that need nothing but the next address
    auto next = [&]() __attribute__((always_inline)) {
        if (!DIRECT && requests == 0) return;               // the last stage's address stays: loads of it that nobody reads
        k_left -= KB;
        --requests;
        if (__builtin_expect(--plain < 0, 0)) {
            if (requests < 0) limit = 0;
            if (k_left <= 0 && requests >= 0) {
                seg = seg + 1 < a.segments ? seg + 1 : 0;
                segment(a.problems == 2 ? prob : seg, 0);
                k_left -= KB;
            }
            if constexpr (DIRECT) {
                if (k_left < KB) {
                    lp.mask(wave * LP, k_left);
                    lq.mask(wave * LQ, k_left);
                }
            }
            plain = max(0, min(requests, k_left / KB - 1));
        }
        pb += pstep;
        qb += qstep;
        if (TWO) ub += pstep;
        if constexpr (DIRECT) {
            pres = resource(pb, limit);
            if (TWO) ures = resource(ub, limit);
            qres = resource(qb, limit);
        }
    };
    auto load = [&](unsigned stage, int i) __attribute__((always_inline)) {
        if constexpr (DIRECT) {
            if (i < LP) line_to_lds(TWO && i >= LP / 2 ? ures : pres, lp.off[i], lds0 + stage + (unsigned)(wave * LP + i) * 1024);
            else line_to_lds(qres, lq.off[i - LP], lds0 + stage + QOFF + (unsigned)(wave * LQ + i - LP) * 1024);
        }
    };
    f16v acc[FC][FR];
#pragma unroll
    for (int i = 0; i < FC; ++i)
#pragma unroll
        for (int j = 0; j < FR; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    v8 fp[2][FC], fq[2][FR];
    auto read = [&](unsigned stage, int step, int set, int i) __attribute__((always_inline)) {
        if (i < FC) fp[set][i] = rp.get(stage, step, i);
        else fq[set][i - FC] = rq.get(stage + QOFF, step, i - FC);
    };
    // A step's multiplications, between them the reads of the step after it (rstep of the stage at rstage) and the requests [l0, l1)
    // for the stage at lstage: a wave that sent them all at once would wait for the memory pipe, and its multiplications with it.
    constexpr int M = FC * FR;
    auto step = [&](int set, bool reads, unsigned rstage, int rstep, unsigned lstage, int l0, int l1) __attribute__((always_inline)) {
        constexpr int RPM = M == 1 ? FC + FR : (FC + FR + M - 2) / (M > 1 ? M - 1 : 1);     // reads in front of a multiplication
        static_for<0, M>([&](auto mc) __attribute__((always_inline)) {
            constexpr int m = decltype(mc)::value, i = m / FR, j = m % FR;
            if (reads) {
#pragma unroll
                for (int r = m * RPM; r < (m + 1) * RPM; ++r)
                    if (r < FC + FR) read(rstage, rstep, set ^ 1, r);
            }
            acc[i][j] = T::mma(fp[set][i], fq[set][j], acc[i][j]);
#pragma unroll
            for (int l = l0 + m * (l1 - l0) / M; l < l0 + (m + 1) * (l1 - l0) / M; ++l) load(lstage, l);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // A stage's requests by the step that they go out in: the last of the stage that makes room for them, and the first of the next.
    constexpr int NL = LP + LQ, L0 = NL / 2;
    if (total > 0) {
        if constexpr (DIRECT) {
#pragma unroll
            for (int i = 0; i < RING; ++i) {
                next();
#pragma unroll
                for (int l = 0; l < (i < RING - 1 ? NL : L0); ++l) load(i * STAGE, l);
            }
            wait_loads<(RING - 2) * NL + L0>();
            asm volatile("s_barrier" ::: "memory");
            unsigned cur = 0, last = (RING - 1) * STAGE;
#pragma unroll
            for (int r = 0; r < FC + FR; ++r) read(cur, 0, 0, r);
            for (int s = 0; s < total - 1; ++s) {
                step(0, true, cur, 1, last, L0, NL);
                next();                                     // (here, where multiplications cover it, not behind the barrier)
                step(1, true, cur, 2, 0, 0, 0);
                step(0, true, cur, 3, 0, 0, 0);
                // this wave's reads of the stage have arrived, and so has its part of the next one
                __builtin_amdgcn_s_waitcnt(WAIT_LOADS_AND_LDS((RING - 2) * NL));
                asm volatile("s_barrier" ::: "memory");
                last = cur;
                cur = cur == (RING - 1) * STAGE ? 0 : cur + STAGE;
                step(1, true, cur, 0, last, 0, L0);
            }
#pragma unroll
            for (int k = 0; k < KS - 1; ++k) step(k & 1, true, cur, k + 1, 0, 0, 0);
            step(1, false, 0, 0, 0, 0, 0);
            wait_loads<0>();
        } else {
            // RING stages on their way in registers: stage s + 1 in set s % RING when stage s is multiplied
            decltype(lp) ps[RING];
            decltype(lq) qs[RING];
#pragma unroll
            for (int d = 0; d < RING; ++d) {
                ps[d] = lp;
                qs[d] = lq;
            }
            auto fetch = [&](int d) __attribute__((always_inline)) {
                next();
                ps[d].load(pb, k_left);
                qs[d].load(qb, k_left);
            };
            auto put = [&](unsigned stage, int d) __attribute__((always_inline)) {
                ps[d].put(stage, wave * LP);
                qs[d].put(stage + QOFF, wave * LQ);
            };
            if (lp.tiny || lq.tiny) {
                // operands of less than eight, element by element: one stage at a time
                for (int s = 0; s < total; ++s) {
                    next();
                    if (lp.tiny) ps[0].load_tiny(pb, wave * LP, k_left);
                    else ps[0].load(pb, k_left);
                    if (lq.tiny) qs[0].load_tiny(qb, wave * LQ, k_left);
                    else qs[0].load(qb, k_left);
                    __syncthreads();
                    put(0, 0);
                    __syncthreads();
#pragma unroll
                    for (int r = 0; r < FC + FR; ++r) read(0, 0, 0, r);
#pragma unroll
                    for (int k = 0; k < KS; ++k) step(k & 1, k + 1 < KS, 0, k + 1, 0, 0, 0);
                }
            } else {
                fetch(0);
                put(0, 0);
#pragma unroll
                for (int d = 0; d < RING; ++d) fetch(d);
                __builtin_amdgcn_s_waitcnt(WAIT_LDS);
                asm volatile("s_barrier" ::: "memory");
#pragma unroll
                for (int r = 0; r < FC + FR; ++r) read(0, 0, 0, r);
                auto turn = [&](int d, bool more) __attribute__((always_inline)) {
                    const unsigned cur = (d & 1) * STAGE;
                    step(0, true, cur, 1, 0, 0, 0);
                    put(STAGE - cur, d);                        // everybody has read what was there before
                    if (more) fetch(d);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int k = 1; k < KS - 1; ++k) step(k & 1, true, cur, k + 1, 0, 0, 0);
                    __builtin_amdgcn_s_waitcnt(WAIT_LDS);
                    asm volatile("s_barrier" ::: "memory");
                    step(1, true, STAGE - cur, 0, 0, 0, 0);
                };
                static_assert(RING % 2 == 0, "two slots of LDS in turn");
                int s = 0;
                for (; s + RING < total; s += RING) static_for<0, RING>([&](auto d) __attribute__((always_inline)) { turn(decltype(d)::value, true); });
                unsigned cur = 0;
                static_for<0, RING - 1>([&](auto d) __attribute__((always_inline)) {
                    if (s + decltype(d)::value + 1 < total) {
                        turn(decltype(d)::value, false);
                        cur = STAGE - cur;
                    }
                });
#pragma unroll
                for (int k = 0; k < KS - 1; ++k) step(k & 1, true, cur, k + 1, 0, 0, 0);
                step(1, false, 0, 0, 0, 0, 0);
            }
        }
    }
    if constexpr (E::OWN) {
        extra.template tile<T, FC, FR, WC>(a, acc, r0 + wr * FR * 32, c0 + wc * FC * 32, wave);
        return;
    }
    // ---- epilogue: JB * 32 rows at a time through an area of LDS that is the wave's own ----
    constexpr int JB = FR == 1 ? 1 : 2, CW = FC * 32, CROW = CW + 4, CO = GATED ? CW / 2 : CW;   // columns of the wave, floats of an LDS row, columns of C
    constexpr int LPR = CO / 8, RPU = 64 / LPR, UNITS = JB * 32 / RPU;         // lanes to a row, rows that they cover at a time
    static_assert(FR % JB == 0, "");
    float* const lf = (float*)ff_lds + wave * (JB * 32 * CROW);
    const int cw = lane % LPR * 8, c = c0 + wc * CO + cw, rw = lane / LPR;
    const float* const src = lf + rw * CROW + (GATED ? (cw >> 5) * 64 + (cw & 31) : cw);
    float* const part = a.part + (int64_t)(split * (GATED ? 2 : a.problems) + prob) * a.nr * a.nc;
    __syncthreads();
    const auto last = extra.ready();
#pragma unroll
    for (int j = 0; j < FR; j += JB) {
#pragma unroll
        for (int b = 0; b < JB; ++b)
#pragma unroll
            for (int i = 0; i < FC; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(f4v*)(lf + (b * 32 + l32) * CROW + i * 32 + q * 8 + lhi * 4) =
                        f4v{acc[i][j + b][q * 4], acc[i][j + b][q * 4 + 1], acc[i][j + b][q * 4 + 2], acc[i][j + b][q * 4 + 3]};
        __builtin_amdgcn_wave_barrier();
        const int r = r0 + (wr * FR + j) * 32 + rw;
        if (a.nc - c >= 8) {
            constexpr int AT = UNITS < 4 ? UNITS : 4;                          // units whose waits are shared
#pragma unroll 1
            for (int u = 0; u < UNITS; u += AT) {
                float v[AT][8], w[AT][8];
#pragma unroll
                for (int k = 0; k < AT; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        *(f4v*)(v[k] + e * 4) = *(const f4v*)(src + (u + k) * RPU * CROW + e * 4);
                        if (GATED) *(f4v*)(w[k] + e * 4) = *(const f4v*)(src + (u + k) * RPU * CROW + 32 + e * 4);
                    }
                if (a.splits > 1) {
#pragma unroll
                    for (int k = 0; k < AT; ++k) {
                        const int ru = r + (u + k) * RPU;
                        if (ru >= a.nr) continue;
                        store_floats(part + (int64_t)ru * a.nc + c, 8, v[k]);
                        if (GATED) store_floats(part + ((int64_t)a.nr + ru) * a.nc + c, 8, w[k]);
                    }
                } else {
                    finish_many<T, GATED, AT>(a, last, prob, r + u * RPU, RPU, c, v, w);
                }
            }
        }
        // columns behind the last eight: a lane to a row
        const int cols = a.nc - c0 - wc * CO, ct = cols & ~7, rt = r0 + (wr * FR + j) * 32 + lane;
        if (cols < CO && (cols & 7) != 0 && cols > 0 && lane < JB * 32 && rt < a.nr) {
            float v[8], w[8];
            const float* const st = lf + lane * CROW + (GATED ? (ct >> 5) * 64 + (ct & 31) : ct);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                *(f4v*)(v + e * 4) = *(const f4v*)(st + e * 4);
                if (GATED) *(f4v*)(w + e * 4) = *(const f4v*)(st + 32 + e * 4);
            }
            const int ca = c0 + wc * CO + ct, n = cols & 7;
            if (a.splits > 1) {
                store_floats(part + (int64_t)rt * a.nc + ca, n, v);
                if (GATED) store_floats(part + ((int64_t)a.nr + rt) * a.nc + ca, n, w);
            } else {
                finish<T, GATED, 8>(a, last, prob, rt, ca, n, v, w);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Column sums: the partial sums of 64 columns added in order, four threads to a column: the result does not depend on which workgroup came
// first.
__device__ __forceinline__ void add_sums(const DlfFfSumArgs& a, int block)
{
    const int l = threadIdx.x & 63, g = threadIdx.x >> 6, per = (a.n + 63) >> 6, z = block / per, col = (block - z * per) * 64 + l;
    float* const part = (float*)ff_lds;
    const float* const p = a.part[z];
    float t = 0.0f;
    if (p != nullptr && col < a.n) {
#pragma unroll 8
        for (int k = g; k < a.chunks; k += 4) t += p[(int64_t)k * a.n + col];
    }
    part[threadIdx.x] = t;
    __syncthreads();
    if (p != nullptr && g == 0 && col < a.n) a.out[z][col] = (part[l] + part[l + 64]) + (part[l + 128] + part[l + 192]);
}

// k_ff_join: the sums over the splits of k, in order, and the epilogue.  Bound by memory: 117 MB in 20 us.  Chosen where it costs less than
// the compute units that the tiles alone leave idle.
template <typename T, bool GATED, typename E> __device__ __forceinline__ void join(const DlfFfArgs& a, const E& extra, int64_t unit)
{
    const int cols = (a.nc + 7) >> 3;
    const int64_t plane = (int64_t)a.nr * a.nc;
    const int64_t row = unit / cols;
    const int c = (int)(unit - row * cols) * 8, n = a.nc - c;
    const int prob = row >= a.nr ? 1 : 0, r = (int)(row - (prob ? a.nr : 0));
    if (prob >= a.problems || r >= a.nr) return;
    const int planes = GATED ? 2 : a.problems;
    const float* p = a.part + prob * plane + (int64_t)r * a.nc + c;
    float v[8], u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = u[i] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        float x[8], y[8];
        load_floats(p + s * planes * plane, n, x);
        if (GATED) load_floats(p + (s * 2 + 1) * plane, n, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] += x[i];
            if (GATED) u[i] += y[i];
        }
    }
    finish<T, GATED, 8>(a, extra.ready(), prob, r, c, n, v, u);
}

// The waves' partial sums of a workgroup's 16 NF features x 16 MR rows meet in LDS, in the order of the waves.
template <typename T, int NF, int MR, bool GATED, typename E>
__device__ __forceinline__ void few_finish(const DlfFfArgs& a, const E& extra, const f4v (&acc)[GATED ? 2 : NF][MR], int c0, int r0, int wave, int waves)
{
    const int lane = threadIdx.x & 63, l16 = lane & 15;
    __syncthreads();
    // [wave][block][lane] four consecutive c of row lane % 16
    f4v* const part = (f4v*)ff_lds;
    constexpr int NP = GATED ? 2 : NF, NB = NP * MR;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < MR; ++j) part[(wave * NB + i * MR + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int b = wave; b < NF * MR; b += waves) {
        const int i = b / MR, j = b - i * MR;
        f4v v = f4v{0.0f, 0.0f, 0.0f, 0.0f}, u = v;
        for (int w = 0; w < waves; ++w) {
            v += part[(w * NB + i * MR + j) * 64 + lane];
            if (GATED) u += part[(w * NB + MR + j) * 64 + lane];
        }
        const int r = r0 + j * 16 + l16, c = c0 + i * 16 + (lane >> 4) * 4;
        if constexpr (E::OWN) {
            extra.few(a, v, r, c);
        } else if (r < a.nr && c < a.nc) {
            float fv[4] = {v.x, v.y, v.z, v.w}, fu[4] = {u.x, u.y, u.z, u.w};
            finish<T, GATED, 4>(a, extra, 0, r, c, a.nc - c, fv, fu);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// k_ff_few: the forward product of few rows: one token, a handful of requests.  Bound by the weights' bytes, or for small layers by the
// launch and one round trip to memory: nothing is staged, every wave reads its operands from memory straight into the registers
// that v_mfma_f32_16x16x32 takes them from.  A workgroup computes 16 NF features (gated: 16 of both projections) for 16 MR rows, its waves
// share k in equal runs of 32-wide steps and meet in LDS, in a fixed order.  A wave keeps D steps requested.  Rows that do not exist are
// read as the last that does and not stored; a last step that is not whole is the last wave's, requested first.  On the operands of
// k_ff_rows, whose figures are below: 5 x 2048 -> 32001 27.0 us, 1 x 4096 -> 2 x 10880 35.4, 16 x 2048 -> 2 x 5632 14.2, 64 x 4096 -> 4096 17.9.
// ------------------------------------------------------------------------------------------------
template <typename T, int NF, int MR, bool GATED, typename E>
__device__ __forceinline__ void few(const DlfFfArgs& a, const E& extra)
{
    typedef typename T::e e;
    typedef typename T::v8 v8;
    constexpr int NP = GATED ? 2 : NF, D = NP + MR == 2 ? 8 : 6;     // W fragments of a step; steps requested ahead
    static_assert(!GATED || NF == 1, "");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int l16 = lane & 15, kg = (lane >> 4) * 8;
    const int bc = (blockIdx.x >> 3) / a.tiles_r * 8 + (blockIdx.x & 7);   // all rows of a feature group on one XCD: they share its weights
    if (bc >= a.tiles_c) return;
    const int c0 = bc * (16 * NF), r0 = (blockIdx.x >> 3) % a.tiles_r * (16 * MR);
    const int steps = a.nk >> 5, s0 = (int)((int64_t)steps * wave / waves), s1 = (int)((int64_t)steps * (wave + 1) / waves);
    const e *wp[NP], *xp[MR];
#pragma unroll
    for (int i = 0; i < NP; ++i)
        wp[i] = (const e*)a.p[GATED ? i : 0] + (int64_t)min(c0 + (GATED ? 0 : i * 16) + l16, a.nc - 1) * a.ldp + kg;
#pragma unroll
    for (int j = 0; j < MR; ++j) xp[j] = (const e*)a.q[0] + (int64_t)min(r0 + j * 16 + l16, a.nr - 1) * a.ldq + kg;
    f4v acc[NP][MR];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < MR; ++j) acc[i][j] = f4v{0.0f, 0.0f, 0.0f, 0.0f};
    const bool last = wave == waves - 1 && (a.nk & 31) != 0;
    v8 tw[NP], tx[MR];
    if (last) {
        const int k = steps * 32, n = a.nk - k - kg;
#pragma unroll
        for (int i = 0; i < NP; ++i) tw[i] = load8<T>(wp[i], k, n);
#pragma unroll
        for (int j = 0; j < MR; ++j) tx[j] = load8<T>(xp[j], k, n);
    }
    if (s0 < s1) {
        v8 w[D][NP], x[D][MR];
        auto request = [&](int s, int slot) __attribute__((always_inline)) {
            const int64_t k = (int64_t)s * 32;
#pragma unroll
            for (int i = 0; i < NP; ++i) __builtin_memcpy(&w[slot][i], wp[i] + k, 16);
#pragma unroll
            for (int j = 0; j < MR; ++j) __builtin_memcpy(&x[slot][j], xp[j] + k, 16);
        };
        auto multiply = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < MR; ++j) acc[i][j] = T::mma16(w[slot][i], x[slot][j], acc[i][j]);
        };
#pragma unroll
        for (int d = 0; d < D; ++d) request(min(s0 + d, s1 - 1), d);
        int s = s0;
        for (; s + 2 * D <= s1; s += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                multiply(d);
                request(s + D + d, d);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int d = 0; d < D; ++d) {
            if (s + d < s1) multiply(d);
            if (s + D + d < s1) request(s + D + d, d);
        }
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (s + D + d < s1) multiply(d);
    }
    if (last) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < MR; ++j) acc[i][j] = T::mma16(tw[i], tx[j], acc[i][j]);
    }
    few_finish<T, NF, MR, GATED>(a, extra, acc, c0, r0, wave, waves);
}

// ------------------------------------------------------------------------------------------------
// k_ff_rows: k_ff_few for operands whose rows are whole 16-byte lines.  There a wave's load takes 64 bytes of each of 16 rows, and pieces
// of many lines cost a compute unit several times their size; here the operands come as whole 128-byte lines, eight rows per
// instruction, into a ring in LDS that belongs to the wave alone: 64 k ("stage") of its features and rows at a time, D stages
// requested ahead, no barrier before the waves meet.  LDS holds a stage as k_ff_tile does.  5 x 2048 -> 32001 takes 24.6 us (5.3 TB/s
// of weights), 1 x 4096 -> 2 x 10880 32 us (5.6), 16 x 2048 -> 2 x 5632 10.1 (4.6), 1 x 1024 -> 1024 3.8 (a launch and a round trip); more rows
// read x oftener: 64 x 2048 -> 2 x 5632 13.0, 64 x 4096 -> 4096 10.9 (3.1).
// ------------------------------------------------------------------------------------------------
template <typename T, int NF, int MR, bool GATED, typename E>
__device__ __forceinline__ void rows_in_lds(const DlfFfArgs& a, const E& extra)
{
    typedef typename T::v8 v8;
    constexpr int NP = GATED ? 2 : NF, D = DLF_FF_ROWS_RING, LW = GATED ? 2 : 2 * NF, L = 2 * (NP + MR);
    constexpr unsigned STAGE = L * 1024, XOFF = 2 * NP * 1024;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int l16 = lane & 15;
    const int bc = (blockIdx.x >> 3) / a.tiles_r * 8 + (blockIdx.x & 7);   // all rows of a feature group on one XCD: they share its weights
    if (bc >= a.tiles_c) return;
    const int c0 = bc * (16 * NF), r0 = (blockIdx.x >> 3) % a.tiles_r * (16 * MR);
    const int stages = (a.nk + 63) >> 6, s0 = (int)((int64_t)stages * wave / waves), s1 = (int)((int64_t)stages * (wave + 1) / waves);
    Loader<LW, 64, false, 64> lw;
    Loader<2 * MR, 64, false, 64> lx;
    lw.template setup<false>(0, a.nc - c0, a.ldp);
    lx.template setup<false>(0, a.nr - r0, a.ldq);
    const char* wb[2] = {(const char*)a.p[0] + (int64_t)c0 * a.ldp * 2, GATED ? (const char*)a.p[1] + (int64_t)c0 * a.ldp * 2 : nullptr};
    const char* xb = (const char*)a.q[0] + (int64_t)r0 * a.ldq * 2;
    const unsigned ring = (unsigned)wave * (D * STAGE), lds0 = (unsigned)(size_t)(lds_char*)ff_lds + ring;
    auto issue = [&](int s) __attribute__((always_inline)) {
        const unsigned slot = lds0 + (unsigned)(s % D) * STAGE;
        const int left = a.nk - s * 64;
        const int64_t at = (int64_t)s * 128;
        if (left >= 64) {
            lw.template issue<false>(resource(wb[0] + at), 0, slot, 64);
            if (GATED) lw.template issue<false>(resource(wb[1] + at), 0, slot + 2048, 64);
            lx.template issue<false>(resource(xb + at), 0, slot + XOFF, 64);
        } else {
            lw.template issue<true>(resource(wb[0] + at), 0, slot, left);
            if (GATED) lw.template issue<true>(resource(wb[1] + at), 0, slot + 2048, left);
            lx.template issue<true>(resource(xb + at), 0, slot + XOFF, left);
        }
    };
    f4v acc[NP][MR];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < MR; ++j) acc[i][j] = f4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (s0 + d < s1) issue(s0 + d);
    unsigned at[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) at[k] = ring + l16 * 128 + (((k * 4 + (lane >> 4)) ^ (l16 >> 1)) << 4);
    for (int s = s0; s < s1; ++s) {
        if (s + D <= s1) wait_loads<(D - 1) * L>();
        else wait_loads<0>();
        const unsigned slot = (unsigned)(s % D) * STAGE;
        v8 w[2][NP], x[2][MR];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int i = 0; i < NP; ++i) w[k][i] = *(const __attribute__((address_space(3))) v8*)((const lds_char*)ff_lds + (slot + at[k] + i * 2048));
#pragma unroll
            for (int j = 0; j < MR; ++j) x[k][j] = *(const __attribute__((address_space(3))) v8*)((const lds_char*)ff_lds + (slot + at[k] + XOFF + j * 2048));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < MR; ++j) acc[i][j] = T::mma16(w[k][i], x[k][j], acc[i][j]);
        if (s + D < s1) {
            __builtin_amdgcn_s_waitcnt(WAIT_LDS);             // the slot has been read
            __builtin_amdgcn_sched_barrier(0);
            issue(s + D);
        }
    }
    few_finish<T, NF, MR, GATED>(a, extra, acc, c0, r0, wave, waves);
}

// A workgroup's waves per SIMD that the registers have to allow: one of 128 x 128 blocks per wave, else two.
#define FF_TILE_BOUNDS __launch_bounds__(WC* WR * 64, BC * BR / (WC * WR) > 8192 ? 1 : 2)
