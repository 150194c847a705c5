// gfx950 (CDNA4) kernels of the cross entropy of a linear layer over many classes, without its logits in memory.  The products are those of dlf_tile.h;
// what is here are their epilogues, and what joins them.
//
//   lse = log sum_c exp z_c: every wave leaves, for each row and its 32 to 128 classes, the maximum m and s = sum exp(z - m), which
//   k_ce_join adds up as sum s exp(m - M).  dz_c = (dloss + dlse) exp(z_c - lse) - dloss [c = target].
#include "dlf_tile.h"
#include "dlf_ce.h"

#define LOG2_E 1.44269504f
#define LN_2 0.693147181f
#define MINUS_INF (-__builtin_inff())
// exp(d).  d is rounded before it is multiplied: a maximum times log2(e), rounded, would shift all of a row's exponentials.
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2_E); }

// ... to the last place: with what the product with log2(e) rounds off.  (-infinity: the difference of two of them would be none.)
__device__ __forceinline__ float exp_of_all(float d)
{
    d = d < -200.0f ? -200.0f : d;
    const float t = d * LOG2_E, off = __builtin_fmaf(d, 1.925963e-8f, __builtin_fmaf(d, LOG2_E, -t)), v = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(v, off * LN_2, v);
}

// Exponentials kept in 16 bits, two to a word: from 0 to 1, an exponent of five bits and eleven bits behind the point, a bit more than fp16, whose sign
// they do not need.  They are bits 12 to 27 of the number times 2^-96 in 32 bits, so that reading one back is a shift and a product with 2^96, both exact
// (as a part of its row's factor 2^96 would make that infinite beside a large gradient, and a lost exponential NaN).  What is below 2^-42 is lost;
// 1 is exact, so that 1 - p of a sure target is.  (NaN is not kept: such a row's sum says so.)
__device__ __forceinline__ uint32_t kept_of(float x0, float x1)
{
    const uint32_t b0 = __builtin_bit_cast(uint32_t, x0 * 0x1p-96f) + 0x800u, b1 = __builtin_bit_cast(uint32_t, x1 * 0x1p-96f) + 0x800u;
    return (b1 & 0x0ffff000u) << 4 | (b0 >> 12 & 0xffffu);
}
__device__ __forceinline__ float from_kept(uint32_t w, int i)
{
    return __builtin_bit_cast(float, (i ? w >> 4 : w << 12) & 0x0ffff000u) * 0x1p96f;
}

// How dz is scaled: products of it are undone by scale_back.  One dloss for all rows is left out of dz but for its sign and comes back as a factor in 32
// bits: rounded with every element, it would bring its own rounding into all of them.  fp16: see k_ce_unit.
__device__ __forceinline__ float the_dloss(const DlfCeGiven& g) { return g.dloss != nullptr ? g.dloss[0] : g.dloss_value; }
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) <= 3.402823466e38f; }
__device__ __forceinline__ float scale_back(const DlfCeGiven& g)
{
    if (g.one > 0.0f) {
        const float d = fabsf(the_dloss(g));
        return is_finite(d) ? d / g.one : 1.0f;
    }
    return g.unit != nullptr ? g.unit[1] : 1.0f;
}
// A row's part of the gradient: dz = total * exp(z - lse) - own at the target.
struct RowGradient {
    float total, own;
};
__device__ __forceinline__ RowGradient row_gradient(const DlfCeGiven& g, int64_t r, int64_t t, int64_t ignore, int nc)
{
    RowGradient q;
    if (g.one > 0.0f) {
        const float d = the_dloss(g);
        q.own = t == ignore || d == 0.0f ? 0.0f : is_finite(d) ? copysignf(g.one, d) : __builtin_nanf("");
        q.total = q.own;
    } else {
        q.own = t == ignore ? 0.0f : g.dloss != nullptr ? g.dloss[r * g.dloss_stride] : g.dloss_value;
        float l = g.dlse != nullptr ? g.dlse[r * g.dlse_stride] : 0.0f;
        if (g.unit != nullptr) {
            const float u = g.unit[0];
            q.own *= u;
            l *= u;
        }
        q.total = q.own + l;
    }
    if (t != ignore && (t < 0 || t >= nc)) q.total = __builtin_nanf("");        // no class: not silently anything
    return q;
}

// What the rounding of eight elements to type T takes from them.
template <typename T> __device__ __forceinline__ void store_low(void* low, int64_t at, const float (&v)[8])
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v[i] - (float)(typename T::e)v[i];
    store_some<T, 8>(low, at, 8, f);
}

// ------------------------------------------------------------------------------------------------
// The epilogues of a tile.  A lane holds, of one row of each block of 32, every other four of the wave's columns: a row's maximum and sum are its own
// and one other lane's, without LDS.  The target's logit lies in one of the lane's registers, which is looked for only where a row of the
// block has its target among the wave's columns.
// ------------------------------------------------------------------------------------------------
template <int MODE> struct Entropy {
    static constexpr bool OWN = true, SUMS = false;
    const DlfCeArgs& e;
    __device__ __forceinline__ const Entropy& ready() const { return *this; }

    template <typename T, int FC, int FR, int WC>
    __device__ __forceinline__ void tile(const DlfFfArgs& a, f16v (&acc)[FC][FR], int row0, int col0, int wave) const
    {
        constexpr int CW = FC * 32, CROW = CW + 4, LPR = CW / 8, RPU = 64 / LPR;   // columns of the wave, floats of an LDS row, lanes to a row, rows of a store
        const int lane = threadIdx.x & 63, l32 = lane & 31, lhi = lane >> 5, left = a.nc - col0;
        if (MODE == DLF_CE_DZ && e.back != nullptr && row0 == 0 && col0 == 0 && lane == 0) *e.back = scale_back(e.given);
        // stores go through an area of LDS that is the wave's own, so that they are whole lines
        float* const lf = (float*)ff_lds + wave * (32 * CROW);
        const int cw = lane % LPR * 8, rw = lane / LPR;
        float sum[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
        if (MODE != DLF_CE_STAT) __syncthreads();
        if (left <= 0) return;                              // a wave behind the last class
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            // One block of 32 rows at a time: the accumulators leave few registers.  (Comparisons and loads of one block are not kept for the next.)
            __builtin_amdgcn_sched_barrier(0);
            int mine = lhi * 4;
            asm volatile("" : "+v"(mine)::"memory");
            float z[FC][16];
#pragma unroll
            for (int i = 0; i < FC; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    z[i][k] = acc[i][j][k];
                    asm volatile("" : "+v"(z[i][k]));       // (read here, not where the product ends)
                }
            if (a.bias[0] != nullptr) {
                const float* const b = a.bias[0] + col0 + mine;
                if (left >= CW) {
#pragma unroll
                    for (int i = 0; i < FC; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float four[4];
                            __builtin_memcpy(four, b + i * 32 + q * 8, 16);
#pragma unroll
                            for (int k = 0; k < 4; ++k) z[i][q * 4 + k] += four[k];
                        }
                } else {
                    const int last = left - 1 - mine;       // (of columns that do not exist any: they are cut)
#pragma unroll
                    for (int i = 0; i < FC; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) z[i][k] += b[min(i * 32 + (k >> 2) * 8 + (k & 3), last)];
                }
            }
            auto cut = [&](float v) __attribute__((always_inline)) {            // columns that do not exist
                if (left >= CW) return;
#pragma unroll
                for (int i = 0; i < FC; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) z[i][k] = i * 32 + (k >> 2) * 8 + (k & 3) >= left - mine ? v : z[i][k];
            };
            const int r = row0 + j * 32 + l32, at = min(r, a.nr - 1);
            const int64_t t = e.target[at];
            const int rel = (t >= 0 && t < a.nc ? (int)t - col0 : -8) - mine;  // the target's place among the lane's columns
            const bool near = r < a.nr && rel >= -4 && rel < CW;
            // f on the target's logit, in the lane that holds it
            auto target = [&](auto&& f) __attribute__((always_inline)) {
                if (__builtin_amdgcn_ballot_w64(near) == 0) return;
#pragma unroll
                for (int i = 0; i < FC; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (near && rel == i * 32 + (k >> 2) * 8 + (k & 3)) z[i][k] = f(z[i][k]);
            };
            auto to_lds = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < FC; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *(f4v*)(lf + l32 * CROW + i * 32 + q * 8 + lhi * 4) = f4v{z[i][q * 4], z[i][q * 4 + 1], z[i][q * 4 + 2], z[i][q * 4 + 3]};
            };
            if constexpr (MODE == DLF_CE_DZ) {
                RowGradient g = row_gradient(e.given, at, t, e.ignore, a.nc);
                if (r >= a.nr) g.total = g.own = 0.0f;
                const float lse = e.lse[at], total = g.total;
                // (to the last place for the bias's gradient only: it is half of this epilogue, which a tile of few stages shows)
                if (e.sums != nullptr) {
#pragma unroll
                    for (int i = 0; i < FC; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) z[i][k] = total * exp_of_all(z[i][k] - lse);
                } else {
#pragma unroll
                    for (int i = 0; i < FC; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) z[i][k] = total * exp_of(z[i][k] - lse);
                }
                if (__builtin_amdgcn_ballot_w64(g.total == 0.0f) != 0) {        // rows without a gradient, whatever their logits are
#pragma unroll
                    for (int i = 0; i < FC; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) z[i][k] = g.total == 0.0f ? 0.0f : z[i][k];
                }
                if (e.rest != nullptr && col0 == 0 && lhi == 0 && r < a.nr && (t < 0 || t >= a.nc)) e.rest[r] = 0.0f;
                target([&](float v) __attribute__((always_inline)) {
                    v -= g.own;
                    if (e.rest != nullptr) e.rest[r] = v - (float)(typename T::e)v;
                    return v;
                });
                cut(0.0f);
            } else {
                float m = MINUS_INF, s = 0.0f;
                cut(MINUS_INF);
                if (MODE == DLF_CE_LOGITS) to_lds();
#pragma unroll
                for (int i = 0; i < FC; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) m = fmaxf(m, z[i][k]);
                m = fmaxf(m, __shfl_xor(m, 32, 64));
                target([&](float v) __attribute__((always_inline)) { return e.at[r] = v; });
                const float from = m == MINUS_INF ? 0.0f : m;
#pragma unroll
                for (int i = 0; i < FC; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        z[i][k] = exp_of(z[i][k] - from);
                        s += z[i][k];
                    }
                s += __shfl_xor(s, 32, 64);
                if (lhi == 0 && r < a.nr) {
                    const float2 both = {m, s};
                    *(float2*)(e.part + ((int64_t)(col0 / CW) * a.nr + r) * 2) = both;
                }
            }
            if constexpr (MODE != DLF_CE_STAT) {
                if (MODE != DLF_CE_LOGITS) to_lds();
                __builtin_amdgcn_wave_barrier();
#pragma unroll 2
                for (int u = 0; u < 32; u += RPU) {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 2; ++k) *(f4v*)(v + k * 4) = *(const f4v*)(lf + (u + rw) * CROW + cw + k * 4);
                    const int ru = row0 + j * 32 + u + rw;
                    const bool in = ru < a.nr && col0 + cw < e.ldz;
                    const int64_t to = (int64_t)ru * e.ldz + col0 + cw;
                    if (MODE == DLF_CE_DZ) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[i] += v[i];             // (zeros in rows that do not exist)
                        // one rounding to the type that the matrix units multiply
                        if (in) store_some<T, 8>(e.dz, to, 8, v);
                        if (in && e.low != nullptr) store_low<T>(e.low, to, v);
                    } else if (MODE == DLF_CE_LOGITS) {
                        if (in) __builtin_memcpy(e.z + to, v, 32);
                    } else {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = kept_of(v[i * 2], v[i * 2 + 1]);
                        if (in) __builtin_memcpy((uint16_t*)e.dz + to, w, 16);
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        if (MODE == DLF_CE_DZ && e.sums != nullptr) {
#pragma unroll
            for (int d = LPR; d < 64; d <<= 1)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += __shfl_xor(sum[i], d, 64);
            const float back = scale_back(e.given);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] *= back;
            const int c = col0 + cw;
            if (lane < LPR && c < a.nc) store_floats(e.sums + (int64_t)(row0 / (FR * 32)) * a.nc + c, a.nc - c, sum);
        }
    }

    // Few rows: a block of 16 classes and 16 rows, a lane's four classes of row lane % 16.
    __device__ __forceinline__ void few(const DlfFfArgs& a, f4v v, int r, int c) const
    {
        float z[4] = {v.x, v.y, v.z, v.w}, m = MINUS_INF, s = 0.0f;
        if (a.bias[0] != nullptr) {
            float b[4];
            load_floats(a.bias[0] + c, a.nc - c, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] += b[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[i] = c + i < a.nc ? z[i] : MINUS_INF;
            m = fmaxf(m, z[i]);
        }
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const float from = m == MINUS_INF ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < 4; ++i) s += exp_of(z[i] - from);
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
        const int first = c & ~15;
        if (r >= a.nr || first >= a.nc) return;
        if (e.z != nullptr && c < e.ldz) *(f4v*)(e.z + (int64_t)r * e.ldz + c) = f4v{z[0], z[1], z[2], z[3]};
        const int64_t t = e.target[r];
        if (t >= c && t < c + 4 && t < a.nc) e.at[r] = t == c ? z[0] : t == c + 1 ? z[1] : t == c + 2 ? z[2] : z[3];
        if (c == first) {
            const float2 both = {m, s};
            *(float2*)(e.part + ((int64_t)(first >> 4) * a.nr + r) * 2) = both;
        }
    }
};

template <typename T, int BC, int BR, int WC, int WR, int KB, int RING, bool DIRECT, int MODE>
__global__ FF_TILE_BOUNDS void k_ce_tile(const DlfCeArgs e)
{
    tile<T, BC, BR, WC, WR, KB, RING, DIRECT, false, false, false>(e.t, Entropy<MODE>{e}, blockIdx.x);
}
template <typename T, int NF, int MR>
__global__ __launch_bounds__(512, NF + MR <= 3 ? 4 : 2) void k_ce_few(const DlfCeArgs e)
{
    few<T, NF, MR, false>(e.t, Entropy<DLF_CE_STAT>{e});
}
template <typename T, int NF, int MR>
__global__ __launch_bounds__(512) void k_ce_rows(const DlfCeArgs e)
{
    rows_in_lds<T, NF, MR, false>(e.t, Entropy<DLF_CE_STAT>{e});
}

// ------------------------------------------------------------------------------------------------
// k_ce_join: a row's parts to its lse and loss.  ROWS of them to a workgroup, its other threads share the parts, in a fixed order.
// ------------------------------------------------------------------------------------------------
// Sums s of exp(z - m) over parts of the classes, brought together.
struct Parts {
    float m = MINUS_INF, s = 0.0f;
    __device__ __forceinline__ void add(float m2, float s2)
    {
        const float top = fmaxf(m, m2), from = top == MINUS_INF ? 0.0f : top;
        s = s * exp_of(m - from) + s2 * exp_of(m2 - from);
        m = top;
    }
    // ... those of parts first, first + step, ... of row r
    __device__ __forceinline__ void take(const float* part, int parts, int nr, int r, int first, int step)
    {
        constexpr int AT = 8;                               // parts whose loads share a wait
        for (int p = first; p < parts; p += AT * step) {
            float2 v[AT];
#pragma unroll
            for (int k = 0; k < AT; ++k) v[k] = *(const float2*)(part + ((int64_t)min(p + k * step, parts - 1) * nr + r) * 2);
            float top = m;
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                if (p + k * step >= parts) v[k] = float2{MINUS_INF, 0.0f};
                top = fmaxf(top, v[k].x);
            }
            const float from = top == MINUS_INF ? 0.0f : top;
            s *= exp_of(m - from);
#pragma unroll
            for (int k = 0; k < AT; ++k) s += v[k].y * exp_of(v[k].x - from);
            m = top;
        }
    }
    __device__ __forceinline__ float lse() const { return m == MINUS_INF ? (s == s ? MINUS_INF : s) : m + __builtin_amdgcn_logf(s) * LN_2; }
};
__device__ __forceinline__ float loss_of(float lse, int64_t t, int64_t ignore, int nc, const float* at)
{
    return t == ignore ? 0.0f : t < 0 || t >= nc ? __builtin_nanf("") : lse - *at;
}
// A row's parts in all of a workgroup's 256 threads, in a fixed order.
__device__ __forceinline__ Parts all_parts(const float* part, int parts, int nr, int r)
{
    __shared__ float2 waves[4];
    Parts q;
    q.take(part, parts, nr, r, threadIdx.x, 256);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const float m = __shfl_xor(q.m, d, 64), s = __shfl_xor(q.s, d, 64);
        // (the same two in the same order in either lane)
        Parts u;
        const bool low = (threadIdx.x & d) == 0;
        u.m = low ? q.m : m;
        u.s = low ? q.s : s;
        u.add(low ? m : q.m, low ? s : q.s);
        q = u;
    }
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = float2{q.m, q.s};
    __syncthreads();
    Parts all;
#pragma unroll
    for (int w = 0; w < 4; ++w) all.add(waves[w].x, waves[w].y);
    return all;
}

template <int ROWS> __global__ __launch_bounds__(256) void k_ce_join(const DlfCeJoinArgs a)
{
    if constexpr (ROWS == 1) {
        const int r = blockIdx.x;
        const Parts q = all_parts(a.part, a.parts, a.nr, r);
        if (threadIdx.x != 0) return;
        const float lse = q.lse();
        if (a.lse != nullptr) a.lse[r] = a.inverse != nullptr ? q.m : lse;
        if (a.inverse != nullptr) a.inverse[r] = 1.0f / q.s;
        if (a.loss != nullptr) a.loss[r] = loss_of(lse, a.target[r], a.ignore, a.nc, a.at + r);
    } else {
        constexpr int GROUPS = 256 / ROWS;
        __shared__ float2 shared[256];
        const int r = blockIdx.x * ROWS + threadIdx.x % ROWS, g = threadIdx.x / ROWS;
        Parts q;
        if (r < a.nr) q.take(a.part, a.parts, a.nr, r, g, GROUPS);
        shared[threadIdx.x] = float2{q.m, q.s};
#pragma unroll
        for (int h = GROUPS / 2; h > 0; h >>= 1) {
            __syncthreads();
            if (g < h) {
                const float2 v = shared[threadIdx.x + h * ROWS];
                q.add(v.x, v.y);
                shared[threadIdx.x] = float2{q.m, q.s};
            }
        }
        if (g != 0 || r >= a.nr) return;
        const float lse = q.lse();
        if (a.lse != nullptr) a.lse[r] = a.inverse != nullptr ? q.m : lse;
        if (a.inverse != nullptr) a.inverse[r] = 1.0f / q.s;
        if (a.loss != nullptr) a.loss[r] = loss_of(lse, a.target[r], a.ignore, a.nc, a.at + r);
    }
}

// ------------------------------------------------------------------------------------------------
// k_ce_dz: dz from the exponentials kept, in their place: each times dloss exp(its part's maximum - the row's) / the row's sum.  A workgroup takes
// a slice of a row.  Where all of them run at once, each forms its row's lse by itself: a launch for that costs more.  Bound by memory: 4096 rows of
// 32000 classes 91 us (5.8 TB/s, some of it from the last-level cache; with 2^96 in `by` and lse alone 87); formed by each workgroup, the call takes 81 longer.
// ------------------------------------------------------------------------------------------------
// LOGITS: from the logits of few rows, which have been kept in 32 bits.
template <typename T, bool FORM, bool LOGITS> __global__ __launch_bounds__(256) void k_ce_dz(const DlfCeDzArgs a)
{
    static_assert(FORM || !LOGITS, "");
    const int r = blockIdx.x / a.slices, c = (blockIdx.x - r * a.slices) * DLF_CE_DZ_COLS + threadIdx.x * 8;
    // the loads first: what follows branches
    const bool in = c < a.ldz;
    const int64_t at = (int64_t)r * a.ldz + c, t = a.target[r];
    uint32_t q[4];
    float z[8], m = 0.0f, by;
    if (in) {
        if (LOGITS) {
            __builtin_memcpy(z, a.z + at, 32);
        } else {
            __builtin_memcpy(q, (const uint16_t*)a.dz + at, 16);
            m = a.part[((int64_t)(c >> __builtin_ctz(a.width)) * a.nr + r) * 2];
        }
    }
    // By the row's maximum and 1 / sum: lse in 32 bits would be off by 2^-24 |lse|, and so would each p, which is all that 1 - p of a sure target is.
    if constexpr (FORM) {
        const Parts all = all_parts(a.part, a.parts, a.nr, r);
        if (c == 0) a.loss[r] = loss_of(all.lse(), t, a.ignore, a.nc, a.at + r);
        by = (LOGITS ? 1.0f : exp_of(m - all.m)) / all.s;
        if (LOGITS) m = all.m;
    } else {
        by = exp_of(m - a.lse[r]) * a.inverse[r];
    }
    if (a.back != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *a.back = scale_back(a.given);
    if (!in) return;
    const RowGradient g = row_gradient(a.given, r, t, a.ignore, a.nc);
    by *= g.total;
    const int64_t rel = t - c;
    float v[8];
    if (c == 0 && (t < 0 || t >= a.nc)) a.rest[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = g.total == 0.0f ? 0.0f : (LOGITS ? exp_of(z[i] - m) : from_kept(q[i >> 1], i & 1)) * by;
        if (c + i >= a.nc) v[i] = 0.0f;
        if (rel == i && c + i < a.nc) {
            if (t != a.ignore) v[i] -= g.own;
            a.rest[r] = v[i] - (float)(typename T::e)v[i];
        }
    }
    store_some<T, 8>(a.dz, at, 8, v);
    if (a.low != nullptr) store_low<T>(a.low, at, v);
}

// k_ce_dz_sums: dz from the logits, kept in 32 bits, and its column sums.  p = exp(z - lse) * inverse.  A workgroup takes 256 classes, four to a
// lane, of 64 rows, its waves every eighth row; their sums meet in LDS, in a fixed order.  Few rows are bound by latency (a wave to all rows took 28 us for 60 of them),
// many by memory: 4096 rows of 32000 classes 155 us (5.1 TB/s).  FORM: a workgroup forms its rows' lse by itself, in a fixed order.
template <typename T, bool FORM> __global__ __launch_bounds__(DLF_CE_DZ_THREADS) void k_ce_dz_sums(const DlfCeDzArgs a)
{
    constexpr int WAVES = DLF_CE_DZ_THREADS / 64;
    static_assert(DLF_CE_DZ_ROWS <= WAVES * 64 && DLF_FF_FEW_ROWS <= DLF_CE_DZ_ROWS, "a thread for each row, one workgroup for few rows");
    struct Row {
        float total, own, lse, zero;
        int t;              // the target's class, or -1
    };
    __shared__ Row rows[DLF_CE_DZ_ROWS];
    __shared__ f4v sums[WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.y * DLF_CE_DZ_ROWS, nr = min(a.nr - first, DLF_CE_DZ_ROWS);
    Parts all;                                              // of row threadIdx.x
    if constexpr (FORM) {
        __shared__ float2 shared[DLF_CE_DZ_THREADS];
        const int groups = dlf_ce_dz_groups(nr), span = DLF_CE_DZ_THREADS / groups, mine = threadIdx.x & (span - 1), group = threadIdx.x / span;
        if (mine < nr) all.take(a.part, a.parts, a.nr, first + mine, group, groups);
        shared[threadIdx.x] = float2{all.m, all.s};
        for (int h = groups / 2; h > 0; h >>= 1) {
            __syncthreads();
            if (group < h) {
                const float2 v = shared[threadIdx.x + h * span];
                all.add(v.x, v.y);
                shared[threadIdx.x] = float2{all.m, all.s};
            }
        }
    }
    if ((int)threadIdx.x < nr) {
        const int r = first + threadIdx.x;
        const int64_t t = a.target[r];
        const RowGradient g = row_gradient(a.given, r, t, a.ignore, a.nc);
        const bool is_class = t >= 0 && t < a.nc;
        const float inverse = FORM ? 1.0f / all.s : a.inverse != nullptr ? a.inverse[r] : 1.0f;
        rows[threadIdx.x] = Row{g.total * inverse, g.own, FORM ? all.m : a.lse[r], g.total, is_class ? (int)t : -1};
        if (FORM && blockIdx.x == 0) a.loss[r] = loss_of(all.lse(), t, a.ignore, a.nc, a.at + r);
        if (blockIdx.x == 0 && !is_class) a.rest[r] = 0.0f;
        if (blockIdx.x == 0 && r == 0 && a.back != nullptr) *a.back = scale_back(a.given);
    }
    __syncthreads();
    const int c = (blockIdx.x * 64 + lane) * 4;
    f4v sum = f4v{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int AT = 4;                                   // rows whose loads share a wait
    for (int r0 = wave; c < a.ldz && r0 < nr; r0 += AT * WAVES) {
        f4v z[AT];
#pragma unroll
        for (int k = 0; k < AT; ++k) z[k] = *(const f4v*)(a.z + (int64_t)(first + min(r0 + k * WAVES, nr - 1)) * a.ldz + c);
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            if (r0 + k * WAVES >= nr) break;
            const Row q = rows[r0 + k * WAVES];
            const int r = first + r0 + k * WAVES;
            const int64_t at = (int64_t)r * a.ldz + c;
            float v[4], low[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = q.zero == 0.0f ? 0.0f : q.total * exp_of_all(z[k][i] - q.lse);
                if (c + i >= a.nc) v[i] = 0.0f;
                if (q.t == c + i) v[i] -= q.own;
                sum[i] += v[i];
                low[i] = v[i] - (float)(typename T::e)v[i];
                if (q.t == c + i) a.rest[r] = low[i];
            }
            store_some<T, 4>(a.dz, at, 4, v);
            if (a.low != nullptr) store_some<T, 4>(a.low, at, 4, low);
        }
    }
    if (a.sums == nullptr) return;
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= a.nc) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += sums[w][lane];
    const float back = scale_back(a.given);
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = sum[i] * back;
    store_floats(a.sums + (int64_t)blockIdx.y * a.nc + c, a.nc - c, f);
}

// k_ce_pack: up to two matrices whose rows start anywhere, copied to rows of whole lines, for the tiles that are loaded directly.
__global__ __launch_bounds__(256) void k_ce_pack(const DlfCePackArgs a)
{
    int64_t line = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t of_first = a.m[0].rows * a.parts;
    const int which = line >= of_first ? 1 : 0;
    const DlfCePack& m = a.m[which];
    if (which) line -= of_first;
    const int64_t r = line / a.parts;
    if (r >= m.rows) return;
    const int c = (int)(line - r * a.parts) * 8;
    const F16::v8 v = load8<F16>(m.from, r * m.stride + c, a.k - c);
    __builtin_memcpy((char*)m.to + line * 16, &v, 16);
}

// ------------------------------------------------------------------------------------------------
// k_ce_unit: for fp16 and gradients of each row's own, the power of two that brings the largest |dloss| + |dlse| to between 2^13 and 2^14: dz, at most
// twice that, stays below 2^15, and classes of probability 2^-28 are numbers of full precision.  dloss is 0 where a row has no target, whatever is there.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void k_ce_unit(const DlfCeUnitArgs a)
{
    __shared__ float waves[16];
    const DlfCeGiven& g = a.given;
    float m = 0.0f;
    const bool one = (g.dloss == nullptr || g.dloss_stride == 0) && (g.dlse == nullptr || g.dlse_stride == 0);
    for (int64_t r = threadIdx.x; r < a.rows; r += 1024) {
        const bool counts = a.target[r] != a.ignore;
        const float l = fabsf(g.dloss != nullptr ? g.dloss[r * g.dloss_stride] : g.dloss_value), e = fabsf(g.dlse != nullptr ? g.dlse[r * g.dlse_stride] : 0.0f);
        const float v = counts ? l + e : e;
        m = v <= 3.402823466e38f ? fmaxf(m, v) : m;         // (what is not finite makes its own row so)
        if (one && counts) break;                           // (all others are the same)
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 16; ++w) m = fmaxf(m, waves[w]);
    // 2^(13 - e) for m = 1.x * 2^e, as far as it and its inverse are normal numbers
    int e = (int)(__builtin_bit_cast(uint32_t, m) >> 23) - 127;
    if (m == 0.0f) e = 13;
    const int k = max(-126, min(126, 13 - e));
    a.unit[0] = __builtin_bit_cast(float, (uint32_t)(127 + k) << 23);
    a.unit[1] = __builtin_bit_cast(float, (uint32_t)(127 - k) << 23);
}

// The epilogue of the gradients' products: scaled by one value in memory, added to sums of 32 bits or left there.
struct Sums {
    static constexpr bool OWN = false, SUMS = true;
    const float* scale;     // or null
    float* sum;             // [nr][nc] or null
    int add, keep;          // what is there is added; the sum goes there and nowhere else
    // What the rounding of dz has taken from a row's target, rest[r], times its class's weights: the largest element of dz by far, whose rounding would be the
    // result's.
    const float* rest;      // [nr] or null
    const int64_t* target;
    const void* w;
    int64_t ldw;
    float by = 1.0f;
    template <typename T, int N, int V> __device__ __forceinline__ void correct(const DlfFfArgs& a, int r, int step, int c, int n, float (*v)[V]) const
    {
        if (rest == nullptr) return;
        float by[N];
        int64_t at[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int row = min(r + k * step, a.nr - 1);
            by[k] = rest[row];
            at[k] = target[row];
        }
        typename Some<T, V>::v q[N];
#pragma unroll
        for (int k = 0; k < N; ++k)                         // (without a class there is no rest)
            q[k] = load_some<T, V>(w, (by[k] != 0.0f ? at[k] : 0) * ldw + c, n);
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = by[k] != 0.0f ? __builtin_fmaf(by[k], (float)q[k][i], v[k][i]) : v[k][i];
    }
    // Where the epilogue begins.  As an instruction, waited for at once: with a load that the compiler knows it waits for all loads in every turn of the main
    // loop, whose registers it takes for the load's (4096 x 4096 over 32000 classes 1745 -> 1913 us).
    __device__ __forceinline__ Sums ready() const
    {
        Sums s = *this;
        if (scale != nullptr) asm volatile("s_load_dword %0, %1, 0x0\n\ts_waitcnt lgkmcnt(0)" : "=s"(s.by) : "s"(scale) : "memory");
        return s;
    }
    // whether the outputs are to be stored
    template <int V> __device__ __forceinline__ bool take(const DlfFfArgs& a, int r, int c, int n, float (&v)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] *= by;
        if (sum == nullptr) return true;
        float* const at = sum + (int64_t)r * a.nc + c;
        if (add != 0) {
            float before[V];
            __builtin_memset(before, 0, sizeof before);
            if (n >= V) {
                __builtin_memcpy(before, at, 4 * V);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < n) before[i] = at[i];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += before[i];
        }
        if (keep == 0) return true;
        if (n >= V) {
            __builtin_memcpy(at, v, 4 * V);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < n) at[i] = v[i];
        }
        return false;
    }
};

// k_ce_back: the products dx = dz weight and dweight = dz^T x with the column sums, as k_ff_back, scaled back and added up over pieces.
template <typename T, int BC, int BR, int WC, int WR, int KB, int RING, bool DIRECT>
__global__ FF_TILE_BOUNDS void k_ce_back(const DlfCeBackArgs e)
{
    const DlfFfBackArgs& a = e.b;
    int b = blockIdx.x;
    if (a.x_first) b = b < a.blocks_x ? b + a.blocks_w : b < a.blocks_x + a.blocks_w ? b - a.blocks_x : b;   // (both multiples of eight)
    if (b < a.blocks_w) {
        tile<T, BC, BR, WC, WR, KB, RING, DIRECT, true, true, false>(a.w, Sums{e.back, e.sum, e.add, e.keep, nullptr, nullptr, nullptr, 0}, b);
        return;
    }
    b -= a.blocks_w;
    if (b < a.blocks_x) {
        tile<T, BC, BR, WC, WR, KB, RING, DIRECT, true, false, false>(a.x, Sums{e.back, nullptr, 0, 0, e.rest, e.target, e.b.x.p[0], e.b.x.ldp}, b);
        return;
    }
    b -= a.blocks_x;
    if (b < a.sum.blocks) add_sums(a.sum, b);
}
template <typename T> __global__ __launch_bounds__(256) void k_ce_join_back(const DlfCeBackArgs e)
{
    const bool w = (int)blockIdx.x < e.b.blocks_w;
    const int64_t unit = (int64_t)(w ? blockIdx.x : blockIdx.x - e.b.blocks_w) * 256 + threadIdx.x;
    if (w) join<T, false>(e.b.w, Sums{e.back, e.sum, e.add, e.keep, nullptr, nullptr, nullptr, 0}, unit);
    else join<T, false>(e.b.x, Sums{e.back, nullptr, 0, 0, e.rest, e.target, e.b.x.p[0], e.b.x.ldp}, unit);
}

// ------------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------------
typedef void (*CeKernel)(const DlfCeArgs);
typedef void (*CeBackKernel)(const DlfCeBackArgs);
template <typename T, int MODE> static CeKernel tile_kernel(int shape)
{
    switch (shape) {
    case DLF_FF_SHAPE_256: return k_ce_tile<T, 256, 256, 2, 2, 64, 2, true, MODE>;
    case DLF_FF_SHAPE_128: return k_ce_tile<T, 128, 128, 2, 2, 64, 2, true, MODE>;
    case DLF_FF_SHAPE_128_DEEP: return k_ce_tile<T, 128, 128, 2, 2, 64, 4, true, MODE>;
    case DLF_FF_SHAPE_ANY64: return k_ce_tile<T, 64, 64, 2, 2, 64, 4, false, MODE>;
    case DLF_FF_SHAPE_ANY64G: return nullptr;
    default: return k_ce_tile<T, 128, 128, 2, 2, 64, 2, false, MODE>;
    }
}
template <typename T> static CeKernel tile_kernel(int shape, int mode)
{
    return mode == DLF_CE_STAT ? tile_kernel<T, DLF_CE_STAT>(shape) : mode == DLF_CE_KEEP ? tile_kernel<T, DLF_CE_KEEP>(shape)
                                : mode == DLF_CE_DZ ? tile_kernel<T, DLF_CE_DZ>(shape) : tile_kernel<T, DLF_CE_LOGITS>(shape);
}
template <typename T> static CeBackKernel back_kernel(int shape)
{
    switch (shape) {
    case DLF_FF_SHAPE_256: return k_ce_back<T, 256, 256, 2, 2, 64, 2, true>;
    case DLF_FF_SHAPE_128: return k_ce_back<T, 128, 128, 2, 2, 64, 2, true>;
    case DLF_FF_SHAPE_128_DEEP: return k_ce_back<T, 128, 128, 2, 2, 64, 4, true>;
    case DLF_FF_SHAPE_ANY64: return k_ce_back<T, 64, 64, 2, 2, 64, 4, false>;
    case DLF_FF_SHAPE_ANY64G: return nullptr;
    default: return k_ce_back<T, 128, 128, 2, 2, 64, 2, false>;
    }
}
template <typename T> static CeKernel few_kernel(int rows, int nf, int mr)
{
    if (rows) return nf == 1 ? mr == 1 ? k_ce_rows<T, 1, 1> : k_ce_rows<T, 1, 2> : k_ce_rows<T, 2, 2>;
    return nf == 1 ? mr == 1 ? k_ce_few<T, 1, 1> : k_ce_few<T, 1, 2> : k_ce_few<T, 2, 2>;
}
static size_t tile_lds(int shape)
{
    const DlfFfShape& s = DLF_FF_SHAPES[shape];
    const size_t ring = (size_t)s.stages * 64 * (s.bc + s.br) * 2, out = (size_t)4 * (s.br < 128 ? 32 : 64) * (s.bc / 2 + 4) * 4;
    return ring > out ? ring : out;
}
extern "C" int dlf_ce_kernels_init(void)
{
    for (int k = 0; k < 6; ++k) {
        const int nf = k / 2 == 2 ? 2 : 1, mr = k / 2 == 0 ? 1 : 2;
        const CeKernel f = (k & 1) ? few_kernel<BF16>(1, nf, mr) : few_kernel<F16>(1, nf, mr);
        const hipError_t e = hipFuncSetAttribute((const void*)f, hipFuncAttributeMaxDynamicSharedMemorySize, DLF_FF_ROWS_LDS(8, nf, mr, 0));
        if (e != hipSuccess) return (int)e;
    }
    for (int shape = 0; shape < DLF_FF_NUM_SHAPES; ++shape)
        for (int k = 0; k < 10; ++k) {
            const void* const f = k < 8 ? (const void*)((k & 1) ? tile_kernel<BF16>(shape, k >> 1) : tile_kernel<F16>(shape, k >> 1))
                                        : (const void*)((k & 1) ? back_kernel<BF16>(shape) : back_kernel<F16>(shape));
            if (f == nullptr) continue;
            const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)tile_lds(shape));
            if (e != hipSuccess) return (int)e;
        }
    return 0;
}
static unsigned tile_blocks(const DlfFfArgs& a) { return (unsigned)((a.tiles_r * a.tiles_c * a.problems * a.splits + 7) / 8 * 8); }
static unsigned join_blocks(const DlfFfArgs& a) { return (unsigned)(((int64_t)a.nr * a.problems * ((a.nc + 7) / 8) + 255) / 256); }
extern "C" int dlf_ce_start_tile(const DlfCeArgs* a, int shape, int dtype, int mode, void* stream)
{
    hipLaunchKernelGGL(dtype == DLF_F16 ? tile_kernel<F16>(shape, mode) : tile_kernel<BF16>(shape, mode), dim3(tile_blocks(a->t)), dim3(256), tile_lds(shape),
                       (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ce_start_few(const DlfCeArgs* a, const DlfFfFew* c, int dtype, void* stream)
{
    DlfCeArgs b = *a;
    b.t.tiles_r = (a->t.nr + 16 * c->mr - 1) / (16 * c->mr);
    b.t.tiles_c = (a->t.nc + 16 * c->nf - 1) / (16 * c->nf);
    const dim3 grid((unsigned)((b.t.tiles_c + 7) / 8 * 8 * b.t.tiles_r)), block((unsigned)c->waves * 64);
    const size_t lds = c->rows ? (size_t)DLF_FF_ROWS_LDS(c->waves, c->nf, c->mr, 0) : (size_t)c->waves * c->nf * c->mr * 1024;
    hipLaunchKernelGGL(dtype == DLF_F16 ? few_kernel<F16>(c->rows, c->nf, c->mr) : few_kernel<BF16>(c->rows, c->nf, c->mr), grid, block, lds,
                       (hipStream_t)stream, b);
    return (int)hipGetLastError();
}
extern "C" int dlf_ce_start_join(const DlfCeJoinArgs* a, void* stream)
{
    if (a->nr <= DLF_CE_JOIN_FEW) hipLaunchKernelGGL(k_ce_join<1>, dim3((unsigned)a->nr), dim3(256), 0, (hipStream_t)stream, *a);
    else
        hipLaunchKernelGGL(k_ce_join<DLF_CE_JOIN_ROWS>, dim3((unsigned)((a->nr + DLF_CE_JOIN_ROWS - 1) / DLF_CE_JOIN_ROWS)), dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ce_start_dz(const DlfCeDzArgs* a, int dtype, void* stream)
{
    const dim3 grid((unsigned)(a->nr * a->slices));
    const bool h = dtype == DLF_F16;
    void (*const f)(const DlfCeDzArgs) = a->z != nullptr     ? h ? k_ce_dz<F16, true, true> : k_ce_dz<BF16, true, true>
                                         : a->lse != nullptr ? h ? k_ce_dz<F16, false, false> : k_ce_dz<BF16, false, false>
                                                             : h ? k_ce_dz<F16, true, false> : k_ce_dz<BF16, true, false>;
    hipLaunchKernelGGL(f, grid, dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ce_start_dz_sums(const DlfCeDzArgs* a, int dtype, void* stream)
{
    const dim3 grid((unsigned)((a->ldz + 255) / 256), (unsigned)((a->nr + DLF_CE_DZ_ROWS - 1) / DLF_CE_DZ_ROWS));
    const bool h = dtype == DLF_F16;
    void (*const f)(const DlfCeDzArgs) = a->lse != nullptr ? h ? k_ce_dz_sums<F16, false> : k_ce_dz_sums<BF16, false>
                                                           : h ? k_ce_dz_sums<F16, true> : k_ce_dz_sums<BF16, true>;
    hipLaunchKernelGGL(f, grid, dim3(DLF_CE_DZ_THREADS), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ce_start_pack(const DlfCePackArgs* a, void* stream)
{
    hipLaunchKernelGGL(k_ce_pack, dim3((unsigned)(((a->m[0].rows + a->m[1].rows) * a->parts + 255) / 256)), dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ce_start_unit(const DlfCeUnitArgs* a, void* stream)
{
    hipLaunchKernelGGL(k_ce_unit, dim3(1), dim3(1024), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ce_start_back(const DlfCeBackArgs* a, int shape, int dtype, void* stream)
{
    DlfCeBackArgs e = *a;
    DlfFfBackArgs& b = e.b;
    b.blocks_w = (int)tile_blocks(b.w);
    b.blocks_x = (int)tile_blocks(b.x);
    hipLaunchKernelGGL(dtype == DLF_F16 ? back_kernel<F16>(shape) : back_kernel<BF16>(shape), dim3((unsigned)(b.blocks_w + b.blocks_x + b.sum.blocks)),
                       dim3(256), tile_lds(shape), (hipStream_t)stream, e);
    b.blocks_w = b.w.splits > 1 ? (int)join_blocks(b.w) : 0;
    b.blocks_x = b.x.splits > 1 ? (int)join_blocks(b.x) : 0;
    if (b.blocks_w + b.blocks_x > 0)
        hipLaunchKernelGGL(dtype == DLF_F16 ? k_ce_join_back<F16> : k_ce_join_back<BF16>, dim3((unsigned)(b.blocks_w + b.blocks_x)), dim3(256), 0,
                           (hipStream_t)stream, e);
    return (int)hipGetLastError();
}
