// gfx950 (CDNA4) kernels of the feed-forward operators: matrix products with bias, activation and residual in the
// epilogue, the gated pair of projections, and their gradients.  What they are made of is in dlf_tile.h.
#include "dlf_tile.h"

template <typename T, int BC, int BR, int WC, int WR, int KB, int RING, bool DIRECT, bool GATED>
__global__ FF_TILE_BOUNDS void k_ff_tile(const DlfFfArgs a)
{
    tile<T, BC, BR, WC, WR, KB, RING, DIRECT, false, false, GATED>(a, Plain(), blockIdx.x);
}

// k_ff_back: both products of a backward pass and the column sums in one launch: their tiles fill the chip together (each alone leaves compute
// units idle in its last round), and small layers, bound by launches, need one instead of three.  The product of the longer sums
// goes first, and what is short fills the gaps.  The products of 4096 x 2048 -> 2048 take 70 us together, 38 and 38 apart; those of 4096 x 2048
// -> 2 x 5632 351 (1.08 PFLOP/s; 372 with the other order), 235 and 243 apart.
template <typename T, int BC, int BR, int WC, int WR, int KB, int RING, bool DIRECT>
__global__ FF_TILE_BOUNDS void k_ff_back(const DlfFfBackArgs a)
{
    int b = blockIdx.x;
    if (a.x_first) b = b < a.blocks_x ? b + a.blocks_w : b < a.blocks_x + a.blocks_w ? b - a.blocks_x : b;   // (both multiples of eight)
    if (b < a.blocks_w) {
        tile<T, BC, BR, WC, WR, KB, RING, DIRECT, true, true, false>(a.w, Plain(), b);
        return;
    }
    b -= a.blocks_w;
    if (b < a.blocks_x) {
        tile<T, BC, BR, WC, WR, KB, RING, DIRECT, true, false, false>(a.x, Plain(), b);
        return;
    }
    b -= a.blocks_x;
    if (b < a.sum.blocks) add_sums(a.sum, b);
}

template <typename T, bool GATED> __global__ __launch_bounds__(256) void k_ff_join(const DlfFfArgs a)
{
    join<T, GATED>(a, Plain(), (int64_t)blockIdx.x * 256 + threadIdx.x);
}
// ... of the two products of a backward pass: workgroups [0, blocks_w) and the others.
template <typename T> __global__ __launch_bounds__(256) void k_ff_join_back(const DlfFfBackArgs a)
{
    const bool w = (int)blockIdx.x < a.blocks_w;
    join<T, false>(w ? a.w : a.x, Plain(), (int64_t)(w ? blockIdx.x : blockIdx.x - a.blocks_w) * 256 + threadIdx.x);
}

template <typename T, int NF, int MR, bool GATED>
__global__ __launch_bounds__(512, (GATED ? 2 : NF) + MR <= 3 ? 4 : 2) void k_ff_few(const DlfFfArgs a)
{
    few<T, NF, MR, GATED>(a, Plain());
}
template <typename T, int NF, int MR, bool GATED>
__global__ __launch_bounds__(512) void k_ff_rows(const DlfFfArgs a)
{
    rows_in_lds<T, NF, MR, GATED>(a, Plain());
}

// ------------------------------------------------------------------------------------------------
// k_ff_dz: the gradient behind the activation, and column sums of it in 32 bits (before it is rounded).  Bound by memory: 8 bytes an
// element, gated 14 (4096 x 2048: 14 us, 4.8 TB/s; gated 4096 x 5632: 67 us, 4.8 TB/s, what a large copy reaches).  A workgroup takes `chunk`
// rows of 256 columns: 32 threads by eight columns, eight rows at a time; their sums meet in LDS, in a fixed order, and k_ff_back adds up
// what the chunks leave.  (At most 64 chunks: up to 512 columns leave half the compute units idle.)
// ------------------------------------------------------------------------------------------------
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_ff_dz(const DlfFfDzArgs a)
{
    constexpr int NZ = GATED ? 2 : 1, TC = 32, THREADS = 256, RT = DLF_FF_CHUNK_ROWS;
    static_assert(RT * TC == THREADS, "");
    __shared__ __attribute__((aligned(16))) float sums[RT][NZ][8 * TC];
    const int tc = threadIdx.x % TC, tr = threadIdx.x / TC;
    const int c = (blockIdx.x * TC + tc) * 8, n = a.n - c;
    const int r0 = blockIdx.y * a.chunk, r1 = min(a.rows, r0 + a.chunk);
    float sum[NZ][8];
#pragma unroll
    for (int z = 0; z < NZ; ++z)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[z][i] = 0.0f;
    if (n > 0) {
        for (int r = r0 + tr; r < r1; r += RT) {
            const typename T::v8 dy = load8<T>(a.dy, (int64_t)r * a.lddy + c, n);
            float d[NZ][8];
            if (a.saved != nullptr) {
                float z[8], u[8];
                load_floats(a.saved + (int64_t)r * a.n + c, n, z);
                if (GATED) load_floats(a.saved + ((int64_t)a.rows + r) * a.n + c, n, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[0][i] = (float)dy[i];
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
                // One rounding to the tensors' type, which the matrix units multiply: gradients are off by 0.0023 of their norm
                // against 0.0017 with dz in 32 bits (bf16; fp16 0.00029 against 0.00021, and its range).  Rows of dz are whole eights, zeros behind
                // column n, so that a thread's eight are one store.
#pragma unroll
                for (int z2 = 0; z2 < NZ; ++z2) {
                    if (n < 8) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[z2][i] = i < n ? d[z2][i] : 0.0f;
                    }
                    store_some<T, 8>(a.dz[z2], (int64_t)r * a.lddz + c, 8, d[z2]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[0][i] = (float)dy[i];
            }
#pragma unroll
            for (int z2 = 0; z2 < NZ; ++z2)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[z2][i] += d[z2][i];
        }
    }
    if (a.sums[0] == nullptr && a.sums[1] == nullptr) return;
#pragma unroll
    for (int z = 0; z < NZ; ++z)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[tr][z][tc * 8 + i] = sum[z][i];
    // pairs of rows, then pairs of pairs ...
    for (int h = RT / 2; h > 0; h >>= 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < h * NZ * 8 * TC; i += THREADS) (&sums[0][0][0])[i] += (&sums[h][0][0])[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < NZ * 8 * TC; i += THREADS) {
        const int z = i / (8 * TC), col = blockIdx.x * 8 * TC + i % (8 * TC);
        if (col < a.n && a.sums[z] != nullptr) a.sums[z][(int64_t)blockIdx.y * a.n + col] = sums[0][z][i % (8 * TC)];
    }
}
// ------------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------------
// The tile kernels by shape (DLF_FF_SHAPE_*): waves across c and r, k of a stage, stages on their way, direct loads.
typedef void (*TileKernel)(const DlfFfArgs);
typedef void (*BackKernel)(const DlfFfBackArgs);
template <typename T> static TileKernel tile_kernel(int shape, int gated)
{
    switch (shape) {
    case DLF_FF_SHAPE_256: return gated ? k_ff_tile<T, 256, 256, 2, 2, 64, 2, true, true> : k_ff_tile<T, 256, 256, 2, 2, 64, 2, true, false>;
    case DLF_FF_SHAPE_128: return gated ? k_ff_tile<T, 128, 128, 2, 2, 64, 2, true, true> : k_ff_tile<T, 128, 128, 2, 2, 64, 2, true, false>;
    case DLF_FF_SHAPE_128_DEEP: return gated ? k_ff_tile<T, 128, 128, 2, 2, 64, 4, true, true> : k_ff_tile<T, 128, 128, 2, 2, 64, 4, true, false>;
    case DLF_FF_SHAPE_ANY64: return gated ? nullptr : k_ff_tile<T, 64, 64, 2, 2, 64, 4, false, false>;
    case DLF_FF_SHAPE_ANY64G: return gated ? k_ff_tile<T, 64, 128, 1, 4, 64, 4, false, true> : nullptr;
    default: return gated ? k_ff_tile<T, 128, 128, 2, 2, 64, 2, false, true> : k_ff_tile<T, 128, 128, 2, 2, 64, 2, false, false>;
    }
}
template <typename T> static BackKernel back_kernel(int shape)
{
    switch (shape) {
    case DLF_FF_SHAPE_256: return k_ff_back<T, 256, 256, 2, 2, 64, 2, true>;
    case DLF_FF_SHAPE_128: return k_ff_back<T, 128, 128, 2, 2, 64, 2, true>;
    case DLF_FF_SHAPE_128_DEEP: return k_ff_back<T, 128, 128, 2, 2, 64, 4, true>;
    case DLF_FF_SHAPE_ANY64: return k_ff_back<T, 64, 64, 2, 2, 64, 4, false>;
    case DLF_FF_SHAPE_ANY64G: return nullptr;
    default: return k_ff_back<T, 128, 128, 2, 2, 64, 2, false>;
    }
}
static size_t tile_lds(int shape)
{
    const DlfFfShape& s = DLF_FF_SHAPES[shape];
    const size_t ring = (size_t)s.stages * 64 * (s.bc + s.br) * 2, out = (size_t)4 * (s.br < 128 ? 32 : 64) * (s.bc / 2 + 4) * 4;
    return ring > out ? ring : out;
}
template <typename T> static void (*rows_kernel(int nf, int mr, int gated))(const DlfFfArgs)
{
    if (gated) return mr == 1 ? k_ff_rows<T, 1, 1, true> : k_ff_rows<T, 1, 2, true>;
    return nf == 1 ? mr == 1 ? k_ff_rows<T, 1, 1, false> : k_ff_rows<T, 1, 2, false> : k_ff_rows<T, 2, 2, false>;
}
template <typename T> static void (*few_kernel(int nf, int mr, int gated))(const DlfFfArgs)
{
    if (gated) return mr == 1 ? k_ff_few<T, 1, 1, true> : k_ff_few<T, 1, 2, true>;
    return nf == 1 ? mr == 1 ? k_ff_few<T, 1, 1, false> : k_ff_few<T, 1, 2, false> : k_ff_few<T, 2, 2, false>;
}
extern "C" int dlf_ff_start_few(const DlfFfArgs* a, const DlfFfFew* c, int dtype, int gated, void* stream)
{
    const int nf = c->nf, mr = c->mr;
    DlfFfArgs b = *a;
    b.tiles_r = (a->nr + 16 * mr - 1) / (16 * mr);
    b.tiles_c = (a->nc + 16 * nf - 1) / (16 * nf);
    const dim3 grid((unsigned)((b.tiles_c + 7) / 8 * 8 * b.tiles_r)), block((unsigned)c->waves * 64);
    if (c->rows)
        hipLaunchKernelGGL(dtype == DLF_F16 ? rows_kernel<F16>(nf, mr, gated) : rows_kernel<BF16>(nf, mr, gated), grid, block,
                           (size_t)DLF_FF_ROWS_LDS(c->waves, nf, mr, gated), (hipStream_t)stream, b);
    else
        hipLaunchKernelGGL(dtype == DLF_F16 ? few_kernel<F16>(nf, mr, gated) : few_kernel<BF16>(nf, mr, gated), grid, block,
                           (size_t)c->waves * nf * mr * (gated ? 2 : 1) * 1024, (hipStream_t)stream, b);
    return (int)hipGetLastError();
}
extern "C" int dlf_ff_kernels_init(void)
{
    for (int k = 0; k < 10; ++k) {
        const int gated = k / 2 < 2, nf = k / 2 == 4 ? 2 : 1, mr = k / 2 == 0 || k / 2 == 2 ? 1 : 2;
        auto f = (k & 1) ? rows_kernel<BF16>(nf, mr, gated) : rows_kernel<F16>(nf, mr, gated);
        const hipError_t e = hipFuncSetAttribute((const void*)f, hipFuncAttributeMaxDynamicSharedMemorySize, DLF_FF_ROWS_LDS(8, nf, mr, gated));
        if (e != hipSuccess) return (int)e;
    }
    for (int shape = 0; shape < DLF_FF_NUM_SHAPES; ++shape)
        for (int k = 0; k < 6; ++k) {
            const void* f = k < 4 ? (const void*)((k & 1) ? tile_kernel<BF16>(shape, k >> 1) : tile_kernel<F16>(shape, k >> 1))
                                  : (const void*)((k & 1) ? back_kernel<BF16>(shape) : back_kernel<F16>(shape));
            if (f == nullptr) continue;
            const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)tile_lds(shape));
            if (e != hipSuccess) return (int)e;
        }
    return 0;
}
static unsigned tile_blocks(const DlfFfArgs& a) { return (unsigned)((a.tiles_r * a.tiles_c * a.problems * a.splits + 7) / 8 * 8); }
static unsigned join_blocks(const DlfFfArgs& a) { return (unsigned)(((int64_t)a.nr * a.problems * ((a.nc + 7) / 8) + 255) / 256); }
extern "C" int dlf_ff_start_tile(const DlfFfArgs* a, int shape, int dtype, int gated, void* stream)
{
    hipLaunchKernelGGL(dtype == DLF_F16 ? tile_kernel<F16>(shape, gated) : tile_kernel<BF16>(shape, gated), dim3(tile_blocks(*a)), dim3(256), tile_lds(shape),
                       (hipStream_t)stream, *a);
    if (a->splits > 1)
        hipLaunchKernelGGL(dtype == DLF_F16 ? (gated ? k_ff_join<F16, true> : k_ff_join<F16, false>) : (gated ? k_ff_join<BF16, true> : k_ff_join<BF16, false>),
                           dim3(join_blocks(*a)), dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
extern "C" int dlf_ff_start_back(const DlfFfBackArgs* a, int shape, int dtype, void* stream)
{
    DlfFfBackArgs b = *a;
    b.blocks_w = (int)tile_blocks(b.w);
    b.blocks_x = (int)tile_blocks(b.x);
    hipLaunchKernelGGL(dtype == DLF_F16 ? back_kernel<F16>(shape) : back_kernel<BF16>(shape), dim3((unsigned)(b.blocks_w + b.blocks_x + b.sum.blocks)),
                       dim3(256), tile_lds(shape), (hipStream_t)stream, b);
    b.blocks_w = b.w.splits > 1 ? (int)join_blocks(b.w) : 0;
    b.blocks_x = b.x.splits > 1 ? (int)join_blocks(b.x) : 0;
    if (b.blocks_w + b.blocks_x > 0)
        hipLaunchKernelGGL(dtype == DLF_F16 ? k_ff_join_back<F16> : k_ff_join_back<BF16>, dim3((unsigned)(b.blocks_w + b.blocks_x)), dim3(256), 0,
                           (hipStream_t)stream, b);
    return (int)hipGetLastError();
}
extern "C" int dlf_ff_start_dz(const DlfFfDzArgs* a, int dtype, int gated, void* stream)
{
    const dim3 grid((unsigned)((a->n + 255) / 256), (unsigned)(a->rows > 0 ? (a->rows + a->chunk - 1) / a->chunk : 1));
    hipLaunchKernelGGL(dtype == DLF_F16 ? (gated ? k_ff_dz<F16, true> : k_ff_dz<F16, false>) : (gated ? k_ff_dz<BF16, true> : k_ff_dz<BF16, false>), grid,
                       dim3(256), 0, (hipStream_t)stream, *a);
    return (int)hipGetLastError();
}
