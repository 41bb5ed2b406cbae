// fbsr_gemm_i8: products of rows of 8-bit integers with 8-bit matrices, a scale for each row of both.  The arithmetic is stated
// in include/fbsr.h: the integer sum is exact in 32 bits, so neither the split of k nor the order of anything changes a result.
//
// Three kernels.
//
// gemv_i8_kernel (up to 4 rows of a): bound by the reading of w.  A warp takes four rows of w (or a share of their columns), lane
// after lane sixteen columns at a time; four columns a dp4a.  The rows of a stay in L1.  Beyond four the reading of a and the dp4a
// weigh more than that of w (w of 4096 x 11008, out of HBM: one row 9.2 us, four 10.3, eight 21.4; the matrix unit 11.1 for any; 11008 x
// 4096: 9.8, 10.8, 18.1 and 12.6).
//
// gemm_i8_kernel (more): tcgen05.mma kind::i8.  The rows of w are the 128 lanes of the accumulator and the rows of a its
// columns: a thread then owns one row of w, with its scale in a register, and a warp writes 32 neighbouring elements of y at a
// time straight from tensor memory, without staging them; and few rows of a cost few columns.  Tiles of w (128 x 128 bytes) and a (BN x 128 bytes)
// come by TMA in the 128-byte swizzle that the unit reads.  One warp copies, one thread issues the products, four warps write the
// tile before from the other half of tensor memory.  Where there are too few tiles to fill the GPU, a cluster of 2, 4 or 8 CTAs shares
// a tile along k and joins its integer sums through distributed shared memory, each CTA a share of the columns.
//
// gemm_i8_pair_kernel (enough tiles of 256 x 256): the same with cta_group::2.  A tile of 128 x 256 wants 96 bytes a clock from L2 at
// the product unit's rate, and a multiprocessor gets 64; two CTAs that share a tile of 256 x 256, each holding half of either
// operand, want 64.  Measured (bfloat16 results; the unit's rate taken as twice the measured bfloat16 one, 3.3 P/s): 8192^3 346 us,
// 4096 x 11008 x 4096 119, 4096^3 48, the unit busy 94 % of the clocks; 512 x 4096 x 4096 17, 64 x 4096 x 4096 9.8.
#include <cmath>

#include "fbsr_answer.cuh"
#include "fbsr_internal.h"
#include "fbsr_tma.cuh"

namespace fbsr {
namespace {

struct GemmArgs {
    const int8_t* a;
    const int8_t* w;
    const float* a_scales;
    const float* w_scales;
    void* y;
    int64_t lda, ldw, ldy;
    uint32_t m, n, k;
    int out_fmt;
    // gemm_i8_kernel
    uint32_t tiles_m, tiles_n, blocks;           // tiles along the rows of a and of w; blocks of 128 columns
    uint32_t group;                              // tiles of a that neighbouring tiles of the schedule share
    // gemv_i8_kernel
    int k_warps;
};

// One element of the result: two rounded products in binary32, then one rounding to the type of y.
__device__ __forceinline__ void store_result(const GemmArgs& g, uint32_t row, uint32_t col, int sum, float scale)
{
    const float v = __fmul_rn(__int2float_rn(sum), scale);
    const int64_t at = (int64_t)row * g.ldy + col;
    if (g.out_fmt == FBSR_FP32) static_cast<float*>(g.y)[at] = v;
    else if (g.out_fmt == FBSR_BF16) static_cast<__nv_bfloat16*>(g.y)[at] = __float2bfloat16_rn(v);
    else static_cast<__half*>(g.y)[at] = __float2half_rn(v);
}

// The same for a type known to the compiler, at the address of the element.
template <int OUT>
__device__ __forceinline__ void put_result(char* at, int sum, float scale)
{
    const float v = __fmul_rn(__int2float_rn(sum), scale);
    if constexpr (OUT == FBSR_FP32) *reinterpret_cast<float*>(at) = v;
    else if constexpr (OUT == FBSR_BF16) *reinterpret_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(v);
    else *reinterpret_cast<__half*>(at) = __float2half_rn(v);
}

// ------------------------------------------------------------------------------------------------ few rows
constexpr int GEMV_WARPS = 4, GEMV_CHANNELS = 4, UNROLL = 2;

template <int M>
__global__ void __launch_bounds__(GEMV_WARPS * 32)
gemv_i8_kernel(const __grid_constant__ GemmArgs g)
{
    __shared__ int part[GEMV_WARPS][M * GEMV_CHANNELS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int along = warp % g.k_warps, group = warp / g.k_warps, groups = GEMV_WARPS / g.k_warps;
    const uint32_t first = (blockIdx.x * groups + group) * GEMV_CHANNELS;
    const uint32_t chunks = g.k / 16, step = 32 * g.k_warps;
    const int8_t* w[GEMV_CHANNELS];
    const int8_t* a[M];
#pragma unroll
    for (int c = 0; c < GEMV_CHANNELS; ++c) w[c] = g.w + (int64_t)min(first + c, g.n - 1) * g.ldw;
#pragma unroll
    for (int i = 0; i < M; ++i) a[i] = g.a + (int64_t)min((uint32_t)i, g.m - 1) * g.lda;
    int sum[M][GEMV_CHANNELS] = {};
    for (uint32_t chunk = along * 32 + lane; chunk < chunks; chunk += step * UNROLL) {
        uint4 x[UNROLL][GEMV_CHANNELS];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const bool real = chunk + u * step < chunks;
#pragma unroll
            for (int c = 0; c < GEMV_CHANNELS; ++c) {
                x[u][c] = make_uint4(0u, 0u, 0u, 0u);
                if (real)
                    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(x[u][c].x), "=r"(x[u][c].y), "=r"(x[u][c].z), "=r"(x[u][c].w)
                                 : "l"(w[c] + (size_t)(chunk + u * step) * 16));
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (chunk + u * step >= chunks) break;
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const uint4 v = __ldg(reinterpret_cast<const uint4*>(a[i] + (size_t)(chunk + u * step) * 16));
#pragma unroll
                for (int c = 0; c < GEMV_CHANNELS; ++c) {
                    int s = sum[i][c];
                    s = __dp4a((int)x[u][c].x, (int)v.x, s);
                    s = __dp4a((int)x[u][c].y, (int)v.y, s);
                    s = __dp4a((int)x[u][c].z, (int)v.z, s);
                    sum[i][c] = __dp4a((int)x[u][c].w, (int)v.w, s);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int c = 0; c < GEMV_CHANNELS; ++c) {
            const int s = __reduce_add_sync(0xFFFFFFFFu, sum[i][c]);
            if (lane == 0) part[warp][i * GEMV_CHANNELS + c] = s;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < groups * M * GEMV_CHANNELS; i += GEMV_WARPS * 32) {
        // neighbouring threads: neighbouring rows of w
        const int row = i / (groups * GEMV_CHANNELS), channel = i % (groups * GEMV_CHANNELS), in = channel % GEMV_CHANNELS;
        const uint32_t col = blockIdx.x * groups * GEMV_CHANNELS + channel;
        if ((uint32_t)row >= g.m || col >= g.n) continue;
        int s = 0;
        for (int j = 0; j < g.k_warps; ++j) s += part[channel / GEMV_CHANNELS * g.k_warps + j][row * GEMV_CHANNELS + in];
        store_result(g, row, col, s, __fmul_rn(g.a_scales[row], g.w_scales[col]));
    }
}

// ------------------------------------------------------------------------------------------------ many rows
constexpr int BM = 128, BK = 128;                // rows of w and columns of a stage
constexpr int GEMM_THREADS = 192, COPY_WARP = 4, PRODUCT_WARP = 5;

template <int BN> struct Shape {
    static constexpr int STAGE = (BM + BN) * BK;
    static constexpr int STAGES = BN == 256 ? 4 : BN == 128 ? 6 : 4;
    static constexpr int RING = STAGES * STAGE;
    static constexpr int SHARED = RING + 1024;   // the ring begins on 1024 bytes
    static constexpr int COLUMNS = 2 * BN;       // of tensor memory: two accumulators
    static_assert(RING >= BN * BM * 4, "the joining of a cluster's sums fits into the ring");
};

// Descriptor of rows of 128 bytes in the 128-byte swizzle, eight rows (1024 bytes) to a group.
__device__ __forceinline__ uint64_t operand(uint32_t address)
{
    return (uint64_t)((address & 0x3FFFFu) >> 4) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

template <int BN>
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, bool add)
{
    // signed 8-bit operands, both along k; sums in 32 bits; 128 x BN
    constexpr uint32_t KIND = 2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(BN >> 3) << 17 | (uint32_t)(BM >> 4) << 24;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(KIND), "r"((uint32_t)add) : "memory");
}

__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}

// The same for a pair of CTAs: the copy completes on a barrier of the even one, 256 x 256 products of both operands' halves, and
// an arrival at the same place in both.
__device__ __forceinline__ void copy_box_pair(uint32_t to, const CUtensorMap* map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :: "r"(to), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}

__device__ __forceinline__ void product_pair(uint32_t d, uint64_t a, uint64_t b, bool add)
{
    constexpr uint32_t KIND = 2u << 4 | 1u << 7 | 1u << 10 | (256u >> 3) << 17 | (256u >> 4) << 24;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(KIND), "r"((uint32_t)add) : "memory");
}

__device__ __forceinline__ void commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" :: "r"(bar), "h"((uint16_t)3) : "memory");
}

// 32 columns of this warp's 32 lanes.
__device__ __forceinline__ void load_columns(uint32_t address, int (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
          "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]),
          "=r"(v[30]), "=r"(v[31])
        : "r"(address) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// 32 elements of a column of y: sums, the scales of their rows, the scale of the column.  `rows` of them exist.
template <int OUT>
__device__ __forceinline__ void put_column(char* to, int64_t step, const int (&v)[32], const float* scales, float w_scale, uint32_t rows)
{
    float f[32];
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        const float4 s = *reinterpret_cast<const float4*>(scales + i);
        f[i] = __fmul_rn(__int2float_rn(v[i]), __fmul_rn(s.x, w_scale));
        f[i + 1] = __fmul_rn(__int2float_rn(v[i + 1]), __fmul_rn(s.y, w_scale));
        f[i + 2] = __fmul_rn(__int2float_rn(v[i + 2]), __fmul_rn(s.z, w_scale));
        f[i + 3] = __fmul_rn(__int2float_rn(v[i + 3]), __fmul_rn(s.w, w_scale));
    }
#pragma unroll
    for (int i = 0; i < 32; i += 2, to += 2 * step) {
        const bool first = (uint32_t)i < rows, second = (uint32_t)i + 1 < rows;
        if constexpr (OUT == FBSR_FP32) {
            if (first) *reinterpret_cast<float*>(to) = f[i];
            if (second) *reinterpret_cast<float*>(to + step) = f[i + 1];
        } else {
            // two to an instruction: a conversion of one takes four times as long
            uint32_t pair;
            if constexpr (OUT == FBSR_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(pair) : "f"(f[i + 1]), "f"(f[i]));
            else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(pair) : "f"(f[i + 1]), "f"(f[i]));
            if (first) *reinterpret_cast<uint16_t*>(to) = (uint16_t)pair;
            if (second) *reinterpret_cast<uint16_t*>(to + step) = (uint16_t)(pair >> 16);
        }
    }
}

// The four writing warps: this tile's scales of rows of a into shared memory.  Asked for before the wait for the sums; a buffer
// for each half of tensor memory, so that none is written while it is still read.
template <int BN>
__device__ __forceinline__ void stage_scales(float* buffer, const GemmArgs& g, uint32_t row)
{
#pragma unroll
    for (int i = threadIdx.x; i < BN; i += 128) buffer[i] = row + i < g.m ? __ldg(g.a_scales + row + i) : 0.0f;
    asm volatile("bar.sync 1, 128;" ::: "memory");
}

// The tile that comes `index`-th: `group` tiles of a side by side, all tiles of w, then the next group.
__device__ __forceinline__ void tile_at(const GemmArgs& g, uint32_t index, uint32_t& tm, uint32_t& tn)
{
    const uint32_t whole = g.group * g.tiles_n, which = index / whole, in = index - which * whole;
    const uint32_t width = min(g.group, g.tiles_m - which * g.group);
    tn = in / width;
    tm = which * g.group + in - tn * width;
}

// SPLIT CTAs of a cluster share each tile along k.
template <int BN, int SPLIT, int OUT>
__global__ void __launch_bounds__(GEMM_THREADS)
gemm_i8_kernel(const __grid_constant__ GemmArgs g, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a)
{
    using S = Shape<BN>;
    constexpr int OUT_BYTES = OUT == FBSR_FP32 ? 4 : 2;
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t bars[2 * S::STAGES + 4];
    __shared__ __align__(16) float scales[2][SPLIT == 1 ? BN : 4];
    __shared__ uint32_t tensor_memory, gave_up;
    const uint32_t ring = (shared_address(dynamic) + 1023u) & ~1023u;
    const uint32_t full = shared_address(bars), empty = full + 8 * S::STAGES, sums = empty + 8 * S::STAGES, freed = sums + 16;
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const uint32_t rank = SPLIT == 1 ? 0 : blockIdx.x % SPLIT, unit = blockIdx.x / SPLIT, units = gridDim.x / SPLIT;
    const uint32_t tiles = g.tiles_m * g.tiles_n;
    const uint32_t from = g.blocks * rank / SPLIT, to = g.blocks * (rank + 1) / SPLIT;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) { barrier_init(sums + 8 * i, 1); barrier_init(freed + 8 * i, 4); }
        gave_up = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == PRODUCT_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(shared_address(&tensor_memory)), "n"(S::COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t acc = tensor_memory;

    if (warp == COPY_WARP) {
        uint32_t it = 0, s = 0, round = 0;       // block, its place in the ring, how often the ring has been round
        bool fine = true;
        for (uint32_t t = unit; t < tiles && fine; t += units) {
            uint32_t tm, tn;
            tile_at(g, t, tm, tn);
            for (uint32_t b = from; b < to; ++b, ++it) {
                if (round > 0) fine = warp_wait(empty + 8 * s, (round - 1) & 1);
                if (!fine) break;
                const uint32_t stage = ring + s * S::STAGE, bar = full + 8 * s;
                if (elected()) {
                    barrier_expect(bar, S::STAGE);
                    copy_box(stage, &map_w, bar, b * BK, tn * BM);
                    copy_box(stage + BM * BK, &map_a, bar, b * BK, tm * BN);
                }
                __syncwarp();
                if (++s == S::STAGES) { s = 0; ++round; }
            }
        }
        if (!fine) {
            gave_up = 1u;
            // copies in flight end before this CTA does
            for (uint32_t back = 1; back <= S::STAGES && back <= it; ++back)
                if (!warp_wait(full + 8 * ((it - back) % S::STAGES), ((it - back) / S::STAGES) & 1)) break;
        }
    } else if (warp == PRODUCT_WARP) {
        uint32_t s = 0, round = 0, turn = 0;
        bool fine = true;
        for (uint32_t t = unit; t < tiles && fine; t += units, ++turn) {
            const uint32_t half = turn & 1, d = acc + half * BN;
            if (turn >= 2) fine = warp_wait(freed + 8 * half, (turn / 2 - 1) & 1);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (uint32_t b = from; b < to && fine; ++b) {
                fine = warp_wait(full + 8 * s, round & 1);
                if (!fine) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t w = operand(ring + s * S::STAGE), a = operand(ring + s * S::STAGE + BM * BK);
                if (elected()) {
#pragma unroll
                    for (int j = 0; j < BK / 32; ++j) product<BN>(d, w + 2 * j, a + 2 * j, b > from || j > 0);      // 32 columns: 2 x 16 bytes on
                    commit(empty + 8 * s);
                }
                __syncwarp();
                if (++s == S::STAGES) { s = 0; ++round; }
            }
            if (fine && elected()) commit(sums + 8 * half);
        }
        if (!fine) gave_up = 1u;
    } else {
        uint32_t turn = 0;
        bool fine = true;                        // once false, the rest is written as NaN without another wait
        for (uint32_t t = unit; t < tiles; t += units, ++turn) {
            const uint32_t half = turn & 1;
            uint32_t tm, tn;
            tile_at(g, t, tm, tn);
            if constexpr (SPLIT == 1) stage_scales<BN>(scales[half], g, tm * BN);
            if (fine) fine = barrier_wait(sums + 8 * half, (turn / 2) & 1);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t col = tn * BM + threadIdx.x;
            const float w_scale = !fine ? __uint_as_float(0x7FC00000u) : col < g.n ? g.w_scales[col] : 0.0f;
            if (!fine) gave_up = 1u;
            const int64_t step = g.ldy * OUT_BYTES;
            char* to = static_cast<char*>(g.y) + (int64_t)tm * BN * step + (int64_t)col * OUT_BYTES;
#pragma unroll 1
            for (int c = 0; c < BN; c += 32) {
                int v[32];
                load_columns(acc + half * BN + c + ((uint32_t)warp << 21), v);         // lanes 32 warp .. of tensor memory
                if constexpr (SPLIT == 1) {
                    const uint32_t row = tm * BN + c;
                    if (row >= g.m) break;
                    if (col < g.n) {
                        if (row + 32 <= g.m) put_column<OUT>(to, step, v, scales[half] + c, w_scale, 32);
                        else put_column<OUT>(to, step, v, scales[half] + c, w_scale, g.m - row);
                    }
                    to += 32 * step;
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        asm volatile("st.shared.u32 [%0], %1;" :: "r"(ring + ((c + i) * BM + threadIdx.x) * 4), "r"(v[i]) : "memory");
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(freed + 8 * half) : "memory");
        }
    }
    __syncwarp();
    if constexpr (SPLIT > 1) {
        // one tile a cluster: its sums lie in the rings, all products done
        cluster_barrier();
        if (warp < 4 && unit < tiles) {
            uint32_t tm, tn;
            tile_at(g, unit, tm, tn);
            const uint32_t col = tn * BM + threadIdx.x;
            uint32_t lost = 0u, base[SPLIT];
#pragma unroll
            for (int p = 0; p < SPLIT; ++p) {
                uint32_t f;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(base[p]) : "r"(ring), "r"(p));
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(f) : "r"(shared_address(&gave_up)), "r"(p));
                asm volatile("ld.shared::cluster.u32 %0, [%0];" : "+r"(f) :: "memory");
                lost |= f;
            }
            const float w_scale = lost ? __uint_as_float(0x7FC00000u) : col < g.n ? g.w_scales[col] : 0.0f;
            constexpr int SHARE = BN / SPLIT, AT_ONCE = 32 / SPLIT;              // loads in flight: 32 in all
#pragma unroll 1
            for (int i = 0; i < SHARE; i += AT_ONCE) {
                const uint32_t c = rank * SHARE + i, row = tm * BN + c;
                if (row >= g.m) break;
                int v[AT_ONCE][SPLIT];
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
                    for (int p = 0; p < SPLIT; ++p)
                        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v[j][p]) : "r"(base[p] + ((c + j) * BM + threadIdx.x) * 4));
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    int sum = 0;
#pragma unroll
                    for (int p = 0; p < SPLIT; ++p) sum += v[j][p];
                    if (col < g.n && row + j < g.m)
                        put_result<OUT>(static_cast<char*>(g.y) + ((int64_t)(row + j) * g.ldy + col) * OUT_BYTES, sum,
                                        __fmul_rn(__ldg(g.a_scales + row + j), w_scale));
                }
            }
        }
        cluster_barrier();                       // nobody leaves while its sums are being read
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == PRODUCT_WARP) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(acc), "n"(S::COLUMNS));
    }
}

// Two CTAs to a tile of 256 rows of w and 256 of a: each holds 128 rows of both and the sums of its rows of w.  The even one issues
// the products for both; its barriers count the copies of both.
constexpr int PAIR_BN = 256, PAIR_STAGE = 2 * BM * BK, PAIR_STAGES = 6, PAIR_SHARED = PAIR_STAGES * PAIR_STAGE + 1024;

template <int OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GEMM_THREADS)
gemm_i8_pair_kernel(const __grid_constant__ GemmArgs g, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a)
{
    constexpr int OUT_BYTES = OUT == FBSR_FP32 ? 4 : 2;
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t bars[2 * PAIR_STAGES + 4];
    __shared__ __align__(16) float scales[2][PAIR_BN];
    __shared__ uint32_t tensor_memory;
    const uint32_t ring = (shared_address(dynamic) + 1023u) & ~1023u;
    const uint32_t full = shared_address(bars), empty = full + 8 * PAIR_STAGES, sums = empty + 8 * PAIR_STAGES, freed = sums + 16;
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1, unit = blockIdx.x >> 1, units = gridDim.x >> 1, tiles = g.tiles_m * g.tiles_n;
    uint32_t first_full, first_freed;            // of the even CTA
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(first_full) : "r"(full), "r"(0));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(first_freed) : "r"(freed), "r"(0));

    if (threadIdx.x == 0) {
        for (int s = 0; s < PAIR_STAGES; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) { barrier_init(sums + 8 * i, 1); barrier_init(freed + 8 * i, 8); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == PRODUCT_WARP) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(shared_address(&tensor_memory)), "n"(2 * PAIR_BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                           // both CTAs' barriers are there
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t acc = tensor_memory;

    if (warp == COPY_WARP) {
        uint32_t it = 0, s = 0, round = 0;
        bool fine = true;
        for (uint32_t t = unit; t < tiles && fine; t += units) {
            uint32_t tm, tn;
            tile_at(g, t, tm, tn);
            for (uint32_t b = 0; b < g.blocks; ++b, ++it) {
                if (round > 0) fine = warp_wait(empty + 8 * s, (round - 1) & 1);
                if (!fine) break;
                const uint32_t stage = ring + s * PAIR_STAGE;
                if (elected()) {
                    if (rank == 0) barrier_expect(full + 8 * s, 2 * PAIR_STAGE);
                    copy_box_pair(stage, &map_w, first_full + 8 * s, b * BK, tn * 256 + rank * 128);
                    copy_box_pair(stage + BM * BK, &map_a, first_full + 8 * s, b * BK, tm * 256 + rank * 128);
                }
                __syncwarp();
                if (++s == PAIR_STAGES) { s = 0; ++round; }
            }
        }
        if (!fine && rank == 0) {
            // copies in flight end before this CTA does
            for (uint32_t back = 1; back <= PAIR_STAGES && back <= it; ++back)
                if (!warp_wait(full + 8 * ((it - back) % PAIR_STAGES), ((it - back) / PAIR_STAGES) & 1)) break;
        }
    } else if (warp == PRODUCT_WARP) {
        if (rank == 0) {
            uint32_t s = 0, round = 0, turn = 0;
            bool fine = true;
            for (uint32_t t = unit; t < tiles && fine; t += units, ++turn) {
                const uint32_t half = turn & 1, d = acc + half * PAIR_BN;
                if (turn >= 2) fine = warp_wait(freed + 8 * half, (turn / 2 - 1) & 1);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (uint32_t b = 0; b < g.blocks && fine; ++b) {
                    fine = warp_wait(full + 8 * s, round & 1);
                    if (!fine) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t w = operand(ring + s * PAIR_STAGE), a = operand(ring + s * PAIR_STAGE + BM * BK);
                    if (elected()) {
#pragma unroll
                        for (int j = 0; j < BK / 32; ++j) product_pair(d, w + 2 * j, a + 2 * j, b > 0 || j > 0);
                        commit_pair(empty + 8 * s);
                    }
                    __syncwarp();
                    if (++s == PAIR_STAGES) { s = 0; ++round; }
                }
                if (fine && elected()) commit_pair(sums + 8 * half);
            }
        }
    } else {
        uint32_t turn = 0;
        bool fine = true;                        // once false, the rest is written as NaN without another wait
        for (uint32_t t = unit; t < tiles; t += units, ++turn) {
            const uint32_t half = turn & 1;
            uint32_t tm, tn;
            tile_at(g, t, tm, tn);
            stage_scales<PAIR_BN>(scales[half], g, tm * PAIR_BN);
            if (fine) fine = barrier_wait(sums + 8 * half, (turn / 2) & 1);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t col = tn * 256 + rank * 128 + threadIdx.x;
            const float w_scale = !fine ? __uint_as_float(0x7FC00000u) : col < g.n ? g.w_scales[col] : 0.0f;
            const int64_t step = g.ldy * OUT_BYTES;
            char* to = static_cast<char*>(g.y) + (int64_t)tm * PAIR_BN * step + (int64_t)col * OUT_BYTES;
#pragma unroll 1
            for (int c = 0; c < PAIR_BN; c += 32, to += 32 * step) {
                const uint32_t row = tm * PAIR_BN + c;
                if (row >= g.m) break;
                int v[32];
                load_columns(acc + half * PAIR_BN + c + ((uint32_t)warp << 21), v);
                if (col < g.n) {
                    if (row + 32 <= g.m) put_column<OUT>(to, step, v, scales[half] + c, w_scale, 32);
                    else put_column<OUT>(to, step, v, scales[half] + c, w_scale, g.m - row);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(first_freed + 8 * half) : "memory");
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                           // neither leaves while the other's products or arrivals may reach it
    if (warp == PRODUCT_WARP) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(acc), "n"(2 * PAIR_BN));
    }
}

// ------------------------------------------------------------------------------------------------ host
// A matrix of `rows` rows of k bytes, ld apart, in tiles of `box` rows of 128.
bool encode(CUtensorMap& map, const int8_t* base, uint32_t rows, uint32_t k, int64_t ld, int box)
{
    const cuuint64_t size[2] = {k, rows}, stride[1] = {(cuuint64_t)ld};
    const cuuint32_t tile[2] = {BK, (cuuint32_t)box};
    return encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, size, stride, tile);
}

template <int BN, int SPLIT, int OUT>
int launch_gemm(const GemmArgs& g, cudaStream_t stream)
{
    static std::atomic<uint64_t> asked{0};
    const auto kernel = gemm_i8_kernel<BN, SPLIT, OUT>;
    if (allow_shared_memory(reinterpret_cast<const void*>(kernel), Shape<BN>::SHARED, asked) != FBSR_OK) return FBSR_ERR_CUDA;
    CUtensorMap map_w, map_a;
    if (!encode(map_w, g.w, g.n, g.k, g.ldw, BM) || !encode(map_a, g.a, g.m, g.k, g.lda, BN)) return FBSR_ERR_CUDA;
    const uint64_t tiles = (uint64_t)g.tiles_m * g.tiles_n;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)(SPLIT > 1 ? tiles * SPLIT : tiles < 148 ? tiles : 148));
    config.blockDim = dim3(GEMM_THREADS);
    config.dynamicSmemBytes = Shape<BN>::SHARED;
    config.stream = stream;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = SPLIT; cluster.val.clusterDim.y = 1; cluster.val.clusterDim.z = 1;
    config.attrs = &cluster;
    config.numAttrs = SPLIT > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&config, kernel, g, map_w, map_a) != cudaSuccess) { cudaGetLastError(); return FBSR_ERR_CUDA; }
    count_launch();
    return FBSR_OK;
}

template <int OUT>
int launch_gemm_pair(const GemmArgs& g, cudaStream_t stream)
{
    static std::atomic<uint64_t> asked{0};
    const auto kernel = gemm_i8_pair_kernel<OUT>;
    if (allow_shared_memory(reinterpret_cast<const void*>(kernel), PAIR_SHARED, asked) != FBSR_OK) return FBSR_ERR_CUDA;
    CUtensorMap map_w, map_a;
    if (!encode(map_w, g.w, g.n, g.k, g.ldw, BM) || !encode(map_a, g.a, g.m, g.k, g.lda, BM)) return FBSR_ERR_CUDA;
    const uint64_t tiles = (uint64_t)g.tiles_m * g.tiles_n;
    kernel<<<(unsigned)(tiles < 74 ? 2 * tiles : 148), GEMM_THREADS, PAIR_SHARED, stream>>>(g, map_w, map_a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}

template <int BN, int OUT>
int launch_gemm_split(const GemmArgs& g, int split, cudaStream_t stream)
{
    switch (split) {
    case 8: return launch_gemm<BN, 8, OUT>(g, stream);
    case 4: return launch_gemm<BN, 4, OUT>(g, stream);
    case 2: return launch_gemm<BN, 2, OUT>(g, stream);
    default: return launch_gemm<BN, 1, OUT>(g, stream);
    }
}

template <int OUT>
int launch_gemm_columns(const GemmArgs& g, int bn, int split, cudaStream_t stream)
{
    if (split == 0) return launch_gemm_pair<OUT>(g, stream);
    switch (bn) {
    case 256: return launch_gemm_split<256, OUT>(g, split, stream);
    case 128: return launch_gemm_split<128, OUT>(g, split, stream);
    case 64: return launch_gemm_split<64, OUT>(g, split, stream);
    default: return launch_gemm_split<32, OUT>(g, split, stream);
    }
}

// Columns of a tile and split of k (0: a pair of CTAs to a tile of 256 x 256): the least of a model of the time, in clocks.  A
// block of 128 columns takes a CTA the longest of 2 BN (the product unit: 8192 products a clock), (128 + BN) 128 bytes at 64 bytes a
// clock (a multiprocessor's share of L2; two CTAs on one share it), and the ring's depth over a latency of about 2000 clocks;
// writing a tile takes about 16 clocks a column.  How many clusters of 2, 4 and 8 the GPU holds at once was asked of the
// runtime: 74, 33 and 15 where a CTA fills a multiprocessor, 148, 71 and 33 where two fit.
struct GemmPlan { int bn, split; };

GemmPlan plan_gemm(uint64_t m, uint64_t n, uint64_t blocks)
{
    GemmPlan best{32, 1};
    double least = 1e300;
    constexpr uint64_t HELD[2][4] = {{148, 74, 33, 15}, {296, 148, 71, 33}};
    for (int bn = 32; bn <= 256; bn *= 2) {
        const uint64_t tiles = (m + bn - 1) / bn * ((n + BM - 1) / BM);
        const int stages = bn == 128 ? 6 : 4, two = bn <= 64;
        for (int i = 0; i < 4; ++i) {
            const uint64_t split = 1ull << i;
            if (split > 1 && blocks < 2 * split) break;
            const uint64_t held = i == 0 ? 148 : HELD[two][i], ctas = tiles * split;
            const double share = ctas > 148 && split > 1 && two ? 2.0 : 1.0;               // CTAs on a multiprocessor
            const double per = fmax(fmax(2.0 * bn, 2.0 * (128 + bn)) * share, 2000.0 / stages);
            const double waves = (double)((tiles + held - 1) / held), mine = (double)((blocks + split - 1) / split);
            const double writing = 16.0 * bn / split + (split > 1 ? 8.0 * bn + 1500.0 : 0.0);
            const double t = waves * (per * mine + (split > 1 ? writing : 500.0)) + (split > 1 ? 0.0 : writing);
            if (t < least) { least = t; best = {bn, (int)split}; }
        }
    }
    const uint64_t pairs = (m + 255) / 256 * ((n + 255) / 256);
    const double t = (double)((pairs + 73) / 74) * (530.0 * blocks + 500.0) + 16.0 * 256 + 1500.0;
    if (t < least) best = {256, 0};
    return best;
}

template <int M>
void launch_gemv(GemmArgs g, cudaStream_t stream)
{
    // warps along k until there are about 16 warps for each multiprocessor, as long as each has a step of 512 columns
    g.k_warps = 1;
    while (g.k_warps < GEMV_WARPS && (uint64_t)(g.n / GEMV_CHANNELS) * g.k_warps < 148 * 16 && g.k / 512 >= 2 * (uint32_t)g.k_warps) g.k_warps *= 2;
    const uint32_t per = GEMV_WARPS / g.k_warps * GEMV_CHANNELS;
    gemv_i8_kernel<M><<<(g.n + per - 1) / per, GEMV_WARPS * 32, 0, stream>>>(g);
    count_launch();
}

inline bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

}  // namespace
}  // namespace fbsr

using namespace fbsr;

extern "C" int fbsr_gemm_i8(const int8_t* a, int64_t lda, size_t m, const float* a_scales, const int8_t* w, int64_t ldw, size_t n,
                            const float* w_scales, size_t k, void* y, int out_fmt, int64_t ldy, void* cuda_stream)
{
    if (out_fmt != FBSR_FP32 && out_fmt != FBSR_BF16 && out_fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    if (k % 16 != 0 || k == 0) return FBSR_ERR_INVALID_ARG;
    if (k >= 131072 || m > 0x7FFFFFFFu || n > 0x7FFFFFFFu) return FBSR_ERR_TOO_LARGE;
    if (m == 0 || n == 0) return FBSR_OK;
    if (a == nullptr || w == nullptr || a_scales == nullptr || w_scales == nullptr || y == nullptr) return FBSR_ERR_INVALID_ARG;
    if (lda < (int64_t)k || ldw < (int64_t)k || ldy < (int64_t)n) return FBSR_ERR_INVALID_ARG;
    if (lda % 16 != 0 || ldw % 16 != 0) return FBSR_ERR_ALIGNMENT;
    const size_t bytes = out_fmt == FBSR_FP32 ? 4 : 2;
    if (off(a, 16) || off(w, 16) || off(a_scales, 4) || off(w_scales, 4) || off(y, bytes)) return FBSR_ERR_ALIGNMENT;
    if (lda >= (int64_t)1 << 40 || ldw >= (int64_t)1 << 40) return FBSR_ERR_TOO_LARGE;          // what a tensor map's stride holds
    const RowSet result(y, ldy, 0, m, 1, n, bytes);
    if (rows_meet(RowSet(a, lda, 0, m, 1, k, 1), result) || rows_meet(RowSet(w, ldw, 0, n, 1, k, 1), result)) return FBSR_ERR_INVALID_ARG;
    GemmArgs g{};
    g.a = a; g.w = w; g.a_scales = a_scales; g.w_scales = w_scales; g.y = y;
    g.lda = lda; g.ldw = ldw; g.ldy = ldy;
    g.m = (uint32_t)m; g.n = (uint32_t)n; g.k = (uint32_t)k; g.out_fmt = out_fmt;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (m <= 4) {
        if (m == 1) launch_gemv<1>(g, stream);
        else if (m == 2) launch_gemv<2>(g, stream);
        else launch_gemv<4>(g, stream);
        return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
    }
    g.blocks = (uint32_t)((k + BK - 1) / BK);
    const GemmPlan p = plan_gemm(m, n, g.blocks);
    g.tiles_m = (uint32_t)((m + p.bn - 1) / p.bn); g.tiles_n = (uint32_t)(p.split == 0 ? (n + 255) / 256 : (n + BM - 1) / BM);
    if ((uint64_t)g.tiles_m * g.tiles_n > 0x7FFFFFFFu / 8) return FBSR_ERR_TOO_LARGE;
    g.group = 8;
    return out_fmt == FBSR_FP32 ? launch_gemm_columns<FBSR_FP32>(g, p.bn, p.split, stream)
         : out_fmt == FBSR_BF16 ? launch_gemm_columns<FBSR_BF16>(g, p.bn, p.split, stream)
                                : launch_gemm_columns<FBSR_FP16>(g, p.bn, p.split, stream);
}
