// fbsr_gemv_w4: y = x W^T for few rows of x and a matrix W held as 4-bit codes with group scales.
// The arithmetic is stated in include/fbsr.h, the order of the codes in fbsr_w4.cuh.
//
// What bounds it is reading W, half a byte an element; at the memory's full rate that is about 50 weights a clock on each
// multiprocessor, so a weight may cost at most two or three instruction slots in all.  A pair of codes becomes a pair of
// binary16 values by one conversion, and the products and sums go to the tensor cores (m16n8k16, binary16 operands,
// binary32 sums): 16 rows of W against 8 rows of x, so that up to 8 rows of x cost what one does.  Each group's partial
// sum is formed in the matrix unit from zero and enters the running binary32 sum multiplied by the group's scale: codes
// stay exact, scales are applied in binary32.  (The fifth-generation unit would take 128-row tiles from shared memory:
// the decoded weights would have to be written there and read back, for a product that is far from compute-bound.)
//
// A warp takes tiles of 16 rows of W in runs of 512 columns, of which it keeps two or three on their way through a ring in shared
// memory: enough bytes in flight for the memory's latency without registers.  Row g of the tile is read by four lanes, 16 bytes
// each, and lane t's words of the four quarters of a block of 128 columns meet x's elements [32 j + 8 t, + 8): the order of k
// inside the matrix instruction is the same permutation on both sides.  Two kernels share this.  Where W has many rows and x
// fits in shared memory, gemv_w4_stream_kernel gives each multiprocessor one CTA of 16 warps that share its rows' runs equally.
// Elsewhere gemv_w4_kernel gives a warp one tile at a time, and where the rows are few, warps of a CTA or CTAs of a cluster share
// the columns of the same rows (see launch).  Both add shared sums in a fixed order.
//
// x is staged in shared memory in binary16, once per CTA.  Each block of 128 columns of a bfloat16 row is first multiplied by
// the power of two that brings its largest finite magnitude to [2^14, 2^15): elements down to 2^-32 of it keep all their 8
// bits, smaller ones are rounded to 2^-40 of it, far below the rounding of the binary32 sums; the block's sum is multiplied
// back as it joins the others.
//
// Measured, one row of x, groups of 32, on the device, W not in L2: 128000 x 4096 50.6 us = 5.51 TB/s (0.84 of the measured copy
// rate), 28672 x 8192 27.1 us, 4096 x 11008 (groups of 128) 9.0 us, 4096 x 4096 5.8 us, 1024 x 4096 3.9 us; eight rows by 11008 x
// 4096 11.9 us, by 128000 x 4096 58.7 us.  What bounds the large ones is the latency of the instructions of 16 warps a
// multiprocessor (102 registers a thread allow no more), 104 of them for a 16 x 128 block of one row of x, 131 of eight: 24 warps
// with half the run, two tiles a warp, bulk copies a row at a time, codes through registers and blocks without the way out
// between them were not faster.  The small ones are a launch, x's way to shared memory and one memory latency.
#include <atomic>

#include <cooperative_groups.h>

#include "../../include/fbsr.h"
#include "fbsr_internal.h"
#include "fbsr_w4.cuh"

namespace cg = cooperative_groups;

namespace fbsr {
namespace {

constexpr int GEMV_WARPS = 8, STREAM_WARPS = 16;
constexpr int GEMV_THREADS = GEMV_WARPS * 32;
constexpr int GEMV_MAX_M = 32;                   // rows of x a launch takes
constexpr int RUN = 4;                           // blocks of 128 columns of a stage
constexpr int TILE = 16;                         // rows of W a warp takes
constexpr int ROW_PITCH = RUN * W4_BLOCK_BYTES;  // of a row of codes in shared memory

struct GemvArgs {
    const uint16_t* x;
    const uint8_t* codes;
    const uint8_t* scales;
    void* y;
    int64_t ldx, ldy;
    uint32_t n, k, blocks;                       // blocks: of 128 columns, one row of W
    uint32_t row_scale_bytes;
    int m, chunk_runs, out_fmt, warps_k;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same into sums that start from zero.
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// A row's scales of a run (SB bytes a block) out of shared memory, and those of block d as numbers.
template <int SB> struct RunScales {
    uint32_t w[SB];                              // RUN SB bytes
    __device__ __forceinline__ void load(const unsigned char* p)
    {
        static_assert(RUN == 4, "a word holds one, two or four bytes of each block");
        if constexpr (SB == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
        if constexpr (SB == 2) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
        if constexpr (SB >= 4) {
#pragma unroll
            for (int i = 0; i < SB; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
                w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
            }
        }
    }
    template <bool BF16_S, int COUNT>
    __device__ __forceinline__ void values(int d, float (&s)[COUNT]) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; i += 2) {     // scales i and i + 1 as bfloat16
            uint32_t pair;
            if constexpr (BF16_S && COUNT == 1) pair = w[d / 2] >> (16 * (d & 1));
            else if constexpr (BF16_S) pair = w[(d * COUNT + i) / 2];
            else pair = e8m0_pair_to_bf16x2(w[(d * COUNT + i) / 4] >> (8 * ((d * COUNT + i) & 3)));
            s[i] = __uint_as_float(pair << 16);
            if constexpr (COUNT > 1) s[i + 1] = __uint_as_float(pair & 0xFFFF0000u);
        }
    }
};

template <int BYTES>
__device__ __forceinline__ void copy_async(unsigned char* smem_dst, const uint8_t* gmem_src)
{
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(smem_dst);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(gmem_src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(gmem_src) : "memory");
}

// Eight elements of a row of x from column k on, zero beyond the row's end.
__device__ __forceinline__ uint4 load_x8(const GemvArgs& a, int row, uint32_t k)
{
    const uint16_t* p = a.x + (int64_t)row * a.ldx + k;
    if (k + 8 <= a.k && reinterpret_cast<uintptr_t>(p) % 16 == 0) return __ldg(reinterpret_cast<const uint4*>(p));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (k + c < a.k) w[c >> 1] |= (uint32_t)__ldg(p + c) << (16 * (c & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void store_y(const GemvArgs& a, int col, uint32_t row, float sum)
{
    if (col >= a.m || row >= a.n) return;
    const int64_t at = (int64_t)col * a.ldy + row;
    if (a.out_fmt == FBSR_FP32) static_cast<float*>(a.y)[at] = sum;
    else if (a.out_fmt == FBSR_BF16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(sum);
    else static_cast<__half*>(a.y)[at] = __float2half_rn(sum);
}

__device__ __forceinline__ uint32_t word_of(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// Largest finite magnitude pattern among eight bfloat16 numbers.
__device__ __forceinline__ uint32_t top_of8(const uint4& v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t top = 0u;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t lo = w[c] & 0x7FFFu, hi = (w[c] >> 16) & 0x7FFFu;
        top = max(top, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
    }
    return top;
}

// `blocks` blocks of 128 columns of x, from block `first` on, to shared memory as binary16; COLS: rows of x provided for.
// Sixteen lanes hold a block of a row, eight elements each; up to four such loads are in flight per thread.
template <bool BF16_X, int COLS, int WARPS>
__device__ __forceinline__ void stage_x(const GemvArgs& a, uint32_t first, uint32_t blocks, __half* xs, int stride, float* factor)
{
    constexpr int FLIGHT = 4, LANES = W4_BLOCK / 8, GROUPS = WARPS * 32 / LANES;
    const uint32_t lane = threadIdx.x % LANES, total = blocks * (COLS == 1 ? 1u : (uint32_t)a.m);
    // group i of sixteen threads takes blocks i, i + GROUPS, ... of all rows' blocks
    uint32_t row = 0, block = threadIdx.x / LANES;
    for (uint32_t done = 0; done < total; done += FLIGHT * GROUPS) {
        uint4 v[FLIGHT];
        uint32_t r[FLIGHT], b[FLIGHT];
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            while (COLS > 1 && block >= blocks && row < (uint32_t)a.m) { block -= blocks; ++row; }
            r[i] = row; b[i] = block;
            const bool inside = COLS > 1 ? row < (uint32_t)a.m : block < blocks;
            if (!inside) r[i] = 0xFFFFFFFFu;
            v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (inside) v[i] = load_x8(a, row, (first + block) * W4_BLOCK + lane * 8);
            block += GROUPS;
        }
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            if (done + i * GROUPS >= total) break;           // the same for all threads
            if constexpr (BF16_X) {
                uint32_t top = top_of8(v[i]);
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                // 2^(14 - e), e the exponent of the largest, as far as binary32 has it; and its inverse
                const int f = min(14 - ((int)(top >> 7) - 127), 126);
                const float up = __uint_as_float((uint32_t)(127 + f) << 23), down = __uint_as_float((uint32_t)(127 - f) << 23);
                uint32_t* w = reinterpret_cast<uint32_t*>(&v[i]);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const __half2 h = __floats2half2_rn(__fmul_rn(__uint_as_float(w[c] << 16), up),
                                                        __fmul_rn(__uint_as_float(w[c] & 0xFFFF0000u), up));
                    w[c] = *reinterpret_cast<const uint32_t*>(&h);
                }
                if (r[i] != 0xFFFFFFFFu && lane == 0) factor[b[i] * COLS + r[i]] = down;
            }
            if (r[i] != 0xFFFFFFFFu) *reinterpret_cast<uint4*>(xs + (size_t)r[i] * stride + b[i] * W4_BLOCK + lane * 8) = v[i];
        }
    }
}

// What a lane adds to the warp-uniform addresses of a stage's codes and scales.  Neighbouring lanes read a row; odd rows have
// neighbouring 64 bytes exchanged so that the lanes that read two rows together meet different banks.  The rows' scales
// follow as words.  Rows beyond the matrix are left as they are: what comes of them is dropped.
template <int SB> struct StageCopy {             // SB: bytes of scales of a block
    static constexpr uint32_t ROW_LANES = ROW_PITCH / 16, ROWS_AT_ONCE = 32 / ROW_LANES;  // lanes to a row's codes
    static constexpr uint32_t WORDS = RUN * SB / 4 > 0 ? RUN * SB / 4 : 1;                // of a row's scales of a stage
    uint32_t lane, pitch, row, piece, from, to, scale_from;
    bool scales_by_4;
    __device__ __forceinline__ StageCopy(const GemvArgs& a, uint32_t lane_)
        : lane(lane_), pitch(a.blocks * W4_BLOCK_BYTES), row(lane_ / ROW_LANES), piece(lane_ % ROW_LANES)
    {
        from = row * pitch + piece * 16;
        to = row * ROW_PITCH + (piece ^ ((row & 1) << 2)) * 16;
        scale_from = lane / WORDS * a.row_scale_bytes + lane % WORDS * 4;
        scales_by_4 = RUN * SB % 4 == 0 && a.row_scale_bytes % 4 == 0 && reinterpret_cast<uintptr_t>(a.scales) % 4 == 0;
    }
    // Run q of the tile whose first row's codes and scales are given.
    __device__ __forceinline__ void stage(const GemvArgs& a, unsigned char* dst, const uint8_t* codes, const uint8_t* scales, uint32_t q,
                                          uint32_t tile_rows) const
    {
        unsigned char* scales_to = dst + TILE * ROW_PITCH;
        const uint8_t* codes_at = codes + q * ROW_PITCH;
        const uint8_t* scales_at = scales + q * (RUN * SB);
        if (tile_rows == TILE && q * RUN + RUN <= a.blocks && scales_by_4) {       // a whole stage
#pragma unroll
            for (int r = 0; r < TILE; r += ROWS_AT_ONCE) copy_async<16>(dst + to + r * ROW_PITCH, codes_at + r * pitch + from);
#pragma unroll
            for (int i = 0; i < TILE * WORDS; i += 32)
                if (TILE * WORDS >= 32 || lane < TILE * WORDS)
                    copy_async<4>(scales_to + (i + lane) * 4, scales_at + i / WORDS * a.row_scale_bytes + scale_from);
        } else {
            const uint32_t here = min((uint32_t)RUN, a.blocks - q * RUN);
#pragma unroll
            for (int r = 0; r < TILE; r += ROWS_AT_ONCE)
                if (piece < here * 4 && r + row < tile_rows) copy_async<16>(dst + to + r * ROW_PITCH, codes_at + r * pitch + from);
            if (scales_by_4) {
#pragma unroll
                for (int i = 0; i < TILE * WORDS; i += 32)
                    if ((i + lane) / WORDS < tile_rows && lane % WORDS * 4 < here * SB)
                        copy_async<4>(scales_to + (i + lane) * 4, scales_at + i / WORDS * a.row_scale_bytes + scale_from);
            } else if (lane < tile_rows) {       // rows of scales off the word grid: byte by byte
                for (uint32_t i = 0; i < here * SB; ++i) scales_to[lane * (RUN * SB) + i] = __ldg(scales_at + lane * a.row_scale_bytes + i);
            }
        }
    }
};

// A stage's `here` blocks against x from block x_block0 of shared memory on, into the lane's sums.
template <bool BF16_X, bool BF16_S, int COUNT, bool ONE, int NT>
__device__ __forceinline__ void run_products(float (&acc)[NT][4], const unsigned char* from, uint32_t here, uint32_t x_block0,
                                             const __half* const (&x_lane)[NT], const float* factor, int g, int t)
{
    constexpr int SB = COUNT * (BF16_S ? 2 : 1), COLS = ONE ? 1 : 8 * NT;
    constexpr int QUARTERS = 4 / COUNT;          // quarters of a block under one scale
    constexpr int STEP = ONE ? 2 : 1;            // of the four sums of a lane, those of column 0 are the first and the third
    const unsigned char* codes_of[2] = {from + g * ROW_PITCH + (g & 1) * 64 + t * 16, from + g * ROW_PITCH + ((g & 1) ^ 1) * 64 + t * 16};
    const unsigned char* scales_of = from + TILE * ROW_PITCH + g * (RUN * SB);
    RunScales<SB> scales_of_row[2];      // blocks that the last run of a row lacks: not used
    scales_of_row[0].load(scales_of);
    scales_of_row[1].load(scales_of + 8 * (RUN * SB));
#pragma unroll
    for (int d = 0; d < RUN; ++d) {
        if (d >= here) break;
        const uint32_t x_block = x_block0 + d;
        uint4 code[2];
        float s[2][COUNT], sum[NT][4];               // scales and sums of the block
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            code[h] = *reinterpret_cast<const uint4*>(codes_of[d & 1] + 8 * h * ROW_PITCH + (d & ~1) * W4_BLOCK_BYTES);
            scales_of_row[h].template values<BF16_S, COUNT>(d, s[h]);
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            float part[NT][4];                       // of the codes under one scale
#pragma unroll
            for (int qu = 0; qu < QUARTERS; ++qu) {
                const int j = i * QUARTERS + qu;
                uint32_t lo[4], hi[4];
                e2m1_word_to_half2(word_of(code[0], j), lo);
                e2m1_word_to_half2(word_of(code[1], j), hi);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 b = *reinterpret_cast<const uint4*>(x_lane[n] + x_block * W4_BLOCK + 32 * j);
                    if (qu == 0) mma_f16_first(part[n], lo[0], hi[0], lo[1], hi[1], b.x, b.y);
                    else mma_f16(part[n], lo[0], hi[0], lo[1], hi[1], b.x, b.y);
                    mma_f16(part[n], lo[2], hi[2], lo[3], hi[3], b.z, b.w);
                }
            }
            float (&into)[NT][4] = BF16_X ? sum : acc;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; c += STEP) {
                    const float sc = s[c >> 1][i];
                    into[n][c] = BF16_X && i == 0 ? __fmul_rn(sc, part[n][c]) : __fmaf_rn(sc, part[n][c], into[n][c]);
                }
        }
        if constexpr (BF16_X) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float f[2];
                if constexpr (ONE) f[0] = factor[x_block];
                else {
                    const float2 both = *reinterpret_cast<const float2*>(factor + x_block * COLS + 8 * n + 2 * t);
                    f[0] = both.x; f[1] = both.y;
                }
#pragma unroll
                for (int c = 0; c < 4; c += STEP) acc[n][c] = __fmaf_rn(f[c & 1], sum[n][c], acc[n][c]);
            }
        }
    }
}

// BF16_X: x holds bfloat16.  BF16_S, COUNT: scales are bfloat16, COUNT of them in a block of 128.  ONE: x is one row, which
// column 0 of the sums stands for alone.  NT: groups of 8 rows of x.  STAGES: of each warp's ring.
template <bool BF16_X, bool BF16_S, int COUNT, bool ONE, int NT, int STAGES>
__global__ void __launch_bounds__(GEMV_THREADS, 2)
gemv_w4_kernel(const __grid_constant__ GemvArgs a)
{
    constexpr int SB = COUNT * (BF16_S ? 2 : 1); // bytes of scales of a block
    constexpr int COLS = ONE ? 1 : 8 * NT;
    constexpr int STAGE = TILE * (ROW_PITCH + RUN * SB);
    extern __shared__ __align__(16) unsigned char smem[];
    const uint32_t lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), g = (int)lane >> 2, t = (int)lane & 3;
    const int rows = GEMV_WARPS * TILE / a.warps_k, warp_row = warp / a.warps_k, warp_k = warp % a.warps_k;
    const uint32_t row0 = blockIdx.x * rows + warp_row * TILE;
    const int stride = a.chunk_runs * (RUN * W4_BLOCK) + 32;       // elements: 64 bytes more, so that two rows meet different banks
    unsigned char* ring = smem + warp * (STAGES * STAGE);
    float* red = reinterpret_cast<float*>(smem);                   // at the end, over the rings: [warps_k][m][rows]
    float* factor = reinterpret_cast<float*>(smem + GEMV_WARPS * STAGES * STAGE);      // BF16_X: [block of the chunk][COLS]
    __half* xs = reinterpret_cast<__half*>(factor + (BF16_X ? (a.chunk_runs * RUN * COLS + 3) / 4 * 4 : 0));

    // this CTA's runs of blocks; warp_k of them is this warp's first, and every warps_k-th after it
    const uint32_t runs = (a.blocks + RUN - 1) / RUN;
    const uint32_t q_begin = (uint32_t)((uint64_t)runs * blockIdx.y / gridDim.y), q_end = (uint32_t)((uint64_t)runs * (blockIdx.y + 1) / gridDim.y);

    const StageCopy<SB> copy(a, lane);
    const uint32_t tile_rows = row0 >= a.n ? 0u : min((uint32_t)TILE, a.n - row0);
    const uint8_t* codes = a.codes + (uint64_t)row0 * copy.pitch;
    const uint8_t* scales = a.scales + (uint64_t)row0 * a.row_scale_bytes;
    auto issue = [&](uint32_t q, int slot) {
        if (q < q_end) copy.stage(a, ring + slot * STAGE, codes, scales, q, tile_rows);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // the first stages are on their way before x is staged
    const uint32_t q_first = q_begin + warp_k;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(q_first + s * a.warps_k, s);

    float acc[NT][4];
    const __half* x_lane[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
        // columns beyond row m are computed and dropped
        x_lane[n] = xs + (size_t)(ONE ? 0 : min(8 * n + g, a.m - 1)) * stride + 8 * t;
    }

    int slot = 0, next_slot = STAGES - 1;
    for (uint32_t q0 = q_begin; q0 < q_end; q0 += a.chunk_runs) {
        const uint32_t q1 = min(q0 + (uint32_t)a.chunk_runs, q_end);
        if (q0 > q_begin) __syncthreads();       // the previous chunk has been read
        stage_x<BF16_X, COLS, GEMV_WARPS>(a, q0 * RUN, (q1 - q0) * RUN, xs, stride, factor);
        __syncthreads();
        for (uint32_t q = q0 + warp_k; q < q1; q += a.warps_k) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();                        // this stage has arrived for all lanes, and all have read the one before it
            issue(q + (STAGES - 1) * a.warps_k, next_slot);
            run_products<BF16_X, BF16_S, COUNT, ONE, NT>(acc, ring + slot * STAGE, min((uint32_t)RUN, a.blocks - q * RUN), (q - q0) * RUN, x_lane,
                                                         factor, g, t);
            slot = slot + 1 == STAGES ? 0 : slot + 1;
            next_slot = next_slot + 1 == STAGES ? 0 : next_slot + 1;
        }
    }
    const bool alone = gridDim.y == 1 && a.warps_k == 1;
    if (!alone) __syncthreads();                 // the rings have been read
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = 8 * n + 2 * t + (i & 1), row = warp_row * TILE + g + 8 * (i >> 1);
            if (col >= a.m) continue;
            if (alone) store_y(a, col, blockIdx.x * rows + row, acc[n][i]);
            else red[(warp_k * a.m + col) * rows + row] = acc[n][i];
        }
    if (alone) return;
    if (gridDim.y == 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < rows * a.m; i += GEMV_THREADS) {
            float total = 0.0f;
            for (int w = 0; w < a.warps_k; ++w) total = __fadd_rn(total, red[w * a.m * rows + i]);
            store_y(a, i / rows, blockIdx.x * rows + i % rows, total);
        }
        return;
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    // each CTA of the cluster adds up its share of the sums
    for (uint32_t i = blockIdx.y * GEMV_THREADS + threadIdx.x; i < (uint32_t)(rows * a.m); i += gridDim.y * GEMV_THREADS) {
        float total = 0.0f;
        for (uint32_t c = 0; c < gridDim.y; ++c) {
            const float* theirs = cluster.map_shared_rank(red, c);
            for (int w = 0; w < a.warps_k; ++w) total = __fadd_rn(total, theirs[w * a.m * rows + i]);
        }
        store_y(a, i / rows, blockIdx.x * rows + i % rows, total);
    }
    cluster.sync();                              // nobody leaves while others read its sums
}

// The same for up to eight rows of x that shared memory holds whole and many rows of W: one CTA a multiprocessor, which
// stages x once and takes `tiles` tiles of 16 rows.  Their runs, tile after tile, are one row of work of which each warp takes an
// equal share, without a pause from tile to tile; a share may begin and end inside a tile.
template <bool BF16_X, bool BF16_S, int COUNT, bool ONE, int STAGES>
__global__ void __launch_bounds__(STREAM_WARPS * 32, 1)
gemv_w4_stream_kernel(const __grid_constant__ GemvArgs a, const uint32_t cta_tiles)
{
    constexpr int SB = COUNT * (BF16_S ? 2 : 1), COLS = ONE ? 1 : 8, WARPS = STREAM_WARPS;
    constexpr int STAGE = TILE * (ROW_PITCH + RUN * SB);
    extern __shared__ __align__(16) unsigned char smem[];
    const uint32_t lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), g = (int)lane >> 2, t = (int)lane & 3;
    const uint32_t runs = (a.blocks + RUN - 1) / RUN, tile0 = blockIdx.x * cta_tiles;
    const uint32_t tiles = min(cta_tiles, (a.n + TILE - 1) / TILE - tile0), items = tiles * runs;
    const int stride = runs * (RUN * W4_BLOCK) + 32;               // as above
    unsigned char* ring = smem + warp * (STAGES * STAGE);
    float* part = reinterpret_cast<float*>(smem);                  // at the end, over the rings: [warp][2][m][TILE]
    float* factor = reinterpret_cast<float*>(smem + WARPS * STAGES * STAGE);
    __half* xs = reinterpret_cast<__half*>(factor + (BF16_X ? (runs * RUN * COLS + 3) / 4 * 4 : 0));

    const uint32_t begin = items * warp / WARPS, end = items * (warp + 1) / WARPS;
    uint32_t tile = begin / runs, q = begin % runs, ahead = begin, ahead_tile = tile, ahead_q = q;      // ahead: what is copied next
    const StageCopy<SB> copy(a, lane);
    auto issue = [&](int slot) {
        if (ahead < end) {
            const uint32_t row = (tile0 + ahead_tile) * TILE;
            copy.stage(a, ring + slot * STAGE, a.codes + (uint64_t)row * copy.pitch, a.scales + (uint64_t)row * a.row_scale_bytes, ahead_q,
                       min((uint32_t)TILE, a.n - row));
            ++ahead;
            if (++ahead_q == runs) { ahead_q = 0; ++ahead_tile; }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(s);                 // on their way before x is staged
    stage_x<BF16_X, COLS, WARPS>(a, 0, runs * RUN, xs, stride, factor);
    __syncthreads();

    // early: the sums of the tile that the share begins inside, where it ends beyond it
    float acc[1][4] = {{0.0f, 0.0f, 0.0f, 0.0f}}, early[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const __half* x_lane[1] = {xs + (size_t)(ONE ? 0 : min(g, a.m - 1)) * stride + 8 * t};
    bool from_start = q == 0;                    // the share holds the tile's first run
    int slot = 0, next_slot = STAGES - 1;
    for (uint32_t item = begin; item < end; ++item) {
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        __syncwarp();                            // this stage has arrived for all lanes, and all have read the one before it
        issue(next_slot);
        run_products<BF16_X, BF16_S, COUNT, ONE, 1>(acc, ring + slot * STAGE, min((uint32_t)RUN, a.blocks - q * RUN), q * RUN, x_lane, factor, g, t);
        slot = slot + 1 == STAGES ? 0 : slot + 1;
        next_slot = next_slot + 1 == STAGES ? 0 : next_slot + 1;
        if (++q == runs) {                       // the tile's last run
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (from_start) store_y(a, 2 * t + (i & 1), (tile0 + tile) * TILE + g + 8 * (i >> 1), acc[0][i]);
                else early[i] = acc[0][i];
                acc[0][i] = 0.0f;
            }
            q = 0;
            ++tile;
            from_start = true;
        }
    }
    // The sums of tiles that warps share, added in the warps' order.  A warp has up to two: of the tile that its share begins
    // inside and of the one that it ends inside; the former alone if the share lies inside one tile.
    __syncthreads();                             // the rings have been read
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = 2 * t + (i & 1);
        if (col < a.m) {
            float* mine = part + (warp * 2 * a.m + col) * TILE + g + 8 * (i >> 1);
            mine[0] = from_start ? early[i] : acc[0][i];
            mine[a.m * TILE] = acc[0][i];
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < tiles * TILE * a.m; i += WARPS * 32) {
        const uint32_t row = i % TILE, col = i / TILE % a.m, of = i / TILE / a.m;
        // the warps that hold the tile's first and last run
        const uint32_t first = ((of * runs + 1) * WARPS - 1) / items, last = ((of + 1) * runs * WARPS - 1) / items;
        if (first == last) continue;
        float total = part[((first * 2 + 1) * a.m + col) * TILE + row];
        for (uint32_t w = first + 1; w <= last; ++w)
            if (items * w / WARPS != items * (w + 1) / WARPS) total = __fadd_rn(total, part[(w * 2 * a.m + col) * TILE + row]);
        store_y(a, col, (tile0 + of) * TILE + row, total);
    }
}

template <bool BF16_X, bool BF16_S, int COUNT, bool ONE, int NT, int STAGES>
int launch(GemvArgs a, cudaStream_t stream)
{
    auto kernel = gemv_w4_kernel<BF16_X, BF16_S, COUNT, ONE, NT, STAGES>;
    constexpr int COLS = ONE ? 1 : 8 * NT, STAGE = TILE * (ROW_PITCH + RUN * COUNT * (BF16_S ? 2 : 1));
    constexpr int RINGS = GEMV_WARPS * STAGES * STAGE, RUN_COLUMNS = RUN * W4_BLOCK;
    static_assert(GEMV_WARPS * TILE * COLS * 4 <= RINGS, "the sums fit over the rings");
    constexpr int SMEM_SM = 227 * 1024, SMEM_CTA = SMEM_SM - 1024;
    const int run_bytes = a.m * RUN_COLUMNS * 2 + (BF16_X ? RUN * COLS * 4 : 0), fixed = RINGS + a.m * 64 + 16;
    const uint32_t runs = (a.blocks + RUN - 1) / RUN;
    // Work for most of the GPU out of few rows of W: several warps of a CTA share rows (warps_k), which costs little but
    // stages the same x against fewer rows; or several CTAs of a cluster do (split), which stages each column of x once but
    // waits for the cluster twice.  One to four rows of x take the first, more the second; what is still too little takes
    // the other as well.  (4096 x 4096, one row of x: 5.8 us with four warps sharing, 7.5 with four CTAs, 11.5 with neither;
    // sixteen rows: 15.5, 11.0, 24.8.)
    constexpr uint32_t ENOUGH = 120;
    uint32_t split = 1;
    a.warps_k = 1;
    auto ctas = [&] { const uint32_t rows = GEMV_WARPS * TILE / a.warps_k; return (a.n + rows - 1) / rows * split; };
    auto share_warps = [&] { while (ctas() < ENOUGH && a.warps_k < GEMV_WARPS && (uint32_t)a.warps_k * split < runs) a.warps_k *= 2; };
    auto share_ctas = [&](uint32_t least) { while (ctas() < ENOUGH && split < 8 && split * 2 * (uint32_t)a.warps_k * least <= runs) split *= 2; };
    if (a.m <= 4) { share_warps(); share_ctas(2); }
    else { share_ctas(1); share_warps(); }
    // A chunk of x is whole rounds of the warps that share rows, so that each goes on with its runs from chunk to chunk.  It
    // leaves room for two CTAs a multiprocessor if a round fits then.
    int fit = ((SMEM_SM - 4096) / 2 - fixed) / run_bytes;
    if (fit < a.warps_k) fit = (SMEM_CTA - fixed) / run_bytes;
    static_assert((SMEM_CTA - RINGS - 8 * NT * 64 - 16) / (8 * NT * RUN_COLUMNS * 2 + RUN * COLS * 4) >= 1, "one run of all rows always fits");
    while (a.warps_k > fit) a.warps_k /= 2;
    const uint32_t rows = GEMV_WARPS * TILE / a.warps_k, row_groups = (a.n + rows - 1) / rows;
    const int runs_of_cta = (int)((runs + split - 1) / split), most = fit / a.warps_k * a.warps_k;
    a.chunk_runs = runs_of_cta < most ? runs_of_cta : most;
    const int bytes = fixed + a.chunk_runs * run_bytes;
    static std::atomic<uint64_t> allowed{0};
    if (int rc = allow_shared_memory((const void*)kernel, SMEM_CTA, allowed)) return rc;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(row_groups, split);
    config.blockDim = dim3(GEMV_THREADS);
    config.dynamicSmemBytes = (size_t)bytes;
    config.stream = stream;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = 1; cluster.val.clusterDim.y = split; cluster.val.clusterDim.z = 1;
    config.attrs = &cluster;
    config.numAttrs = split > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&config, kernel, a) != cudaSuccess) return FBSR_ERR_CUDA;
    count_launch();
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}

// Whether the call suits the stream kernel: x fits beside the rings, every multiprocessor has a tile, every warp two runs or
// more, and no more than a quarter of the warps' time is lost to shares that are a run longer than others.  It stages x once a
// multiprocessor and has no pause between tiles, the other kernel finer shares: 128000 x 4096 50.6 us against 55.0, with four rows
// of x 51.8 against 63.0, with eight 58.7 against 75.8; 4096 x 11008 (0.79 of the time filled) 9.0 against 9.9, 14336 x 4096 (0.76)
// 11.2 against 11.7; 20000 x 2048 (0.70) 9.5 against 9.2, 4096 x 4096 (one run a warp) 6.0 against 5.8.
template <bool BF16_X, bool BF16_S, int COUNT, bool ONE, int STAGES>
bool launch_stream(const GemvArgs& a, cudaStream_t stream, int* status)
{
    auto kernel = gemv_w4_stream_kernel<BF16_X, BF16_S, COUNT, ONE, STAGES>;
    constexpr int COLS = ONE ? 1 : 8, STAGE = TILE * (ROW_PITCH + RUN * COUNT * (BF16_S ? 2 : 1)), RINGS = STREAM_WARPS * STAGES * STAGE;
    constexpr uint32_t SMS = 148, SMEM_CTA = 226 * 1024;
    static_assert(STREAM_WARPS * 2 * TILE * COLS * 4 <= RINGS, "the partial sums fit over the rings");
    const uint32_t tiles = (a.n + TILE - 1) / TILE, runs = (a.blocks + RUN - 1) / RUN;
    const uint64_t bytes = RINGS + (BF16_X ? (uint64_t)runs * RUN * COLS * 4 : 0) + (uint64_t)a.m * (runs * (RUN * W4_BLOCK) + 32) * 2 + 16;
    if (tiles < SMS || bytes > SMEM_CTA) return false;
    const uint32_t cta_tiles = (tiles + SMS - 1) / SMS;
    const uint64_t share = ((uint64_t)cta_tiles * runs + STREAM_WARPS - 1) / STREAM_WARPS;
    if (share * STREAM_WARPS >= (1u << 27) || share < 2 || (uint64_t)tiles * runs * 4 < share * STREAM_WARPS * SMS * 3) return false;
    static std::atomic<uint64_t> allowed{0};
    *status = allow_shared_memory((const void*)kernel, SMEM_CTA, allowed);
    if (*status != FBSR_OK) return true;
    kernel<<<(tiles + cta_tiles - 1) / cta_tiles, STREAM_WARPS * 32, bytes, stream>>>(a, cta_tiles);
    count_launch();
    *status = cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
    return true;
}
template <bool BF16_X, bool BF16_S, int COUNT>
int launch_rows(const GemvArgs& a, cudaStream_t stream)
{
    int status;
    if (a.m == 1)
        return launch_stream<BF16_X, BF16_S, COUNT, true, 3>(a, stream, &status) ? status : launch<BF16_X, BF16_S, COUNT, true, 1, 3>(a, stream);
    if (a.m <= 8 && launch_stream<BF16_X, BF16_S, COUNT, false, 2>(a, stream, &status)) return status;
    if (a.m <= 8) return launch<BF16_X, BF16_S, COUNT, false, 1, 2>(a, stream);
    if (a.m <= 16) return launch<BF16_X, BF16_S, COUNT, false, 2, 2>(a, stream);
    return launch<BF16_X, BF16_S, COUNT, false, 4, 2>(a, stream);
}

typedef int (*launch_fn)(const GemvArgs&, cudaStream_t);
// [x is bfloat16][scales are bfloat16][group 32, 64, 128]
const launch_fn kLaunch[2][2][3] = {
    {{launch_rows<false, false, 4>, launch_rows<false, false, 2>, launch_rows<false, false, 1>},
     {launch_rows<false, true, 4>, launch_rows<false, true, 2>, launch_rows<false, true, 1>}},
    {{launch_rows<true, false, 4>, launch_rows<true, false, 2>, launch_rows<true, false, 1>},
     {launch_rows<true, true, 4>, launch_rows<true, true, 2>, launch_rows<true, true, 1>}}};

inline bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

}  // namespace
}  // namespace fbsr

using namespace fbsr;

extern "C" int fbsr_gemv_w4(const void* x, int x_fmt, int64_t ldx, size_t m, const uint8_t* codes, const void* scales, int scale_fmt,
                            int group, size_t n, size_t k, void* y, int out_fmt, int64_t ldy, void* cuda_stream)
{
    if (x_fmt != FBSR_BF16 && x_fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    if (out_fmt != FBSR_FP32 && out_fmt != FBSR_BF16 && out_fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    if ((group != 32 && group != 64 && group != 128) || (scale_fmt != FBSR_SCALE_E8M0 && scale_fmt != FBSR_SCALE_BF16))
        return FBSR_ERR_UNSUPPORTED;
    if (m == 0 || n == 0) return FBSR_OK;
    if (y == nullptr || ldy < (int64_t)n) return FBSR_ERR_INVALID_ARG;
    const size_t out_bytes = out_fmt == FBSR_FP32 ? 4 : 2;
    if (off(y, out_bytes)) return FBSR_ERR_ALIGNMENT;
    if (k > 0 && (x == nullptr || codes == nullptr || scales == nullptr || ldx < (int64_t)k)) return FBSR_ERR_INVALID_ARG;
    if (n > ((size_t)1 << 31) - 64 || k > ((size_t)1 << 28) || m > ((size_t)1 << 31)) return FBSR_ERR_TOO_LARGE;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (k == 0) {                                // an empty sum
        return cudaMemset2DAsync(y, (size_t)ldy * out_bytes, 0, n * out_bytes, m, stream) == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
    }
    const uint32_t scale_bytes = scale_fmt == FBSR_SCALE_BF16 ? 2 : 1;
    GemvArgs a{};
    a.codes = codes; a.scales = static_cast<const uint8_t*>(scales);
    a.ldx = ldx; a.ldy = ldy;
    a.n = (uint32_t)n; a.k = (uint32_t)k; a.blocks = (uint32_t)(fbsr_w4_padded(k) / W4_BLOCK);
    const uint32_t block_scale_bytes = W4_BLOCK / (uint32_t)group * scale_bytes;
    a.row_scale_bytes = a.blocks * block_scale_bytes;
    a.out_fmt = out_fmt;
    const launch_fn launch_m = kLaunch[x_fmt == FBSR_BF16][scale_fmt == FBSR_SCALE_BF16][group == 32 ? 0 : group == 64 ? 1 : 2];
    if (off(x, 2) || off(codes, 16) || off(scales, block_scale_bytes)) return FBSR_ERR_ALIGNMENT;
    if (y == x) return FBSR_ERR_INVALID_ARG;
    for (size_t at = 0; at < m; at += GEMV_MAX_M) {
        a.x = static_cast<const uint16_t*>(x) + (int64_t)at * ldx;
        a.y = static_cast<char*>(y) + (int64_t)at * ldy * (int64_t)out_bytes;
        a.m = (int)(m - at < (size_t)GEMV_MAX_M ? m - at : (size_t)GEMV_MAX_M);
        const int rc = launch_m(a, stream);
        if (rc != FBSR_OK) return rc;
    }
    return FBSR_OK;
}
