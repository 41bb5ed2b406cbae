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
// A CTA takes up to 128 rows of W, 16 to a warp, and a range of the columns.  Each warp keeps three stages of 16 rows by 512
// columns on their way through shared memory (two where x is more than a row): enough bytes in flight for the memory's
// latency without registers.  Row g of the warp's tile is read by four lanes, 16 bytes each, and lane t's words of the four
// quarters of a block of 128 columns meet x's elements [32 j + 8 t, + 8): the order of k inside the matrix instruction is the
// same permutation on both sides.  Where the rows are few, warps of a CTA or CTAs of a cluster share the columns of the same
// rows and add their sums in a fixed order (see launch).
//
// x is staged in shared memory in binary16, once per CTA.  Each block of 128 columns of a bfloat16 row is first multiplied by
// the power of two that brings its largest finite magnitude to [2^14, 2^15): elements down to 2^-32 of it keep all their 8
// bits, smaller ones are rounded to 2^-40 of it, far below the rounding of the binary32 sums; the block's sum is multiplied
// back as it joins the others.
//
// Measured, one row of x, bfloat16, groups of 32, on the device: 128000 x 4096 55 us = 5.06 TB/s (0.77 of the measured copy
// rate), 28672 x 8192 31 us, 4096 x 11008 9.6 us, 4096 x 4096 5.8 us, 1024 x 4096 4.0 us; eight rows by 11008 x 4096 14.3 us.
// What bounds the large ones is issue latency, not memory (16 warps a multiprocessor, 111 instructions for a 16 x 128 block,
// 51 % of the issue slots): 24 warps with half the stage gained 3 % there and lost 14 % at 8192 columns; two tiles a warp, bulk
// copies a row at a time, codes through registers and blocks without the way out between them were slower.
#include <atomic>

#include <cooperative_groups.h>

#include "../../include/fbsr.h"
#include "fbsr_internal.h"
#include "fbsr_w4.cuh"

namespace cg = cooperative_groups;

namespace fbsr {
namespace {

constexpr int GEMV_WARPS = 8;
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
template <bool BF16_X, int COLS>
__device__ __forceinline__ void stage_x(const GemvArgs& a, uint32_t first, uint32_t blocks, __half* xs, int stride, float* factor)
{
    constexpr int FLIGHT = 4, LANES = W4_BLOCK / 8, GROUPS = GEMV_THREADS / LANES;
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

// BF16_X: x holds bfloat16.  BF16_S, COUNT: scales are bfloat16, COUNT of them in a block of 128.  ONE: x is one row, which
// column 0 of the sums stands for alone.  NT: groups of 8 rows of x.  STAGES: of each warp's ring.
template <bool BF16_X, bool BF16_S, int COUNT, bool ONE, int NT, int STAGES>
__global__ void __launch_bounds__(GEMV_THREADS, 2)
gemv_w4_kernel(const __grid_constant__ GemvArgs a)
{
    constexpr int SB = COUNT * (BF16_S ? 2 : 1); // bytes of scales of a block
    constexpr int COLS = ONE ? 1 : 8 * NT;
    constexpr int QUARTERS = 4 / COUNT;          // quarters of a block under one scale
    constexpr int STEP = ONE ? 2 : 1;            // of the four sums of a lane, those of column 0 are the first and the third
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

    // Each warp fills its own ring, neighbouring lanes to a row; odd rows have neighbouring 64 bytes exchanged so that
    // the lanes that read two rows together meet different banks.  The rows' scales follow as words.  Rows beyond the matrix
    // are left as they are: what comes of them is dropped.
    const uint32_t tile_rows = row0 >= a.n ? 0u : min((uint32_t)TILE, a.n - row0), pitch = a.blocks * W4_BLOCK_BYTES;
    // warp-uniform addresses, and what the lane adds to them
    const uint8_t* codes = a.codes + (uint64_t)row0 * pitch;
    const uint8_t* scales = a.scales + (uint64_t)row0 * a.row_scale_bytes;
    constexpr uint32_t ROW_LANES = ROW_PITCH / 16, ROWS_AT_ONCE = 32 / ROW_LANES;  // lanes to a row's codes
    const uint32_t lane_row = lane / ROW_LANES, lane_piece = lane % ROW_LANES;
    const uint32_t copy_from = lane_row * pitch + lane_piece * 16;
    const uint32_t copy_to = lane_row * ROW_PITCH + (lane_piece ^ ((lane_row & 1) << 2)) * 16;
    constexpr uint32_t WORDS = RUN * SB / 4 > 0 ? RUN * SB / 4 : 1;                // of a row's scales of a stage
    const uint32_t scale_from = lane / WORDS * a.row_scale_bytes + lane % WORDS * 4;
    const bool scales_by_4 = RUN * SB % 4 == 0 && a.row_scale_bytes % 4 == 0 && reinterpret_cast<uintptr_t>(a.scales) % 4 == 0;
    auto issue = [&](uint32_t q, int slot) {
        if (q < q_end) {
            unsigned char* to = ring + slot * STAGE;
            unsigned char* scales_to = to + TILE * ROW_PITCH;
            const uint8_t* from = codes + q * ROW_PITCH;
            const uint8_t* scales_at = scales + q * (RUN * SB);
            if (tile_rows == TILE && q * RUN + RUN <= a.blocks && scales_by_4) {   // a whole stage
#pragma unroll
                for (int r = 0; r < TILE; r += ROWS_AT_ONCE) copy_async<16>(to + copy_to + r * ROW_PITCH, from + r * pitch + copy_from);
#pragma unroll
                for (int i = 0; i < TILE * WORDS; i += 32)
                    if (TILE * WORDS >= 32 || lane < TILE * WORDS)
                        copy_async<4>(scales_to + (i + lane) * 4, scales_at + i / WORDS * a.row_scale_bytes + scale_from);
            } else {
                const uint32_t here = min((uint32_t)RUN, a.blocks - q * RUN);
#pragma unroll
                for (int r = 0; r < TILE; r += ROWS_AT_ONCE)
                    if (lane_piece < here * 4 && r + lane_row < tile_rows)
                        copy_async<16>(to + copy_to + r * ROW_PITCH, from + r * pitch + copy_from);
                if (scales_by_4) {
#pragma unroll
                    for (int i = 0; i < TILE * WORDS; i += 32)
                        if ((i + lane) / WORDS < tile_rows && lane % WORDS * 4 < here * SB)
                            copy_async<4>(scales_to + (i + lane) * 4, scales_at + i / WORDS * a.row_scale_bytes + scale_from);
                } else if (lane < tile_rows) {                     // rows of scales off the word grid: byte by byte
                    for (uint32_t i = 0; i < here * SB; ++i) scales_to[lane * (RUN * SB) + i] = __ldg(scales_at + lane * a.row_scale_bytes + i);
                }
            }
        }
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
        stage_x<BF16_X, COLS>(a, q0 * RUN, (q1 - q0) * RUN, xs, stride, factor);
        __syncthreads();
        for (uint32_t q = q0 + warp_k; q < q1; q += a.warps_k) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();                        // this stage has arrived for all lanes, and all have read the one before it
            issue(q + (STAGES - 1) * a.warps_k, next_slot);
            const unsigned char* from = ring + slot * STAGE;
            const unsigned char* codes_of[2] = {from + g * ROW_PITCH + (g & 1) * 64 + t * 16, from + g * ROW_PITCH + ((g & 1) ^ 1) * 64 + t * 16};
            const unsigned char* scales_of = from + TILE * ROW_PITCH + g * (RUN * SB);
            const uint32_t here = min((uint32_t)RUN, a.blocks - q * RUN);
            RunScales<SB> scales_of_row[2];      // blocks that the last run of a row lacks: not used
            scales_of_row[0].load(scales_of);
            scales_of_row[1].load(scales_of + 8 * (RUN * SB));
#pragma unroll
            for (int d = 0; d < RUN; ++d) {
                if (d >= here) break;
                const uint32_t x_block = (q - q0) * RUN + d;
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

template <bool BF16_X, bool BF16_S, int COUNT>
int launch_rows(const GemvArgs& a, cudaStream_t stream)
{
    if (a.m == 1) return launch<BF16_X, BF16_S, COUNT, true, 1, 3>(a, stream);
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
    for (size_t at = 0; at < m; at += GEMV_MAX_M) {
        a.x = static_cast<const uint16_t*>(x) + (int64_t)at * ldx;
        a.y = static_cast<char*>(y) + (int64_t)at * ldy * (int64_t)out_bytes;
        a.m = (int)(m - at < (size_t)GEMV_MAX_M ? m - at : (size_t)GEMV_MAX_M);
        const int rc = launch_m(a, stream);
        if (rc != FBSR_OK) return rc;
    }
    return FBSR_OK;
}
