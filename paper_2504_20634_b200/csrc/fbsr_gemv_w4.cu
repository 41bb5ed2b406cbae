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
// A CTA takes 16 RT rows of W; its eight warps share out the row's blocks of 128 columns and add their sums in shared
// memory in a fixed order.  Row g of a 16-row tile is read by four lanes, 16 bytes each, and lane t's words of the four
// quarters of the block meet x's elements [32 j + 8 t, + 8): the order of k inside the matrix instruction is the same
// permutation on both sides.
//
// x is staged in shared memory in binary16.  bfloat16 rows are first multiplied by the power of two that brings the row's
// largest finite magnitude to [2^14, 2^15): elements down to 2^-32 of it keep all their 8 bits, smaller ones are rounded
// to 2^-40 of it, far below the rounding of the binary32 sums; the sum is multiplied back at the end.
#include <cmath>

#include "../../include/fbsr.h"
#include "fbsr_internal.h"
#include "fbsr_w4.cuh"

namespace fbsr {
namespace {

constexpr int GEMV_WARPS = 8;
constexpr int GEMV_THREADS = GEMV_WARPS * 32;
constexpr int GEMV_MAX_M = 32;                   // rows of x a launch takes
constexpr int X_SMEM = 72 * 1024;                // shared memory for a chunk of x
constexpr int CHUNK_GRAIN = W4_BLOCK * GEMV_WARPS;

struct GemvArgs {
    const uint16_t* x;
    const uint8_t* codes;
    const uint8_t* scales;
    void* y;
    int64_t ldx, ldy;
    uint32_t n, k, blocks;                       // blocks: of 128 columns, one row of W
    uint32_t row_scale_bytes, block_scale_bytes; // bytes of scales of a row / of a block of 128
    int m, chunk, out_fmt, scale_bf16;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The scales of one block of one row as stored: one, two, four or eight bytes.
__device__ __forceinline__ uint2 load_scales(const uint8_t* p, uint32_t bytes)
{
    uint2 r = make_uint2(0u, 0u);
    if (bytes == 4) r.x = __ldg(reinterpret_cast<const uint32_t*>(p));
    else if (bytes == 8) r = __ldg(reinterpret_cast<const uint2*>(p));
    else if (bytes == 2) r.x = __ldg(reinterpret_cast<const uint16_t*>(p));
    else r.x = __ldg(p);
    return r;
}

// The scale of quarter j (32 elements) of the block.
__device__ __forceinline__ float quarter_scale(const uint2& raw, int j, const GemvArgs& a)
{
    if (a.scale_bf16) {
        // 8, 4 or 2 bytes: four, two or one scales
        const int i = a.block_scale_bytes == 8 ? j : a.block_scale_bytes == 4 ? j >> 1 : 0;
        const uint32_t w = i >= 2 ? raw.y : raw.x;
        return __uint_as_float((i & 1) ? (w & 0xFFFF0000u) : (w << 16));
    }
    const int i = a.block_scale_bytes == 4 ? j : a.block_scale_bytes == 2 ? j >> 1 : 0;
    return e8m0_value((raw.x >> (8 * i)) & 0xFFu);
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

// Power of two that brings a row whose largest finite magnitude has the bfloat16 pattern `top` to [2^14, 2^15).
__device__ __forceinline__ float row_factor(uint32_t top)
{
    const int e = (int)(top >> 7) - 127;                           // subnormal or zero: -127
    return __uint_as_float((uint32_t)(min(14 - e, 127) + 127) << 23);
}

template <bool BF16_X, int NT, int RT>
__global__ void __launch_bounds__(GEMV_THREADS)
gemv_w4_kernel(const __grid_constant__ GemvArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t row_top[GEMV_MAX_M];
    __half* xs = reinterpret_cast<__half*>(smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t row0 = blockIdx.x * (16 * RT);
    const int stride = a.chunk + 32;             // elements: 64 bytes more, so that two rows' quarters meet different banks

    if constexpr (BF16_X) {
        if (threadIdx.x < GEMV_MAX_M) row_top[threadIdx.x] = 0u;
        __syncthreads();
        const uint32_t units = a.blocks * (W4_BLOCK / 8);
        for (int row = 0; row < a.m; ++row) {
            uint32_t top = 0u;
            for (uint32_t u = threadIdx.x; u < units; u += GEMV_THREADS) {
                const uint4 v = load_x8(a, row, u * 8);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t lo = w[c] & 0x7FFFu, hi = (w[c] >> 16) & 0x7FFFu;
                    top = max(top, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
                }
            }
            top = __reduce_max_sync(0xFFFFFFFFu, top);
            if (lane == 0) atomicMax(&row_top[row], top);
        }
    }

    float acc[RT][NT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[r][n][i] = 0.0f;

    // this lane's two rows of each tile; rows beyond the matrix read its last row and are dropped at the end
    const uint8_t* code_row[RT][2];
    const uint8_t* scale_row[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t row = min(row0 + 16 * r + 8 * h + g, a.n - 1);
            code_row[r][h] = a.codes + (uint64_t)row * a.blocks * W4_BLOCK_BYTES + t * 16;
            scale_row[r][h] = a.scales + (uint64_t)row * a.row_scale_bytes;
        }

    const uint32_t padded = a.blocks * W4_BLOCK;
    for (uint32_t k0 = 0; k0 < padded; k0 += a.chunk) {
        const uint32_t len = min((uint32_t)a.chunk, padded - k0);
        __syncthreads();                         // the previous chunk has been read (first: the rows' maxima are complete)
        for (int row = 0; row < a.m; ++row) {
            float factor = 1.0f;
            if constexpr (BF16_X) factor = row_factor(row_top[row]);
            for (uint32_t u = threadIdx.x; u < len / 8; u += GEMV_THREADS) {
                uint4 v = load_x8(a, row, k0 + u * 8);
                if constexpr (BF16_X) {
                    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const __half2 h = __floats2half2_rn(__fmul_rn(__uint_as_float(w[c] << 16), factor),
                                                            __fmul_rn(__uint_as_float(w[c] & 0xFFFF0000u), factor));
                        w[c] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                }
                *reinterpret_cast<uint4*>(xs + (size_t)row * stride + u * 8) = v;
            }
        }
        __syncthreads();
        for (uint32_t s = warp; s < len / W4_BLOCK; s += GEMV_WARPS) {
            const uint32_t block = k0 / W4_BLOCK + s;
            uint4 b[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    b[n][j] = make_uint4(0u, 0u, 0u, 0u);
                    if (8 * n + g < a.m)
                        b[n][j] = *reinterpret_cast<const uint4*>(xs + (size_t)(8 * n + g) * stride + s * W4_BLOCK + 32 * j + 8 * t);
                }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const uint4 lo = __ldg(reinterpret_cast<const uint4*>(code_row[r][0] + (uint64_t)block * W4_BLOCK_BYTES));
                const uint4 hi = __ldg(reinterpret_cast<const uint4*>(code_row[r][1] + (uint64_t)block * W4_BLOCK_BYTES));
                const uint2 s_lo = load_scales(scale_row[r][0] + (uint64_t)block * a.block_scale_bytes, a.block_scale_bytes);
                const uint2 s_hi = load_scales(scale_row[r][1] + (uint64_t)block * a.block_scale_bytes, a.block_scale_bytes);
                const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t pl[4], ph[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        pl[p] = e2m1_pair_to_half2(wl[j] >> (8 * p));
                        ph[p] = e2m1_pair_to_half2(wh[j] >> (8 * p));
                    }
                    const float sl = quarter_scale(s_lo, j, a), sh = quarter_scale(s_hi, j, a);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_f16(part, pl[0], ph[0], pl[1], ph[1], b[n][j].x, b[n][j].y);
                        mma_f16(part, pl[2], ph[2], pl[3], ph[3], b[n][j].z, b[n][j].w);
                        acc[r][n][0] = __fmaf_rn(sl, part[0], acc[r][n][0]);
                        acc[r][n][1] = __fmaf_rn(sl, part[1], acc[r][n][1]);
                        acc[r][n][2] = __fmaf_rn(sh, part[2], acc[r][n][2]);
                        acc[r][n][3] = __fmaf_rn(sh, part[3], acc[r][n][3]);
                    }
                }
            }
        }
    }

    // the warps' sums, [warp][x row][W row], over the staged x
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);
    constexpr int ROWS = 16 * RT, TILE = ROWS * 8 * NT;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                red[warp * TILE + (8 * n + 2 * t + (i & 1)) * ROWS + 16 * r + g + 8 * (i >> 1)] = acc[r][n][i];
    __syncthreads();
    for (int i = threadIdx.x; i < TILE; i += GEMV_THREADS) {
        const int col = i / ROWS;
        const uint32_t row = row0 + i % ROWS;
        if (col >= a.m || row >= a.n) continue;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < GEMV_WARPS; ++w) sum = __fadd_rn(sum, red[w * TILE + i]);
        if constexpr (BF16_X) sum = __fdiv_rn(sum, row_factor(row_top[col]));        // a power of two
        const int64_t at = (int64_t)col * a.ldy + row;
        if (a.out_fmt == FBSR_FP32) static_cast<float*>(a.y)[at] = sum;
        else if (a.out_fmt == FBSR_BF16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(sum);
        else static_cast<__half*>(a.y)[at] = __float2half_rn(sum);
    }
}

template <bool BF16_X, int NT, int RT>
int launch(GemvArgs a, cudaStream_t stream)
{
    auto kernel = gemv_w4_kernel<BF16_X, NT, RT>;
    const int padded = (int)(a.blocks * W4_BLOCK);
    a.chunk = (X_SMEM / (2 * a.m) - 32) / CHUNK_GRAIN * CHUNK_GRAIN;
    if (a.chunk > padded) a.chunk = padded;
    const int x_bytes = a.m * (a.chunk + 32) * 2, red_bytes = GEMV_WARPS * 16 * RT * 8 * NT * 4;
    const int bytes = x_bytes > red_bytes ? x_bytes : red_bytes;
    if (bytes > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess)
        return FBSR_ERR_CUDA;
    const unsigned grid = (a.n + 16 * RT - 1) / (16 * RT);
    kernel<<<grid, GEMV_THREADS, bytes, stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}

template <bool BF16_X>
int launch_rows(const GemvArgs& a, cudaStream_t stream)
{
    if (a.m <= 8) return launch<BF16_X, 1, 1>(a, stream);
    if (a.m <= 16) return launch<BF16_X, 2, 1>(a, stream);
    return launch<BF16_X, 4, 1>(a, stream);
}

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
    a.block_scale_bytes = W4_BLOCK / (uint32_t)group * scale_bytes;
    a.row_scale_bytes = a.blocks * a.block_scale_bytes;
    a.out_fmt = out_fmt; a.scale_bf16 = scale_fmt == FBSR_SCALE_BF16;
    if (off(x, 2) || off(codes, 16) || off(scales, a.block_scale_bytes)) return FBSR_ERR_ALIGNMENT;
    for (size_t at = 0; at < m; at += GEMV_MAX_M) {
        a.x = static_cast<const uint16_t*>(x) + (int64_t)at * ldx;
        a.y = static_cast<char*>(y) + (int64_t)at * ldy * (int64_t)out_bytes;
        a.m = (int)(m - at < (size_t)GEMV_MAX_M ? m - at : (size_t)GEMV_MAX_M);
        const int rc = x_fmt == FBSR_BF16 ? launch_rows<true>(a, stream) : launch_rows<false>(a, stream);
        if (rc != FBSR_OK) return rc;
    }
    return FBSR_OK;
}
