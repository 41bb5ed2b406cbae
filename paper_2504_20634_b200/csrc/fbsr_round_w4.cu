// fbsr_round_w4: a matrix rounded to 4 bits (E2M1) with one scale per group of 32, 64 or 128 elements of a row.
// The arithmetic is stated in include/fbsr.h, the order of the codes in fbsr_w4.cuh.
//
// The tile structure is that of the bandwidth kernel: a warp owns a tile of whole generator calls, a lane 8 consecutive
// elements of a row of 256 (two blocks of codes, 16 lanes each), variant and k are compile-time so that fields are
// taken and added by fixed shifts.  A group is 4, 8 or 16 neighbouring lanes: its maximum takes two to four shuffles.
// Tiles are laid over the draw stream (offset + row * padded columns + column), so that offset, a multiple of 128,
// only shifts which blocks a tile holds.
#include <array>
#include <cmath>
#include <utility>

#include "../../include/fbsr.h"
#include "fbsr_internal.h"
#include "fbsr_w4.cuh"

namespace fbsr {
namespace {

struct RoundW4Args {
    const void* src;
    uint8_t* codes;
    void* scales;
    void* values;
    int64_t src_ld, values_ld;
    uint64_t offset, blocks;                     // blocks: of 128 elements, all rows
    uint32_t cols, row_blocks;                   // row_blocks: blocks of one row
    uint32_t k0, k1;
    int type, group_lanes, scale_bf16;           // group_lanes: 4, 8 or 16
    float scale_max;                             // bf16 scales: the largest whose sixfold the source's type holds
};

__device__ __forceinline__ void load_row8(const RoundW4Args& a, uint64_t row, uint32_t c0, int valid, float (&x)[8])
{
    if (a.type == FBSR_FP32) {
        const float* p = static_cast<const float*>(a.src) + (int64_t)row * a.src_ld + c0;
        if (valid == 8 && reinterpret_cast<uintptr_t>(p) % 32 == 0) {
            unpack(load_f8_stream(p), x);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) x[c] = c < valid ? p[c] : 0.0f;
        }
        return;
    }
    const uint16_t* p = static_cast<const uint16_t*>(a.src) + (int64_t)row * a.src_ld + c0;
    uint32_t w[4];
    if (valid == 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4*>(p));
        w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            w[c] = (2 * c < valid ? (uint32_t)p[2 * c] : 0u) | (2 * c + 1 < valid ? (uint32_t)p[2 * c + 1] << 16 : 0u);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if (a.type == FBSR_BF16) {
            x[2 * c] = __uint_as_float(w[c] << 16);
            x[2 * c + 1] = __uint_as_float(w[c] & 0xFFFF0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[c]));
            x[2 * c] = f.x; x[2 * c + 1] = f.y;
        }
    }
}

// The values that the codes of `word` stand for, rounded once to the source's type.
__device__ __forceinline__ void store_values8(const RoundW4Args& a, uint64_t row, uint32_t c0, int valid, uint32_t word, float scale)
{
    float v[8];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t h = e2m1_pair_to_half2(word >> (8 * c));
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        v[2 * c] = __fmul_rn(f.x, scale); v[2 * c + 1] = __fmul_rn(f.y, scale);
    }
    if (a.type == FBSR_FP32) {
        float* p = static_cast<float*>(a.values) + (int64_t)row * a.values_ld + c0;
        if (valid == 8 && reinterpret_cast<uintptr_t>(p) % 32 == 0) {
            store_f8(p, v);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < valid) p[c] = v[c];
        }
        return;
    }
    uint32_t w[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if (a.type == FBSR_BF16) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * c], v[2 * c + 1]);
            w[c] = *reinterpret_cast<const uint32_t*>(&b);
        } else {
            const __half2 b = __floats2half2_rn(v[2 * c], v[2 * c + 1]);
            w[c] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
    uint16_t* p = static_cast<uint16_t*>(a.values) + (int64_t)row * a.values_ld + c0;
    if (valid == 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c < valid) p[c] = (uint16_t)(w[c >> 1] >> (16 * (c & 1)));
    }
}

__device__ __forceinline__ uint32_t group_max(uint32_t m, int lanes)
{
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    if (lanes >= 8) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
    if (lanes >= 16) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
    return m;
}

template <int VAR, int K>
__global__ void __launch_bounds__(CTA_THREADS, MIN_CTAS_ROUND)
round_w4_kernel(const __grid_constant__ RoundW4Args a, const uint64_t first_tile, const uint64_t n_tiles)
{
    using T = Tile<K>;
    constexpr bool DRAWS = VAR < RTNE;
    constexpr bool OWN_CALL = T::DPW == 2;
    constexpr int ROWS = T::ELEMS / ROW_ELEMS;
    __shared__ __align__(16) uint32_t wordbuf[WARPS_PER_CTA][!DRAWS || OWN_CALL ? 4 : T::BUFFER_WORDS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t index = (uint64_t)blockIdx.x * WARPS_PER_CTA + warp;
    if (index >= n_tiles) return;
    const uint64_t tile = first_tile + index, call0 = tile * T::CALLS;
    uint32_t* wb = wordbuf[warp];

    if constexpr (DRAWS && !OWN_CALL) {
#pragma unroll
        for (int j = 0; j < (T::CALLS + 31) / 32; ++j) {
            const int c = j * 32 + lane;
            if (T::CALLS % 32 == 0 || c < T::CALLS)
                Draws8<K>::store_call(wb + Draws8<K>::WORDS_PER_CALL * c, philox_block(call0 + c, a.k0, a.k1));
        }
        __syncwarp();
    }
    // this lane's block in the tile's first row: the stream's first blocks may lie before the matrix
    int64_t block = ((int64_t)(tile * T::ELEMS) - (int64_t)a.offset) / W4_BLOCK + (lane >> 4);
    int64_t row = block / (int64_t)a.row_blocks;
    int64_t in_row = block - row * (int64_t)a.row_blocks;
    const int place = lane & 15;

#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const bool inside = block >= 0 && (uint64_t)block < a.blocks;
        const uint32_t c0 = (uint32_t)in_row * W4_BLOCK + place * 8;
        const int valid = !inside || c0 >= a.cols ? 0 : a.cols - c0 >= 8 ? 8 : (int)(a.cols - c0);
        float x[8] = {};
        if (valid > 0) load_row8(a, (uint64_t)row, c0, valid, x);

        uint32_t m = 0u;
#pragma unroll
        for (int c = 0; c < 8; ++c) m = max(m, __float_as_uint(x[c]) & 0x7FFFFFFFu);
        m = group_max(m, a.group_lanes);
        const bool is_nan = m > 0x7F800000u;
        if (__any_sync(0xFFFFFFFFu, m >= 0x7F800000u)) {          // rare: the largest FINITE magnitude sets the scale
            m = 0u;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint32_t b = __float_as_uint(x[c]) & 0x7FFFFFFFu;
                m = max(m, b < 0x7F800000u ? b : 0u);
            }
            m = group_max(m, a.group_lanes);
        }
        float scale, inv;
        uint32_t scale_code;
        if (a.scale_bf16) {
            const uint32_t q = __float_as_uint(__fmul_rn(__uint_as_float(m), 1.0f / 6.0f));
            scale = fminf(fmaxf(__uint_as_float((q + 0xFFFFu) & 0xFFFF0000u), 0x1p-126f), a.scale_max);
            inv = __fdiv_rn(1.0f, scale);
            if (is_nan) scale = __uint_as_float(0x7FC00000u);
            scale_code = __float_as_uint(scale) >> 16;
        } else {
            const int e = max((int)(m >> 23) - 127 - 2, -127);    // floor(log2 amax) - floor(log2 6)
            const uint32_t field = (uint32_t)(127 - e);           // never 0: e is at most 125
            inv = __uint_as_float(field << 23);
            scale_code = is_nan ? 255u : (uint32_t)(e + 127);
            scale = e8m0_value(scale_code);
        }
        float y[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) y[c] = __fmul_rn(x[c], inv);
        Draws8<K> d;
        if constexpr (DRAWS && OWN_CALL) d.from_call(philox_block(call0 + r * 32 + lane, a.k0, a.k1));
        else if constexpr (DRAWS) d.from_normalised(wb, r * ROW_ELEMS + lane * 8);
        uint32_t t[8];
        round_row_fast<E2M1, VAR, K>(y, d, t);                    // infinities saturate like any value beyond 6
        uint32_t word = 0u;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            word = (word >> 4) | (t[c] & 0x70000000u) | (__float_as_uint(y[c]) & 0x80000000u);
        if (is_nan) word = 0u;
        if (inside) {
            reinterpret_cast<uint32_t*>(a.codes)[(uint64_t)block * 16 + (place & 3) * 4 + (place >> 2)] = word;
            if (lane % a.group_lanes == 0) {
                const uint64_t g = ((uint64_t)block * 16 + place) / (uint32_t)a.group_lanes;
                if (a.scale_bf16) static_cast<uint16_t*>(a.scales)[g] = (uint16_t)scale_code;
                else static_cast<uint8_t*>(a.scales)[g] = (uint8_t)scale_code;
            }
            if (a.values != nullptr && valid > 0) store_values8(a, (uint64_t)row, c0, valid, word, scale);
        }
        block += 2;
        in_row += 2;
        while (in_row >= (int64_t)a.row_blocks) { in_row -= a.row_blocks; ++row; }
    }
}

typedef void (*launch_fn)(const RoundW4Args&, cudaStream_t);

template <int VAR, int K>
void launch(const RoundW4Args& a, cudaStream_t stream)
{
    constexpr uint64_t ELEMS = Tile<K>::ELEMS;
    const uint64_t first = a.offset / ELEMS, last = (a.offset + a.blocks * W4_BLOCK - 1) / ELEMS, n = last - first + 1;
    round_w4_kernel<VAR, K><<<(unsigned)((n + WARPS_PER_CTA - 1) / WARPS_PER_CTA), CTA_THREADS, 0, stream>>>(a, first, n);
    count_launch();
}

template <int VAR, int... K>
constexpr std::array<launch_fn, 16> per_k(std::integer_sequence<int, K...>) { return {launch<VAR, K + 1>...}; }
const std::array<launch_fn, 16> kStochastic[3] = {per_k<SRFF>(std::make_integer_sequence<int, 16>{}),
                                                  per_k<SRF>(std::make_integer_sequence<int, 16>{}),
                                                  per_k<SRC>(std::make_integer_sequence<int, 16>{})};
const launch_fn kDeterministic[3] = {launch<RTNE, 4>, launch<RTA, 4>, launch<RTO, 4>};      // k is ignored

inline bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

}  // namespace
}  // namespace fbsr

using namespace fbsr;

extern "C" size_t fbsr_w4_padded(size_t cols) { return (cols + W4_BLOCK - 1) / W4_BLOCK * W4_BLOCK; }

extern "C" int fbsr_round_w4(const void* src, int src_fmt, int64_t src_ld, size_t rows, size_t cols, uint8_t* codes, void* scales,
                             int scale_fmt, int group, void* values, int64_t values_ld, int variant, int k_bits, uint64_t seed,
                             uint64_t offset, void* cuda_stream)
{
    if (variant < 0 || variant > 5 || k_bits < 1 || k_bits > 16) return FBSR_ERR_INVALID_ARG;
    if (src_fmt != FBSR_FP32 && src_fmt != FBSR_BF16 && src_fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    if ((group != 32 && group != 64 && group != 128) || (scale_fmt != FBSR_SCALE_E8M0 && scale_fmt != FBSR_SCALE_BF16))
        return FBSR_ERR_UNSUPPORTED;
    if (offset % W4_BLOCK != 0 || offset > (1ull << 62)) return FBSR_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return FBSR_OK;
    if (src == nullptr || codes == nullptr || scales == nullptr) return FBSR_ERR_INVALID_ARG;
    if (src_ld < (int64_t)cols || (values != nullptr && values_ld < (int64_t)cols)) return FBSR_ERR_INVALID_ARG;
    const size_t bytes = src_fmt == FBSR_FP32 ? 4 : 2;
    if (off(src, bytes) || off(values, bytes) || off(codes, 16) || off(scales, scale_fmt == FBSR_SCALE_BF16 ? 2 : 1)) return FBSR_ERR_ALIGNMENT;
    if (cols > ((size_t)1 << 31) || rows > ((size_t)1 << 40)) return FBSR_ERR_TOO_LARGE;
    const uint64_t row_blocks = fbsr_w4_padded(cols) / W4_BLOCK;
    if (rows > ((uint64_t)1 << 36) / row_blocks) return FBSR_ERR_TOO_LARGE;
    RoundW4Args a{};
    a.src = src; a.codes = codes; a.scales = scales; a.values = values;
    a.src_ld = src_ld; a.values_ld = values_ld;
    a.offset = offset; a.blocks = rows * row_blocks;
    a.cols = (uint32_t)cols; a.row_blocks = (uint32_t)row_blocks;
    a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32);
    a.type = src_fmt; a.group_lanes = group / 8; a.scale_bf16 = scale_fmt == FBSR_SCALE_BF16;
    a.scale_max = src_fmt == FBSR_FP16 ? 10880.0f : 0x1.54p125f;   // 6 * 10880 <= 65504; 6 * 0x1.54p125 = the largest bf16
    if (variant < FBSR_RTNE) kStochastic[variant][k_bits - 1](a, static_cast<cudaStream_t>(cuda_stream));
    else kDeterministic[variant - FBSR_RTNE](a, static_cast<cudaStream_t>(cuda_stream));
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}
