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

struct RoundW4Args {
    const void* src;
    uint8_t* codes;
    void* scales;
    void* values;
    int64_t src_ld, values_ld;
    uint64_t offset;
    uint32_t blocks, cols, row_blocks;           // blocks: of 128 elements, all rows; of one row
    uint32_t k0, k1;
    int group_lanes, scale_bf16;           // group_lanes: 4, 8 or 16
    float scale_max;                             // bf16 scales: the largest whose sixfold the source's type holds
};

namespace {

// Eight elements of a row as they lie in memory: TYPE is FBSR_FP32, FBSR_BF16 or FBSR_FP16.
template <int TYPE> struct Raw8 { uint32_t w[TYPE == FBSR_FP32 ? 8 : 4]; };

template <int TYPE>
__device__ __forceinline__ void load_raw8(const RoundW4Args& a, int64_t row, uint32_t c0, int valid, Raw8<TYPE>& out)
{
    if constexpr (TYPE == FBSR_FP32) {
        const float* p = static_cast<const float*>(a.src) + row * a.src_ld + c0;
        if (valid == 8 && reinterpret_cast<uintptr_t>(p) % 32 == 0) {
            float x[8];
            unpack(load_f8_stream(p), x);
#pragma unroll
            for (int c = 0; c < 8; ++c) out.w[c] = __float_as_uint(x[c]);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) out.w[c] = c < valid ? __float_as_uint(p[c]) : 0u;
        }
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(a.src) + row * a.src_ld + c0;
        if (valid == 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(out.w[0]), "=r"(out.w[1]), "=r"(out.w[2]), "=r"(out.w[3]) : "l"(p));
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                out.w[c] = (2 * c < valid ? (uint32_t)p[2 * c] : 0u) | (2 * c + 1 < valid ? (uint32_t)p[2 * c + 1] << 16 : 0u);
        }
    }
}

template <int TYPE>
__device__ __forceinline__ void widen(const Raw8<TYPE>& r, float (&x)[8])
{
    if constexpr (TYPE == FBSR_FP32) {
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = __uint_as_float(r.w[c]);
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if constexpr (TYPE == FBSR_BF16) {
                x[2 * c] = __uint_as_float(r.w[c] << 16);
                x[2 * c + 1] = __uint_as_float(r.w[c] & 0xFFFF0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r.w[c]));
                x[2 * c] = f.x; x[2 * c + 1] = f.y;
            }
        }
    }
}

// The values that the codes of `word` stand for, rounded once to the source's type.
template <int TYPE>
__device__ __forceinline__ void store_values8(const RoundW4Args& a, int64_t row, uint32_t c0, int valid, uint32_t word, float scale)
{
    float v[8];
    uint32_t h[4];
    e2m1_word_to_half2(word, h);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[c]));
        v[2 * c] = __fmul_rn(f.x, scale); v[2 * c + 1] = __fmul_rn(f.y, scale);
    }
    if constexpr (TYPE == FBSR_FP32) {
        float* p = static_cast<float*>(a.values) + row * a.values_ld + c0;
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
        if constexpr (TYPE == FBSR_BF16) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * c], v[2 * c + 1]);
            w[c] = *reinterpret_cast<const uint32_t*>(&b);
        } else {
            const __half2 b = __floats2half2_rn(v[2 * c], v[2 * c + 1]);
            w[c] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
    uint16_t* p = static_cast<uint16_t*>(a.values) + row * a.values_ld + c0;
    if (valid == 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c < valid) p[c] = (uint16_t)(w[c >> 1] >> (16 * (c & 1)));
    }
}

// Largest magnitude of eight values as a pattern; a NaN is larger than all.
__device__ __forceinline__ uint32_t amax8(const float (&x)[8])
{
    float m = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; c += 2) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(x[c]), "f"(x[c + 1]));
    return __float_as_uint(m);
}

__device__ __forceinline__ uint32_t group_max(uint32_t m, int lanes)
{
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    if (lanes >= 8) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
    if (lanes >= 16) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
    return m;
}

// Where a lane's eight elements are.
struct Octet {
    uint32_t block, row, c0;                     // block of the matrix, its row and the first column
    int valid;                                   // how many of the eight the matrix has; -1: the block is none of its blocks
};

// Rows of 256 whose loads are in flight before the first is used, and resident CTAs the compiler must allow: 4096 x 11008
// binary32 with values, k = 4, took 63 us (6.1 TB/s) with 2 and 4, 73 with 1 and 4, 64 with 4 and 4 or 2 and 5, 70 with three
// CTAs.  Without values it takes 57 us for 31 us of bytes and from bfloat16 64 us for 31: then it is the instructions that bound it
// (33 and 38 issue slots an element, 37 with values from binary32; issue 76 to 79 % busy).
constexpr int W4_BATCH = 2, W4_CTAS = 4;

template <int TYPE, int VAR, int K>
__global__ void __launch_bounds__(CTA_THREADS, W4_CTAS)
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

    // This lane's block in the tile's first row.  The stream's first blocks may lie before the matrix (first < 0); blocks are
    // counted modulo 2^32 then, and none below a.blocks is met before the matrix begins.
    const int place = lane & 15;
    const int64_t first = ((int64_t)(tile * T::ELEMS) - (int64_t)a.offset) / W4_BLOCK + (lane >> 4);
    uint32_t block = (uint32_t)first, row = first < 0 ? 0u : block / a.row_blocks, in_row = first < 0 ? 0u : block - row * a.row_blocks;
    auto next = [&] {                            // the place in the tile's next row of 256 elements
        Octet o;
        o.block = block; o.row = row; o.c0 = in_row * W4_BLOCK + place * 8;
        o.valid = block >= a.blocks ? -1 : (int)min(max(a.cols, o.c0) - o.c0, 8u);      // cols may be 2^31
        // two blocks on; out of the stream before the matrix into its first or second block
        const bool before = (int32_t)block < 0 && first < 0;
        block += 2;
        if (before) { in_row = block < 2u ? block : 0u; row = 0u; }
        else in_row += 2;
        while (in_row >= a.row_blocks) { in_row -= a.row_blocks; ++row; }
        return o;
    };
    Raw8<TYPE> raw[W4_BATCH];
    Octet octet[W4_BATCH];
    auto fetch = [&](int j) {
        octet[j] = next();
#pragma unroll
        for (int c = 0; c < (TYPE == FBSR_FP32 ? 8 : 4); ++c) raw[j].w[c] = 0u;
        if (octet[j].valid > 0) load_raw8<TYPE>(a, octet[j].row, octet[j].c0, octet[j].valid, raw[j]);
    };
#pragma unroll
    for (int j = 0; j < W4_BATCH; ++j) fetch(j);

    // the generator runs in the shadow of the first loads
    if constexpr (DRAWS && !OWN_CALL) {
#pragma unroll
        for (int j = 0; j < (T::CALLS + 31) / 32; ++j) {
            const int c = j * 32 + lane;
            if (T::CALLS % 32 == 0 || c < T::CALLS)
                Draws8<K>::store_call(wb + Draws8<K>::WORDS_PER_CALL * c, philox_block(call0 + c, a.k0, a.k1));
        }
        __syncwarp();
    }

#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const Octet at = octet[r % W4_BATCH];
        float x[8];
        widen<TYPE>(raw[r % W4_BATCH], x);
        if (r + W4_BATCH < ROWS) fetch(r % W4_BATCH);

        uint32_t m = group_max(amax8(x), a.group_lanes);
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
            // the top four bits of (sign of y, code) enter from the right, the eighth element first
            word = __funnelshift_l((t[7 - c] & 0x7FFFFFFFu) | (__float_as_uint(y[7 - c]) & 0x80000000u), word, 4);
        if (is_nan) word = 0u;
        if (at.valid >= 0) {
            reinterpret_cast<uint32_t*>(a.codes)[(uint64_t)at.block * 16 + (place & 3) * 4 + (place >> 2)] = word;
            if (lane % a.group_lanes == 0) {
                const uint64_t g = ((uint64_t)at.block * 16 + place) / (uint32_t)a.group_lanes;
                if (a.scale_bf16) static_cast<uint16_t*>(a.scales)[g] = (uint16_t)scale_code;
                else static_cast<uint8_t*>(a.scales)[g] = (uint8_t)scale_code;
            }
            if (a.values != nullptr && at.valid > 0) store_values8<TYPE>(a, at.row, at.c0, at.valid, word, scale);
        }
    }
}

typedef void (*launch_fn)(const RoundW4Args&, cudaStream_t);

template <int TYPE, int VAR, int K>
void launch(const RoundW4Args& a, cudaStream_t stream)
{
    constexpr uint64_t ELEMS = Tile<K>::ELEMS;
    const uint64_t first = a.offset / ELEMS, last = (a.offset + (uint64_t)a.blocks * W4_BLOCK - 1) / ELEMS, n = last - first + 1;
    round_w4_kernel<TYPE, VAR, K><<<(unsigned)((n + WARPS_PER_CTA - 1) / WARPS_PER_CTA), CTA_THREADS, 0, stream>>>(a, first, n);
    count_launch();
}

template <int TYPE, int VAR, int... K>
constexpr std::array<launch_fn, 16> per_k(std::integer_sequence<int, K...>) { return {launch<TYPE, VAR, K + 1>...}; }

}  // namespace

// The launch for one source type; this file is compiled once per type for it (FBSR_W4_TYPE), and once without for the entry
// point.
#ifdef FBSR_W4_TYPE
#define FBSR_NAME2(t) round_w4_##t
#define FBSR_NAME(t) FBSR_NAME2(t)
void FBSR_NAME(FBSR_W4_TYPE)(const RoundW4Args& a, int variant, int k, cudaStream_t stream)
{
    constexpr int TYPE = FBSR_W4_TYPE;
    static const std::array<launch_fn, 16> stochastic[3] = {per_k<TYPE, SRFF>(std::make_integer_sequence<int, 16>{}),
                                                            per_k<TYPE, SRF>(std::make_integer_sequence<int, 16>{}),
                                                            per_k<TYPE, SRC>(std::make_integer_sequence<int, 16>{})};
    static const launch_fn deterministic[3] = {launch<TYPE, RTNE, 4>, launch<TYPE, RTA, 4>, launch<TYPE, RTO, 4>};      // k is ignored
    if (variant < FBSR_RTNE) stochastic[variant][k - 1](a, stream);
    else deterministic[variant - FBSR_RTNE](a, stream);
}
}  // namespace fbsr
#else
void round_w4_0(const RoundW4Args&, int, int, cudaStream_t);
void round_w4_1(const RoundW4Args&, int, int, cudaStream_t);
void round_w4_32(const RoundW4Args&, int, int, cudaStream_t);

namespace {

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
    if (rows > ((uint64_t)1 << 30) / row_blocks) return FBSR_ERR_TOO_LARGE;         // 2^37 elements
    if (values == src) return FBSR_ERR_INVALID_ARG;
    RoundW4Args a{};
    a.src = src; a.codes = codes; a.scales = scales; a.values = values;
    a.src_ld = src_ld; a.values_ld = values_ld;
    a.offset = offset; a.blocks = (uint32_t)(rows * row_blocks);
    a.cols = (uint32_t)cols; a.row_blocks = (uint32_t)row_blocks;
    a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32);
    a.group_lanes = group / 8; a.scale_bf16 = scale_fmt == FBSR_SCALE_BF16;
    a.scale_max = src_fmt == FBSR_FP16 ? 10880.0f : 0x1.54p125f;   // 6 * 10880 <= 65504; 6 * 0x1.54p125 = the largest bf16
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (src_fmt == FBSR_FP32) round_w4_32(a, variant, k_bits, stream);
    else if (src_fmt == FBSR_BF16) round_w4_0(a, variant, k_bits, stream);
    else round_w4_1(a, variant, k_bits, stream);
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}
#endif
