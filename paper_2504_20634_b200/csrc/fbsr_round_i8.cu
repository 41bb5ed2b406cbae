// fbsr_round_i8: rows of a matrix rounded to 8-bit integers with a scale each.  The arithmetic is stated in include/fbsr.h.
//
// A row's largest magnitude is needed before its first code, so the row stays in registers between the two: one warp holds rows
// of up to 1024 elements, four, eight or sixteen warps rows of up to 16384 (one octet of eight elements a thread and step; the
// number of steps is compile-time, so that all loads of a row are in flight at once).  Longer rows are read twice, the second
// time mostly from L2.
//
// To nearest this is bound by memory: 4096 x 11008 from bfloat16 (135 MB) 20.8 us (6.5 TB/s), with values (225 MB) 34.9.  Stochastic
// rounding is bound by instructions, 25 an element at 75 % of the issue rate (integer units 67 %), two fifths of the time in the
// generator, one call of which serves eight elements: SRF 44.8 us and 54.7 with values, SRC 54.6 and 64.8.
#include <cfloat>

#include "fbsr_answer.cuh"
#include "fbsr_internal.h"

namespace fbsr {
namespace {

struct RoundI8Args {
    const void* src;
    int8_t* codes;
    float* scales;
    void* values;
    int64_t src_ld, values_ld;
    uint64_t rows, offset;
    uint32_t cols, octets;                       // octets: of a padded row
    uint32_t k0, k1;
    int whole, values_whole;                     // eight elements of src (of values) may be moved at a time
    float scale_max;
    uint32_t base, base_hi;                      // PLAIN: the pattern of 128 and the half step; the same before the high draw's rotation
    RoundRule rule;
};

// EVEN: y is added to 1.5 2^23.  Otherwise |y|, at most 127, is added to 128: the sum's pattern holds the integer in bits 16 to 22 and sixteen fraction bits below, cut off
// by the rounding mode.  That is enough for k random bits and half a step up to k = 15, and for a pre-round to k bits with its tie
// and a sticky bit up to k = 14; wider draws (WIDE) go through an integer of eighteen fraction bits.
constexpr int I8_SH0 = 16, I8_WIDE_SH0 = 18;

inline int i8_kind(int variant, int k)
{
    if ((variant == SRF && k > 15) || (variant == SRC && k > 14)) return RULE_WIDE;
    return rule_kind(variant);
}

// The pattern of 128 + the integer that |y| is rounded to, with anything in its lower sixteen bits; EVEN: of 1.5 2^23 + the
// integer that y is rounded to, whose lowest byte is the code.
template <int KIND>
__device__ __forceinline__ uint32_t round_to_integer(float y, const uint4& draws, int c, const RoundI8Args& a)
{
    const RoundRule& r = a.rule;
    if constexpr (KIND == RULE_EVEN) return __float_as_uint(__fadd_rn(y, 12582912.0f));
    const float t = fminf(fabsf(y), 127.0f);
    if constexpr (KIND == RULE_PLAIN) {
        // 128 + draw + half a step is itself a number of sixteen fraction bits: one addition, cut off, is the rounding
        const uint32_t word = c < 2 ? draws.x : c < 4 ? draws.y : c < 6 ? draws.z : draws.w;
        uint32_t d;
        if (c & 1) { d = (word & r.mask_hi) | a.base_hi; d = __funnelshift_l(d, d, r.rot); }
        else d = (word & r.mask_lo) * r.mul + a.base;
        return __float_as_uint(__fadd_rz(t, __uint_as_float(d)));
    } else if constexpr (KIND == RULE_NEAREST) {
        uint32_t u = __float_as_uint(__fadd_rz(t, 128.0f));
        u |= (u ^ __float_as_uint(__fadd_ru(t, 128.0f))) & 1u;
        return u + (((u >> r.pos) & 1u) ^ r.flip) + placed_draw<false>(draws, c, r) + r.add;
    } else {
        const float f = __fmul_rn(t, 0x1p18f);                 // exact
        uint32_t u = __float2uint_rz(f);
        u |= __uint2float_rn(u) != f ? 1u : 0u;
        // SRF: no parity is asked for, and the sticky bit lies two below its half step
        if (r.flip == 2u) u += placed_draw<true>(draws, c, r);
        else u += (((u >> r.pos) & 1u) ^ r.flip) + placed_draw<false>(draws, c, r) + r.add;
        return 0x43000000u + (u >> I8_WIDE_SH0 << 16);
    }
}

// A row's scale and its inverse from the largest finite magnitude.
struct RowScale { float scale, inv; bool is_nan, has_inf; };

__device__ __forceinline__ RowScale scale_of(uint32_t finite, bool is_nan, float scale_max)
{
    RowScale s;
    s.is_nan = is_nan;
    s.scale = fminf(fmaxf(__fmul_rn(__uint_as_float(finite), 1.0f / 127.0f), 0x1p-126f), scale_max);
    s.inv = __fdiv_rn(1.0f, s.scale);
    return s;
}

// The top bit of each word eight times, in the two low bytes.
__device__ __forceinline__ uint32_t top_bits(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, 0x00FB;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <int TYPE, int KIND, bool VALUES>
__device__ __forceinline__ void write_octet(const RoundI8Args& a, uint64_t row, uint32_t octet, const float (&x)[8], const RowScale& s)
{
    uint4 d = make_uint4(0u, 0u, 0u, 0u);
    if (a.rule.mask_lo != 0u) {
        const uint64_t call = a.offset / 8 + row * a.octets + octet;
        d = philox4x32_10((uint32_t)call, (uint32_t)(call >> 32), DRAWS_I8, 0u, a.k0, a.k1);
    }
    // what lies behind the row's end was read as zeros, and zero rounds to zero
    uint32_t t[8], y[8];
    if (KIND == RULE_EVEN && s.has_inf) {
        float clamped[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) clamped[c] = fminf(fmaxf(__fmul_rn(x[c], s.inv), -127.0f), 127.0f);
#pragma unroll
        for (int c = 0; c < 8; ++c) { y[c] = __float_as_uint(clamped[c]); t[c] = round_to_integer<KIND>(clamped[c], d, c, a); }
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float f = __fmul_rn(x[c], s.inv);
            y[c] = __float_as_uint(f);
            t[c] = round_to_integer<KIND>(f, d, c, a);
        }
    }
    uint32_t word[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t* p = t + 4 * h;
        const uint32_t* q = y + 4 * h;
        if constexpr (KIND == RULE_EVEN) {
            word[h] = s.is_nan ? 0u : gather_bytes<0>(p[0], p[1], p[2], p[3]);
            continue;
        }
        const uint32_t m = gather_bytes<2>(p[0], p[1], p[2], p[3]);
        // bytes of ones where y is negative (a byte's sign repeated), then each byte's two's complement: no carry leaves a byte
        const uint32_t n = __byte_perm(top_bits(q[0], q[1]), top_bits(q[2], q[3]), 0x5410);
        word[h] = (((m ^ n) & 0x7F7F7F7Fu) + (n & 0x01010101u)) ^ (n & 0x80808080u);
        if (s.is_nan) word[h] = 0u;
    }
    reinterpret_cast<uint2*>(a.codes)[row * a.octets + octet] = make_uint2(word[0], word[1]);
    if constexpr (VALUES) {
        if (octet * 8 >= a.cols) return;
        // an integer has one zero: the sum with +0 makes +0 of -0 and changes nothing else
        float v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            if constexpr (KIND == RULE_EVEN) v[c] = __fmul_rn(__fsub_rn(__uint_as_float(t[c]), 12582912.0f), s.scale);
            else v[c] = __fmaf_rn(copysignf(__fsub_rn(__uint_as_float(t[c] & 0xFFFF0000u), 128.0f), __uint_as_float(y[c])), s.scale, 0.0f);
        }
        const int valid = (int)min(a.cols - octet * 8, 8u);
        store8<TYPE>(a.values, (int64_t)row * a.values_ld + octet * 8, valid, a.values_whole && valid == 8, v);
    }
}

__device__ __forceinline__ uint32_t warp_max(uint32_t m) { return __reduce_max_sync(0xFFFFFFFFu, m); }

// The maximum over the WARPS warps of a row; `buffer` holds a word for each.
template <int WARPS>
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* buffer)
{
    m = warp_max(m);
    if constexpr (WARPS > 1) {
        __syncthreads();                         // the last maximum has been read by all
        if ((threadIdx.x & 31) == 0) buffer[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) m = max(m, buffer[w]);
    }
    return m;
}

// WARPS warps to a row, STEPS octets a thread; STEPS = 0: as many as the row has, read twice.
template <int TYPE, int KIND, bool VALUES, int WARPS, int STEPS>
__global__ void __launch_bounds__(WARPS == 1 ? 128 : WARPS * 32)
round_i8_kernel(const __grid_constant__ RoundI8Args a)
{
    __shared__ uint32_t buffer[WARPS];
    constexpr int LANES = WARPS * 32;
    const uint64_t row = WARPS == 1 ? (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= a.rows) return;
    const uint32_t lane = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x;
    auto load = [&](uint32_t octet, Octet8<TYPE>& o) {
        const uint32_t c0 = octet * 8;
        const int valid = c0 < a.cols ? (int)min(a.cols - c0, 8u) : 0;
        load_octet<TYPE>(a.src, (int64_t)row * a.src_ld + c0, valid, a.whole && valid == 8, o);
    };
    constexpr int HELD = STEPS > 0 ? STEPS : 1;
    Octet8<TYPE> held[HELD];
    const uint32_t steps = STEPS > 0 ? STEPS : (a.octets + LANES - 1) / LANES;
    float x[8];
    uint32_t m = 0u;
    if constexpr (STEPS > 0) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) load(i * LANES + lane, held[i]);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) m = join_amax<TYPE>(m, amax8<TYPE>(held[i]));
    } else {
#pragma unroll 4
        for (uint32_t i = 0; i < steps; ++i) {
            load(i * LANES + lane, held[0]);
            m = join_amax<TYPE>(m, amax8<TYPE>(held[0]));
        }
    }
    m = row_max<WARPS>(amax_pattern<TYPE>(m), buffer);
    const bool is_nan = m > 0x7F800000u, has_inf = m >= 0x7F800000u;
    if (has_inf) {                      // rare, and the same for all of the row: the largest FINITE magnitude sets the scale
        m = 0u;
        for (uint32_t i = 0; i < steps; ++i) {
            load(i * LANES + lane, held[0]);
            widen<TYPE>(held[0], x);
            m = max(m, finite_amax8_pattern(x));
        }
        m = row_max<WARPS>(m, buffer);
        if constexpr (STEPS > 0) load(lane, held[0]);
    }
    RowScale s = scale_of(m, is_nan, a.scale_max);
    s.has_inf = has_inf;
    if (is_nan) s.scale = __uint_as_float(0x7FC00000u);
    if (lane == 0) a.scales[row] = s.scale;
    if constexpr (STEPS > 0) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const uint32_t octet = i * LANES + lane;
            widen<TYPE>(held[i], x);
            if (octet < a.octets) write_octet<TYPE, KIND, VALUES>(a, row, octet, x, s);
        }
    } else {
#pragma unroll 2
        for (uint32_t octet = lane; octet < a.octets; octet += LANES) {
            load(octet, held[0]);
            widen<TYPE>(held[0], x);
            write_octet<TYPE, KIND, VALUES>(a, row, octet, x, s);
        }
    }
}

// Up to two rows a multiprocessor: sixteen warps to a row, for its latency.
constexpr uint64_t FEW_ROWS = 296;

template <int TYPE, int KIND, bool VALUES>
void launch(const RoundI8Args& a, cudaStream_t stream)
{
    const unsigned rows = (unsigned)a.rows, quarter = (unsigned)((a.rows + 3) / 4);
    const uint32_t n = a.octets * 8;
    if (KIND == RULE_WIDE) round_i8_kernel<TYPE, KIND, VALUES, 8, 0><<<rows, 256, 0, stream>>>(a);
    else if (n <= 256) round_i8_kernel<TYPE, KIND, VALUES, 1, 1><<<quarter, 128, 0, stream>>>(a);
    else if (n <= 1024) round_i8_kernel<TYPE, KIND, VALUES, 1, 4><<<quarter, 128, 0, stream>>>(a);
    else if (a.rows <= FEW_ROWS && n <= 8192) round_i8_kernel<TYPE, KIND, VALUES, 16, 2><<<rows, 512, 0, stream>>>(a);
    else if (a.rows <= FEW_ROWS && n <= 16384) round_i8_kernel<TYPE, KIND, VALUES, 16, 4><<<rows, 512, 0, stream>>>(a);
    else if (n <= 2048) round_i8_kernel<TYPE, KIND, VALUES, 4, 2><<<rows, 128, 0, stream>>>(a);
    else if (n <= 4096) round_i8_kernel<TYPE, KIND, VALUES, 4, 4><<<rows, 128, 0, stream>>>(a);
    else if (n <= 8192) round_i8_kernel<TYPE, KIND, VALUES, 8, 4><<<rows, 256, 0, stream>>>(a);
    else if (n <= 12288) round_i8_kernel<TYPE, KIND, VALUES, 8, 6><<<rows, 256, 0, stream>>>(a);
    else if (n <= 16384) round_i8_kernel<TYPE, KIND, VALUES, 8, 8><<<rows, 256, 0, stream>>>(a);
    else round_i8_kernel<TYPE, KIND, VALUES, 8, 0><<<rows, 256, 0, stream>>>(a);
    count_launch();
}

template <int TYPE>
void launch_kind(const RoundI8Args& a, int kind, cudaStream_t stream)
{
    const bool values = a.values != nullptr;
    if (kind == RULE_PLAIN) values ? launch<TYPE, RULE_PLAIN, true>(a, stream) : launch<TYPE, RULE_PLAIN, false>(a, stream);
    else if (kind == RULE_EVEN) values ? launch<TYPE, RULE_EVEN, true>(a, stream) : launch<TYPE, RULE_EVEN, false>(a, stream);
    else if (kind == RULE_NEAREST) values ? launch<TYPE, RULE_NEAREST, true>(a, stream) : launch<TYPE, RULE_NEAREST, false>(a, stream);
    else values ? launch<TYPE, RULE_WIDE, true>(a, stream) : launch<TYPE, RULE_WIDE, false>(a, stream);
}

inline bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

}  // namespace
}  // namespace fbsr

using namespace fbsr;

extern "C" size_t fbsr_i8_padded(size_t cols) { return (cols + 127) / 128 * 128; }

extern "C" int fbsr_round_i8(const void* src, int src_fmt, int64_t src_ld, size_t rows, size_t cols, int8_t* codes, float* scales,
                             void* values, int64_t values_ld, int variant, int k_bits, uint64_t seed, uint64_t offset, void* cuda_stream)
{
    if (variant < 0 || variant > 5 || k_bits < 1 || k_bits > 16) return FBSR_ERR_INVALID_ARG;
    if (src_fmt != FBSR_FP32 && src_fmt != FBSR_BF16 && src_fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    if (offset % 128 != 0 || offset > (1ull << 62)) return FBSR_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return FBSR_OK;
    if (src == nullptr || codes == nullptr || scales == nullptr) return FBSR_ERR_INVALID_ARG;
    if (src_ld < (int64_t)cols || (values != nullptr && values_ld < (int64_t)cols)) return FBSR_ERR_INVALID_ARG;
    const size_t bytes = src_fmt == FBSR_FP32 ? 4 : 2;
    if (off(src, bytes) || off(values, bytes) || off(codes, 16) || off(scales, 4)) return FBSR_ERR_ALIGNMENT;
    if (rows > 0x7FFFFFFFu || cols > 0x7FFFFF00u) return FBSR_ERR_TOO_LARGE;
    if (values != nullptr && rows_meet(RowSet(src, src_ld, 0, rows, 1, cols, bytes), RowSet(values, values_ld, 0, rows, 1, cols, bytes)))
        return FBSR_ERR_INVALID_ARG;
    RoundI8Args a{};
    a.src = src; a.codes = codes; a.scales = scales; a.values = values;
    a.src_ld = src_ld; a.values_ld = values_ld;
    a.rows = rows; a.cols = (uint32_t)cols; a.octets = (uint32_t)(fbsr_i8_padded(cols) / 8);
    a.offset = offset;
    a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32);
    const size_t step = 8 * bytes;
    a.whole = !off(src, step) && src_ld * bytes % step == 0;
    a.values_whole = !off(values, step) && values_ld * bytes % step == 0;
    a.scale_max = 0x1.020406p+121f;              // the largest binary32 number whose 127-fold is finite
    static_assert(127.0 * 0x1.020406p+121 <= (double)FLT_MAX && 127.0 * 0x1.020408p+121 > (double)FLT_MAX, "scale_max");
    const int kind = i8_kind(variant, k_bits);
    a.rule = round_rule(kind == RULE_WIDE ? I8_WIDE_SH0 : I8_SH0, 0, variant, k_bits);
    a.base = 0x43000000u | a.rule.add;
    a.base_hi = a.base >> a.rule.rot | a.base << (32 - a.rule.rot);          // rot is 16 to 32, taken modulo 32
    if (a.rule.rot == 0) a.base_hi = a.base;
    if (kind == RULE_WIDE && variant == SRF) a.rule.flip = 2u;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (src_fmt == FBSR_FP32) launch_kind<FBSR_FP32>(a, kind, stream);
    else if (src_fmt == FBSR_BF16) launch_kind<FBSR_BF16>(a, kind, stream);
    else launch_kind<FBSR_FP16>(a, kind, stream);
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}
