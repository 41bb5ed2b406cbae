// fbsr_adamw_multi: one AdamW step over many tensors, with binary32 or 8-bit moments and the stochastically
// rounded low-precision copy of the weights.  The arithmetic is stated in include/fbsr.h.
//
// The tensor table travels as a kernel argument (up to 400 tensors a launch): nothing is uploaded, nothing has to
// outlive the call, and gradients may lie elsewhere at every step.  A warp owns up to 1024 consecutive elements of one
// tensor and finds the tensor by bisection over the table's running tile counts, so that a tensor of one element
// costs one warp and a tensor of 2^25 elements spreads over the whole GPU.
#include <cmath>
#include <type_traits>

#include "../../include/fbsr.h"
#include "fbsr_internal.h"
#include "fbsr_kernels.cuh"

namespace fbsr {

// What rounding a row needs to know of variant and draw width, formed on the host (see round_row).
struct RowConstants {
    int at;                                      // bit where the draw's field is added
    uint32_t field;                              // the field's bits there
    uint32_t add, cap;                           // what is added besides, before the shift by L; the code of M with it
    uint32_t use_lsb, flip;                      // PREROUND, NEAREST: 1 << L or 0 for ties away; 1 << L for ties to odd
    int fits;                                    // whether round_row holds for this draw width
};

// Everything a launch needs besides the tensors; shared by the units that this file is compiled into.
struct AdamwHyper {
    float beta1, beta2, eps, neg_c1, c2, a1, a2, decay;
    const float* grad_scale;
    uint32_t k0, k1;
    int variant, k, ieee;
    // the weights' draws: per word, elements of a call, log2 of that or 0, (1 << k) - 1, 65536 / per_word + 1
    int per_word, per_call, per_call_log2;
    uint32_t mask, recip;
    RowConstants weights, state;
};

namespace {

constexpr int TILE = 1024;                       // elements of a warp: 4 rows of 256 (one where there are few, see launch_chunk)
constexpr int STATE_BLOCK = 256;                 // elements that share a scale of the 8-bit state: one row
static_assert(STATE_BLOCK == ROW_ELEMS, "a row is a block");
constexpr int DRAW_WORDS = 4 * (TILE / 8 + 1);   // words of the generator calls that cover a tile, at most

template <int CAP> struct AdamwTable {
    fbsr_adamw_tensor t[CAP];
    uint32_t first_tile[CAP + 1];
    uint32_t count, tile_rows;                   // rows of a warp's tile: 4 or 1
};

enum { GRAD_FP32, GRAD_BF16, GRAD_FP16 };

// The variants in three classes; within a class they differ by constants.
enum { ADD = 0 /* SRFF, SRF */, PREROUND = 1 /* SRC */, NEAREST = 2 /* the deterministic modes */ };

// ---------------------------------------------------------------------------- rounding with a run-time draw width
// The row rounder of the bandwidth kernel (round_row_fast) with k as run-time data: the value is rescaled so that the
// target's exponent range starts where binary32's does, the draw is added where the excess bits end, the code comes out in
// the top K bits.  It holds while the draw and the half step fit under the 24 - P excess bits of the rescaled pattern: k <= 22 - P,
// 14 for bfloat16 and 11 for binary16.  Wider draws round element by element, as the IEEE overflow option does: 62 M parameters,
// binary32 state, 277 us in the row form, 279 with bfloat16 at k = 16, 283 with IEEE overflow, 292 with binary16 at k = 13; 8-bit
// state 219, 276 with IEEE overflow.
template <int FMT> struct Row {
    using F = Format<FMT>;
    static constexpr int SH0 = 24 - F::P, L = FMT == BF16 ? 0 : 31 - (F::K - 1) - SH0;
    static RowConstants constants(int cls, int variant, int k)
    {
        RowConstants rc{};
        rc.fits = cls == NEAREST || k <= SH0 - 2;
        if (!rc.fits) k = 1;
        rc.at = (cls == NEAREST ? SH0 : SH0 - k) + L;
        rc.field = ((1u << k) - 1u) << (cls == NEAREST ? 0 : rc.at);
        const uint32_t half = 1u << (rc.at - 1);
        rc.add = (cls == ADD ? (variant == SRF ? half : 0u) : variant == RTA ? half : half - (1u << L)) >> L;
        rc.cap = (F::MAXCODE << SH0) + rc.add;
        rc.use_lsb = variant == RTA ? 0u : 1u << L;
        rc.flip = variant == RTO ? 1u << L : 0u;
        return rc;
    }
};

// Codes of y in the top K bits of t (bfloat16 with its sign); draw[c]: the field moved to bit `at`.  Holds for finite values
// (and infinities, where the format has none); bfloat16: up to the largest value.
template <int FMT, int CLS>
__device__ __forceinline__ void round_row(const float (&y)[8], const uint32_t (&draw)[8], const RowConstants& rc, uint32_t (&t)[8])
{
    using F = Format<FMT>;
    using R = Row<FMT>;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        uint32_t u;
        if constexpr (FMT == BF16) {
            u = __float_as_uint(y[c]);
        } else {
            const float rescale = __uint_as_float((uint32_t)(128 - F::EMINB) << 23);                // 2^(1 - EMINB)
            u = __float_as_uint(__fmul_rz(fabsf(y[c]), rescale));
            if constexpr (CLS != ADD) u |= (u ^ __float_as_uint(__fmul_ru(fabsf(y[c]), rescale))) & 1u;   // sticky
        }
        uint32_t lsb = 0u;                       // of the kept part, saturated like it
        if constexpr (CLS != ADD) {
            const uint32_t kept = FMT == BF16 ? u : min(u, F::MAXCODE << R::SH0);
            lsb = (((kept << R::L) >> (rc.at - R::L)) & rc.use_lsb) ^ rc.flip;
        }
        u += rc.add;
        if constexpr (FMT != BF16) u = min(u, rc.cap);
        t[c] = (u << R::L) + lsb + (CLS == NEAREST ? 0u : draw[c]);
    }
}

// Element by element: the same result, for rows that hold special values and for wide draws.
struct Values8 { float y[8]; uint32_t n[8]; };
struct Packed8 { uint32_t w[4]; };

template <int FMT>
__device__ __noinline__ Packed8 round_values_exact(Values8 x, int variant, int k, int ieee)
{
    uint32_t code[8];
    Packed8 out;
#pragma unroll
    for (int c = 0; c < 8; ++c) code[c] = round_core<FMT, false>(arith_bits(x.y[c]), x.n[c], variant, k, nullptr, ieee != 0);
    pack_codes8<FMT>(code, out.w);
    return out;
}

// By value, so that no array of the fast path needs an address (and with it a place in local memory).
template <int FMT>
__device__ __forceinline__ void round_row_exact(const float (&y)[8], const uint32_t (&n)[8], int variant, int k, int ieee, uint32_t* packed)
{
    Values8 x;
#pragma unroll
    for (int c = 0; c < 8; ++c) { x.y[c] = y[c]; x.n[c] = n[c]; }
    const Packed8 out = round_values_exact<FMT>(x, variant, k, ieee);
#pragma unroll
    for (int i = 0; i < WordsPerOctet<FMT>::value; ++i) packed[i] = out.w[i];
}

__device__ __forceinline__ uint32_t rotate(uint32_t w, int by) { return __funnelshift_l(w, w, by); }

// The k-bit draws of the weights' rounding for `count` elements of a warp: word w of generator call c lies at 4 c + w.
// Returns the place of the tile's first element in the first call.
__device__ __forceinline__ uint32_t fill_draws(uint32_t* words, uint64_t g0, int count, const AdamwHyper& h, int lane)
{
    const uint64_t call0 = h.per_call_log2 ? g0 >> h.per_call_log2 : g0 / (uint32_t)h.per_call;
    const uint32_t base = (uint32_t)(g0 - call0 * (uint32_t)h.per_call);
    const int calls = (int)(base + count + h.per_call - 1) / h.per_call;
    for (int c = lane; c < calls; c += 32) reinterpret_cast<uint4*>(words)[c] = philox_block(call0 + c, h.k0, h.k1);
    __syncwarp();
    return base;
}

// The fields of the eight elements from p on (a multiple of 8), each moved to bit `at`; field: its bits there.
__device__ __forceinline__ void take_draws(const uint32_t* words, uint32_t base, uint32_t p, int at, uint32_t field, const AdamwHyper& h, uint32_t (&d)[8])
{
    if (h.per_call_log2) {                       // base is 0: a tensor starts at a multiple of 256 of the stream
        if (h.per_word >= 8) {
            const uint32_t first = p & (h.per_word - 1), w = words[(p - first) >> (h.per_call_log2 - 2)] >> (first * h.k);
#pragma unroll
            for (int c = 0; c < 8; ++c) d[c] = rotate(w, at - c * h.k) & field;
        } else if (h.per_word == 4) {
            const uint2 w = *reinterpret_cast<const uint2*>(words + p / 4);
#pragma unroll
            for (int c = 0; c < 8; ++c) d[c] = rotate(c < 4 ? w.x : w.y, at - (c & 3) * h.k) & field;
        } else {
            const uint4 w = *reinterpret_cast<const uint4*>(words + p / 2);
#pragma unroll
            for (int c = 0; c < 8; ++c) d[c] = rotate(c < 2 ? w.x : c < 4 ? w.y : c < 6 ? w.z : w.w, at - (c & 1) * h.k) & field;
        }
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint32_t pos = base + p + c, q = (pos * h.recip) >> 16;      // pos / per_word (pos < 2^11)
            d[c] = rotate(words[q], at - (int)((pos - q * (uint32_t)h.per_word) * (uint32_t)h.k)) & field;
        }
    }
}

// ---------------------------------------------------------------------------- roots and quotients without branches
// Correctly rounded results from the hardware's approximations by iterations in fused multiply-adds (Markstein, "Computation
// of elementary functions on the IBM RISC System/6000 processor", 1990): the compiler's own forms test every operand for
// special cases, sixteen branches a row, which kept the 8-bit step from overlapping its elements.

// Square root of 2^-96 <= v <= 2^126 (where the residual v - g g is exact); NaN for NaN.  Equal to the rounded root for every number of
// [1, 4), [2^-96, 2^-94) and [2^124, 2^126), which the tests go through.
__device__ __forceinline__ float root_in_range(float v)
{
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(v));
    const float g = __fmul_rn(v, y);
    return __fmaf_rn(__fmaf_rn(-g, g, v), __fmul_rn(0.5f, y), g);
}

// m / d for 2^-126 <= |d|; |d| beyond 2^126 counts as infinite (an overflowing second moment: zero for finite m).  Quotients whose
// residual m - q d is below binary32's range (|m| below 2^-100, subnormal quotients) may be one unit off.  NaN where d is zero or
// subnormal, m infinite or the quotient beyond binary32: the step does those again with the general division.
__device__ __forceinline__ float quotient(float m, float d)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(d));          // zero for an infinite d, and zero it stays
    asm("min.NaN.f32 %0, %0, 0f7E800000;" : "+f"(d));
    y = __fmaf_rn(y, __fmaf_rn(-d, y, 1.0f), y);
    const float q = __fmul_rn(m, y);
    return __fmaf_rn(__fmaf_rn(-d, q, m), y, q);
}

__device__ __forceinline__ void roots8(const float (&v)[8], float (&r)[8])
{
    float low = v[0], high = v[0];
#pragma unroll
    for (int c = 0; c < 8; ++c) r[c] = root_in_range(v[c]);
#pragma unroll
    for (int c = 0; c < 8; c += 2) {
        asm("min.f32 %0, %0, %1, %2;" : "+f"(low) : "f"(v[c]), "f"(v[c + 1]));
        asm("max.f32 %0, %0, %1, %2;" : "+f"(high) : "f"(v[c]), "f"(v[c + 1]));
    }
    if (!(low >= 0x1p-96f && high <= 0x1p126f)) {
#pragma unroll
        for (int c = 0; c < 8; ++c) r[c] = __fsqrt_rn(v[c]);
    }
}

// ---------------------------------------------------------------------------- 8-bit state
// Largest finite magnitude of the warp's 256 values.
__device__ __forceinline__ float row_amax(const float (&x)[8])
{
    float m = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; c += 2) asm("max.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(x[c]), "f"(x[c + 1]));      // ignores NaN
    const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m));
    if (all < 0x7F800000u) return __uint_as_float(all);
    m = 0.0f;                                    // an infinity in the row (rare, the same for all lanes)
#pragma unroll
    for (int c = 0; c < 8; ++c) m = fmaxf(m, fabsf(x[c]) < __uint_as_float(0x7F800000u) ? fabsf(x[c]) : 0.0f);
    return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m)));
}

// Codes of a row of state, packed: scale from the row's maximum, then the few-bit rounding with the field at bit `shift` of each
// halfword of the draws; redo: a value may be a NaN.  POSITIVE: a value above zero never takes the zero code (a zero second
// moment under a non-zero first one would blow the next step up).
template <int CLS, bool POSITIVE>
__device__ __forceinline__ float round_state(const float (&x)[8], const uint4& draws, int shift, const AdamwHyper& h, bool redo, uint32_t (&packed)[2])
{
    const RowConstants& rc = h.state;
    const float scale = fmaxf(__fmul_rn(row_amax(x), 1.0f / 448.0f), 0x1p-126f), inv = __frcp_rn(scale);
    const uint32_t w[4] = {draws.x, draws.y, draws.z, draws.w};
    float y[8];
    uint32_t d[8] = {};
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        y[c] = __fmul_rn(x[c], inv);
        if constexpr (CLS != NEAREST) d[c] = rotate(w[c >> 1], rc.at - (16 * (c & 1) + shift)) & rc.field;
    }
    if (!redo) {
        uint32_t t[8];
        round_row<E4M3, CLS>(y, d, rc, t);
        if constexpr (POSITIVE) {                // a root above zero is above 2^-75, its pattern above that of code 1
#pragma unroll
            for (int c = 0; c < 8; ++c) t[c] = max(t[c], min(__float_as_uint(x[c]), 1u << (Row<E4M3>::SH0 + Row<E4M3>::L)));
        }
        if constexpr (POSITIVE) {                // no signs to take along
#pragma unroll
            for (int j = 0; j < 2; ++j)
                packed[j] = __byte_perm(__byte_perm(t[4 * j], t[4 * j + 1], 0x7373), __byte_perm(t[4 * j + 2], t[4 * j + 3], 0x7373), 0x5410);
        } else {
            pack_row_fast<E4M3>(t, y, packed);
        }
    } else {
        uint32_t n[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) n[c] = CLS == NEAREST ? 0u : d[c] >> rc.at;
        round_row_exact<E4M3>(y, n, h.variant, h.k, 0, packed);
        if constexpr (POSITIVE) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (x[c] > 0.0f && ((packed[c >> 2] >> (8 * (c & 3))) & 0xFFu) == 0u) packed[c >> 2] |= 1u << (8 * (c & 3));
        }
    }
    return scale;
}

// ---------------------------------------------------------------------------- the kernel
template <int BYTES>
__device__ __forceinline__ void copy_async(unsigned char* smem_dst, const void* gmem_src)
{
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(smem_dst);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(gmem_src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(gmem_src) : "memory");
}

// A row's inputs on their way through shared memory, copied in runs of 512 bytes a warp.  Arrays of four bytes an element
// have every second run of eight 16-byte pieces exchanged pairwise, so that the lanes' 32-byte parts meet all banks.
template <int BITS, int G> struct Stage {
    static constexpr int W = 0, GRAD = 1024, M = GRAD + (G == GRAD_FP32 ? 1024 : 512), V = M + (BITS == 32 ? 1024 : 256);
    static constexpr int SCALES = V + (BITS == 32 ? 1024 : 256);                 // 8-bit state: m's and v's
    static constexpr int BYTES = SCALES + (BITS == 32 ? 0 : 16);
    __device__ __forceinline__ static int wide(int piece) { return (piece ^ ((piece >> 3) & 1)) * 16; }      // place of a 16-byte piece
};

template <int BYTES_A_ROW>
__device__ __forceinline__ void copy_row(unsigned char* to, const void* from, int lane)
{
    using St = Stage<32, GRAD_FP32>;
#pragma unroll
    for (int i = 0; i < BYTES_A_ROW / 512; ++i) {
        const int piece = i * 32 + lane;
        copy_async<16>(to + (BYTES_A_ROW == 1024 ? St::wide(piece) : piece * 16), static_cast<const unsigned char*>(from) + piece * 16);
    }
}

// A warp's place in a tensor: its pointers stand at the first element of the row that `row` counts from.
template <int FMT, int BITS, int G> struct Place {
    using Grad = std::conditional_t<G == GRAD_FP32, uint32_t, uint16_t>;
    using S = std::conditional_t<BITS == 32, uint32_t, uint8_t>;
    using C = std::conditional_t<Format<FMT>::K == 16, uint16_t, uint8_t>;
    float* w; const Grad* g; S* m; S* v; C* lp;
    float* m_scale; float* v_scale;
    int left;                                    // elements of the tensor from here on, at most 2^30
    bool copies, vec, has_lp;                    // pointers allow: 16-byte copies; vector stores of eight elements

    __device__ __forceinline__ void set(const fbsr_adamw_tensor& t, uint64_t e0)
    {
        w = t.w + e0; g = static_cast<const Grad*>(t.g) + e0; m = static_cast<S*>(t.m) + e0; v = static_cast<S*>(t.v) + e0;
        lp = static_cast<C*>(t.w_lp) + e0;
        if constexpr (BITS == 8) { m_scale = t.m_scale + e0 / STATE_BLOCK; v_scale = t.v_scale + e0 / STATE_BLOCK; }
        left = t.n - e0 > (1u << 30) ? 1 << 30 : (int)(t.n - e0);
        has_lp = t.w_lp != nullptr;
        const uintptr_t state = reinterpret_cast<uintptr_t>(m) | reinterpret_cast<uintptr_t>(v);
        copies = (reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(g) | state) % 16 == 0;
        vec = (reinterpret_cast<uintptr_t>(w) % 32 | state % (8 * sizeof(S)) | (has_lp ? reinterpret_cast<uintptr_t>(lp) % (8 * sizeof(C)) : 0)) == 0;
    }
    __device__ __forceinline__ void advance()
    {
        w += ROW_ELEMS; g += ROW_ELEMS; m += ROW_ELEMS; v += ROW_ELEMS; lp += ROW_ELEMS;
        if constexpr (BITS == 8) { ++m_scale; ++v_scale; }
        left -= ROW_ELEMS;
    }
    // elements of the eight of this lane that the tensor has
    __device__ __forceinline__ int valid(int row, uint32_t lane) const { return min(max(left - row * ROW_ELEMS - (int)lane * 8, 0), 8); }

    // Sends a row's inputs to a stage.
    __device__ __forceinline__ void fetch(int row, unsigned char* stage, uint32_t lane) const
    {
        using St = Stage<BITS, G>;
        const int at = row * ROW_ELEMS;
        if (copies && left - at >= ROW_ELEMS) {
            copy_row<1024>(stage + St::W, w + at, lane);
            copy_row<G == GRAD_FP32 ? 1024 : 512>(stage + St::GRAD, g + at, lane);
            if constexpr (BITS == 32) {
                copy_row<1024>(stage + St::M, m + at, lane);
                copy_row<1024>(stage + St::V, v + at, lane);
            } else {
                copy_async<16>(stage + St::M + lane * 16, (lane < 16 ? m : v) + at + (lane & 15) * 16);
            }
        } else {                                 // unaligned tensors and the end of a tensor, element by element; zeros beyond it
            const int ok = valid(row, lane);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const bool there = c < ok;
                const int four = St::wide(2 * lane + (c >> 2)) + (c & 3) * 4, e = lane * 8 + c;
                *reinterpret_cast<float*>(stage + St::W + four) = there ? w[at + e] : 0.0f;
                *reinterpret_cast<Grad*>(stage + St::GRAD + (G == GRAD_FP32 ? four : e * 2)) = there ? g[at + e] : (Grad)0;
                *reinterpret_cast<S*>(stage + St::M + (BITS == 32 ? four : e)) = there ? m[at + e] : (S)0;
                *reinterpret_cast<S*>(stage + St::V + (BITS == 32 ? four : e)) = there ? v[at + e] : (S)0;
            }
        }
        if constexpr (BITS == 8) {
            if (lane < 2) copy_async<4>(stage + St::SCALES + lane * 4, (lane ? v_scale : m_scale) + row);
        }
    }
};

__device__ __forceinline__ void take_floats(const unsigned char* array, int lane, float (&x)[8])
{
    using St = Stage<32, GRAD_FP32>;
    const float4 p = *reinterpret_cast<const float4*>(array + St::wide(2 * lane)), q = *reinterpret_cast<const float4*>(array + St::wide(2 * lane + 1));
    x[0] = p.x; x[1] = p.y; x[2] = p.z; x[3] = p.w; x[4] = q.x; x[5] = q.y; x[6] = q.z; x[7] = q.w;
}

template <class T>
__device__ __forceinline__ void store_first(T* p, int count, const uint32_t* packed)
{
    constexpr int PER = 4 / sizeof(T);
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (c < count) p[c] = (T)(packed[c / PER] >> (8 * (int)sizeof(T) * (c % PER)));
}

__device__ __forceinline__ void store_floats(float* p, bool whole, int count, const float (&x)[8])
{
    if (whole) {
        store_f8(p, x);
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c < count) p[c] = x[c];
    }
}

// Rows of a warp's ring, and resident CTAs the compiler must allow.  62 M parameters, k = 4, bfloat16 copies: binary32 state and
// gradients 274 us (6.77 TB/s: memory bounds it) with two rows and two or three CTAs; 8-bit state and bfloat16 gradients 212 us
// (4.69 TB/s: issue slots 85 % busy, 103 instructions an element) with two rows and three CTAs.  Before the last
// instructions were saved it was 222, with two CTAs 250 and with three rows 225.
constexpr int RING = 2, CTAS_32 = 2, CTAS_8 = 3;

template <int FMT, int BITS, int G, int CLS, int CAP>
__global__ void __launch_bounds__(CTA_THREADS, BITS == 32 ? CTAS_32 : CTAS_8)
adamw_multi_kernel(const __grid_constant__ AdamwTable<CAP> tab, const __grid_constant__ AdamwHyper h)
{
    __shared__ __align__(16) uint32_t wordbuf[WARPS_PER_CTA][CLS == NEAREST ? 4 : DRAW_WORDS];
    const uint32_t lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);             // the same for the warp, and known to be
    const uint32_t tile = blockIdx.x * (blockDim.x / 32) + warp;
    if (tile >= tab.first_tile[tab.count]) return;

    uint32_t lo = 0, hi = tab.count;             // first_tile[lo] <= tile < first_tile[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (tab.first_tile[mid] <= tile) lo = mid; else hi = mid;
    }
    const fbsr_adamw_tensor& t = tab.t[lo];
    const uint64_t e0 = (uint64_t)(tile - tab.first_tile[lo]) * (tab.tile_rows * ROW_ELEMS);
    const uint64_t g0 = t.offset + e0;           // of the stream of draws
    const int rows = t.n - e0 >= tab.tile_rows * ROW_ELEMS ? (int)tab.tile_rows : (int)(t.n - e0 + ROW_ELEMS - 1) / ROW_ELEMS;
    Place<FMT, BITS, G> at;
    at.set(t, e0);

    using St = Stage<BITS, G>;
    extern __shared__ __align__(16) unsigned char stages[];
    unsigned char* ring = stages + warp * (RING * St::BYTES);
#pragma unroll
    for (int j = 0; j < RING - 1; ++j) {
        if (j < rows) at.fetch(j, ring + j * St::BYTES, lane);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }

    // the generator runs in the shadow of the first loads
    uint32_t draw_base = 0;
    if (CLS != NEAREST && at.has_lp) draw_base = fill_draws(wordbuf[warp], g0, rows * ROW_ELEMS, h, lane);
    const float gs = h.grad_scale ? __ldg(h.grad_scale) : 1.0f;

    for (int row = 0; row < rows; ++row) {
        // the row that will be needed RING - 1 rows from now takes the place of the one before this, which all lanes have read
        __syncwarp();
        if (row + RING - 1 < rows) at.fetch(RING - 1, ring + (row + RING - 1) % RING * St::BYTES, lane);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
        __syncwarp();
        const unsigned char* in = ring + row % RING * St::BYTES;
        float w[8], m[8], v[8], r[8], g[8];
        take_floats(in + St::W, lane, w);
        if constexpr (BITS == 32) {
            take_floats(in + St::M, lane, m);
            take_floats(in + St::V, lane, v);
        } else {
            const uint2 cm = *reinterpret_cast<const uint2*>(in + St::M + lane * 8), cv = *reinterpret_cast<const uint2*>(in + St::V + lane * 8);
            const float2 scales = *reinterpret_cast<const float2*>(in + St::SCALES);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float x[4];
                decode4<E4M3>(q ? cm.y : cm.x, x);
#pragma unroll
                for (int c = 0; c < 4; ++c) m[4 * q + c] = __fmul_rn(x[c], scales.x);
                decode4<E4M3>(q ? cv.y : cv.x, x);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float root = __fmul_rn(x[c], scales.y);
                    v[4 * q + c] = __fmul_rn(root, root);
                }
            }
        }
        if constexpr (G == GRAD_FP32) {
            take_floats(in + St::GRAD, lane, g);
        } else {
            const uint4 q = *reinterpret_cast<const uint4*>(in + St::GRAD + lane * 16);
            const uint32_t x[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if constexpr (G == GRAD_BF16) {
                    g[2 * c] = __uint_as_float(x[c] << 16);
                    g[2 * c + 1] = __uint_as_float(x[c] & 0xFFFF0000u);
                } else {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[c]));
                    g[2 * c] = f.x; g[2 * c + 1] = f.y;
                }
            }
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            g[c] = __fmul_rn(g[c], gs);
            if constexpr (BITS == 32) {
                m[c] = __fmaf_rn(h.beta1, m[c], __fmul_rn(h.a1, g[c]));
                v[c] = __fmaf_rn(h.beta2, v[c], __fmul_rn(__fmul_rn(h.a2, g[c]), g[c]));
            } else {
                m[c] = __fadd_rn(__fmul_rn(h.beta1, m[c]), __fmul_rn(h.a1, g[c]));
                v[c] = __fadd_rn(__fmul_rn(h.beta2, v[c]), __fmul_rn(__fmul_rn(h.a2, g[c]), g[c]));
            }
        }
        if constexpr (BITS == 8) roots8(v, r);
        // a NaN or an infinity anywhere among the eight weights (a NaN in a moment makes one of its weight)
        float poison = 0.0f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            if constexpr (BITS == 32) r[c] = __fsqrt_rn(v[c]);
            const float d = __fadd_rn(__fmul_rn(r[c], h.c2), h.eps);
            const float q = BITS == 32 ? __fdiv_rn(m[c], d) : quotient(m[c], d);
            w[c] = __fmaf_rn(h.neg_c1, q, __fmul_rn(w[c], h.decay));
            poison = __fmaf_rn(w[c], 0.0f, poison);
        }
        const bool special = poison != poison;
        if (BITS == 8 && special) {              // rare: out of the fast quotient's range, or special by the formula
            take_floats(in + St::W, lane, w);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float d = __fadd_rn(__fmul_rn(r[c], h.c2), h.eps);
                w[c] = __fmaf_rn(h.neg_c1, __fdiv_rn(m[c], d), __fmul_rn(w[c], h.decay));
            }
        }
        const int valid = at.valid(0, lane);
        const bool whole = at.vec && valid == 8;
        store_floats(at.w + lane * 8, whole, valid, w);
        if constexpr (BITS == 32) {
            store_floats(reinterpret_cast<float*>(at.m) + lane * 8, whole, valid, m);
            store_floats(reinterpret_cast<float*>(at.v) + lane * 8, whole, valid, v);
        } else {
            // what lies beyond the tensor's end must not be noticed by a maximum (0 * grad_scale may be a NaN)
            if (valid < 8) {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c >= valid) { m[c] = 0.0f; r[c] = 0.0f; }
            }
            uint4 bits = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (CLS != NEAREST) {
                const uint64_t i = (g0 >> 3) + row * (ROW_ELEMS / 8) + lane;
                bits = philox4x32_10((uint32_t)i, (uint32_t)(i >> 32), 1u, 0u, h.k0, h.k1);
            }
            uint32_t cm[2], cr[2];
            const float sm = round_state<CLS, false>(m, bits, 0, h, special, cm);
            const float sr = round_state<CLS, true>(r, bits, 8, h, special, cr);
            if (whole) {
                *reinterpret_cast<uint2*>(at.m + lane * 8) = make_uint2(cm[0], cm[1]);
                *reinterpret_cast<uint2*>(at.v + lane * 8) = make_uint2(cr[0], cr[1]);
            } else {
                store_first(at.m + lane * 8, valid, cm);
                store_first(at.v + lane * 8, valid, cr);
            }
            if (lane == 0) { *at.m_scale = sm; *at.v_scale = sr; }
        }
        if (at.has_lp) {
            constexpr int WPO = WordsPerOctet<FMT>::value;
            const uint32_t p = row * ROW_ELEMS + lane * 8;
            uint32_t packed[WPO], d[8] = {}, code[8];
            bool redo = special || !h.weights.fits || h.ieee;
            if constexpr (FMT == BF16) {         // beyond M too, which a draw could carry past the exponent
                float over = 0.0f;
#pragma unroll
                for (int c = 0; c < 8; c += 2) asm("max.abs.f32 %0, %0, %1, %2;" : "+f"(over) : "f"(w[c]), "f"(w[c + 1]));
                redo |= over > __uint_as_float(0x7F7F0000u);
            }
            if (!redo) {
                if constexpr (CLS != NEAREST) take_draws(wordbuf[warp], draw_base, p, h.weights.at, h.weights.field, h, d);
                round_row<FMT, CLS>(w, d, h.weights, code);
                pack_row_fast<FMT>(code, w, packed);
            } else {
                if constexpr (CLS != NEAREST) take_draws(wordbuf[warp], draw_base, p, 0, h.mask, h, d);
                round_row_exact<FMT>(w, d, h.variant, h.k, h.ieee, packed);
            }
            if (whole) store_words<WPO>(at.lp + lane * 8, packed);
            else store_first(at.lp + lane * 8, valid, packed);
        }
        at.advance();
    }
}

// Four rows to a warp share its generator calls and keep its copies ahead of it; where that leaves most of the GPU idle, a warp
// takes one row, and a CTA four warps.  8-bit state, bfloat16 gradients: 110,000 elements 8.4 us with four rows, 3.9 with one;
// 0.45 M 8.4 and 5.4; 0.93 M (six tiles a multiprocessor) 8.3 and 8.1; 1.8 M 11.3 and 12.6.  binary32 state: 0.45 M 8.4 and 5.6,
// 0.93 M 8.4 and 8.8, 1.8 M 10.4 and 12.4.
constexpr int FEW_TILES = 6 * 148, FEW_WARPS = 4;

template <int FMT, int BITS, int G, int CLS, int CAP>
int launch_chunk(const fbsr_adamw_tensor* t, size_t count, const AdamwHyper& h, cudaStream_t stream)
{
    AdamwTable<CAP> tab;
    uint64_t tiles = 0;
    for (size_t i = 0; i < count; ++i) tiles += (t[i].n + TILE - 1) / TILE;
    const bool few = tiles < FEW_TILES;
    tab.tile_rows = few ? 1 : TILE / ROW_ELEMS;
    const uint32_t tile = tab.tile_rows * ROW_ELEMS;
    tab.count = 0;
    tiles = 0;
    for (size_t i = 0; i < count; ++i) {
        if (t[i].n == 0) continue;
        tab.t[tab.count] = t[i];
        tab.first_tile[tab.count++] = (uint32_t)tiles;
        tiles += (t[i].n + tile - 1) / tile;
    }
    tab.first_tile[tab.count] = (uint32_t)tiles;
    if (tiles == 0) return FBSR_OK;
    const int warps = few ? FEW_WARPS : WARPS_PER_CTA;
    const unsigned grid = (unsigned)((tiles + warps - 1) / warps);
    constexpr int WARP_BYTES = RING * Stage<BITS, G>::BYTES;
    auto kernel = adamw_multi_kernel<FMT, BITS, G, CLS, CAP>;
    static std::atomic<uint64_t> allowed{0};
    if (int rc = allow_shared_memory((const void*)kernel, WARPS_PER_CTA * WARP_BYTES, allowed)) return rc;
    kernel<<<grid, warps * 32, warps * WARP_BYTES, stream>>>(tab, h);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}

constexpr int CAP_MANY = 400;                    // 72 + 4 bytes a tensor: under the 32,764 bytes of kernel arguments
constexpr int CAP_FEW = 48;                      // with the scalars under 4 KB of argument: a call from Python 7.3 us for 48 tensors, 10.7 for 49

template <int FMT, int BITS, int G, int CLS>
int launch_all(const fbsr_adamw_tensor* t, size_t count, const AdamwHyper& h, cudaStream_t stream)
{
    for (size_t at = 0; at < count; at += CAP_MANY) {
        const size_t len = count - at < (size_t)CAP_MANY ? count - at : (size_t)CAP_MANY;
        const int rc = len <= (size_t)CAP_FEW ? launch_chunk<FMT, BITS, G, CLS, CAP_FEW>(t + at, len, h, stream)
                                              : launch_chunk<FMT, BITS, G, CLS, CAP_MANY>(t + at, len, h, stream);
        if (rc != FBSR_OK) return rc;
    }
    return FBSR_OK;
}

}  // namespace

// The launch for one target format; this file is compiled once per format for it, and once without for the entry point.
#ifdef FBSR_FMT
template <int BITS, int G>
static int launch_class(int cls, const fbsr_adamw_tensor* t, size_t count, const AdamwHyper& h, cudaStream_t stream)
{
    return cls == ADD ? launch_all<FBSR_FMT, BITS, G, ADD>(t, count, h, stream)
         : cls == PREROUND ? launch_all<FBSR_FMT, BITS, G, PREROUND>(t, count, h, stream)
                           : launch_all<FBSR_FMT, BITS, G, NEAREST>(t, count, h, stream);
}
template <int G>
static int launch_state(int state_bits, int cls, const fbsr_adamw_tensor* t, size_t count, const AdamwHyper& h, cudaStream_t stream)
{
    return state_bits == 32 ? launch_class<32, G>(cls, t, count, h, stream) : launch_class<8, G>(cls, t, count, h, stream);
}
#define FBSR_NAME2(f) adamw_multi_##f
#define FBSR_NAME(f) FBSR_NAME2(f)
int FBSR_NAME(FBSR_FMT)(const fbsr_adamw_tensor* t, size_t count, int state_bits, int g_fmt, AdamwHyper h, cudaStream_t stream)
{
    const int cls = h.variant <= FBSR_SRF ? ADD : h.variant == FBSR_SRC ? PREROUND : NEAREST;
    h.weights = Row<FBSR_FMT>::constants(cls, h.variant, h.k);
    h.state = Row<E4M3>::constants(cls, h.variant, cls == NEAREST ? 1 : h.k);
    return g_fmt == FBSR_FP32 ? launch_state<GRAD_FP32>(state_bits, cls, t, count, h, stream)
         : g_fmt == FBSR_BF16 ? launch_state<GRAD_BF16>(state_bits, cls, t, count, h, stream)
                              : launch_state<GRAD_FP16>(state_bits, cls, t, count, h, stream);
}
}  // namespace fbsr
#else
int adamw_multi_0(const fbsr_adamw_tensor*, size_t, int, int, AdamwHyper, cudaStream_t);
int adamw_multi_1(const fbsr_adamw_tensor*, size_t, int, int, AdamwHyper, cudaStream_t);
int adamw_multi_2(const fbsr_adamw_tensor*, size_t, int, int, AdamwHyper, cudaStream_t);
int adamw_multi_3(const fbsr_adamw_tensor*, size_t, int, int, AdamwHyper, cudaStream_t);
int adamw_multi_4(const fbsr_adamw_tensor*, size_t, int, int, AdamwHyper, cudaStream_t);

namespace {

typedef int (*launch_fn)(const fbsr_adamw_tensor*, size_t, int, int, AdamwHyper, cudaStream_t);
const launch_fn kLaunch[5] = {adamw_multi_0, adamw_multi_1, adamw_multi_2, adamw_multi_3, adamw_multi_4};

inline bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

}  // namespace
}  // namespace fbsr

using namespace fbsr;

extern "C" int fbsr_adamw_multi(const fbsr_adamw_tensor* tensors, size_t count, int state_bits, int g_fmt, int fmt, int variant,
                                int k_bits, uint64_t seed, double lr, double beta1, double beta2, double eps,
                                double weight_decay, int step, const float* grad_scale, void* cuda_stream)
{
    const int ieee = (fmt & FBSR_OVF_IEEE) ? 1 : 0;
    fmt &= ~FBSR_OVF_IEEE;
    if (fmt < 0 || fmt > 4 || variant < 0 || variant > 5 || k_bits < 1 || k_bits > 16 || step < 1) return FBSR_ERR_INVALID_ARG;
    if (g_fmt != FBSR_FP32 && g_fmt != FBSR_BF16 && g_fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    if (state_bits != 32 && state_bits != 8) return FBSR_ERR_UNSUPPORTED;
    if (state_bits == 8 && variant < FBSR_RTNE && k_bits > 8) return FBSR_ERR_UNSUPPORTED;
    if (count > 0 && tensors == nullptr) return FBSR_ERR_INVALID_ARG;
    if (off(grad_scale, 4)) return FBSR_ERR_ALIGNMENT;
    const size_t g_bytes = g_fmt == FBSR_FP32 ? 4 : 2, state_bytes = state_bits == 32 ? 4 : 1, lp_bytes = fmt <= FBSR_FP16 ? 2 : 1;
    uint64_t tiles = 0;
    for (size_t i = 0; i < count; ++i) {
        const fbsr_adamw_tensor& t = tensors[i];
        if (t.offset % STATE_BLOCK != 0) return FBSR_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (!t.w || !t.g || !t.m || !t.v || (state_bits == 8 && (!t.m_scale || !t.v_scale))) return FBSR_ERR_INVALID_ARG;
        if (off(t.w, 4) || off(t.g, g_bytes) || off(t.m, state_bytes) || off(t.v, state_bytes) || off(t.w_lp, lp_bytes) ||
            (state_bits == 8 && (off(t.m_scale, 4) || off(t.v_scale, 4)))) return FBSR_ERR_ALIGNMENT;
        if (t.n > ((uint64_t)1 << 40)) return FBSR_ERR_TOO_LARGE;
        tiles += (t.n + TILE - 1) / TILE;
        if (tiles > 0xFFFFFFFFull - 2 * WARPS_PER_CTA) return FBSR_ERR_TOO_LARGE;
    }
    AdamwHyper h{};
    h.beta1 = (float)beta1; h.beta2 = (float)beta2; h.eps = (float)eps;
    // pow and not the products of fbsr_adam_scalars, which cost 53 us at step 100,000 (beta2 0.999; 138 with 0.9999): more than a step
    h.neg_c1 = -(float)(lr / (1.0 - std::pow(beta1, step)));
    h.c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, step)));
    h.a1 = (float)(1.0 - beta1); h.a2 = (float)(1.0 - beta2);
    h.decay = (float)(1.0 - lr * weight_decay);
    h.grad_scale = grad_scale;
    h.k0 = (uint32_t)seed; h.k1 = (uint32_t)(seed >> 32);
    h.variant = variant; h.k = k_bits; h.ieee = ieee;
    h.per_word = 32 / k_bits; h.per_call = 4 * h.per_word; h.per_call_log2 = 0;
    for (int i = 3; i <= 7; ++i)
        if (h.per_call == 1 << i) h.per_call_log2 = i;
    h.mask = (1u << k_bits) - 1u; h.recip = 65536u / (uint32_t)h.per_word + 1u;
    return kLaunch[fmt](tensors, count, state_bits, g_fmt, h, static_cast<cudaStream_t>(cuda_stream));
}
#endif
