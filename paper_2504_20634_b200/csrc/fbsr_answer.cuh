// What the operators that answer with few-bit numbers share: eight elements of a row in and out, the draws of sixteen bits,
// and the round-up predicates with run-time variant and width.
//
// The variant and k are arguments here and not template parameters: an octet of elements takes one generator call whatever k
// is (sixteen bits an element), so no layout depends on k, and within a kind (see RULE_PLAIN) the predicates differ in constants
// alone.
#pragma once
#include "../../include/fbsr.h"
#include "fbsr_w4.cuh"

namespace fbsr {

// Third word of the generator's counter for each use of these draws (0 and 1 belong to weights and moments).
enum { DRAWS_KEYS = 2, DRAWS_VALUES = 3, DRAWS_I8 = 4 };

// Eight elements of a row as they lie in memory.
template <int TYPE> struct Octet8 { uint32_t w[TYPE == FBSR_FP32 ? 8 : 4]; };

// `whole`: all eight exist and the address is aligned to what eight of them take (32 or 16 bytes).
template <int TYPE>
__device__ __forceinline__ void load_octet(const void* base, int64_t at, int valid, bool whole, Octet8<TYPE>& o)
{
    if constexpr (TYPE == FBSR_FP32) {
        const float* p = static_cast<const float*>(base) + at;
        if (whole) {
            float x[8];
            unpack(load_f8_stream(p), x);
#pragma unroll
            for (int c = 0; c < 8; ++c) o.w[c] = __float_as_uint(x[c]);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) o.w[c] = c < valid ? __float_as_uint(p[c]) : 0u;
        }
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
        if (whole) {
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(o.w[0]), "=r"(o.w[1]), "=r"(o.w[2]), "=r"(o.w[3]) : "l"(p));
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                o.w[c] = (2 * c < valid ? (uint32_t)p[2 * c] : 0u) | (2 * c + 1 < valid ? (uint32_t)p[2 * c + 1] << 16 : 0u);
        }
    }
}

template <int TYPE>
__device__ __forceinline__ void widen(const Octet8<TYPE>& o, float (&x)[8])
{
    if constexpr (TYPE == FBSR_FP32) {
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = __uint_as_float(o.w[c]);
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if constexpr (TYPE == FBSR_BF16) {
                x[2 * c] = __uint_as_float(o.w[c] << 16);
                x[2 * c + 1] = __uint_as_float(o.w[c] & 0xFFFF0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&o.w[c]));
                x[2 * c] = f.x; x[2 * c + 1] = f.y;
            }
        }
    }
}

// Eight binary32 values, each rounded once to TYPE.
template <int TYPE>
__device__ __forceinline__ void store8(void* base, int64_t at, int valid, bool whole, const float (&v)[8])
{
    if constexpr (TYPE == FBSR_FP32) {
        float* p = static_cast<float*>(base) + at;
        if (whole) {
            store_f8(p, v);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < valid) p[c] = v[c];
        }
    } else {
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
        uint16_t* p = static_cast<uint16_t*>(base) + at;
        if (whole) {
            __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < valid) p[c] = (uint16_t)(w[c >> 1] >> (16 * (c & 1)));
        }
    }
}

// Four E4M3 codes to two pairs of binary16 values (every one of them is a binary16 number).
__device__ __forceinline__ void e4m3_word_to_half2(uint32_t word, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(word));
}

// Largest magnitude of an octet, as a number that grows with it: the pattern of a binary32 source, of a 16-bit one its two halves
// apart (`amax_pattern` makes the binary32 pattern of it).  A NaN is larger than all.
template <int TYPE>
__device__ __forceinline__ uint32_t amax8(const Octet8<TYPE>& o)
{
    if constexpr (TYPE == FBSR_FP32) {
        float m = 0.0f;
#pragma unroll
        for (int c = 0; c < 8; c += 2)
            asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(__uint_as_float(o.w[c])), "f"(__uint_as_float(o.w[c + 1])));
        return __float_as_uint(m);
    } else {
        return __vmaxu2(__vmaxu2(o.w[0] & 0x7FFF7FFFu, o.w[1] & 0x7FFF7FFFu), __vmaxu2(o.w[2] & 0x7FFF7FFFu, o.w[3] & 0x7FFF7FFFu));
    }
}

template <int TYPE>
__device__ __forceinline__ uint32_t join_amax(uint32_t a, uint32_t b) { return TYPE == FBSR_FP32 ? max(a, b) : __vmaxu2(a, b); }

template <int TYPE>
__device__ __forceinline__ uint32_t amax_pattern(uint32_t m)
{
    if constexpr (TYPE == FBSR_FP32) return m;
    m = max(m & 0xFFFFu, m >> 16);
    if constexpr (TYPE == FBSR_BF16) return m << 16;
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));       // a NaN stays one
}

// The same over the finite values alone, as a binary32 pattern.
__device__ __forceinline__ uint32_t finite_amax8_pattern(const float (&x)[8])
{
    uint32_t m = 0u;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint32_t b = __float_as_uint(x[c]) & 0x7FFFFFFFu;
        m = max(m, b < 0x7F800000u ? b : 0u);
    }
    return m;
}

// Quotients by a number known to the host: n / d = (n * mul) >> (31 + shift) for n < 2^31 and d > 1 (Granlund and Montgomery, "Division
// by invariant integers using multiplication"); d = 1 is handled apart.
struct Divider { uint32_t mul, shift, d; };

inline Divider divider(uint32_t d)
{
    uint32_t shift = 0;
    while (shift < 31 && (1u << shift) < d) ++shift;          // 2^(shift - 1) < d <= 2^shift
    // the smallest multiplier of 31 + shift bits that is not below the quotient; it has 32 bits at most
    const uint64_t mul = d == 1 ? 0 : ((1ull << (31 + shift)) + d - 1) / d;
    return Divider{(uint32_t)mul, shift, d};
}

__device__ __forceinline__ uint32_t divide(uint32_t n, const Divider& d)
{
    return d.d == 1 ? n : __umulhi(n, d.mul) >> (d.shift - 1);
}

// FBSR_OK, or what is wrong with a cache's description.
int check_kv_cache(const fbsr_kv_cache* cache);

// How a variant rounds.  PLAIN (SRFF, SRF, ties away): floor(sigma~ + draw 2^-k + c), nothing is asked about what is cut off.
// NEAREST (SRC's pre-round, ties to even, ties to odd): the parity of what is kept and a sticky bit for what is cut off.
// EVEN (ties to even): what the hardware's conversions do.
enum { RULE_PLAIN = 0, RULE_NEAREST = 1, RULE_WIDE = 2, RULE_EVEN = 3 };

// A predicate as constants, filled in by the host.  The value comes as an integer of SH0 fraction bits, moved L bits to the left; a
// draw's lowest bit goes to bit P = pos + L, pos = SH0 - k (SH0 where there is no draw).  Element c's draw is halfword c of its
// octet's generator call, low half of word 0 first.
struct RoundRule {
    uint32_t mask_lo, mask_hi;                   // the k bits in the low and the high halfword
    uint32_t half_hi;                            // half a step, below the high halfword's draw
    uint32_t mul, rot;                           // bit 0 to bit P; bit 16 to bit P (a rotation)
    uint32_t add;                                // half a step, or one unit less, at its place
    uint32_t pos, flip;                          // NEAREST: the parity bit before the shift by L, inverted or not
};

inline int rule_kind(int variant)
{
    return variant == RTNE ? RULE_EVEN : variant == SRC || variant == RTO ? RULE_NEAREST : RULE_PLAIN;
}

inline RoundRule round_rule(int sh0, int l, int variant, int k)
{
    const bool drawn = variant < RTNE;
    RoundRule r{};
    r.pos = (uint32_t)(drawn ? sh0 - k : sh0);
    const uint32_t p = r.pos + l, mask = drawn ? (1u << k) - 1u : 0u;
    r.mask_lo = mask; r.mask_hi = mask << 16;
    r.mul = 1u << p; r.rot = (p + 16) & 31;
    if (variant == SRF || variant == RTA) { r.add = p > 0 ? 1u << (p - 1) : 0u; r.half_hi = 0x8000u; }
    if (rule_kind(variant) == RULE_NEAREST) { r.add = ((1u << (r.pos - 1)) - 1u) << l; r.flip = variant == RTO; }
    return r;
}

// Element c's draw at its place; with HALF also the half step of SRF and ties away.
template <bool HALF>
__device__ __forceinline__ uint32_t placed_draw(const uint4& w, int c, const RoundRule& r)
{
    const uint32_t word = c < 2 ? w.x : c < 4 ? w.y : c < 6 ? w.z : w.w;
    if (c & 1) {
        const uint32_t d = HALF ? (word & r.mask_hi) | r.half_hi : word & r.mask_hi;
        return __funnelshift_l(d, d, r.rot);
    }
    return HALF ? (word & r.mask_lo) * r.mul + r.add : (word & r.mask_lo) * r.mul;
}

// The magnitude code of y in FMT, in the top bits below the sign (from bit 30 down); what exceeds the largest value saturates,
// infinities too.  The rescaling multiply is that of round_row_fast, pos at least 4.
template <int FMT> constexpr int RULE_L = 31 - (Format<FMT>::K - 1) - (24 - Format<FMT>::P);

template <int FMT, int KIND>
__device__ __forceinline__ uint32_t round_by_rule(float y, const uint4& draws, int c, const RoundRule& r)
{
    using F = Format<FMT>;
    constexpr int SH0 = 24 - F::P, L = RULE_L<FMT>;
    const float rescale = __uint_as_float((uint32_t)(128 - F::EMINB) << 23);       // 2^(1 - EMINB)
    uint32_t u = __float_as_uint(__fmul_rz(fabsf(y), rescale));
    if constexpr (KIND == RULE_PLAIN) {
        u = min(u, F::MAXCODE << SH0);
        return u * (1u << L) + placed_draw<true>(draws, c, r);
    } else {
        u |= (u ^ __float_as_uint(__fmul_ru(fabsf(y), rescale))) & 1u;             // sticky
        u = min(u, F::MAXCODE << SH0);
        u += ((u >> r.pos) & 1u) ^ r.flip;
        return u * (1u << L) + placed_draw<false>(draws, c, r) + r.add;
    }
}

// Bytes `byte` of four words as one word.
template <int BYTE>
__device__ __forceinline__ uint32_t gather_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __byte_perm(__byte_perm(a, b, BYTE | (BYTE + 4) << 4), __byte_perm(c, d, BYTE | (BYTE + 4) << 4), 0x5410);
}

}  // namespace fbsr
