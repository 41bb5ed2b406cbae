// What the 4-bit operators share: the format E2M1, the order in which the codes of a row lie in memory, and the two
// kinds of group scale.
//
// E2M1 = (K, P, B; M) = (4, 2, 1; 6): 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; no infinity, no NaN.
//
// Order of a row: padded with zeros to whole blocks of 128 elements, 64 bytes each.  A 32-bit word holds 8 consecutive
// elements, element i in bits [4 i, 4 i + 4).  Word t (0..3) of the block's quarter j (0..3; 32 elements) lies at place
// 4 t + j: a matrix instruction sums over four lanes at a time, each with its own k, so the four lanes of a row must
// hold the SAME 32 elements' worth of k at every step or the sum would run across groups with different scales; with
// this order lane t finds its word of each of the four quarters in one aligned 16-byte load.
#pragma once
#include "fbsr_kernels.cuh"

namespace fbsr {

constexpr int E2M1 = 5;                          // names Format<E2M1>; not a value of fbsr_fmt
template <> struct Format<E2M1> {
    static constexpr bool SINGLE_ZERO = false, HAS_INF = false;
    static constexpr int K = 4, P = 2, EMINB = 127;
    static constexpr uint32_t MAXBITS = 0x40C00000u;
    static constexpr uint32_t MAXCODE = 7u, INFCODE = 7u, NANCODE = 7u;          // NaN is carried by the group's scale
};

constexpr int W4_BLOCK = 128;                    // elements of a block of codes
constexpr int W4_BLOCK_BYTES = 64;

// Eight codes (a word of the stored order) to four pairs of binary16 values.
__device__ __forceinline__ void e2m1_word_to_half2(uint32_t word, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(word));
}

// 2^(byte - 127) of a power-of-two scale; 255 is the NaN scale.
__device__ __forceinline__ float e8m0_value(uint32_t byte)
{
    const uint32_t p = byte << 23;
    return __uint_as_float(byte == 0u ? 0x00400000u : byte == 255u ? 0x7FC00000u : p);
}

// The same for the two low bytes, as a pair of bfloat16 (which holds every one of these values).
__device__ __forceinline__ uint32_t e8m0_pair_to_bf16x2(uint32_t bytes)
{
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.bf16x2.ue8m0x2 %0, lo;\n\t}" : "=r"(r) : "r"(bytes));
    return r;
}

}  // namespace fbsr
