// fbsr_round_kv: keys and values rounded to 8 or 4 bits as they are written to a paged cache; fbsr_read_kv: rows of the cache as
// numbers again.  The arithmetic and the layout are stated in include/fbsr.h.
//
// 2 (or 4) bytes an element on one side, 1 or 1/2 on the other, and no reuse: reading and rounding to nearest are bound by memory.
// Stochastic rounding is bound by instructions, 30 an element: a generator call for eight of
// them is two fifths of the time, the rest is the maximum, the draws put in place, signs and packing (76 % of the issue rate, the
// integer units busy 67 %).  8192 tokens of 8 heads of 128 from bfloat16 to 8 bits (50.7 MB): nearest 10.6 us (4.8 TB/s), SRF 20.0, SRC 22.9.  A thread owns the same
// eight elements of a token's key and value, so two loads are in flight before the first generator call (one call serves eight
// elements); neighbouring threads own neighbouring octets of a head, then the next head, so a warp reads whole rows of the source
// and writes rows of 32 to 128 bytes, one per head, as the cache's layout (token after token of a head) makes them.  A scale's
// maximum is taken over 4 (4 bits), 8 or 16 (8 bits) neighbouring lanes.
#include <cstring>

#include "fbsr_answer.cuh"
#include "fbsr_internal.h"

namespace fbsr {
namespace {

constexpr int THREADS = 256;

struct KvArgs {
    const void* k;                               // rounding: sources; reading: results
    const void* v;
    int64_t k_token, k_head, v_token, v_head;    // strides in elements
    uint8_t* k_codes;
    uint8_t* v_codes;
    uint16_t* k_scales;
    uint16_t* v_scales;
    const int64_t* slots;
    uint64_t capacity;                           // slots of the cache
    uint32_t octets;                             // of the call, each of keys and values
    Divider by_heads;
    uint64_t offset;
    uint32_t k0, k1;
    int heads, page_shift, whole;                // whole: rows may be moved eight elements at a time
    float scale_max;
    RoundRule rule;
};

// Lanes that share a scale.
template <int BITS, int DIM> constexpr int GROUP_LANES = BITS == 8 ? DIM / 8 : 4;

template <int TYPE, int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t m)
{
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) m = join_amax<TYPE>(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    return m;
}

// Nearest codes, ties to even, saturating: the hardware's conversion is the definition's.
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d)
{
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
        : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

__device__ __forceinline__ uint32_t to_e2m1x8(const float (&y)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return r;
}

// Rounds one octet and writes it: `row` is its row of the cache (a head of a token), negative where nothing is written.
template <int TYPE, int BITS, int DIM, int KIND>
__device__ __forceinline__ void round_octet(const KvArgs& a, const Octet8<TYPE>& raw, const uint4& draws, int64_t row, int octet,
                                            uint8_t* codes, uint16_t* scales)
{
    constexpr int FMT = BITS == 8 ? (int)E4M3 : (int)E2M1, LANES = GROUP_LANES<BITS, DIM>;
    float x[8];
    widen<TYPE>(raw, x);
    uint32_t m = amax_pattern<TYPE>(lanes_max<TYPE, LANES>(amax8<TYPE>(raw)));
    const bool is_nan = m > 0x7F800000u;
    if (__any_sync(0xFFFFFFFFu, m >= 0x7F800000u))            // rare: the largest FINITE magnitude sets the scale
        m = lanes_max<FBSR_FP32, LANES>(finite_amax8_pattern(x));
    // amax / M, rounded up to bfloat16
    const uint32_t q = __float_as_uint(__fmul_rn(__uint_as_float(m), BITS == 8 ? 1.0f / 448.0f : 1.0f / 6.0f));
    const float scale = fminf(fmaxf(__uint_as_float((q + 0xFFFFu) & 0xFFFF0000u), 0x1p-126f), a.scale_max);
    const float inv = __fdiv_rn(1.0f, scale);
    uint32_t word[2];
    if constexpr (KIND == RULE_EVEN) {
        float y[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) y[c] = __fmul_rn(x[c], inv);
        if constexpr (BITS == 8) { word[0] = to_e4m3x4(y[0], y[1], y[2], y[3]); word[1] = to_e4m3x4(y[4], y[5], y[6], y[7]); }
        else word[0] = to_e2m1x8(y);
    } else {
        uint32_t t[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float y = __fmul_rn(x[c], inv);
            t[c] = round_by_rule<FMT, KIND>(y, draws, c, a.rule) | (__float_as_uint(y) & 0x80000000u);
        }
        if constexpr (BITS == 8) {
            word[0] = gather_bytes<3>(t[0], t[1], t[2], t[3]);
            word[1] = gather_bytes<3>(t[4], t[5], t[6], t[7]);
        } else {
            word[0] = 0u;
#pragma unroll
            for (int c = 7; c >= 0; --c) word[0] = __funnelshift_l(t[c], word[0], 4);  // the top four bits enter from the right
        }
    }
    if (is_nan) word[0] = word[BITS == 8] = 0u;
    if (row < 0) return;
    if constexpr (BITS == 8) *reinterpret_cast<uint2*>(codes + row * DIM + octet * 8) = make_uint2(word[0], word[1]);
    else *reinterpret_cast<uint32_t*>(codes + row * (DIM / 2) + octet * 4) = word[0];
    if (octet % LANES == 0) scales[row * (DIM / 8 / LANES) + octet / LANES] = is_nan ? (uint16_t)0x7FC0u : (uint16_t)(__float_as_uint(scale) >> 16);
}

// Row of the cache for a token's head, or -1 where the slot is not one of the cache's.
__device__ __forceinline__ int64_t cache_row(const KvArgs& a, int64_t slot, int head)
{
    if ((uint64_t)slot >= a.capacity) return -1;               // negative ones too
    const int64_t page = slot >> a.page_shift, place = slot - (page << a.page_shift);
    return (((page * a.heads + head) << a.page_shift)) + place;
}

template <int TYPE, int BITS, int DIM, int KIND>
__global__ void __launch_bounds__(THREADS)
round_kv_kernel(const __grid_constant__ KvArgs a)
{
    constexpr uint32_t OCTETS = DIM / 8;
    const uint32_t index = blockIdx.x * THREADS + threadIdx.x;
    const bool mine = index < a.octets;                        // the rest of the warp takes part in the shuffles
    const uint32_t at = mine ? index : a.octets - 1;
    const uint32_t row = at / OCTETS, token = divide(row, a.by_heads);        // row: token * heads + head
    const int octet = (int)(at % OCTETS), head = (int)(row - token * (uint32_t)a.heads);
    Octet8<TYPE> k, v;
    load_octet<TYPE>(a.k, (int64_t)token * a.k_token + head * a.k_head + octet * 8, 8, a.whole, k);
    load_octet<TYPE>(a.v, (int64_t)token * a.v_token + head * a.v_head + octet * 8, 8, a.whole, v);
    const int64_t slot = mine ? a.slots[token] : -1;
    uint4 dk = make_uint4(0u, 0u, 0u, 0u), dv = dk;
    if (KIND != RULE_EVEN && a.rule.mask_lo != 0u) {
        const uint64_t call = a.offset / 8 + at;
        dk = philox4x32_10((uint32_t)call, (uint32_t)(call >> 32), DRAWS_KEYS, 0u, a.k0, a.k1);
        dv = philox4x32_10((uint32_t)call, (uint32_t)(call >> 32), DRAWS_VALUES, 0u, a.k0, a.k1);
    }
    const int64_t to = cache_row(a, slot, head);
    round_octet<TYPE, BITS, DIM, KIND>(a, k, dk, to, octet, a.k_codes, a.k_scales);
    round_octet<TYPE, BITS, DIM, KIND>(a, v, dv, to, octet, a.v_codes, a.v_scales);
}

// Eight codes with the pattern of their scale; zeros for a row that is not in the cache (negative).
template <int BITS> struct Codes8 { uint32_t w[BITS / 4], scale; };

template <int BITS, int DIM>
__device__ __forceinline__ Codes8<BITS> read_codes(int64_t row, int octet, const uint8_t* codes, const uint16_t* scales)
{
    constexpr int LANES = GROUP_LANES<BITS, DIM>;
    Codes8<BITS> r{};
    if (row >= 0) {
        r.scale = scales[row * (DIM / 8 / LANES) + octet / LANES];
        if constexpr (BITS == 8) {
            const uint2 w = __ldcs(reinterpret_cast<const uint2*>(codes + row * DIM + octet * 8));
            r.w[0] = w.x; r.w[1] = w.y;
        } else {
            r.w[0] = __ldcs(reinterpret_cast<const uint32_t*>(codes + row * (DIM / 2) + octet * 4));
        }
    }
    return r;
}

template <int BITS>
__device__ __forceinline__ void numbers_of(const Codes8<BITS>& r, float (&x)[8])
{
    uint32_t h[4];
    if constexpr (BITS == 8) { e4m3_word_to_half2(r.w[0], h[0], h[1]); e4m3_word_to_half2(r.w[1], h[2], h[3]); }
    else e2m1_word_to_half2(r.w[0], h);
    const float scale = __uint_as_float(r.scale << 16);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[c]));
        x[2 * c] = __fmul_rn(f.x, scale); x[2 * c + 1] = __fmul_rn(f.y, scale);
    }
}

// Octets that a thread reads, THREADS apart: their slots, then their codes are all asked for before the first is used.  30011 tokens
// of 8 heads of 128 in 4 bits (157 MB) take 33.1 us (4.8 TB/s), 39.7 with one.
constexpr int READ_AT_ONCE = 4;

template <int TYPE, int BITS, int DIM>
__global__ void __launch_bounds__(THREADS)
read_kv_kernel(const __grid_constant__ KvArgs a)
{
    constexpr uint32_t OCTETS = DIM / 8;
    const uint32_t first = blockIdx.x * (THREADS * READ_AT_ONCE) + threadIdx.x;
    uint32_t token[READ_AT_ONCE];
    int head[READ_AT_ONCE];
    int64_t row[READ_AT_ONCE];
    const int octet = (int)(first % OCTETS);                   // the same for all of them: THREADS is a multiple of OCTETS
#pragma unroll
    for (int i = 0; i < READ_AT_ONCE; ++i) {
        const uint32_t at = first + i * THREADS, r = at / OCTETS;
        token[i] = divide(r, a.by_heads);
        head[i] = (int)(r - token[i] * (uint32_t)a.heads);
        row[i] = at < a.octets ? a.slots[token[i]] : -1;
    }
    Codes8<BITS> k[READ_AT_ONCE], v[READ_AT_ONCE];
#pragma unroll
    for (int i = 0; i < READ_AT_ONCE; ++i) {
        row[i] = cache_row(a, row[i], head[i]);
        k[i] = read_codes<BITS, DIM>(row[i], octet, a.k_codes, a.k_scales);
        v[i] = read_codes<BITS, DIM>(row[i], octet, a.v_codes, a.v_scales);
    }
#pragma unroll
    for (int i = 0; i < READ_AT_ONCE; ++i) {
        if (first + i * THREADS >= a.octets) return;
        float x[8];
        numbers_of<BITS>(k[i], x);
        store8<TYPE>(const_cast<void*>(a.k), (int64_t)token[i] * a.k_token + head[i] * a.k_head + octet * 8, 8, a.whole, x);
        numbers_of<BITS>(v[i], x);
        store8<TYPE>(const_cast<void*>(a.v), (int64_t)token[i] * a.v_token + head[i] * a.v_head + octet * 8, 8, a.whole, x);
    }
}

// KIND: of the rounding rule; negative: reading.
template <int TYPE, int KIND>
void launch(const KvArgs& a, int bits, int dim, cudaStream_t stream)
{
    constexpr uint32_t PER = KIND >= 0 ? THREADS : THREADS * READ_AT_ONCE;
    const unsigned grid = (a.octets + PER - 1) / PER;
#define FBSR_KV(b, d) \
    if (bits == b && dim == d) { \
        if constexpr (KIND >= 0) round_kv_kernel<TYPE, b, d, KIND><<<grid, THREADS, 0, stream>>>(a); \
        else read_kv_kernel<TYPE, b, d><<<grid, THREADS, 0, stream>>>(a); \
    }
    FBSR_KV(8, 128) FBSR_KV(8, 64) FBSR_KV(4, 128) FBSR_KV(4, 64)
#undef FBSR_KV
    count_launch();
}

template <int KIND>
void launch_type(const KvArgs& a, int fmt, int bits, int dim, cudaStream_t stream)
{
    if (fmt == FBSR_FP32) launch<FBSR_FP32, KIND>(a, bits, dim, stream);
    else if (fmt == FBSR_BF16) launch<FBSR_BF16, KIND>(a, bits, dim, stream);
    else launch<FBSR_FP16, KIND>(a, bits, dim, stream);
}

inline bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// What both calls check, and the arguments they share; `done` is set where there is nothing to do.
int fill(KvArgs& a, const fbsr_kv_cache* cache, const void* k, int64_t k_token, int64_t k_head, const void* v, int64_t v_token,
         int64_t v_head, int fmt, size_t tokens, const int64_t* slots, bool& done)
{
    const int status = check_kv_cache(cache);
    if (status != FBSR_OK) return status;
    if (fmt != FBSR_FP32 && fmt != FBSR_BF16 && fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    done = tokens == 0;
    if (done) return FBSR_OK;
    if (k == nullptr || v == nullptr || slots == nullptr) return FBSR_ERR_INVALID_ARG;
    const size_t bytes = fmt == FBSR_FP32 ? 4 : 2;
    if (off(k, bytes) || off(v, bytes) || off(slots, 8)) return FBSR_ERR_ALIGNMENT;
    if (tokens > (((size_t)1 << 31) - 65536) / (cache->dim / 8) / cache->heads) return FBSR_ERR_TOO_LARGE;     // octets in 31 bits
    a.k = k; a.v = v;
    a.k_token = k_token; a.k_head = k_head; a.v_token = v_token; a.v_head = v_head;
    a.k_codes = static_cast<uint8_t*>(cache->k_codes); a.v_codes = static_cast<uint8_t*>(cache->v_codes);
    a.k_scales = static_cast<uint16_t*>(cache->k_scales); a.v_scales = static_cast<uint16_t*>(cache->v_scales);
    a.slots = slots;
    a.octets = (uint32_t)(tokens * cache->heads * (cache->dim / 8));
    a.by_heads = divider((uint32_t)cache->heads);
    a.capacity = cache->pages * (uint64_t)cache->page;
    a.heads = cache->heads;
    a.page_shift = __builtin_ctz(cache->page);
    const int64_t step = 8 * (int64_t)bytes;                   // 32 or 16 bytes
    a.whole = !off(k, step) && !off(v, step) && k_token * (int64_t)bytes % step == 0 && k_head * (int64_t)bytes % step == 0 &&
              v_token * (int64_t)bytes % step == 0 && v_head * (int64_t)bytes % step == 0;
    return FBSR_OK;
}

}  // namespace

int check_kv_cache(const fbsr_kv_cache* c)
{
    if (c == nullptr) return FBSR_ERR_INVALID_ARG;
    if ((c->bits != 8 && c->bits != 4) || (c->dim != 64 && c->dim != 128)) return FBSR_ERR_UNSUPPORTED;
    if (c->page < 8 || c->page > 65536 || (c->page & (c->page - 1)) != 0) return FBSR_ERR_UNSUPPORTED;
    if (c->heads < 1 || c->pages < 1) return FBSR_ERR_INVALID_ARG;
    if (c->heads > 65536 || c->pages > ((uint64_t)1 << 31)) return FBSR_ERR_TOO_LARGE;
    if (c->k_codes == nullptr || c->v_codes == nullptr || c->k_scales == nullptr || c->v_scales == nullptr) return FBSR_ERR_INVALID_ARG;
    if (c->k_codes == c->v_codes || c->k_scales == c->v_scales) return FBSR_ERR_INVALID_ARG;
    if (off(c->k_codes, 16) || off(c->v_codes, 16) || off(c->k_scales, 16) || off(c->v_scales, 16)) return FBSR_ERR_ALIGNMENT;
    return FBSR_OK;
}

}  // namespace fbsr

using namespace fbsr;

extern "C" int fbsr_round_kv(const fbsr_kv_cache* cache, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                             int64_t v_token_stride, int64_t v_head_stride, int src_fmt, size_t tokens, const int64_t* slots, int variant,
                             int k_bits, uint64_t seed, uint64_t offset, void* cuda_stream)
{
    if (variant < 0 || variant > 5 || k_bits < 1 || k_bits > 16) return FBSR_ERR_INVALID_ARG;
    if (offset % 8 != 0 || offset > (1ull << 62)) return FBSR_ERR_INVALID_ARG;
    KvArgs a{};
    bool done = false;
    const int status = fill(a, cache, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, src_fmt, tokens, slots, done);
    if (status != FBSR_OK || done) return status;
    a.offset = offset;
    a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32);
    // the largest bfloat16 whose multiple by the format's largest value is finite in the source's type
    const double largest = src_fmt == FBSR_FP16 ? 65504.0 : src_fmt == FBSR_BF16 ? 0x1.FEp127 : 0x1.FFFFFEp127;
    const float top = (float)(largest / (cache->bits == 8 ? 448.0 : 6.0));
    uint32_t bits;
    std::memcpy(&bits, &top, 4);
    bits &= 0xFFFF0000u;
    std::memcpy(&a.scale_max, &bits, 4);
    a.rule = cache->bits == 8 ? round_rule(24 - Format<E4M3>::P, RULE_L<E4M3>, variant, k_bits) : round_rule(24 - Format<E2M1>::P, RULE_L<E2M1>, variant, k_bits);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (rule_kind(variant) == RULE_EVEN) launch_type<RULE_EVEN>(a, src_fmt, cache->bits, cache->dim, stream);
    else if (rule_kind(variant) == RULE_PLAIN) launch_type<RULE_PLAIN>(a, src_fmt, cache->bits, cache->dim, stream);
    else launch_type<RULE_NEAREST>(a, src_fmt, cache->bits, cache->dim, stream);
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}

extern "C" int fbsr_read_kv(const fbsr_kv_cache* cache, const int64_t* slots, size_t tokens, void* k, int64_t k_token_stride,
                            int64_t k_head_stride, void* v, int64_t v_token_stride, int64_t v_head_stride, int out_fmt, void* cuda_stream)
{
    KvArgs a{};
    bool done = false;
    const int status = fill(a, cache, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, out_fmt, tokens, slots, done);
    if (status != FBSR_OK || done) return status;
    const size_t bytes = out_fmt == FBSR_FP32 ? 4 : 2, heads = (size_t)cache->heads, dim = (size_t)cache->dim;
    if (rows_meet(RowSet(k, k_token_stride, k_head_stride, tokens, heads, dim, bytes), RowSet(v, v_token_stride, v_head_stride, tokens, heads, dim, bytes)))
        return FBSR_ERR_INVALID_ARG;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    launch_type<-1>(a, out_fmt, cache->bits, cache->dim, stream);
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}
