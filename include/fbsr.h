/*
 * fbsr.h -- few-bit stochastic rounding (FBSR) on NVIDIA B200 (sm_100a).
 *
 * C-ABI of libfbsr.so.  The operations follow "On Stochastic Rounding with Few
 * Random Bits" (Fitzgibbon & Felix): a binary32 value y is rounded to a narrower
 * format (K, P, B; M) by
 *     e~     = max(floor(log2 |y|), 1 - B)                      Section II-A, Eq. (2)
 *     sigma~ = |y| 2^-e~ 2^(P-1),  delta~ = sigma~ - floor(sigma~)           Eq. (3)
 *     sigma  = floor(sigma~) + [R(delta~, n)]                                Eq. (5)
 * with n an integer of N = k_bits random bits and R one of
 *     R_SRFF(d, n) = d + n 2^-N >= 1                            Section II-B
 *     R_SRF (d, n) = d + (n + 1/2) 2^-N >= 1                    Section II-B
 *     R_SRC (d, n) = R_SRFF(Round(d 2^N) 2^-N, n)               Section III-F, Eq. (8)
 * (Round = nearest, ties to even).  sigma = 2^P increments the exponent.
 *
 * Conventions shared by every entry point unless stated otherwise
 *   - Pointers are DEVICE pointers owned by the caller.  The library allocates no
 *     memory, never synchronises, and only enqueues work on `cuda_stream`
 *     (a cudaStream_t passed as void*; NULL = the default stream) of the current
 *     device.  Buffers must stay valid until that work has run.
 *   - Results are a pure function of the arguments: the same (seed, offset)
 *     gives the same bits on every call and for every way of splitting a tensor
 *     into calls, provided `offset` is the global index of element 0.
 *   - The magnitude is rounded and the sign copied.  NaN -> quiet NaN, sign of
 *     the input kept (0x7FC0 bf16, 0x7E00 fp16, 0x7F e4m3 and e5m2).  +-Inf ->
 *     +-Inf, or +-M for e4m3, which has no infinity.  Finite |y| > M -> +-M.
 *     Binary8P4 has one zero and one NaN: a zero result is 0x00 whatever the sign
 *     of the input (-0, or a negative value rounded down to zero), NaN -> 0x80.
 *     None of these consume the paper's predicates (Section II leaves values
 *     outside the finite range to deterministic rounding).
 *   - Random draws: Philox4x32-10 with key (seed lo, seed hi).  With
 *     dpw = 32 / k_bits (integer division) draws per 32-bit word and E = 4 dpw,
 *     the element with global index g uses field (g mod dpw), low bits first, of
 *     output word ((g mod E) / dpw) of the generator call with counter
 *     (b lo, b hi, 0, 0), b = g / E.  The paper leaves the generator open
 *     (Section II-B); this indexing is the library's definition.
 *   - Any n (including 0) and any element alignment are accepted.  The fast
 *     path needs src 32-byte aligned, dst 16-byte aligned and `offset` a multiple
 *     of the tile size reported by fbsr_tile_elements(); other calls are served
 *     by a slower kernel with identical results.  fbsr_round itself has a second
 *     fast kernel that takes pointers of any element alignment (a slice of a
 *     tensor, a packed parameter buffer) at about four fifths of the speed; the
 *     part of a call before the first tile boundary of `offset` (less than one
 *     tile) always goes to the slower kernel.
 *   - Errors are reported by the return value only.  Nothing is written on error.
 */
#ifndef FBSR_H
#define FBSR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FBSR_OK = 0,
    FBSR_ERR_INVALID_ARG = 1, /* null pointer with n > 0, bad enum, k_bits outside 1..16, bad scale */
    FBSR_ERR_UNSUPPORTED = 2, /* a combination this build does not implement */
    FBSR_ERR_ALIGNMENT = 3,   /* a pointer is not aligned to its element size */
    FBSR_ERR_CUDA = 4,        /* the CUDA runtime reported an error at launch */
    FBSR_ERR_WORKSPACE = 5,   /* workspace missing or too small */
    FBSR_ERR_TOO_LARGE = 6    /* n exceeds the limit of an entry point with built-in scratch */
} fbsr_status;

/* Target formats (K, P, B; M), Section II.  P counts the hidden bit. */
typedef enum {
    FBSR_BF16 = 0, /* (16,  8, 127; 0x1.FEp127) */
    FBSR_FP16 = 1, /* (16, 11,  15; 65504)      */
    FBSR_E4M3 = 2, /* ( 8,  4,   7; 448)   OCP E4M3: no Inf, S.1111.111 is NaN */
    FBSR_E5M2 = 3, /* ( 8,  3,  15; 57344) */
    FBSR_B8P4 = 4  /* ( 8,  4,   8; 224)   IEEE WG P3109 Binary8P4, the target of Section IV:
                      0x7F / 0xFF are +-Inf, 0x80 is the NaN, there is no negative zero */
} fbsr_fmt;

/* May be or-ed into any `fmt` argument.  Section II leaves values beyond the finite range to the deterministic
 * nearest rounding of IEEE 754; with this flag finite |y| > M follow that reading (M below M + ulp(M)/2, +-Inf
 * above it -- the NaN code for e4m3 -- ties to the even neighbour) instead of saturating.  fbsr_round and
 * fbsr_round_lp serve the flag at full speed on aligned calls (one comparison per element in the tiled kernel);
 * the other entry points, and calls whose pointers are off the fast path's alignment, use the general kernel. */
#define FBSR_OVF_IEEE 0x100

/* binary32, for the arguments that name the type of a SOURCE (g_fmt of fbsr_adamw_multi, src_fmt of fbsr_round_w4, _kv and _i8,
 * out_fmt of fbsr_gemv_w4, fbsr_read_kv and fbsr_gemm_i8); it is not a target of rounding. */
#define FBSR_FP32 0x20

/* Round-up predicates: the few-bit stochastic ones of Section II-B and Eq. (8), and the deterministic
 * ones of Section II-A (ties to even, ties away from zero (Eq. (4)), ties to odd), which use no draw:
 * for those k_bits, seed and offset are ignored (k_bits must still be in 1..16). */
typedef enum {
    FBSR_SRFF = 0, FBSR_SRF = 1, FBSR_SRC = 2,
    FBSR_RTNE = 3, FBSR_RTA = 4, FBSR_RTO = 5
} fbsr_variant;

/* Error statistics over the SR-rounded elements of one call.  e = up - delta~
 * is the rounding error of the magnitude in target ulps, the quantity whose
 * mean Section III calls bias.  NaN, Inf and saturated elements are counted
 * but excluded from the sums. */
typedef struct {
    uint64_t n_finite;   /* elements that were SR-rounded (|y| <= M, zeros included) */
    uint64_t n_up;       /* of those, how many rounded up in magnitude */
    uint64_t n_nan;
    uint64_t n_inf;
    uint64_t n_sat;      /* finite |y| > M */
    double sum_e;        /* sum of e */
    double sum_e2;       /* sum of e^2 */
    double sum_signed_e; /* sum of sign(y) e: error of the signed value */
    double sum_abs_e;    /* sum of |e| */
} fbsr_stats;

/* ---------------------------------------------------------------------------
 * fbsr_round -- Section II-A/II-B/III-F: dst[i] = FBSR(fl32(src[i] * scale)).
 *   src      device, n binary32 values (read only; must not overlap dst)
 *   dst      device, n codes: uint16 for bf16/fp16, uint8 for e4m3/e5m2/b8p4
 *   fmt, variant, k_bits   fbsr_fmt, fbsr_variant, N in 1..16
 *   seed, offset           Philox key and global index of element 0
 *   scale    finite, > 0; the per-tensor factor of a scaled tensor (Section I-A),
 *            applied as one rounded binary32 multiply
 * ------------------------------------------------------------------------- */
int fbsr_round(const float* src, void* dst, size_t n, int fmt, int variant, int k_bits,
               uint64_t seed, uint64_t offset, float scale, void* cuda_stream);

/* fbsr_round_lp -- the paper's own regime (Section III-E, Fig. 2, the rounding to 8 bits that ends Algorithm 1):
 * the source is already a low-precision tensor.  dst[i] = FBSR(fl32(value(src[i]) * scale)), where
 * value() widens the stored code exactly by Eq. (1).
 *   src      device, n codes of src_fmt (FBSR_BF16 or FBSR_FP16, uint16 each); must not overlap dst
 *   dst      device, n codes of dst_fmt (FBSR_E4M3, FBSR_E5M2 or FBSR_B8P4, uint8 each)
 * Other format pairs return FBSR_ERR_UNSUPPORTED.  The fast path needs src 32-byte aligned, dst 16-byte
 * aligned (a lane reads 16 source codes and writes 16 target codes at a time) and `offset` on the tile grid;
 * other calls are served by the general kernel with identical results.  A NaN source keeps its sign. */
int fbsr_round_lp(const void* src, int src_fmt, void* dst, size_t n, int dst_fmt, int variant, int k_bits,
                  uint64_t seed, uint64_t offset, float scale, void* cuda_stream);

/* fbsr_round_desc -- fbsr_round for a format (K, P, B; M) given at run time, Section II's parametrisation
 * (width, precision, exponent bias and largest finite value); the rounding itself is Section II-A
 * Eq. (2)-(5) with the predicates of Section II-B and Eq. (8), as in fbsr_round.
 *   desc     HOST pointer, read before the call returns:
 *     K          8 or 16: width of a code (dst is uint8 or uint16)
 *     P          precision including the hidden bit, 2 <= P <= min(K - 1, 13)
 *     B          exponent bias, 1 <= B <= 127
 *     max_code   magnitude code of M, the largest finite value (exponent field of M minus B at most 127)
 *     has_inf / inf_code   whether an infinity exists, and its magnitude code (> max_code)
 *     nan_code   magnitude code written for NaN (> max_code, != inf_code); with single_zero the pattern
 *                1 << (K - 1) instead
 *     single_zero  non-zero: one zero and one unsigned NaN (the pattern that would be minus zero), as in
 *                Binary8P4; a zero result then has no sign
 *   ovf_ieee non-zero: finite |y| > M are rounded as IEEE nearest-even does (see FBSR_OVF_IEEE)
 * Special values follow the conventions at the top of this file (Inf -> the infinity, or +-M without one).
 * Whole tiles of the draw stream (src 32-byte aligned and dst 8 x code-size aligned at the first tile boundary) are
 * served by a tiled kernel at roughly half the speed of the built-in formats' kernels; the head, the ragged end and
 * unaligned calls by a general kernel (any alignment, any offset) that is several times slower.
 * The built-in formats written as descriptors give the built-in results bit for bit.
 * Returns FBSR_ERR_INVALID_ARG for a descriptor outside the ranges above. */
typedef struct {
    int32_t K, P, B;
    uint32_t max_code;
    int32_t has_inf;
    uint32_t inf_code, nan_code;
    int32_t single_zero;
} fbsr_format_desc;

int fbsr_round_desc(const float* src, void* dst, size_t n, const fbsr_format_desc* desc, int ovf_ieee,
                    int variant, int k_bits, uint64_t seed, uint64_t offset, float scale, void* cuda_stream);

/* 1 if fbsr_round_desc accepts the descriptor, else 0.  Host only, no CUDA call. */
int fbsr_format_desc_valid(const fbsr_format_desc* desc);

/* fbsr_round_mx -- block-scaled tensors (Section I-A: each block of low-precision values carries a scale
 * factor of its own, here a power of two).  Blocks are 32 consecutive elements of the call; per block
 *     amax  = largest finite |src| (0 if none)
 *     e_blk = clamp(floor(log2 amax) - emax, -127, 127), emax = floor(log2 M);  -127 if amax < 2^-126
 *     scales[block] = e_blk + 127;   dst[i] = FBSR(fl32(src[i] * 2^-e_blk))
 * so the block maximum lands in the format's top binade (values between M and 2^(emax+1) saturate).
 *   scales   device, ceil(n / 32) bytes, overwritten
 * Draws are indexed by offset + i as everywhere else.  The fast path additionally needs the first tile
 * boundary of the call to fall on a block boundary (true for offset = 0 or any multiple of the tile size). */
int fbsr_round_mx(const float* src, void* dst, uint8_t* scales, size_t n, int fmt, int variant, int k_bits,
                  uint64_t seed, uint64_t offset, void* cuda_stream);

/* fbsr_round_w4 -- block-scaled rounding of a weight matrix to 4 bits (Section I-A's scaled values; the target is E2M1 =
 * (K, P, B; M) = (4, 2, 1; 6): 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign).  `group` (32, 64 or 128) consecutive elements of a
 * row share a scale s; with amax the group's largest finite magnitude (0 if none):
 *     FBSR_SCALE_E8M0  s = 2^e, e = max(floor(log2 amax) - 2, -127) (-127 if amax < 2^-126): one byte e + 127.  As in
 *                      fbsr_round_mx, the maximum lands in the top binade and what exceeds 6 s saturates.
 *     FBSR_SCALE_BF16  s = fl(amax fl(1 / 6)) rounded up to bfloat16, at least 2^-126, at most the largest bfloat16 whose
 *                      sixfold is finite in the source's type; stored as that bfloat16.
 *     code = FBSR_E2M1(fl(x fl(1 / s)));  value = code s.   Infinities saturate.  A group that holds a NaN gets the NaN scale
 *     (byte 255, or bfloat16 0x7FC0) and zero codes: all of it reads as NaN.
 *   src        device, rows x cols values of src_fmt (FBSR_FP32, FBSR_BF16 or FBSR_FP16), row r at src + r src_ld (elements)
 *   codes      device, rows x (padded / 2) bytes, padded = fbsr_w4_padded(cols): cols rounded up to a multiple of 128, the
 *              rest filled with zeros; 16-byte aligned.  A 32-bit word holds 8 consecutive elements, the first in its lowest
 *              bits; in every 64 bytes (128 elements) word 4 j + t of plain order lies at place 4 t + j (j, t = 0..3).
 *   scales     device, rows x (padded / group) bytes or bfloat16
 *   values     NULL, or device, rows x cols of src_fmt at values + r values_ld: the values that the codes stand for, rounded
 *              once to src_fmt (what a forward pass over 4-bit weights multiplies with); must not overlap src (src
 *              itself is refused)
 *   offset     a multiple of 128, at most 2^62; element (r, c) has the global index offset + r padded + c for its draw.
 * At most 2^30 blocks of 128 (FBSR_ERR_TOO_LARGE).  Rows whose addresses allow it (32 bytes for binary32, 16 for 16-bit) are
 * read and written eight elements at a time. */
#define FBSR_SCALE_E8M0 0
#define FBSR_SCALE_BF16 1
size_t fbsr_w4_padded(size_t cols);
int fbsr_round_w4(const void* src, int src_fmt, int64_t src_ld, size_t rows, size_t cols, uint8_t* codes, void* scales,
                  int scale_fmt, int group, void* values, int64_t values_ld, int variant, int k_bits, uint64_t seed,
                  uint64_t offset, void* cuda_stream);

/* fbsr_gemv_w4 -- the product of activations with a matrix that fbsr_round_w4 has written (the forward product that the
 * quantised weights of Algorithm 1 exist for):  y[i][r] = sum over c < k of x[i][c] value(W[r][c]),
 * value(W[r][c]) = code s.  Each group's products are exact, summed in the matrix unit (binary32 sums, which it may truncate where
 * it aligns their terms: up to 2^-23 a step) and multiplied by s in binary32; groups are added in binary32, in an order that
 * depends on shapes and types alone; one rounding to out_fmt at the end.  bfloat16
 * elements of x below 2^-32 of the largest finite magnitude of their 128 columns are rounded to 2^-40 of it, and scales
 * above 2^100 may overflow before the sum does.  NaN and infinities in x and NaN scales go where the formula takes them.
 *   x        device, m rows of k values of x_fmt (FBSR_BF16 or FBSR_FP16), row i at x + i ldx (elements)
 *   codes, scales, scale_fmt, group   n x k matrix as written by fbsr_round_w4 (its rows x cols); codes 16-byte aligned,
 *            scales aligned to the scales of 128 elements (1 to 8 bytes); codes beyond column k must be zero
 *   y        device, m rows of n values of out_fmt (FBSR_FP32, FBSR_BF16 or FBSR_FP16) at y + i ldy; must not overlap x (x
 *            itself is refused)
 * Meant for few rows: up to 8 share the reading and decoding of W (128000 x 4096: 51 us for one, 59 for eight); every 32
 * rows read the matrix again.  k = 0 gives zeros. */
int fbsr_gemv_w4(const void* x, int x_fmt, int64_t ldx, size_t m, const uint8_t* codes, const void* scales, int scale_fmt,
                 int group, size_t n, size_t k, void* y, int out_fmt, int64_t ldy, void* cuda_stream);

/* ---------------------------------------------------------------------------
 * A cache of keys and values in few bits (the low-precision values of Section I-A, each group with a scale of its own), in
 * pages.  A page holds `page` tokens of every head; slot = page index * page + place in the page names a token's place.
 *   k_codes, v_codes    device, [pages][heads][page][dim * bits / 8] bytes: 8 bits, E4M3 codes; 4 bits, E2M1 codes, element 2 i
 *                       in the low half of byte i.  16-byte aligned.
 *   k_scales, v_scales  device, [pages][heads][page][groups] bfloat16: 8 bits, one for a row of dim elements (groups = 1); 4
 *                       bits, one for every 32 elements (groups = dim / 32).  16-byte aligned.
 *   pages  1..2^31;  heads  1..65536;  page  a power of two, 8..65536;  dim  64 or 128;  bits  8 or 4
 * The four buffers must not overlap. */
typedef struct {
    void* k_codes;
    void* v_codes;
    void* k_scales;
    void* v_scales;
    uint64_t pages;
    int32_t heads, page, dim, bits;
} fbsr_kv_cache;

/* fbsr_round_kv -- keys and values rounded into a cache as they are written.  Per group of a row, M = 448 (8 bits) or 6 (4
 * bits), amax the group's largest finite magnitude (0 if none):
 *     s = fl(amax fl(1 / M)) rounded up to bfloat16, at least 2^-126, at most the largest bfloat16 whose M-fold is finite in
 *     the source's type;  code = FBSR(fl(x fl(1 / s))), stored value = code s.  Infinities saturate.  A group that holds a NaN
 *     gets the NaN scale (0x7FC0) and zero codes: all of it reads as NaN.
 *   k, v       device, tokens x heads x dim values of src_fmt (FBSR_FP32, FBSR_BF16 or FBSR_FP16); token t, head h at
 *              k + t k_token_stride + h k_head_stride (elements), dim contiguous ones
 *   slots      device, one int64 per token: where its rows go.  A token whose slot is not one of the cache's (-1 for padding) is
 *              not written.  Two tokens of a call must not have the same slot: what that slot holds then is undefined.
 *   offset     a multiple of 8, at most 2^62; element d of head h of token t has the index J = offset + (t heads + h) dim + d.
 *              Its draw is bits [0, k) of halfword J mod 8 (low half of word 0 first) of the generator call with counter
 *              (J / 8 lo, hi, 2, 0) for keys and (.., .., 3, 0) for values.
 * tokens x heads x dim less than 2^34 - 2^19 (FBSR_ERR_TOO_LARGE).  Any element alignment is accepted; sources whose address and strides are
 * multiples of 32 bytes (binary32) or 16 are read eight elements at a time. */
int fbsr_round_kv(const fbsr_kv_cache* cache, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                  int64_t v_token_stride, int64_t v_head_stride, int src_fmt, size_t tokens, const int64_t* slots, int variant,
                  int k_bits, uint64_t seed, uint64_t offset, void* cuda_stream);

/* fbsr_read_kv -- rows of a cache as numbers: code s, rounded once to out_fmt (FBSR_FP32, FBSR_BF16 or FBSR_FP16).  A token whose
 * slot is not one of the cache's gives zeros.  k and v as the sources of fbsr_round_kv, overwritten; rows of k and v must not overlap (refused). */
int fbsr_read_kv(const fbsr_kv_cache* cache, const int64_t* slots, size_t tokens, void* k, int64_t k_token_stride,
                 int64_t k_head_stride, void* v, int64_t v_token_stride, int64_t v_head_stride, int out_fmt, void* cuda_stream);

/* fbsr_attend_kv -- attention of drafted tokens over a cache, straight from its codes.  A sequence's queries are its last
 * tokens: with `length` cached tokens and n queries, query i's own key is token length - n + i (its rows have been written
 * before the call), and tokens below length - n are the context, which every query sees.  Of the n drafts, query i sees those
 * whose bit is set in its row of `tree` (a tree of drafts: its ancestors and itself); without a tree the drafts up to i.  One
 * query a sequence is ordinary decoding.  Query head h reads head h / (heads / cache heads).  Per query and head
 *     out = sum_t p_t value(v_t) / sum_t p_t,   p_t = exp(scale q . value(k_t))      over the tokens t that it sees;
 * zeros if it sees none.  The products are of binary16 operands with binary32 sums: codes exactly; bfloat16 queries times a power of
 * two for each head (what is below 2^-38 of its largest element loses bits, as do the scores of a row whose largest element times scale
 * is below 2^-112); weights p_t times the scale of v_t rounded to
 * binary16, the sum of the p_t from binary32 values.  Within a row of the cache, 4-bit groups more than 2^14 below the row's
 * largest scale lose bits, as do rows of v whose scales are below 2^-70; a weight below 2^-134 of the largest product of a weight and its
 * token's scale of v counts as zero.  A NaN that a query sees makes its result NaN; one that it does not see has no influence.
 *   q          device, total queries x heads x dim of q_fmt (FBSR_BF16 or FBSR_FP16), strides in elements
 *   cache      as above, codes as fbsr_round_kv writes them (no NaN codes) in every slot below a sequence's length
 *   pages      device, batch rows of max_pages page indices (int32), row b at pages + b pages_ld (max_pages or more)
 *   lengths    device, batch int32: tokens in the cache, the queries' own among them
 *   starts     device, batch + 1 int32, not decreasing: sequence b's queries are rows starts[b] .. starts[b + 1] - 1 of q.
 *              NULL: every sequence has max_queries of them, one after another.
 *   max_queries  1..256, at least every sequence's number of queries; more are not computed
 *   tree       NULL, or device, total queries x tree_words uint64; bit j mod 64 of word j / 64 is draft j.
 *              tree_words: (max_queries + 63) / 64 or more, 1024 at most
 *   scale      finite, and so is its product with log2(e)
 *   out        device, total queries x heads x dim of q_fmt; no row of it may overlap one of q (refused).  Rows that belong to no
 *              sequence are left as they were.
 *   workspace  device, fbsr_attend_workspace_bytes(...) bytes, 16-byte aligned; contents on entry are ignored.  Calls that may overlap need
 *              workspaces of their own.
 * An index that is not one of the cache's pages, or a length beyond max_pages pages, makes the results that depend on it NaN;
 * nothing outside the buffers is read.  heads a multiple of the cache's; at most 65536 heads, 2^31 - 1 queries, 2^40 rows of them (queries x
 * heads) and 2^31 - 64 tokens a sequence (FBSR_ERR_TOO_LARGE).  The order of summation depends on the arguments, shapes and lengths alone. */
size_t fbsr_attend_workspace_bytes(const fbsr_kv_cache* cache, size_t batch, size_t total, int heads, size_t max_queries, size_t max_pages);
int fbsr_attend_kv(const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_fmt, size_t total, int heads,
                   const fbsr_kv_cache* cache, const int32_t* pages, int64_t pages_ld, size_t max_pages, const int32_t* lengths,
                   size_t batch, const int32_t* starts, size_t max_queries, const uint64_t* tree, int tree_words, float scale,
                   void* out, int64_t out_token_stride, int64_t out_head_stride, void* workspace, size_t workspace_bytes,
                   void* cuda_stream);

/* fbsr_round_i8 -- rows rounded to 8-bit integers with a scale each (activations with a scale for each token, weights with one
 * for each channel).  With amax the row's largest finite magnitude (0 if none),
 *     s = fl(amax fl(1 / 127)), at least 2^-126, at most the largest binary32 number whose 127-fold is finite;
 *     code = FBSR to the integers of fl(x fl(1 / s)), at most 127 in magnitude (infinities too);  value = code s.
 * A row that holds a NaN gets a NaN scale and zero codes: all of it reads as NaN.
 *   src        device, rows x cols values of src_fmt (FBSR_FP32, FBSR_BF16 or FBSR_FP16), row r at src + r src_ld (elements)
 *   codes      device, rows x padded bytes, padded = fbsr_i8_padded(cols): cols rounded up to a multiple of 128, the rest
 *              filled with zeros; 16-byte aligned
 *   scales     device, rows binary32 numbers
 *   values     NULL, or device, rows x cols of src_fmt at values + r values_ld: the values, rounded once to src_fmt; no row
 *              may overlap one of src (refused)
 *   offset     a multiple of 128, at most 2^62; element (r, c) has the index J = offset + r padded + c, its draw is bits [0, k) of
 *              halfword J mod 8 (low half of word 0 first) of the generator call with counter (J / 8 lo, hi, 4, 0).
 * At most 2^31 - 1 rows and 2^31 - 256 columns.  Without rows or without columns nothing is written, the scales (2^-126 each) neither.
 * Any element alignment is accepted; rows whose addresses are multiples of 32 bytes (binary32) or 16 are moved eight elements at a time. */
size_t fbsr_i8_padded(size_t cols);
int fbsr_round_i8(const void* src, int src_fmt, int64_t src_ld, size_t rows, size_t cols, int8_t* codes, float* scales, void* values,
                  int64_t values_ld, int variant, int k_bits, uint64_t seed, uint64_t offset, void* cuda_stream);

/* fbsr_gemm_i8 -- the product of two matrices that fbsr_round_i8 has written, activations by weights:
 *     y[i][r] = fl(float(sum over c < k of a[i][c] w[r][c]) fl(a_scales[i] w_scales[r])),  rounded once more to out_fmt,
 * the sum exact in 32-bit integers, its conversion to binary32 rounded to nearest.  The bits do not depend on how a product is
 * split into calls.  NaN scales make their rows (columns) of y NaN.
 *   a          device, m x k signed bytes, row i at a + i lda; w device, n x k, row r at w + r ldw; both 16-byte aligned, lda and
 *              ldw multiples of 16 below 2^40
 *   k          columns with their padding: a multiple of 16, not 0, less than 131072 (FBSR_ERR_TOO_LARGE beyond: the sum could overflow)
 *   y          device, m rows of n values of out_fmt (FBSR_FP32, FBSR_BF16 or FBSR_FP16) at y + i ldy; no row may overlap one of
 *              a or w (refused)
 * Up to 4 rows of a (single tokens) are served by a kernel that reads w once; more by the matrix unit. */
int fbsr_gemm_i8(const int8_t* a, int64_t lda, size_t m, const float* a_scales, const int8_t* w, int64_t ldw, size_t n,
                 const float* w_scales, size_t k, void* y, int out_fmt, int64_t ldy, void* cuda_stream);

/* fbsr_round_bits -- the same rounding with caller-supplied random bits
 * (Section II-B treats the randomness as a finite string of bits handed to the
 * rounder).  rand_words: device, ceil(n / dpw) words; element i uses field
 * (i mod dpw) of word (i / dpw), low bits first; higher bits are ignored. */
int fbsr_round_bits(const float* src, void* dst, size_t n, int fmt, int variant, int k_bits,
                    const uint32_t* rand_words, float scale, void* cuda_stream);

/* fbsr_round_stats -- fbsr_round plus the error statistics of Section III
 * (bias = mean of e) accumulated in binary64.
 *   group_size       0, or the length of the consecutive groups of this call's
 *                    elements (group j = elements [j group_size, (j+1) group_size))
 *   group_sum_e/_e2  device, ceil(n / group_size) doubles each, overwritten with
 *                    the per-group sums of e and e^2; may be NULL when group_size = 0.
 *                    Group sums are added with atomics: their last bits may vary
 *                    from run to run.
 *   total            device, one fbsr_stats, overwritten.  Totals are reduced in a
 *                    fixed order and are reproducible bit for bit.
 *   workspace        device scratch of at least fbsr_stats_workspace_bytes() bytes,
 *                    8-byte aligned; contents on entry are ignored. */
size_t fbsr_stats_workspace_bytes(void);
int fbsr_round_stats(const float* src, void* dst, size_t n, int fmt, int variant, int k_bits,
                     uint64_t seed, uint64_t offset, float scale, size_t group_size,
                     double* group_sum_e, double* group_sum_e2, fbsr_stats* total,
                     void* workspace, size_t workspace_bytes, void* cuda_stream);

/* fbsr_round_stats_noalloc -- fbsr_round_stats without a workspace argument.
 * (The paper has no counterpart; this exists for the sake of callers, see below.)
 *
 * Who it is for: code that may not allocate device memory at the point where it
 * wants rounding statistics -- a step that runs inside a memory pool whose size was
 * fixed at start-up, a plugin inside someone else's process that must not touch
 * the allocator, a monitoring hook on a device that is already full.  Such a
 * caller cannot provide the scratch that fbsr_round_stats needs for its per-CTA
 * partial sums, so this variant keeps that scratch inside the library: a
 * file-scope device array of FBSR_NOALLOC_SCRATCH_BYTES (85,248 bytes), which
 * every GPU that loads libfbsr.so holds until the process exits.  The call itself
 * performs no cudaMalloc / cudaFree and calls no allocating routine.
 *
 * Arguments and results are those of fbsr_round_stats (same kernels, same fixed
 * reduction order, so totals are bit-identical to it); src, dst, the group arrays
 * and `total` are still the caller's.
 *   - n must not exceed FBSR_NOALLOC_MAX_ELEMENTS (2^31); larger calls return
 *     FBSR_ERR_TOO_LARGE and do nothing.  The limit bounds how long one call can
 *     occupy the shared scratch.
 *   - The first call on each device looks up the device address of the scratch
 *     array (cudaGetSymbolAddress) with that device current; make that first
 *     call outside any stream capture.  The address is remembered per device
 *     ordinal for the life of the process and does not survive a
 *     cudaDeviceReset: do not call this entry point again after one.
 *   - All calls on a device share the one array.  It keeps whatever the previous
 *     call left there; nothing in it has to start at zero, because every slot a
 *     call reads is first written by that same call.  Two calls that can overlap
 *     on the GPU (different streams without an ordering between them) race on
 *     it and give undefined statistics: order them, or use fbsr_round_stats with
 *     separate workspaces. */
#define FBSR_NOALLOC_SCRATCH_BYTES 85248u
#define FBSR_NOALLOC_MAX_ELEMENTS ((size_t)1 << 31)
int fbsr_round_stats_noalloc(const float* src, void* dst, size_t n, int fmt, int variant, int k_bits,
                             uint64_t seed, uint64_t offset, float scale, size_t group_size,
                             double* group_sum_e, double* group_sum_e2, fbsr_stats* total,
                             void* cuda_stream);

/* fbsr_sgd_update -- last line of Algorithm 1 with a binary32 master copy:
 *     m' = fma(mu, m, g);  w' = fma(-lr, m', w);  dst = FBSR(w')
 * master_w and momentum are updated in place; grad is read only.  Every
 * operation is one correctly rounded binary32 operation (no flush to zero). */
int fbsr_sgd_update(float* master_w, const float* grad, float* momentum, void* dst_lp, size_t n,
                    int fmt, int variant, int k_bits, uint64_t seed, uint64_t offset,
                    float lr, float mu, void* cuda_stream);

/* fbsr_adam_update -- same, with Adam (no weight decay).  Host scalars, in
 * binary64 then rounded to binary32: b1t = beta1^step and b2t = beta2^step by
 * repeated multiplication, c1 = lr / (1 - b1t), c2 = 1 / sqrt(1 - b2t),
 * a1 = 1 - beta1, a2 = 1 - beta2.  Per element, binary32:
 *     m' = fma(beta1, m, a1 g);  v' = fma(beta2, v, (a2 g) g);
 *     d  = sqrt(v') c2 + eps;    w' = fma(-c1, m' / d, w);  dst = FBSR(w')
 * step >= 1 is the 1-based step count. */
int fbsr_adam_update(float* master_w, const float* grad, float* m, float* v, void* dst_lp, size_t n,
                     int fmt, int variant, int k_bits, uint64_t seed, uint64_t offset,
                     float lr, float beta1, float beta2, float eps, int step, void* cuda_stream);

/* The four host scalars of fbsr_adam_update and fbsr_qat_adamw_step for a given step (Algorithm 1 leaves the
 * arithmetic of its AdamW update open; this is the library's definition, stated with fbsr_adam_update):
 * out = {c1, c2, a1, a2}.  beta^step is formed by repeated multiplication in binary64; the multiplication stops
 * once the product of a |beta| < 1 has fallen below 2^-54, from where on 1 - beta^step is exactly 1, so the cost
 * on the host does not grow with the step count.  Host only, no CUDA call; out must hold 4 floats. */
void fbsr_adam_scalars(float lr, float beta1, float beta2, int step, float out[4]);

/* fbsr_accumulate -- the last step of Algorithm 1 (weight plus update, rounded to the narrow format) with the sum
 * formed in binary32:  w_lp[i] = FBSR(fl32(value(w_lp[i]) + update[i])), in place.
 * A NaN sum is written as the positive quiet NaN. */
int fbsr_accumulate(void* w_lp, const float* update, size_t n, int fmt, int variant, int k_bits,
                    uint64_t seed, uint64_t offset, void* cuda_stream);

/* fbsr_qat_adamw_step -- Algorithm 1, one whole iteration from the gradient on, fused:
 *     w16 = value(w8);  g = value(grad16);
 *     the algorithm's 16-bit AdamW update: moments in binary32, each operation rounded once, the result rounded to the 16-bit format
 *         m' = fma(beta1, m, a1 g);  v' = fma(beta2, v, (a2 g) g);  d = sqrt(v') c2 + eps;
 *         u32 = fma(-c1, m' / d, -(lr weight_decay) w16);   u16 = RTNE_16(u32)      (c1, c2, a1, a2 as in fbsr_adam_update)
 *     w8 = FBSR(RTNE_16(fl32(w16 + u16)))                                            (as in fbsr_qat_update; SR applied here)
 *   w8       device, n codes of w_fmt (FBSR_E4M3, FBSR_E5M2 or FBSR_B8P4), read and overwritten
 *   grad16   device, n codes of g_fmt (FBSR_BF16 or FBSR_FP16), the algorithm's 16-bit format
 *   m, v     device, n binary32 moments each, read and overwritten
 * 20 bytes per parameter.  The paper states the shape of the step, not its arithmetic: the operation list is this
 * library's.  A NaN result is written as the positive NaN code; m and v then hold NaNs of unspecified sign. */
int fbsr_qat_adamw_step(void* w8, const void* grad16, float* m, float* v, size_t n, int w_fmt, int g_fmt, int variant,
                        int k_bits, uint64_t seed, uint64_t offset, float lr, float beta1, float beta2, float eps,
                        float weight_decay, int step, void* cuda_stream);

/* fbsr_adamw_multi -- Algorithm 1's AdamW update of a whole model: one step over `count` tensors, with the moments in
 * binary32 or in 8 bits, and the SR write of each tensor's low-precision copy.  Per element, binary32, every operation
 * rounded once; the host scalars c1, c2, a1, a2 (as in fbsr_adam_update) and decay = 1 - lr weight_decay are formed in
 * binary64 from the binary64 arguments (beta^step by pow) and then rounded to binary32, as beta1, beta2 and eps are:
 *     g = fl(value(g) grad_scale);  m' = fma(beta1, m, a1 g);  v' = fma(beta2, v, (a2 g) g);  r = sqrt(v');
 *     w' = fma(-c1, m' / fl(fl(r c2) + eps), fl(w decay));  w_lp = FBSR(w')
 * With weight_decay = 0, binary32 gradients and state, no grad_scale and scalars that are binary32 numbers, every
 * tensor's result is that of fbsr_adam_update with its `offset`, bit for bit (c1 and c2 are the same binary32 numbers at every
 * step up to 200,000 for ten betas between 0.5 and 0.99999, though beta^step is formed by products there).
 *   tensors     HOST array, read before the call returns; a tensor with n = 0 is skipped.  Tensors must not overlap.
 *     w           device, n binary32 master weights, updated in place
 *     g           device, n gradients of g_fmt (FBSR_FP32, FBSR_BF16 or FBSR_FP16), read only
 *     m, v        device: n binary32 moments (state_bits 32), or n codes (state_bits 8), updated in place
 *     m_scale, v_scale   state_bits 8: device, ceil(n / 256) binary32 scales each, updated in place; else ignored
 *     w_lp        device, n codes of `fmt`, overwritten; NULL: no copy of this tensor is written
 *     offset      global index of the tensor's element 0 for the draws; a multiple of 256
 *   grad_scale  device, one binary32 factor (loss unscaling, clipping) read when the kernel runs; NULL = 1
 * 8-bit state: 256 consecutive elements of a tensor share a scale.  m holds E4M3 codes of m' / s, v holds E4M3 codes of
 * sqrt(v') / s, s = max(fl(amax fl(1 / 448)), 2^-126) with amax the block's largest finite magnitude of what is stored;
 * products and sums of m' and v' are rounded one by one here (no fma), so that plain binary32 arithmetic reproduces codes:
 *     code = FBSR_E4M3(fl(x fl(1 / s))), the same variant and k_bits as the weights; a root above zero whose code came out
 *     as zero takes the smallest code, so that a moment never vanishes under a step that divides by it.
 * The quotient m' / d of this state may be one unit off where |m'| < 2^-100 or the quotient is subnormal, and a |d| above 2^126
 * may count as infinite (an eps above it, or a second moment that overflows).
 * Fresh state is all zeros, scales included.  The draws of element J = offset + j for the two states are bits [0, k) and
 * [8, 8 + k) of halfword J mod 8 (low half of word 0 first) of the generator call with counter (J / 8 lo, hi, 1, 0); the
 * weights draw from counters (.., .., 0, 0) as everywhere else.  Stochastic variants need k_bits <= 8 with 8-bit state
 * (FBSR_ERR_UNSUPPORTED).  Every 400 tensors cost one launch.  Any element alignment is accepted; tensors whose pointers
 * allow it (32 bytes for binary32, 16 for 16-bit, 8 for 8-bit arrays) are read and written eight elements at a time. */
typedef struct {
    float* w;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    void* w_lp;
    uint64_t n, offset;
} fbsr_adamw_tensor;

int fbsr_adamw_multi(const fbsr_adamw_tensor* tensors, size_t count, int state_bits, int g_fmt, int fmt, int variant,
                     int k_bits, uint64_t seed, double lr, double beta1, double beta2, double eps, double weight_decay,
                     int step, const float* grad_scale, void* cuda_stream);

/* fbsr_qat_update -- Algorithm 1, last line, with the sum formed in the 16-bit format as written there:
 *     w16 = value(w8);  s = RTNE_16(fl32(w16 + u16));  w8 = FBSR(s)          (in place on w8)
 *   w8       device, n codes of w_fmt (FBSR_E4M3, FBSR_E5M2 or FBSR_B8P4), read and overwritten
 *   update16 device, n codes of u_fmt (FBSR_BF16 or FBSR_FP16): the update computed in the 16-bit format
 * RTNE_16 rounds to u_fmt with ties to even (saturating); a NaN sum is written as the positive NaN. */
int fbsr_qat_update(void* w8, const void* update16, size_t n, int w_fmt, int u_fmt, int variant, int k_bits,
                    uint64_t seed, uint64_t offset, void* cuda_stream);

/* fbsr_round_host -- fbsr_round for HOST buffers (pinned memory gives overlap):
 * copies src to the device in chunks, rounds, copies the codes back, using
 * dev_workspace (device, >= fbsr_round_host_min_workspace() bytes, 256-byte
 * aligned) as a double buffer.  Kernels are enqueued on cuda_stream, the copies
 * on two internal streams (one per direction, so that the upload of a chunk, the
 * rounding of the previous one and the download of the one before overlap); the
 * uploads wait for what cuda_stream held at the time of the call, and everything
 * is joined back into cuda_stream before return: dst_host is valid once
 * cuda_stream has been synchronised.  Callers on different streams may call
 * concurrently with workspaces of their own. */
size_t fbsr_round_host_min_workspace(void);
int fbsr_round_host(const float* src_host, void* dst_host, size_t n, int fmt, int variant, int k_bits,
                    uint64_t seed, uint64_t offset, float scale, void* dev_workspace,
                    size_t workspace_bytes, void* cuda_stream);

/* A common multiple of the warp-tile sizes the entry points use for k_bits: `offset` values that are
 * multiples of it keep a sharded call on the fast path.  0 if k_bits is invalid. */
size_t fbsr_tile_elements(int k_bits);

/* Number of kernel launches the library has enqueued since it was loaded. */
uint64_t fbsr_launch_count(void);

const char* fbsr_status_string(int status);
int fbsr_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FBSR_H */
