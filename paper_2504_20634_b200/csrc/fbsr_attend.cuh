// What the kernels of fbsr_attend_kv share: the arguments, what a CTA works on, the layout of a tile of codes, scales.
#pragma once
#include <cuda.h>

#include "fbsr_answer.cuh"
#include "fbsr_internal.h"
#include "fbsr_tma.cuh"

namespace fbsr {

constexpr int TILE = 64;                         // tokens of a stage
constexpr float LOWEST = -3.0e38f, HEADROOM = 8.0f;

struct AttendArgs {
    const void* q;
    void* out;
    int64_t q_token, q_head, o_token, o_head;
    const uint8_t* k_codes;
    const uint8_t* v_codes;
    const uint16_t* k_scales;
    const uint16_t* v_scales;
    const int32_t* table;
    int64_t table_ld;
    const int32_t* lengths;
    const int32_t* starts;
    const uint64_t* tree;
    float* part_o;                               // [splits][total * heads][dim]
    float2* part_ml;                             // [splits][total * heads]: maximum, sum
    uint64_t pages;
    int kv_heads, share, page_shift, capacity;      // share: query heads of a cache head; capacity: tokens of a table row
    int total, max_queries, row_tiles, splits, chunk, tree_words;     // chunk: tokens of a split, a multiple of TILE
    Divider by_share;
    int q_whole;                                 // addresses of q are multiples of 16 bytes
    int clustered;                               // the splits of a sequence are a cluster, which joins them
    float scale_log2;
};

template <int DIM, int BITS> struct Layout {
    static constexpr int ROW = DIM * BITS / 8;                 // bytes of a row of codes
    static constexpr int GROUPS = BITS == 8 ? 1 : DIM / 32;
    static constexpr int LINE_ROWS = 128 / ROW;                // rows in 128 bytes: the banks
    static constexpr int CHUNKS = ROW / 16;
    static constexpr int CODES = TILE * ROW;
    static constexpr int SCALES = TILE * GROUPS * 2;
    static constexpr int STAGE = 2 * (CODES + 1024);           // scales in a kilobyte of their own: tiles begin on 1024 bytes
    static constexpr int STAGES = ROW == 128 ? 3 : 5;
    static_assert(SCALES <= 1024, "");
    // Byte of a tile's row at `byte`, as the swizzle puts it: 16-byte chunks of a line of 128 bytes, moved by the line's number.
    static __device__ __forceinline__ int at(int row, int byte)
    {
        const int line = row / LINE_ROWS, chunk = (row % LINE_ROWS) * CHUNKS + (byte >> 4);
        return line * 128 + ((chunk ^ (line & 7)) << 4) + (byte & 15);
    }
    // Which token of sixteen is row r of the left operand, so that the lanes of a load meet different banks: keys are read from rows
    // g, values from rows 2 t (and 2 t + 1, 2 t + 8, 2 t + 9), a piece of each.
    static __device__ __forceinline__ int token(int r)
    {
        if constexpr (LINE_ROWS == 1) return r;
        if constexpr (LINE_ROWS == 2) return (r & 6) * 2 + (r & 1) + (r >> 3) * 2;
        return ((r & 6) >> 1) + (r & 1) * 4 + (r >> 3) * 8;
    }
    template <int NR> static constexpr int shared()
    {
        constexpr int combine = 4 * 8 * NR * (DIM + 4) * 4 + 5 * 8 * NR * 8, ring = STAGES * STAGE;
        return (ring > combine ? ring : combine) + 1024;
    }
};

// 2^x; the largest negative number stands for nothing seen and gives zero.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float log2_fast(float x)
{
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b)
{
    const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}

__device__ __forceinline__ uint32_t half2_of(float lo, float hi)
{
    const __half2 r = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// A token's scales as other lanes read them: what follows, with the rest in binary16.
struct __align__(16) ScaleEntry { float scale; uint16_t rest[4]; };

// A token's scales.  8 bits: its one scale.  4 bits: 2^(largest exponent), and the scales of its groups over that, in binary16.  A
// pattern that is no finite non-negative number makes the scale NaN and the rest zero, so that codes times rest stay finite (a place
// behind the sequence's end may hold anything).
template <int GROUPS> struct RowScale {
    float scale, inv;                            // 4 bits: 2^e, and 2^-e or zero
    uint32_t w[GROUPS > 2 ? 2 : 1];

    __device__ __forceinline__ explicit RowScale(const uint16_t* s)
    {
        if constexpr (GROUPS == 1) {
            scale = bf16_value(*s);
        } else {
            if constexpr (GROUPS == 4) { const uint2 v = *reinterpret_cast<const uint2*>(s); w[0] = v.x; w[1] = v.y; }
            else w[0] = *reinterpret_cast<const uint32_t*>(s);
            uint32_t m = w[0];
            if constexpr (GROUPS == 4) m = __vmaxu2(m, w[1]);
            m = max(m & 0xFFFFu, m >> 16);
            const uint32_t e = m & 0x7F80u;
            const bool sound = m < 0x7F80u;
            scale = sound ? bf16_value(e) : __uint_as_float(0x7FC00000u);
            inv = sound ? __uint_as_float((0x7F00u - e) << 16) : 0.0f;
        }
    }

    __device__ __forceinline__ ScaleEntry entry() const
    {
        uint32_t r[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < GROUPS / 2; ++i)
            r[i] = half2_of(__fmul_rn(bf16_value(w[i] & 0xFFFFu), inv), __fmul_rn(__uint_as_float(w[i] & 0xFFFF0000u), inv));
        if (inv == 0.0f) r[0] = r[1] = 0u;       // zero times what is no number
        ScaleEntry e;
        *reinterpret_cast<uint4*>(&e) = make_uint4(__float_as_uint(scale), r[0], r[1], 0u);
        return e;
    }

    // What multiplies the codes of group `group`, twice.
    __device__ __forceinline__ uint32_t rest(int group) const
    {
        const uint32_t own = w[GROUPS > 2 ? group >> 1 : 0] >> (16 * (group & 1));
        const float r = inv == 0.0f ? 0.0f : __fmul_rn(bf16_value(own & 0xFFFFu), inv);      // zero times what is no number
        return half2_of(r, r);
    }
};

// What a CTA works on.
struct Work {
    int batch, head, first_row, rows;            // rows: of this sequence and cache head; first_row: of this CTA
    int start, queries, length, context;         // query rows [start, start + queries); tokens; the queries' keys begin at context
    int from, to;                                // tokens of this split
    bool beyond;                                 // the length passes the table's end
};

__device__ __forceinline__ Work work_of(const AttendArgs& a, int row_tile, int head, int batch, int split, int tile_rows)
{
    Work w;
    w.batch = batch; w.head = head;
    int start, end;
    if (a.starts != nullptr) {
        start = min(max(a.starts[batch], 0), a.total);
        end = min(max(a.starts[batch + 1], start), a.total);
    } else {
        start = (int)min((int64_t)batch * a.max_queries, (int64_t)a.total);
        end = (int)min((int64_t)start + a.max_queries, (int64_t)a.total);
    }
    w.start = start;
    const int all = end - start;                 // the drafts are this many whether or not all of them are computed
    w.queries = min(all, a.max_queries);
    w.rows = w.queries * a.share;
    w.first_row = row_tile * tile_rows;
    const int length = max(a.lengths[batch], 0);
    w.beyond = length > a.capacity;
    w.length = min(length, a.capacity);
    w.context = length - all;                    // may be negative: such keys do not exist
    w.from = (int)min((int64_t)split * a.chunk, (int64_t)w.length);
    w.to = (int)min((int64_t)w.from + a.chunk, (int64_t)w.length);
    return w;
}

// Chunks that a sequence of `length` tokens has, one at least.  Lengths and chunks together may pass 31 bits.
__device__ __forceinline__ int splits_of(int length, int chunk) { return length > 0 ? (length - 1) / chunk + 1 : 1; }

// The joining kernel may be launched once every CTA has come here; it waits for what they write.
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// A row of queries, or `count` of its elements: bfloat16 ones times a power of two that `score` takes back.
template <int N>
__device__ __forceinline__ void load_query(const uint16_t* p, bool real, uint32_t (&x)[N / 2])
{
    if (real && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
        uint4 v[N / 8];                          // all asked for before the first is used
#pragma unroll
        for (int j = 0; j < N / 8; ++j) v[j] = *reinterpret_cast<const uint4*>(p + 8 * j);
#pragma unroll
        for (int j = 0; j < N / 8; ++j) { x[4 * j] = v[j].x; x[4 * j + 1] = v[j].y; x[4 * j + 2] = v[j].z; x[4 * j + 3] = v[j].w; }
    } else if (real) {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) x[j] = p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
    } else {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) x[j] = 0u;
    }
}

// Largest finite bfloat16 pattern among the elements.
template <int N>
__device__ __forceinline__ uint32_t query_amax(const uint32_t (&x)[N / 2])
{
    uint32_t m = 0u;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) m = __vmaxu2(m, x[j] & 0x7FFF7FFFu);
    m = max(m & 0xFFFFu, m >> 16);
    if (m >= 0x7F80u) {                          // rare: infinities or NaN among them
        m = 0u;
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const uint32_t lo = x[j] & 0x7FFFu, hi = (x[j] >> 16) & 0x7FFFu;
            m = max(m, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
        }
    }
    return m;
}

// bfloat16 to binary16, times the power of two that puts the largest finite element (pattern m) into [2^14, 2^15); what turns a sum of
// products into a score in units of log 2 is divided by it.
template <int N>
__device__ __forceinline__ float query_to_half(uint32_t (&x)[N / 2], uint32_t m, float score)
{
    const int e = max((int)(m >> 7), 1) - 127;                            // exponent of the largest, 127 at most
    const int up = 14 - e;                                                // -113 .. 140, in two factors
    const float f0 = __uint_as_float((uint32_t)(127 + up / 2) << 23), f1 = __uint_as_float((uint32_t)(127 + up - up / 2) << 23);
#pragma unroll
    for (int j = 0; j < N / 2; ++j)
        x[j] = half2_of(__fmul_rn(__fmul_rn(__uint_as_float(x[j] << 16), f0), f1), __fmul_rn(__fmul_rn(__uint_as_float(x[j] & 0xFFFF0000u), f0), f1));
    return __fmul_rn(__fmul_rn(score, __uint_as_float((uint32_t)(127 - up / 2) << 23)), __uint_as_float((uint32_t)(127 - (up - up / 2)) << 23));
}

// The copies of tiles of codes into stages of the ring, by one warp, tile after tile.  A piece is what one copy brings: a page, or 64
// tokens of a larger one.  The table is read for 32 pieces at a time, and those to come are asked for before the present ones are
// used.  All that the warp computes is the same for its lanes, and one of them issues the copies.
template <int DIM, int BITS> struct TileCopy {
    using L = Layout<DIM, BITS>;
    const AttendArgs& a;
    const Work& w;
    const CUtensorMap* k_map;
    const CUtensorMap* v_map;
    const int32_t* table;
    int piece_shift, pieces, now, next;

    __device__ __forceinline__ TileCopy(const AttendArgs& a, const Work& w, const CUtensorMap* k_map, const CUtensorMap* v_map)
        : a(a), w(w), k_map(k_map), v_map(v_map), table(a.table + w.batch * a.table_ld), piece_shift(min(a.page_shift, 6)), pieces(TILE >> piece_shift),
          now(-2), next(-2) {}

    __device__ __forceinline__ void start() { next = pages_from(0); }

    // The page of piece `first` + lane; -1: one that the cache does not have; -2: nothing to copy.
    __device__ __forceinline__ int pages_from(int first) const
    {
        const int64_t token = w.from + ((int64_t)(first + (threadIdx.x & 31)) << piece_shift);
        if (token >= w.to) return -2;
        const int p = table[token >> a.page_shift];
        return (uint32_t)p < a.pages ? p : -1;
    }

    // `bad`, a word of shared memory, receives a bit for each piece on a page that the cache does not have.
    __device__ __forceinline__ void operator()(int tile, uint32_t stage, uint32_t bar, uint32_t* bad)
    {
        const int first = tile * pieces, in = first & 31, tokens = 1 << piece_shift;
        if (in == 0) { now = next; next = pages_from(first + 32); }
        const uint32_t these = (pieces == 8 ? 0xFFu : (1u << pieces) - 1u) << in;
        const uint32_t real = (__ballot_sync(0xFFFFFFFFu, now >= 0) & these) >> in, missing = (__ballot_sync(0xFFFFFFFFu, now == -1) & these) >> in;
        if (elected()) {
            *bad = missing;
            barrier_expect(bar, __popc(real) * tokens * 2 * (L::ROW + L::GROUPS * 2));
        }
        __syncwarp();
#pragma unroll 1
        for (int piece = 0; piece < pieces; ++piece) {
            const int page = __shfl_sync(0xFFFFFFFFu, now, in + piece);
            if (page < 0) continue;
            const int token = w.from + ((first + piece) << piece_shift);
            const int64_t row = (((int64_t)page * a.kv_heads + w.head) << a.page_shift) + (token & ((1 << a.page_shift) - 1));
            const uint32_t to = stage + (piece << piece_shift) * L::ROW, scales = stage + 2 * L::CODES + (piece << piece_shift) * L::GROUPS * 2;
            if (elected()) {
                copy_box(to, k_map, bar, 0, (int)(row / L::LINE_ROWS));
                copy_box(to + L::CODES, v_map, bar, 0, (int)(row / L::LINE_ROWS));
                copy_bytes(scales, a.k_scales + row * L::GROUPS, tokens * L::GROUPS * 2, bar);
                copy_bytes(scales + 1024, a.v_scales + row * L::GROUPS, tokens * L::GROUPS * 2, bar);
            }
            __syncwarp();
        }
    }
};

// Eight elements of partial sums, times f, added to v.
__device__ __forceinline__ void add_scaled(const float* from, float f, float (&v)[8])
{
    const float4 x = reinterpret_cast<const float4*>(from)[0], y = reinterpret_cast<const float4*>(from)[1];
    v[0] = __fmaf_rn(x.x, f, v[0]); v[1] = __fmaf_rn(x.y, f, v[1]); v[2] = __fmaf_rn(x.z, f, v[2]); v[3] = __fmaf_rn(x.w, f, v[3]);
    v[4] = __fmaf_rn(y.x, f, v[4]); v[5] = __fmaf_rn(y.y, f, v[5]); v[6] = __fmaf_rn(y.z, f, v[6]); v[7] = __fmaf_rn(y.w, f, v[7]);
}

// Sums over the sum of the weights, rounded once; zeros where nothing was seen.
template <int DIM, bool BF16Q>
__device__ __forceinline__ void write_result(const AttendArgs& a, int query, int head, int octet, float l, float (&v)[8])
{
    const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = __fmul_rn(v[c], inv);
    const int64_t at = (int64_t)query * a.o_token + head * a.o_head + octet * 8;
    const bool whole = (reinterpret_cast<uintptr_t>(a.out) + 2 * at) % 16 == 0;
    store8<BF16Q ? FBSR_BF16 : FBSR_FP16>(a.out, at, 8, whole, v);
}

// The ROWS rows of a CTA joined from PARTS partial sums that lie ROWS rows apart in shared memory (rows of DIM + 4 numbers, maxima
// and sums beside) by COUNT threads; put(r, octet, m, l, v) takes eight elements of row r with its maximum and sum.
template <int DIM, int ROWS, int PARTS, int COUNT, class Put>
__device__ __forceinline__ void join_parts(const Work& w, const float* so, const float2* sml, int thread, const Put& put)
{
    constexpr int OCTETS = DIM / 8, PITCH = DIM + 4;
#pragma unroll 1
    for (int i = thread; i < ROWS * OCTETS; i += COUNT) {
        const int r = i / OCTETS, octet = i % OCTETS;
        if (w.first_row + r >= w.rows) break;
        float m = LOWEST;
#pragma unroll
        for (int n = 0; n < PARTS; ++n) m = fmaxf(m, sml[n * ROWS + r].x);
        float l = 0.0f, v[8] = {};
#pragma unroll
        for (int n = 0; n < PARTS; ++n) {
            const float2 ml = sml[n * ROWS + r];
            const float f = exp2_fast(__fsub_rn(ml.x, m));
            l = __fmaf_rn(ml.y, f, l);
            add_scaled(so + (n * ROWS + r) * PITCH + octet * 8, f, v);
        }
        put(r, octet, m, l, v);
    }
}

// The same, written out, or as a split's share to the workspace.
template <int DIM, bool BF16Q, int ROWS, int PARTS, int COUNT>
__device__ __forceinline__ void write_rows(const AttendArgs& a, const Work& w, int split, const float* so, const float2* sml, int thread)
{
    join_parts<DIM, ROWS, PARTS, COUNT>(w, so, sml, thread, [&](int r, int octet, float m, float l, float (&v)[8]) {
        const int row = w.first_row + r, qi = (int)divide((uint32_t)row, a.by_share), head = w.head * a.share + row - qi * a.share;
        if (a.splits == 1) {
            write_result<DIM, BF16Q>(a, w.start + qi, head, octet, l, v);
        } else {
            const int64_t at = ((int64_t)split * a.total + w.start + qi) * (a.kv_heads * a.share) + head;
            float4* dst = reinterpret_cast<float4*>(a.part_o + at * DIM + octet * 8);
            dst[0] = make_float4(v[0], v[1], v[2], v[3]);
            dst[1] = make_float4(v[4], v[5], v[6], v[7]);
            if (octet == 0) a.part_ml[at] = make_float2(m, l);
        }
    });
}

// Kernels of many rows (more than 16 for a head of the cache): fbsr_attend_rows.cu.  `copies`: how often the rows are repeated along
// the 128 lanes of a tile, 1, 2 or 4.
int attend_rows(const AttendArgs& a, const CUtensorMap& k_map, const CUtensorMap& v_map, int dim, int bits, bool bf16, int copies, size_t batch, cudaStream_t stream);

}  // namespace fbsr
