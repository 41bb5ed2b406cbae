// fbsr_attend_kv for many rows (queries x heads that share a head of the cache, more than 16): trees of drafted tokens.
//
// The same single pass on the fifth-generation matrix unit.  128 rows of queries are the lanes of tensor memory: a thread owns a
// row, so that a softmax needs no shuffle.  One warp copies tiles of 64 tokens' codes (TMA), four widen the keys' and four the values' to
// binary16 in the layout that the unit reads (two warps the even tiles, two the odd ones), one or two threads issue the products, and two
// groups of four warps (a thread a row) make weights of scores, each of every other tile and with sums of its own.  Queries and weights
// are left operands out of tensor memory, so only widened codes pass through shared memory: 16 KB each of keys and values a tile,
// written once and read once, where queries in shared memory would be read again for every tile.
//
//     S = Q K^T (128 x 64), keys with their elements along k;   O += P V (128 x dim), values with their tokens along k: the same rows
//     of 128 bytes as the keys, read as the transposed operand.
//
// The products of a tile, the softmax of two others and the widening of the next run side by side, with two of S, P and O and three or
// four of the widened keys and values: what one stage waits for is then two or three tiles old.  (With two of everything and one
// group of widening warps for both, a tile took 3000 clocks, whichever stage was left out.)
//
// Fewer rows.  Up to 32 (64) rows are laid along the lanes four times (twice), and each copy takes every fourth (second) tile of its
// group: its warps alone make weights of it, and the other lanes of O are left out of the product.  So the softmax, which bounds the
// work of a full tile of rows, stays spread over all four schedulers.  Groups and copies are joined at the end like the chunks of a sequence.
//
// So a copy's lanes of S, P and O are written by the products of its own tiles alone, and up to eight tiles are between scores and sums.
//
// What bounds it.  A tile of 64 tokens of dim 128 takes 1350 clocks with 128 rows (the softmax of two warps a scheduler: 512 for the
// exponentials, the rest for their instructions and waits), 870 with 24 (the products need 440; a warp that issues both kinds
// needs 1000).  Start and end of a CTA take 7 us.  65536 tokens of 8 heads in 8 bits with 128 rows: 52 us, of which the products are 20.7 and
// the bytes 20.9; 131000 tokens of 4 heads with 40 rows: 40 us, and 45 with the joining, of 20.9.  No unit is saturated: issue slots 59 and 57 %, the
// product unit 38 and 51 %, the exponential unit 39 and 27 %, memory 34 and 46 %.
//
// Scales and weights are as in fbsr_attend_kv.cu; a row's maximum moves only when a weight would pass 2^15, and then the row of O is
// read, scaled and written back by its thread.
#include "fbsr_attend.cuh"

namespace fbsr {
namespace {

// Warps 0..7 softmax, 8..11 keys, 12..15 values, then one each; the last only fills its group of four.  Registers are moved to the
// softmax, which holds 64 scores and 32 pairs of weights: 256 x 152 + 256 x 64 + 128 x 48 = 61440, the 640 x 96 that the launch has.
constexpr int THREADS = 640, WIDEN_WARP = 8, COPY_WARP = 16, PRODUCT_WARP = 17, SUM_WARP = 18;
constexpr int KEYS = 3;                          // widened tiles of the keys

// Tensor memory: columns of 32 bits.
constexpr int COL_S = 0, COL_O = 128, COL_Q = 384, COL_P = 448, COLUMNS = 512;      // two of S (64 each), O (128) and P (32)

template <int DIM, int BITS> struct Rows {
    using L = Layout<DIM, BITS>;
    // Tiles of codes, and widened tiles of the values.  The ring of codes is what keeps enough bytes under way (rows of 128 bytes, 24 rows of
    // queries, 12000 tokens: 98 us with six and three, 109 with four and four).
    static constexpr int STAGES = 6, VALUES = L::ROW == 128 ? 3 : 4;
    static_assert(STAGES % 2 == 0, "a warp that widens sees every second tile, and has to see every round of a stage");
    static constexpr int WIDE = TILE * DIM * 2;                // bytes of a widened tile: blocks of 64 elements, [64 tokens][128 bytes]
    static constexpr int RING = STAGES * L::STAGE, K_AT = RING, V_AT = K_AT + KEYS * WIDE, END = V_AT + VALUES * WIDE;
    static constexpr int COMBINE = 256 * (DIM + 4) * 4 + 256 * 8;
    static constexpr int SHARED = (END > COMBINE ? END : COMBINE) + 1024;
};

// Descriptors of rows of 128 bytes in the 128-byte swizzle, eight rows (1024 bytes) to a group: k along the rows' bytes, or along the
// rows (then the next 64 elements of the other dimension lie a block of 64 rows on).
__device__ __forceinline__ uint64_t along_bytes(uint32_t address)
{
    return (uint64_t)((address & 0x3FFFFu) >> 4) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

__device__ __forceinline__ uint64_t along_rows(uint32_t address)
{
    return (uint64_t)((address & 0x3FFFFu) >> 4) | (uint64_t)(TILE * 128 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// 128 x N x 16 of binary16, sums in binary32; the left operand in tensor memory.  Lanes whose bit in `off` is set are left as they are.
template <int N, bool TRANSPOSED>
__device__ __forceinline__ void product(uint32_t d, uint32_t a, uint64_t b, bool add, const uint32_t (&off)[4])
{
    constexpr uint32_t KIND = 1u << 4 | (TRANSPOSED ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (128u >> 4) << 24;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %6, %7, %8}, p;\n\t}"
                 :: "r"(d), "r"(a), "l"(b), "r"(KIND), "r"((uint32_t)add), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]) : "memory");
}

__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}

__device__ __forceinline__ void arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}

#define FBSR_32(v) \
    v(0), v(1), v(2), v(3), v(4), v(5), v(6), v(7), v(8), v(9), v(10), v(11), v(12), v(13), v(14), v(15), \
    v(16), v(17), v(18), v(19), v(20), v(21), v(22), v(23), v(24), v(25), v(26), v(27), v(28), v(29), v(30), v(31)
#define FBSR_LIST32 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}"

// 32 columns of this warp's 32 lanes; loads and stores are waited for by the caller.
__device__ __forceinline__ void load32(uint32_t address, float* x)
{
#define FBSR_OUT(i) "=f"(x[i])
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " FBSR_LIST32 ", [%32];" : FBSR_32(FBSR_OUT) : "r"(address) : "memory");
#undef FBSR_OUT
}

__device__ __forceinline__ void store32(uint32_t address, const uint32_t* x)
{
#define FBSR_IN(i) "r"(x[i])
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], " FBSR_LIST32 ";" :: FBSR_32(FBSR_IN), "r"(address) : "memory");
#undef FBSR_IN
}

__device__ __forceinline__ void loads_done() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// Two binary32 numbers as one operand.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}

__device__ __forceinline__ void parts_of(uint64_t p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Which of the 64 tokens from `first` on a row's query sees: a bit each.
__device__ __forceinline__ uint64_t seen_by(const AttendArgs& a, const Work& w, int first, int query)
{
    if (query < 0) return 0ull;
    const int draft = first - w.context;         // of the first token; negative: the context
    auto drafts_from = [&](int j) -> uint64_t {  // bits of drafts j .. j + 63
        if (a.tree == nullptr) {
            const int n = query - j + 1;
            return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
        }
        const uint64_t* row = a.tree + (int64_t)(w.start + query) * a.tree_words;
        const int word = j >> 6, shift = j & 63;
        const uint64_t lo = word < a.tree_words ? row[word] : 0ull, hi = shift != 0 && word + 1 < a.tree_words ? row[word + 1] : 0ull;
        return shift == 0 ? lo : lo >> shift | hi << (64 - shift);
    };
    uint64_t seen = draft <= -64 ? ~0ull : draft < 0 ? ((1ull << -draft) - 1) | drafts_from(0) << -draft : drafts_from(draft);
    const int left = w.to - first;
    if (left < 64) seen &= (1ull << left) - 1;
    return seen;
}

template <int DIM, int BITS, int COPIES, bool BF16Q>
__global__ void __launch_bounds__(THREADS, 1)
attend_rows_kv_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    using L = Layout<DIM, BITS>;
    using R = Rows<DIM, BITS>;
    constexpr int GROUP_ROWS = 128 / COPIES, GROUP_WARPS = 4 / COPIES, AHEAD = COPIES == 1 ? 2 : 4;
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t bars[2 * R::STAGES + 6 * 8 + 2];
    __shared__ __align__(16) float k_scale[8][TILE], v_scale[8][TILE], v_log[8][TILE];       // v_log: log2 of v_scale, -60 at least
    __shared__ float row_score[128];
    __shared__ uint32_t bad_pieces[R::STAGES], tensor_memory;
    const uint32_t base = (shared_address(dynamic) + 1023u) & ~1023u;
    uint8_t* const shared = dynamic + (base - shared_address(dynamic));
    const uint32_t full = shared_address(bars), empty = full + 8 * R::STAGES;             // codes
    // Eight barriers of each kind, tile i the (i mod 8)-th: the softmax warps of a copy wait for their own tiles alone, every eighth
    // at most, and a barrier that served others in between could not tell them a phase from the one two before.
    const uint32_t keys_wide = empty + 8 * R::STAGES, values_wide = keys_wide + 64, scored = values_wide + 64, taken = scored + 64;
    const uint32_t weighed = taken + 64, summed = weighed + 64, finished = summed + 64, asked = finished + 8;
    auto wait = [](uint32_t kind, int i) { return barrier_wait(kind + 8 * (i & 7), (i >> 3) & 1); };
    const int warp = warp_number(), lane = threadIdx.x & 31;
    let_next_kernel_start();

    uint32_t block = blockIdx.x;
    const int split = block % a.splits; block /= a.splits;
    const int row_tile = block % a.row_tiles; block /= a.row_tiles;
    const int kv_head = block % a.kv_heads;
    const Work w = work_of(a, row_tile, kv_head, block / a.kv_heads, split, GROUP_ROWS);
    if (w.first_row >= w.rows || (split > 0 && w.from >= w.to)) return;
    const int tiles = (w.to - w.from + TILE - 1) / TILE;

    TileCopy<DIM, BITS> copy(a, w, &k_map, &v_map);
    if (warp == COPY_WARP) {
        copy.start();
        if (lane < R::STAGES) { barrier_init(full + 8 * lane, 1); barrier_init(empty + 8 * lane, 4); }
        if (lane < 8) {
            barrier_init(keys_wide + 8 * lane, 2); barrier_init(values_wide + 8 * lane, 2);
            barrier_init(scored + 8 * lane, 1); barrier_init(summed + 8 * lane, 1);
            barrier_init(taken + 8 * lane, GROUP_WARPS); barrier_init(weighed + 8 * lane, GROUP_WARPS);
        }
        if (lane == 0) { barrier_init(finished, 1); barrier_init(asked, 4); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == PRODUCT_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(shared_address(&tensor_memory)), "n"(COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tm = tensor_memory;

    if (warp >= COPY_WARP) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        if (warp == COPY_WARP) {
            bool fine = true;
            for (int i = 0, s = 0, round = 0; i < tiles; ++i) {
                if (round > 0) fine = warp_wait(empty + 8 * s, (round - 1) & 1);
                if (!fine) break;                              // the others give up too
                copy(i, base + s * L::STAGE, full + 8 * s, bad_pieces + s);
                if (++s == R::STAGES) { s = 0; ++round; }
            }
        } else if (warp <= SUM_WARP) {
            auto all_wait = [](uint32_t kind, int i) { return warp_wait(kind + 8 * (i & 7), (i >> 3) & 1); };
            auto others = [](int i, uint32_t (&off)[4]) {      // the lanes whose tile i is not
#pragma unroll
                for (int q = 0; q < 4; ++q) off[q] = q / GROUP_WARPS == (i >> 1) % COPIES ? 0u : 0xFFFFFFFFu;
            };
            bool fine = tiles == 0 || warp_wait(asked, 0);
            auto score = [&](int i) {            // S = Q K^T of tile i
                if (fine) fine = all_wait(keys_wide, i);
                // S has been read.  With copies the lanes of S are free for longer, and it is the scales of four tiles before that have
                // to be: what the ring of scales takes next is written over them.
                if (fine && i >= AHEAD) fine = all_wait(COPIES == 1 ? taken : weighed, i - AHEAD);
                if (!fine) return;
                after_sync();
                uint32_t off[4];
                others(i, off);
                const uint64_t keys = along_bytes(base + R::K_AT + i % KEYS * R::WIDE);
                if (elected()) {
#pragma unroll
                    for (int j = 0; j < DIM / 16; ++j)         // 16 elements: 32 bytes, or the next block of 64
                        product<TILE, false>(tm + COL_S + (i & 1) * TILE, tm + COL_Q + 8 * j, keys + j / 4 * (TILE * 128 / 16) + 2 * (j % 4), j > 0, off);
                    commit(scored + 8 * (i & 7));
                }
                __syncwarp();
            };
            auto sum_up = [&](int i) {           // O += P V of tile i
                if (fine) fine = all_wait(values_wide, i);
                if (fine) fine = all_wait(weighed, i);
                if (!fine) return;
                after_sync();
                uint32_t off[4];
                others(i, off);
                const uint64_t values = along_rows(base + R::V_AT + i % R::VALUES * R::WIDE);
                if (elected()) {
#pragma unroll
                    for (int j = 0; j < TILE / 16; ++j)        // 16 tokens: 2048 bytes
                        product<DIM, true>(tm + COL_O + (i & 1) * 128, tm + COL_P + (i & 1) * (TILE / 2) + 8 * j, values + 128 * j, i >= 2 * COPIES || j > 0, off);
                    commit(summed + 8 * (i & 7));
                }
                __syncwarp();
            };
            // One warp spends 1000 clocks on a tile's waits and products.  With copies that bounds the tile, and each product has a warp
            // (131000 tokens, 40 rows, 8 bits: 45 us against 51); without, the softmax does, and scores that run ahead of the sums
            // delay it (128 rows: 55 us against 53): the sums follow two tiles behind the scores in one warp.
            if (warp == PRODUCT_WARP) {
                for (int i = 0; i < tiles && fine; ++i) {
                    score(i);
                    if (COPIES == 1 && i >= 2) sum_up(i - 2);
                }
            }
            if (warp == (COPIES == 1 ? PRODUCT_WARP : SUM_WARP)) {
                for (int i = COPIES == 1 ? max(tiles - 2, 0) : 0; i < tiles && fine; ++i) sum_up(i);
                if (tiles > 0 && fine && elected()) commit(finished);
            }
        }
    } else if (warp >= WIDEN_WARP) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ---- widening: a thread has a token, of the keys or of the values; two warps have the even tiles and two the odd ones
        const bool v = warp >= WIDEN_WARP + 4;
        const int token = threadIdx.x & 63;
        constexpr int HALF = DIM / 2, BYTES = HALF * BITS / 8;                   // elements at a time; bytes of codes
        const int piece_shift = min(a.page_shift, 6);
        bool fine = true;
        for (int i = (warp >> 1) & 1; i < tiles; i += 2) {
            const int s = i % R::STAGES, round = i / R::STAGES;
            if (fine) fine = barrier_wait(full + 8 * s, round & 1);
            const uint8_t* codes = shared + s * L::STAGE;
            const RowScale<L::GROUPS> scale(reinterpret_cast<const uint16_t*>(codes + 2 * L::CODES) + (v ? 512 : 0) + token * L::GROUPS);
            const uint32_t bad = bad_pieces[s];
            float number = scale.scale;
            bool nothing = false, missing = false;
            if (bad != 0u || w.to - w.from - i * TILE < TILE) {
                // what was not copied, or lies behind the end, may be anything: a weight of zero must make nothing of it
                missing = (bad >> (token >> piece_shift)) & 1;
                nothing = missing || w.from + i * TILE + token >= w.to;
                if (missing) number = __uint_as_float(0x7FC00000u);
            }
            uint8_t* to = shared + (v ? R::V_AT + i % R::VALUES * R::WIDE : R::K_AT + i % KEYS * R::WIDE) + token * 128;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint4 u[BYTES / 16];
#pragma unroll
                for (int c = 0; c < BYTES / 16; ++c) {
                    u[c] = *reinterpret_cast<const uint4*>(codes + (v ? L::CODES : 0) + L::at(token, half * BYTES + 16 * c));
                    if (nothing) u[c] = make_uint4(0u, 0u, 0u, 0u);
                }
                if (half == 0) {
                    // the products that read what is written over
                    if (!v && fine && i >= KEYS) fine = wait(scored, i - KEYS);
                    if (v && fine && i >= R::VALUES) fine = wait(summed, i - R::VALUES);
                    if (v && fine && i >= R::VALUES - 16384 / R::WIDE && i < R::VALUES) fine = barrier_wait(asked, 0);     // where the queries passed
                    if (!v) {
                        const RowScale<L::GROUPS> of_value(reinterpret_cast<const uint16_t*>(codes + 2 * L::CODES) + 512 + token * L::GROUPS);
                        const float value = missing ? number : of_value.scale;
                        k_scale[i & 7][token] = number; v_scale[i & 7][token] = value; v_log[i & 7][token] = fmaxf(log2_fast(value), -60.0f);
                    }
                }
#pragma unroll
                for (int c = 0; c < BYTES / 16; ++c) {
                    const uint32_t word[4] = {u[c].x, u[c].y, u[c].z, u[c].w};
                    const int element = half * HALF + c * 128 / BITS;
                    uint8_t* block = to + element / 64 * (TILE * 128);
                    const int chunk = element % 64 / 8;        // of eight elements
                    if constexpr (BITS == 8) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            uint4 o;
                            e4m3_word_to_half2(word[2 * q], o.x, o.y);
                            e4m3_word_to_half2(word[2 * q + 1], o.z, o.w);
                            *reinterpret_cast<uint4*>(block + (((chunk + q) ^ (token & 7)) << 4)) = o;
                        }
                    } else {
                        const uint32_t r = scale.rest(element / 32);             // sixteen bytes are a group of 32
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint32_t h[4];
                            e2m1_word_to_half2(word[q], h);
                            *reinterpret_cast<uint4*>(block + (((chunk + q) ^ (token & 7)) << 4)) =
                                make_uint4(mul_half2(h[0], r), mul_half2(h[1], r), mul_half2(h[2], r), mul_half2(h[3], r));
                        }
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) { arrive(empty + 8 * s); arrive((v ? values_wide : keys_wide) + 8 * (i & 7)); }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
        // ---- softmax: a thread has a row.  Queries into tensor memory first: rows are read by neighbouring lanes, by way of
        // the last 16 KB of the widened values (a thread that read its own row from memory took 5000 clocks)
        const int my_row = w.first_row + threadIdx.x % GROUP_ROWS;
        const int query = my_row < w.rows ? (int)divide((uint32_t)my_row, a.by_share) : -1;
        if (warp < 4) {
            uint8_t* const stage = shared + R::END - 16384;    // [128 rows][128 bytes], swizzled
            uint32_t x[DIM / 2];
            const uint16_t* from[8];                           // eight lanes a row, four rows an instruction
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = w.first_row + (warp * 32 + i * 4 + (lane >> 3)) % GROUP_ROWS;
                const int qi = (int)divide((uint32_t)min(row, w.rows - 1), a.by_share), head = kv_head * a.share + min(row, w.rows - 1) - qi * a.share;
                from[i] = static_cast<const uint16_t*>(a.q) + (int64_t)(w.start + qi) * a.q_token + head * a.q_head + (lane & 7) * 8;
            }
            uint4 y[DIM / 64][8];
            if (a.q_whole) {
#pragma unroll
                for (int h = 0; h < DIM / 64; ++h)
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[h][i] = *reinterpret_cast<const uint4*>(from[i] + h * 64);      // all in flight at once
            } else {
#pragma unroll
                for (int h = 0; h < DIM / 64; ++h)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint16_t* e = from[i] + h * 64;
                        y[h][i] = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
                    }
            }
#pragma unroll
            for (int h = 0; h < DIM / 64; ++h) {               // 64 elements of each row at a time
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = warp * 32 + i * 4 + (lane >> 3);
                    *reinterpret_cast<uint4*>(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4)) = y[h][i];
                }
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint4 u = *reinterpret_cast<const uint4*>(stage + threadIdx.x * 128 + ((c ^ (threadIdx.x & 7)) << 4));
                    const bool real = query >= 0;
                    x[32 * h + 4 * c] = real ? u.x : 0u; x[32 * h + 4 * c + 1] = real ? u.y : 0u;
                    x[32 * h + 4 * c + 2] = real ? u.z : 0u; x[32 * h + 4 * c + 3] = real ? u.w : 0u;
                }
                __syncwarp();
            }
            float score = a.scale_log2;
            if constexpr (BF16Q) score = query_to_half<DIM>(x, query_amax<DIM>(x), score);
            row_score[threadIdx.x] = score;
#pragma unroll
            for (int c = 0; c < DIM / 2; c += 32) store32(tm + COL_Q + c + ((uint32_t)warp << 21), x + c);
            stores_done();
            before_sync();
            __syncwarp();
            if (lane == 0) arrive(asked);
        }
        if (tiles > 0) barrier_wait(asked, 0);
        const float to_score = row_score[threadIdx.x & 127];
        const uint32_t lanes = (uint32_t)(warp & 3) << 21, b = warp >> 2;        // b: which of S, O and P
        const int first_tile = (int)b + 2 * ((warp & 3) / GROUP_WARPS);
        float top = LOWEST, sum = w.beyond ? __uint_as_float(0x7FC00000u) : 0.0f;
        bool fine = true;
        for (int i = first_tile; i < tiles; i += 2 * COPIES) {
            if (fine) fine = wait(scored, i);
            if (fine) fine = wait(keys_wide, i);                                 // the scales
            after_sync();
            float x[TILE];
            load32(tm + COL_S + b * TILE + lanes, x);
            load32(tm + COL_S + b * TILE + 32 + lanes, x + 32);
            loads_done();
            if constexpr (COPIES == 1) {
                before_sync();
                __syncwarp();
                if (lane == 0) arrive(taken + 8 * (i & 7));
            }
            const int first = w.from + i * TILE;
            const bool masked = first + TILE > min(w.context, w.to);
            const uint64_t seen = masked ? seen_by(a, w, first, query) : ~0ull;
            const float* ks = k_scale[i & 7];
            const float* vs = v_scale[i & 7];
            const float* vl = v_log[i & 7];
            // two scores an instruction; both factors first, since a sum of products times one of them may be out of range
            const uint64_t to_score2 = pair_of(to_score, to_score);
#pragma unroll
            for (int c = 0; c < TILE; c += 4) {
                const ulonglong2 k2 = *reinterpret_cast<const ulonglong2*>(ks + c);
                parts_of(mul2(pair_of(x[c], x[c + 1]), mul2(to_score2, k2.x)), x[c], x[c + 1]);
                parts_of(mul2(pair_of(x[c + 2], x[c + 3]), mul2(to_score2, k2.y)), x[c + 2], x[c + 3]);
            }
            if (masked) {
#pragma unroll
                for (int c = 0; c < TILE; ++c)
                    if (!((seen >> c) & 1)) x[c] = -__uint_as_float(0x7F800000u);
            }
            float m = top;
#pragma unroll
            for (int c = 0; c < TILE; c += 4) {
                const ulonglong2 l2 = *reinterpret_cast<const ulonglong2*>(vl + c);
                float w0, w1, w2, w3;
                parts_of(add2(pair_of(x[c], x[c + 1]), l2.x), w0, w1);
                parts_of(add2(pair_of(x[c + 2], x[c + 3]), l2.y), w2, w3);
                m = fmaxf(fmaxf(m, w0), w1);
                m = fmaxf(fmaxf(m, w2), w3);
            }
            // P is free, and O at rest, once the products of the group's last tile are done
            if (fine && i >= 2 * COPIES) fine = wait(summed, i - 2 * COPIES);
            after_sync();
            if (__any_sync(0xFFFFFFFFu, m > __fadd_rn(top, 15.0f - HEADROOM))) {
                const float f = exp2_fast(__fsub_rn(top, m));
                top = m;
                sum = __fmul_rn(sum, f);
                if (i >= 2 * COPIES) {
#pragma unroll 1
                    for (int c = 0; c < DIM; c += 32) {
                        float o[32];
                        load32(tm + COL_O + b * 128 + c + lanes, o);
                        loads_done();
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = __fmul_rn(o[j], f);
                        store32(tm + COL_O + b * 128 + c + lanes, reinterpret_cast<const uint32_t*>(o));
                    }
                    stores_done();
                }
            }
            const float lift = __fsub_rn(HEADROOM, top);
            const uint64_t lift2 = pair_of(lift, lift);
            uint32_t p[TILE / 2];
            uint64_t parts[2] = {0ull, 0ull};
#pragma unroll
            for (int c = 0; c < TILE; c += 4) {
                const ulonglong2 v2 = *reinterpret_cast<const ulonglong2*>(vs + c);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float lo, hi;
                    parts_of(add2(pair_of(x[c + 2 * j], x[c + 2 * j + 1]), lift2), lo, hi);
                    const uint64_t e = pair_of(exp2_fast(lo), exp2_fast(hi));
                    parts[j] = add2(parts[j], e);
                    parts_of(mul2(e, j ? v2.y : v2.x), lo, hi);
                    p[c / 2 + j] = half2_of(lo, hi);
                }
            }
            if (masked) {                        // a weight of zero times a scale that is no number
#pragma unroll
                for (int c = 0; c < TILE / 2; ++c) {
                    if (!((seen >> (2 * c)) & 1)) p[c] &= 0xFFFF0000u;
                    if (!((seen >> (2 * c + 1)) & 1)) p[c] &= 0x0000FFFFu;
                }
            }
            {
                float lo, hi;
                parts_of(add2(parts[0], parts[1]), lo, hi);
                sum = __fadd_rn(sum, __fadd_rn(lo, hi));
            }
            store32(tm + COL_P + b * (TILE / 2) + lanes, p);
            stores_done();
            before_sync();
            __syncwarp();
            if (lane == 0) arrive(weighed + 8 * (i & 7));
        }
        // ---- the rows of O into shared memory, whose tiles have all been read, and out
        if (tiles > 0 && fine) fine = barrier_wait(finished, 0);
        after_sync();
        if (!fine) sum = __uint_as_float(0x7FC00000u);                           // a copy or a product that never came
        float* so = reinterpret_cast<float*>(shared);
        float2* sml = reinterpret_cast<float2*>(so + 256 * (DIM + 4));
        const bool some = first_tile < tiles;    // otherwise nothing has been written to this row of O
#pragma unroll 1
        for (int c = 0; c < DIM; c += 32) {
            float o[32];
            load32(tm + COL_O + b * 128 + c + lanes, o);
            loads_done();
            float4* to = reinterpret_cast<float4*>(so + threadIdx.x * (DIM + 4) + c);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                to[j] = some ? make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        sml[threadIdx.x] = make_float2(top, sum);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        write_rows<DIM, BF16Q, GROUP_ROWS, 2 * COPIES, 256>(a, w, split, so, sml, threadIdx.x);
    }
    __syncwarp();
    before_sync();
    __syncthreads();
    if (warp == PRODUCT_WARP) {
        after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tm), "n"(COLUMNS));
    }
}

template <int DIM, int BITS, int COPIES, bool BF16Q>
int launch(const AttendArgs& a, const CUtensorMap& k_map, const CUtensorMap& v_map, uint64_t grid, cudaStream_t stream)
{
    static std::atomic<uint64_t> asked{0};
    const auto kernel = attend_rows_kv_kernel<DIM, BITS, COPIES, BF16Q>;
    constexpr int SHARED = Rows<DIM, BITS>::SHARED;
    if (allow_shared_memory(reinterpret_cast<const void*>(kernel), SHARED, asked) != FBSR_OK) return FBSR_ERR_CUDA;
    kernel<<<(unsigned)grid, THREADS, SHARED, stream>>>(a, k_map, v_map);
    count_launch();
    return FBSR_OK;
}

template <int DIM, int BITS, bool BF16Q>
int launch_copies(const AttendArgs& a, const CUtensorMap& k_map, const CUtensorMap& v_map, int copies, uint64_t grid, cudaStream_t stream)
{
    return copies == 4 ? launch<DIM, BITS, 4, BF16Q>(a, k_map, v_map, grid, stream) : copies == 2 ? launch<DIM, BITS, 2, BF16Q>(a, k_map, v_map, grid, stream)
                                                                                                   : launch<DIM, BITS, 1, BF16Q>(a, k_map, v_map, grid, stream);
}

}  // namespace

int attend_rows(const AttendArgs& a, const CUtensorMap& k_map, const CUtensorMap& v_map, int dim, int bits, bool bf16, int copies, size_t batch, cudaStream_t stream)
{
    const uint64_t grid = (uint64_t)batch * a.kv_heads * a.row_tiles * a.splits;
    if (grid > 0x7FFFFFFFu) return FBSR_ERR_TOO_LARGE;
#define FBSR_ROWS(d, b) \
    if (dim == d && bits == b) \
        return bf16 ? launch_copies<d, b, true>(a, k_map, v_map, copies, grid, stream) : launch_copies<d, b, false>(a, k_map, v_map, copies, grid, stream);
    FBSR_ROWS(128, 8) FBSR_ROWS(128, 4) FBSR_ROWS(64, 8) FBSR_ROWS(64, 4)
#undef FBSR_ROWS
    return FBSR_ERR_UNSUPPORTED;
}

}  // namespace fbsr
