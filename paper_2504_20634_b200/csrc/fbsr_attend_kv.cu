// fbsr_attend_kv: attention of drafted tokens over a few-bit cache.  The arithmetic is stated in include/fbsr.h.
//
// One pass over the cache with the running maximum and sum of a softmax.  A row is one head of one query; the rows that share a
// head of the cache (queries x heads per cache head) go through the matrix unit together (mma.sync m16n8k16, binary16 operands from
// decoded codes, binary32 sums).  Sixteen tokens are the LEFT operand of the first product and sixteen elements of their values that
// of the second, eight rows the right one: codes are decoded once for all rows of a warp, and eight rows (one token of a model
// that shares a cache head among eight) waste nothing.  A CTA of four warps takes one chunk of a sequence's tokens: WR warps along
// the rows, 8 NR of them each, and 4 / WR along the tokens, with a maximum and sum of their own, joined through shared memory at
// the end.  Chunks of one sequence are joined by their cluster or by a second kernel, in a fixed order.
//
// Tiles of 64 tokens come by TMA, a page (or 64 tokens of it) a copy, in the 128-byte swizzle.
//
// Operand layout without a shuffle or a transpose of halves.  The order of a contraction is free, so lane t of a quad takes the
// contiguous dim / 4 elements [t dim / 4, ..) of a key row, and of the query to match; and lane group g takes the contiguous
// dim / 8 elements of a value row as rows g and g + 8 of each of its tiles.  Pairs of neighbouring tokens, which the second product
// contracts over, are made by interleaving the CODES of two rows (bytes by prmt, nibbles by masks) before they are widened.
// The first product's sums lie with tokens along the lanes and want them along the registers: one movmatrix for eight of them.
//
// Scales.  8 bits: a key's scale multiplies its scores, a value's its weight.  4 bits: the largest exponent of a row's group
// scales does, and scale / 2^exponent, a number of eight bits, multiplies the widened pairs (exact in binary16).
//
// Weights.  e = 2^(x - m + 8), p = e * scale of v rounded to binary16, with x the score in units of log 2 and m the maximum over
// what has been seen of x + log2(scale of v).  m moves only when a p would pass 2^15 (checked by a vote), so a tile usually takes
// no shuffle and no rescaling of the sums.
//
// 8 bits, up to 8 rows: bound by memory (131000 tokens of 8 heads of 128, 270 MB: 48 us, 5.6 TB/s).  4 bits: by instructions
// (unpacking, scales of groups): the same tokens take 47 us for half the bytes (53 when every lane made the scales that it needs itself).
#include <cmath>

#include "fbsr_attend.cuh"

namespace fbsr {
namespace {

constexpr int WARPS = 4, THREADS = WARPS * 32;

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The 8 x 8 matrix of 16-bit values that the warp holds, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t a)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// The same place of shared memory in CTA `rank` of the cluster.
template <class T>
__device__ __forceinline__ T* in_cta(T* p, int rank)
{
    uint64_t r;
    asm("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
    return reinterpret_cast<T*>(r);
}

constexpr int MOST_CLUSTERED = 8;                // CTAs of a cluster that every launch can have

template <int DIM, int BITS, int NR, bool BF16Q>
__global__ void __launch_bounds__(THREADS, NR == 1 ? 4 : 3)
attend_kv_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    using L = Layout<DIM, BITS>;
    constexpr int TILE_ROWS = 8 * NR;            // a warp has sixteen tokens of a tile
    constexpr int KD = DIM / 4, VD = DIM / 8, KSTEPS = DIM / 16, MT = DIM / 16;  // a lane's elements of a key, of a value
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t bars[L::STAGES];
    __shared__ uint32_t bad_pieces[L::STAGES];
    __shared__ ScaleEntry row_scales[WARPS][BITS == 4 ? 32 : 1];
    const uint32_t ring = (shared_address(dynamic) + 1023u) & ~1023u;
    uint8_t* const shared = dynamic + (ring - shared_address(dynamic));
    const int lane = threadIdx.x & 31, warp = warp_number(), g = lane >> 2, t = lane & 3;

    let_next_kernel_start();
    uint32_t block = blockIdx.x;
    const int split = block % a.splits; block /= a.splits;
    const int row_tile = block % a.row_tiles; block /= a.row_tiles;
    const int kv_head = block % a.kv_heads;
    const Work w = work_of(a, row_tile, kv_head, block / a.kv_heads, split, TILE_ROWS);
    if (w.first_row >= w.rows || (split > 0 && w.from >= w.to)) return;          // the joining kernel knows how many splits there are

    // ---- the ring of tiles
    const uint32_t full = shared_address(bars);
    if (threadIdx.x == 0) {
        for (int s = 0; s < L::STAGES; ++s) barrier_init(full + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const int tiles = (w.to - w.from + TILE - 1) / TILE;
    TileCopy<DIM, BITS> copy(a, w, &k_map, &v_map);
    auto copy_tile = [&](int tile) {
        const int s = tile % L::STAGES;
        copy(tile, ring + s * L::STAGE, full + 8 * s, bad_pieces + s);
    };
    if (warp == 0) {
        copy.start();
#pragma unroll 1
        for (int s = 0; s < L::STAGES - 1 && s < tiles; ++s) copy_tile(s);
    }

    // ---- this warp's rows of queries, in binary16: right operands
    uint32_t q[NR][KSTEPS][2];
    float to_score[NR][2];                       // rows 2 t and 2 t + 1: what turns a sum of products into a score in units of log 2
    int query[NR][2];                            // of the sequence; -1: no such row
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int row = w.first_row + 8 * n + g;
        const bool real = row < w.rows;
        const int mine = real ? (int)divide((uint32_t)row, a.by_share) : 0, head = kv_head * a.share + (real ? row - mine * a.share : 0);
        const uint16_t* p = static_cast<const uint16_t*>(a.q) + (int64_t)(w.start + mine) * a.q_token + head * a.q_head + t * KD;
        uint32_t x[KD / 2];
        load_query<KD>(p, real, x);
        float score = a.scale_log2;
        if constexpr (BF16Q) {
            uint32_t m = query_amax<KD>(x);
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
            score = query_to_half<KD>(x, m, score);
        }
#pragma unroll
        for (int j = 0; j < KSTEPS; ++j) { q[n][j][0] = x[2 * j]; q[n][j][1] = x[2 * j + 1]; }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            to_score[n][r] = __shfl_sync(0xFFFFFFFFu, score, (2 * t + r) * 4);
            const int other = w.first_row + 8 * n + 2 * t + r;
            query[n][r] = other < w.rows ? (int)divide((uint32_t)other, a.by_share) : -1;
        }
    }

    float o[MT][NR][4] = {}, top[NR][2], sum[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        top[n][0] = top[n][1] = LOWEST;
        sum[n][0] = sum[n][1] = w.beyond ? __uint_as_float(0x7FC00000u) : 0.0f;
    }

    bool fine = true;
    for (int tile = 0; tile < tiles; ++tile) {
        const int s = tile % L::STAGES;
        if (fine) fine = barrier_wait(full + 8 * s, (tile / L::STAGES) & 1);
        __syncthreads();                         // the stage refilled next has been read by all
        if (warp == 0 && tile + L::STAGES - 1 < tiles) copy_tile(tile + L::STAGES - 1);

        uint8_t* keys = shared + s * L::STAGE;
        uint8_t* values = keys + L::CODES;
        uint16_t* k_scales = reinterpret_cast<uint16_t*>(values + L::CODES);
        uint16_t* v_scales = k_scales + 512;
        const int left = w.to - (w.from + tile * TILE);        // tokens of the tile that exist, or more
        const uint32_t bad = bad_pieces[s];
        if (left < TILE || bad != 0u) {
            // Rows that were not copied, or lie behind the end, may hold anything: codes of values become zeros, so that a weight of
            // zero makes nothing of them; a token on a page that the cache does not have gets a scale that is no number.
            for (int i = threadIdx.x; i < TILE * L::CHUNKS; i += THREADS) {
                const int row = i / L::CHUNKS;
                const bool missing = (bad >> (row >> copy.piece_shift)) & 1;
                if (row >= left || missing) *reinterpret_cast<uint4*>(values + L::at(row, i % L::CHUNKS * 16)) = make_uint4(0u, 0u, 0u, 0u);
                if (missing && i % L::CHUNKS == 0)
                    for (int c = 0; c < L::GROUPS; ++c) k_scales[row * L::GROUPS + c] = 0x7FC0u;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncthreads();
        }
        {
            const int base = warp * 16, first = w.from + tile * TILE + base;     // of the tile; of the sequence
            if (first >= w.to) continue;
            const int mine[2] = {base + L::token(g), base + L::token(g + 8)};    // this lane's tokens of the scores
            const ScaleEntry* const vr = row_scales[warp];
            const ScaleEntry* const kr = vr + (BITS == 4 ? 16 : 0);
            if constexpr (BITS == 4) {           // a lane makes the scales of one row, of values or of keys, for the whole warp
                const RowScale<L::GROUPS> row((lane < 16 ? v_scales : k_scales) + (base + L::token(lane & 15)) * L::GROUPS);
                __syncwarp();                    // the last ones have been read
                row_scales[warp][lane] = row.entry();
                __syncwarp();
            }

            // ---- scores of 16 tokens
            float x[NR][4] = {};
            {
                uint32_t words[2][KD * BITS / 32];
                uint32_t rest2[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    constexpr int BYTES = KD * BITS / 8;
                    if constexpr (BYTES >= 16) {
#pragma unroll
                        for (int i = 0; i < BYTES / 16; ++i) {
                            const uint4 v = *reinterpret_cast<const uint4*>(keys + L::at(mine[h], t * BYTES + 16 * i));
                            words[h][4 * i] = v.x; words[h][4 * i + 1] = v.y; words[h][4 * i + 2] = v.z; words[h][4 * i + 3] = v.w;
                        }
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2*>(keys + L::at(mine[h], t * BYTES));
                        words[h][0] = v.x; words[h][1] = v.y;
                    }
                    if constexpr (BITS == 4) {
                        const uint32_t rest = kr[g + 8 * h].rest[t * KD / 32];
                        rest2[h] = __byte_perm(rest, 0u, 0x1010);
                    }
                }
                if constexpr (BITS == 8) {
#pragma unroll
                    for (int j = 0; j < KSTEPS; ++j) {
                        uint32_t f[4];
                        e4m3_word_to_half2(words[0][j], f[0], f[2]);
                        e4m3_word_to_half2(words[1][j], f[1], f[3]);
#pragma unroll
                        for (int n = 0; n < NR; ++n) mma16816(x[n], f, q[n][j][0], q[n][j][1]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < KSTEPS / 2; ++j) {
                        uint32_t h0[4], h1[4];
                        e2m1_word_to_half2(words[0][j], h0);
                        e2m1_word_to_half2(words[1][j], h1);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t f[4] = {mul_half2(h0[2 * i], rest2[0]), mul_half2(h1[2 * i], rest2[1]),
                                                   mul_half2(h0[2 * i + 1], rest2[0]), mul_half2(h1[2 * i + 1], rest2[1])};
#pragma unroll
                            for (int n = 0; n < NR; ++n) mma16816(x[n], f, q[n][2 * j + i][0], q[n][2 * j + i][1]);
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {       // both factors first: a sum of products times one of them may be out of range
                    const float ks = BITS == 4 ? kr[g + 8 * h].scale : bf16_value(k_scales[mine[h]]);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        x[n][2 * h] = __fmul_rn(x[n][2 * h], __fmul_rn(to_score[n][0], ks));
                        x[n][2 * h + 1] = __fmul_rn(x[n][2 * h + 1], __fmul_rn(to_score[n][1], ks));
                    }
                }
            }

            // ---- weights
            float vs[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) vs[h] = BITS == 4 ? vr[g + 8 * h].scale : bf16_value(v_scales[mine[h]]);
            uint32_t weights[NR][2];
            // who sees whom: asked only where the block reaches the drafts or the end
            const bool masked = first + 16 > min(w.context, w.to);
            uint32_t seen = 0xFFFFFFFFu;         // bit 4 n + 2 h + r
            if (masked) {
                seen = 0u;
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int token = w.from + tile * TILE + mine[i >> 1], draft = token - w.context, me = query[n][i & 1];
                        bool see = token < w.to && me >= 0;
                        if (see && draft >= 0) {
                            if (a.tree == nullptr) see = draft <= me;
                            else see = (draft >> 6) < a.tree_words && (a.tree[(int64_t)(w.start + me) * a.tree_words + (draft >> 6)] >> (draft & 63)) & 1;
                        }
                        seen |= (uint32_t)see << (4 * n + i);
                        if (!see) x[n][i] = -__uint_as_float(0x7F800000u);
                    }
            }
            float e[NR][4], p[NR][4];
            auto weigh = [&] {
                float most = 0.0f;
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const float lift[2] = {__fsub_rn(HEADROOM, top[n][0]), __fsub_rn(HEADROOM, top[n][1])};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e[n][i] = exp2_fast(__fadd_rn(x[n][i], lift[i & 1]));
                        p[n][i] = __fmul_rn(e[n][i], vs[i >> 1]);
                        most = fmaxf(most, fmaxf(p[n][i], __fmul_rn(e[n][i], 0x1p-60f)));
                    }
                }
                if (masked) {                    // a weight of zero times a scale that is no number
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!((seen >> (4 * n + i)) & 1)) p[n][i] = 0.0f;
                }
                return most;
            };
            if (__any_sync(0xFFFFFFFFu, weigh() > 32768.0f)) {
                const float lv[2] = {fmaxf(log2_fast(vs[0]), -60.0f), fmaxf(log2_fast(vs[1]), -60.0f)};
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float m = top[n][r];
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if ((seen >> (4 * n + 2 * h + r)) & 1) m = fmaxf(m, __fadd_rn(x[n][2 * h + r], lv[h]));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                        const float f = exp2_fast(__fsub_rn(top[n][r], m));
                        top[n][r] = m;
                        sum[n][r] = __fmul_rn(sum[n][r], f);
#pragma unroll
                        for (int j = 0; j < MT; ++j) { o[j][n][r] = __fmul_rn(o[j][n][r], f); o[j][n][2 + r] = __fmul_rn(o[j][n][2 + r], f); }
                    }
                weigh();
            }
#pragma unroll
            for (int n = 0; n < NR; ++n) {
#pragma unroll
                for (int r = 0; r < 2; ++r) sum[n][r] = __fadd_rn(sum[n][r], __fadd_rn(e[n][r], e[n][2 + r]));
                weights[n][0] = transposed(half2_of(p[n][0], p[n][1]));
                weights[n][1] = transposed(half2_of(p[n][2], p[n][3]));
            }

            // ---- values: pairs of tokens in rows 2 t, 2 t + 1 and 2 t + 8, 2 t + 9 of the operand
            const int from[4] = {base + L::token(2 * t), base + L::token(2 * t + 1), base + L::token(2 * t + 8), base + L::token(2 * t + 9)};
            if constexpr (BITS == 8) {
                uint32_t v[4][VD / 4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (VD == 16) {
                        const uint4 u = *reinterpret_cast<const uint4*>(values + L::at(from[j], g * VD));
                        v[j][0] = u.x; v[j][1] = u.y; v[j][2] = u.z; v[j][3] = u.w;
                    } else {
                        const uint2 u = *reinterpret_cast<const uint2*>(values + L::at(from[j], g * VD));
                        v[j][0] = u.x; v[j][1] = u.y;
                    }
                }
#pragma unroll
                for (int i = 0; i < VD / 4; ++i) {               // four elements: two tiles
                    uint32_t lo[4], hi[4];
                    e4m3_word_to_half2(__byte_perm(v[0][i], v[1][i], 0x5140), lo[0], lo[1]);
                    e4m3_word_to_half2(__byte_perm(v[0][i], v[1][i], 0x7362), lo[2], lo[3]);
                    e4m3_word_to_half2(__byte_perm(v[2][i], v[3][i], 0x5140), hi[0], hi[1]);
                    e4m3_word_to_half2(__byte_perm(v[2][i], v[3][i], 0x7362), hi[2], hi[3]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t f[4] = {lo[2 * j], lo[2 * j + 1], hi[2 * j], hi[2 * j + 1]};
#pragma unroll
                        for (int n = 0; n < NR; ++n) mma16816(o[2 * i + j][n], f, weights[n][0], weights[n][1]);
                    }
                }
            } else {
                uint32_t rest[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) rest[j] = vr[2 * t + (j & 1) + 8 * (j >> 1)].rest[g * VD / 32];
                const uint32_t r0 = __byte_perm(rest[0], rest[1], 0x5410), r1 = __byte_perm(rest[2], rest[3], 0x5410);
                uint32_t v[4][VD / 8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (VD == 16) {
                        const uint2 u = *reinterpret_cast<const uint2*>(values + L::at(from[j], g * (VD / 2)));
                        v[j][0] = u.x; v[j][1] = u.y;
                    } else {
                        v[j][0] = *reinterpret_cast<const uint32_t*>(values + L::at(from[j], g * (VD / 2)));
                    }
                }
#pragma unroll
                for (int i = 0; i < VD / 8; ++i) {               // eight elements: four tiles
                    uint32_t lo[2][4], hi[2][4];                 // even and odd elements
                    constexpr uint32_t EVEN = 0x0F0F0F0Fu;
                    e2m1_word_to_half2((v[0][i] & EVEN) | ((v[1][i] << 4) & ~EVEN), lo[0]);
                    e2m1_word_to_half2(((v[0][i] >> 4) & EVEN) | (v[1][i] & ~EVEN), lo[1]);
                    e2m1_word_to_half2((v[2][i] & EVEN) | ((v[3][i] << 4) & ~EVEN), hi[0]);
                    e2m1_word_to_half2(((v[2][i] >> 4) & EVEN) | (v[3][i] & ~EVEN), hi[1]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t f[4] = {mul_half2(lo[0][c], r0), mul_half2(lo[1][c], r0), mul_half2(hi[0][c], r1), mul_half2(hi[1][c], r1)};
#pragma unroll
                        for (int n = 0; n < NR; ++n) mma16816(o[4 * i + c][n], f, weights[n][0], weights[n][1]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (!fine) sum[n][r] = __uint_as_float(0x7FC00000u);                 // a copy that never came
            sum[n][r] = __fadd_rn(sum[n][r], __shfl_xor_sync(0xFFFFFFFFu, sum[n][r], 4));
            sum[n][r] = __fadd_rn(sum[n][r], __shfl_xor_sync(0xFFFFFFFFu, sum[n][r], 8));
            sum[n][r] = __fadd_rn(sum[n][r], __shfl_xor_sync(0xFFFFFFFFu, sum[n][r], 16));
        }
    __syncthreads();                             // the ring is free: every copy has been waited for

    // ---- the warps along the tokens joined: their sums in shared memory, rows of DIM + 4 to spread the banks
    constexpr int PITCH = DIM + 4;
    float* so = reinterpret_cast<float*>(shared);
    float2* sml = reinterpret_cast<float2*>(so + WARPS * TILE_ROWS * PITCH);
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int at = warp * TILE_ROWS + 8 * n + 2 * t + r;
            float* row = so + at * PITCH + g * VD;
#pragma unroll
            for (int j = 0; j < MT; j += 2)
                *reinterpret_cast<float4*>(row + 2 * j) = make_float4(o[j][n][r], o[j][n][2 + r], o[j + 1][n][r], o[j + 1][n][2 + r]);
            if (g == 0) sml[at] = make_float2(top[n][r], sum[n][r]);
        }
    __syncthreads();
    if (!a.clustered) {
        write_rows<DIM, BF16Q, TILE_ROWS, WARPS, THREADS>(a, w, split, so, sml, threadIdx.x);
        return;
    }

    // ---- the splits of a cluster joined, each CTA's rows read by the others.  What a thread puts back is what it alone has read; the
    // maxima and sums go behind the parts'.  CTAs without tokens have left: they count as arrived, and nothing of theirs is read.
    float2* const ml = sml + WARPS * TILE_ROWS;
    join_parts<DIM, TILE_ROWS, WARPS, THREADS>(w, so, sml, threadIdx.x, [&](int r, int octet, float m, float l, float (&v)[8]) {
        float4* dst = reinterpret_cast<float4*>(so + r * PITCH + octet * 8);
        dst[0] = make_float4(v[0], v[1], v[2], v[3]);
        dst[1] = make_float4(v[4], v[5], v[6], v[7]);
        if (octet == 0) ml[r] = make_float2(m, l);
    });
    cluster_barrier();
    constexpr int OCTETS = DIM / 8;
    const int splits = splits_of(w.length, a.chunk);
#pragma unroll 1
    for (int i = split * THREADS + threadIdx.x; i < TILE_ROWS * OCTETS; i += splits * THREADS) {
        const int r = i / OCTETS, octet = i % OCTETS, row = w.first_row + r;
        if (row >= w.rows) break;
        float2 theirs[MOST_CLUSTERED];
        float m = LOWEST;
#pragma unroll
        for (int s = 0; s < MOST_CLUSTERED; ++s) {
            theirs[s] = s < splits ? *in_cta(ml + r, s) : make_float2(LOWEST, 0.0f);
            m = fmaxf(m, theirs[s].x);
        }
        float l = 0.0f, v[8] = {};
#pragma unroll
        for (int s = 0; s < MOST_CLUSTERED; ++s) {
            if (s >= splits) break;
            const float f = exp2_fast(__fsub_rn(theirs[s].x, m));
            l = __fmaf_rn(theirs[s].y, f, l);
            add_scaled(in_cta(so + r * PITCH + octet * 8, s), f, v);
        }
        const int qi = (int)divide((uint32_t)row, a.by_share), head = w.head * a.share + row - qi * a.share;
        write_result<DIM, BF16Q>(a, w.start + qi, head, octet, l, v);
    }
    cluster_barrier();                           // nobody leaves while it is read
}

// A joining kernel is launched while the last CTAs of the kernel before it still run, and waits here, in every thread, until all of
// their writes can be seen (8192 tokens of 8 heads: 9.5 us against 10.3).
__device__ __forceinline__ void wait_for_kernel_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// The splits of a row joined.  Few of them: DIM / 8 threads a row, eight elements each.
template <int DIM, bool BF16Q>
__global__ void __launch_bounds__(THREADS)
join_few_kernel(const __grid_constant__ AttendArgs a)
{
    constexpr int OCTETS = DIM / 8, ROWS = THREADS / OCTETS;
    uint32_t block = blockIdx.x;
    const int row_tiles = (a.max_queries * a.share + ROWS - 1) / ROWS;
    const int row_tile = block % row_tiles; block /= row_tiles;
    const int kv_head = block % a.kv_heads;
    const Work w = work_of(a, row_tile, kv_head, block / a.kv_heads, 0, ROWS);
    wait_for_kernel_before();
    const int row = w.first_row + threadIdx.x / OCTETS, octet = threadIdx.x % OCTETS;
    if (row >= w.rows) return;
    const int splits = splits_of(w.length, a.chunk);
    const int qi = row / a.share, heads = a.kv_heads * a.share, head = kv_head * a.share + row - qi * a.share;
    const int64_t at = (int64_t)(w.start + qi) * heads + head, step = (int64_t)a.total * heads;
    float m = LOWEST;
    for (int s = 0; s < splits; ++s) m = fmaxf(m, a.part_ml[at + s * step].x);
    float l = 0.0f, v[8] = {};
    for (int s = 0; s < splits; ++s) {
        const float2 ml = a.part_ml[at + s * step];
        const float f = exp2_fast(__fsub_rn(ml.x, m));
        l = __fmaf_rn(ml.y, f, l);
        add_scaled(a.part_o + (at + s * step) * DIM + octet * 8, f, v);
    }
    write_result<DIM, BF16Q>(a, w.start + qi, head, octet, l, v);
}

// Many of them: a CTA to a row.  A thread has a split's maximum and sum (or every 128th one's), then eight elements of every PARTS-th
// split, four of them asked for at a time; parts are added in their order.
constexpr int MOST_SPLITS = 1536;

template <int DIM, bool BF16Q>
__global__ void __launch_bounds__(THREADS)
join_many_kernel(const __grid_constant__ AttendArgs a)
{
    constexpr int OCTETS = DIM / 8, PARTS = THREADS / OCTETS;
    __shared__ float part[PARTS][DIM + 4], factor[MOST_SPLITS], buffer[2][WARPS];
    uint32_t block = blockIdx.x;
    const int row_tile = block % (a.max_queries * a.share); block /= a.max_queries * a.share;
    const int kv_head = block % a.kv_heads;
    const Work w = work_of(a, row_tile, kv_head, block / a.kv_heads, 0, 1);
    wait_for_kernel_before();
    const int row = w.first_row, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (row >= w.rows) return;
    const int splits = splits_of(w.length, a.chunk);
    const int qi = row / a.share, heads = a.kv_heads * a.share, head = kv_head * a.share + row - qi * a.share;
    const int64_t at = (int64_t)(w.start + qi) * heads + head, step = (int64_t)a.total * heads;
    float m = LOWEST;
    for (int s = threadIdx.x; s < splits; s += THREADS) {
        factor[s] = a.part_ml[at + s * step].x;
        m = fmaxf(m, factor[s]);
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if (lane == 0) buffer[0][warp] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) m = fmaxf(m, buffer[0][i]);
    float l = 0.0f;
    for (int s = threadIdx.x; s < splits; s += THREADS) {
        factor[s] = exp2_fast(__fsub_rn(factor[s], m));
        l = __fmaf_rn(a.part_ml[at + s * step].y, factor[s], l);
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) l = __fadd_rn(l, __shfl_xor_sync(0xFFFFFFFFu, l, d));
    if (lane == 0) buffer[1][warp] = l;
    __syncthreads();
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) l = __fadd_rn(l, buffer[1][i]);
    const int octet = threadIdx.x % OCTETS, mine = threadIdx.x / OCTETS;
    float v[8] = {};
#pragma unroll 4
    for (int s = mine; s < splits; s += PARTS) add_scaled(a.part_o + (at + s * step) * DIM + octet * 8, factor[s], v);
#pragma unroll
    for (int c = 0; c < 8; ++c) part[mine][octet * 8 + c] = v[c];
    __syncthreads();
    if (mine != 0) return;
#pragma unroll
    for (int p = 1; p < PARTS; ++p)
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = __fadd_rn(v[c], part[p][octet * 8 + c]);
    write_result<DIM, BF16Q>(a, w.start + qi, head, octet, l, v);
}

// How a call is cut: rows of a CTA (8 nr, or 128 / copies with the kernels of many rows), and tokens of a chunk.
struct Plan { int nr, copies, row_tiles, splits, chunk, clustered; };

// Up to 16 rows go through mma.sync: one warp's operand holds them (9 to 16 with the kernels of many rows instead: one sequence of 32768
// tokens 25 us against 22, 32 of 4000 75 against 66, 148 of 6144 55 against 60).  The table's capacity is cut into equal chunks, for every sequence
// and head as many as give each place that the GPU has one CTA.  Places: three on a multiprocessor with few rows, four (what registers
// and shared memory hold) with up to eight where there are several sequences or few bytes a token (32 sequences of 1 to 8192 tokens: 61
// us against 67; one of 131000 in 4 bits: 47 against 51, but in 8 bits 51 against 48); one with the kernels of many rows, whose start
// and end cost as much as ten tiles.  Several sequences differ in length and leave some of their CTAs without tokens: with few rows
// three times as many (32 sequences of 1 to 8192 tokens: 64 us with four times, 71 with twice; four models, 4 to 128 sequences of up to 2048, 8192 and
// 32768 tokens, from all lengths to nearly equal ones: once to six times are within 7 % of one another in the mean, once is better for
// lengths that are alike and four times for those that are not), and with many two chunks rather than one although the places do not hold them, as long as
// what the second round of CTAs starts and ends is little beside a chunk: up to a number of (sequence, head, tile of rows) that grows
// with the table, the line on which both choices cross.  Times of two chunks over those of one, geometric means over 32 to 252 rows and lengths
// spread from an eighth or a half of the longest: tables of 2048 tokens 0.98 with 80 of them and 1.20 with 88, 3000: 0.92 with 88 and 1.08
// with 96, 4096: 0.97 with 96 and 1.14 with 104, 8192: 0.90 with 112 and 1.08 with 120; 1024: 1.17 with 80.  Not shorter
// than MIN_CHUNK tokens.  With few rows, where the cache is what is read, writing and reading a chunk's sums (8 dim bytes a row) should
// not pass a tenth of reading its tokens: there they are made longer, but not so long that the GPU is no longer full.  (Cutting by the
// lengths themselves, in the kernel, took longer: every CTA reads them all, and many more have nothing to do.)
//
// Short tables of few rows wait for launches and latencies, not for bytes: there the chunks of a sequence are a cluster, which joins
// them without a second kernel or a workspace (one sequence of 700 tokens, 2 heads of the cache, dim 64: 6.5 us against 8.6 on the
// device, 10.9 against 15.7 as calls in a row).  Up to eight CTAs, as many as 1.5 on each multiprocessor allow, of up to CLUSTER_CHUNK
// tokens each (8 heads: 2048 tokens 8.1 us as eight of 256, 7.8 as sixteen and a second launch; 4000 tokens 10.7 as eight, 9.0 as sixteen).
constexpr int64_t MULTIPROCESSORS = 148, MIN_CHUNK = 256, CLUSTER_PLACES = MULTIPROCESSORS * 3 / 2, CLUSTER_CHUNK = 256;

Plan plan_of(const fbsr_kv_cache& c, size_t batch, int heads, size_t max_queries, int64_t capacity)
{
    Plan p;
    const int64_t rows = (int64_t)max_queries * (heads / c.heads);
    p.nr = rows <= 8 ? 1 : 2;
    p.copies = rows <= 16 ? 0 : rows <= 32 ? 4 : rows <= 64 ? 2 : 1;
    const int64_t tile = p.copies ? 128 / p.copies : 8 * p.nr, resident = MULTIPROCESSORS * (p.copies ? 1 : p.nr == 1 && (batch > 1 || c.bits == 4) ? 4 : 3);
    p.row_tiles = (int)((rows + tile - 1) / tile);
    const int64_t units = (int64_t)batch * c.heads * p.row_tiles, used = rows < tile ? rows : tile;
    const int64_t together = CLUSTER_PLACES / units < MOST_CLUSTERED ? CLUSTER_PLACES / units : MOST_CLUSTERED;
    const int64_t full = (capacity * units + resident - 1) / resident;
    int64_t pieces = resident / units;
    if (batch > 1 && !p.copies) pieces = 3 * resident / units;
    else if (batch > 1 && pieces < 2 && units <= resident && units <= resident * (0.55 + 0.118 * std::log2(capacity / 2048.0))) pieces = 2;
    pieces = pieces < 1 ? 1 : pieces;
    int64_t chunk = (capacity + pieces - 1) / pieces;
    const int64_t worth = p.copies ? 0 : used * c.dim * 8 * 10 / (2 * c.dim * c.bits / 8), longer = worth < full ? worth : full;
    chunk = chunk < longer ? longer : chunk;
    const int64_t shortest = (capacity + MOST_SPLITS - 1) / MOST_SPLITS;
    chunk = chunk < shortest ? shortest : chunk;
    chunk = chunk < MIN_CHUNK ? MIN_CHUNK : chunk;
    if (!p.copies && together > 1 && capacity <= together * CLUSTER_CHUNK) chunk = capacity < 1 ? 1 : (capacity + together - 1) / together;
    chunk = (chunk + TILE - 1) / TILE * TILE;
    p.chunk = (int)(chunk > (int64_t)1 << 30 ? (int64_t)1 << 30 : chunk);
    p.splits = (int)((capacity + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    p.clustered = !p.copies && p.splits > 1 && p.splits <= MOST_CLUSTERED && units * p.splits <= resident;
    return p;
}

// FBSR_OK, or what is wrong with the shapes.
int check_shapes(const fbsr_kv_cache* cache, size_t batch, size_t total, int heads, size_t max_queries, size_t max_pages)
{
    const int status = check_kv_cache(cache);
    if (status != FBSR_OK) return status;
    if (heads < 1 || heads % cache->heads != 0 || max_queries < 1 || max_queries > 256) return FBSR_ERR_INVALID_ARG;
    if (heads > 65536 || total > 0x7FFFFFFFu || batch > 0x7FFFFFFFu || (uint64_t)total * heads > (uint64_t)1 << 40) return FBSR_ERR_TOO_LARGE;
    if (max_pages > (((size_t)1 << 31) - 64) / cache->page) return FBSR_ERR_TOO_LARGE;
    return FBSR_OK;
}

size_t workspace_bytes_of(const Plan& p, size_t total, int heads, int dim)
{
    return p.splits == 1 || p.clustered ? 0 : (size_t)p.splits * total * heads * (dim * sizeof(float) + sizeof(float2));
}

// A cache's codes as lines of 128 bytes, copied `lines` at a time.
bool encode_codes(CUtensorMap& map, const void* codes, uint64_t total_lines, int lines)
{
    const cuuint64_t size[2] = {128, total_lines}, stride[1] = {128};
    const cuuint32_t box[2] = {128, (cuuint32_t)lines};
    return encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, codes, size, stride, box);
}

template <int DIM, int BITS, int NR, bool BF16Q>
int launch(const AttendArgs& a, const CUtensorMap& k_map, const CUtensorMap& v_map, size_t batch, cudaStream_t stream)
{
    static std::atomic<uint64_t> asked{0};
    constexpr int SHARED = Layout<DIM, BITS>::template shared<NR>();
    const auto kernel = attend_kv_kernel<DIM, BITS, NR, BF16Q>;
    if (allow_shared_memory(reinterpret_cast<const void*>(kernel), SHARED, asked) != FBSR_OK) return FBSR_ERR_CUDA;
    const uint64_t grid = (uint64_t)batch * a.kv_heads * a.row_tiles * a.splits;
    if (grid > 0x7FFFFFFFu) return FBSR_ERR_TOO_LARGE;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)grid);
    config.blockDim = dim3(THREADS);
    config.dynamicSmemBytes = SHARED;
    config.stream = stream;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = (unsigned)a.splits; cluster.val.clusterDim.y = 1; cluster.val.clusterDim.z = 1;
    config.attrs = &cluster;
    config.numAttrs = a.clustered ? 1 : 0;
    if (cudaLaunchKernelEx(&config, kernel, a, k_map, v_map) != cudaSuccess) { cudaGetLastError(); return FBSR_ERR_CUDA; }
    count_launch();
    return FBSR_OK;
}

template <int DIM, bool BF16Q>
int launch_join(const AttendArgs& a, size_t batch, cudaStream_t stream)
{
    if (a.splits == 1 || a.clustered) return FBSR_OK;
    const bool few = a.splits <= 4;
    const int rows = few ? THREADS / (DIM / 8) : 1;
    const uint64_t grid = (uint64_t)batch * a.kv_heads * ((a.max_queries * a.share + rows - 1) / rows);
    if (grid > 0x7FFFFFFFu) return FBSR_ERR_TOO_LARGE;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)grid);
    config.blockDim = dim3(THREADS);
    config.stream = stream;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &early;
    config.numAttrs = 1;
    if (cudaLaunchKernelEx(&config, few ? join_few_kernel<DIM, BF16Q> : join_many_kernel<DIM, BF16Q>, a) != cudaSuccess) { cudaGetLastError(); return FBSR_ERR_CUDA; }
    count_launch();
    return FBSR_OK;
}

template <int DIM, int BITS, bool BF16Q>
int launch_rows(const AttendArgs& a, const Plan& p, const fbsr_kv_cache& c, size_t batch, cudaStream_t stream)
{
    using L = Layout<DIM, BITS>;
    const uint64_t lines = c.pages * (uint64_t)c.heads * (uint64_t)c.page / L::LINE_ROWS;
    if (lines > 0x7FFFFFFFu) return FBSR_ERR_TOO_LARGE;                            // a coordinate of the copies
    const int piece = (c.page < TILE ? c.page : TILE) / L::LINE_ROWS;
    CUtensorMap k_map, v_map;
    if (!encode_codes(k_map, c.k_codes, lines, piece) || !encode_codes(v_map, c.v_codes, lines, piece)) return FBSR_ERR_CUDA;
    int status;
    if (p.copies) status = attend_rows(a, k_map, v_map, DIM, BITS, BF16Q, p.copies, batch, stream);
    else if (p.nr == 1) status = launch<DIM, BITS, 1, BF16Q>(a, k_map, v_map, batch, stream);
    else status = launch<DIM, BITS, 2, BF16Q>(a, k_map, v_map, batch, stream);
    if (status == FBSR_OK) status = launch_join<DIM, BF16Q>(a, batch, stream);
    return status != FBSR_OK ? status : cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}

inline bool off(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

}  // namespace
}  // namespace fbsr

using namespace fbsr;

extern "C" size_t fbsr_attend_workspace_bytes(const fbsr_kv_cache* cache, size_t batch, size_t total, int heads, size_t max_queries, size_t max_pages)
{
    if (check_shapes(cache, batch, total, heads, max_queries, max_pages) != FBSR_OK || batch == 0 || total == 0) return 0;
    return workspace_bytes_of(plan_of(*cache, batch, heads, max_queries, (int64_t)max_pages * cache->page), total, heads, cache->dim);
}

extern "C" int fbsr_attend_kv(const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_fmt, size_t total, int heads,
                              const fbsr_kv_cache* cache, const int32_t* pages, int64_t pages_ld, size_t max_pages, const int32_t* lengths,
                              size_t batch, const int32_t* starts, size_t max_queries, const uint64_t* tree, int tree_words, float scale,
                              void* out, int64_t out_token_stride, int64_t out_head_stride, void* workspace, size_t workspace_bytes,
                              void* cuda_stream)
{
    if (q_fmt != FBSR_BF16 && q_fmt != FBSR_FP16) return FBSR_ERR_UNSUPPORTED;
    const int status = check_shapes(cache, batch, total, heads, max_queries, max_pages);
    if (status != FBSR_OK) return status;
    const float scale_log2 = (float)((double)scale * 1.4426950408889634);
    if (!(scale_log2 - scale_log2 == 0.0f)) return FBSR_ERR_INVALID_ARG;          // finite
    if (tree != nullptr && (tree_words < (int)((max_queries + 63) / 64) || tree_words > 1024)) return FBSR_ERR_INVALID_ARG;
    if (batch == 0 || total == 0) return FBSR_OK;
    if (q == nullptr || out == nullptr || lengths == nullptr || (pages == nullptr && max_pages > 0)) return FBSR_ERR_INVALID_ARG;
    if (pages_ld < (int64_t)max_pages && batch > 1) return FBSR_ERR_INVALID_ARG;
    if (off(q, 2) || off(out, 2) || off(pages, 4) || off(lengths, 4) || off(starts, 4) || off(tree, 8)) return FBSR_ERR_ALIGNMENT;
    if (rows_meet(RowSet(q, q_token_stride, q_head_stride, total, (size_t)heads, (size_t)cache->dim, 2),
                  RowSet(out, out_token_stride, out_head_stride, total, (size_t)heads, (size_t)cache->dim, 2))) return FBSR_ERR_INVALID_ARG;
    const int64_t capacity = (int64_t)max_pages * cache->page;
    const Plan p = plan_of(*cache, batch, heads, max_queries, capacity);
    const size_t need = workspace_bytes_of(p, total, heads, cache->dim);
    if (need > workspace_bytes || (need > 0 && workspace == nullptr)) return FBSR_ERR_WORKSPACE;
    if (need > 0 && off(workspace, 16)) return FBSR_ERR_ALIGNMENT;
    AttendArgs a{};
    a.q = q; a.out = out;
    a.q_token = q_token_stride; a.q_head = q_head_stride; a.o_token = out_token_stride; a.o_head = out_head_stride;
    a.k_codes = static_cast<const uint8_t*>(cache->k_codes); a.v_codes = static_cast<const uint8_t*>(cache->v_codes);
    a.k_scales = static_cast<const uint16_t*>(cache->k_scales); a.v_scales = static_cast<const uint16_t*>(cache->v_scales);
    a.table = pages; a.table_ld = pages_ld; a.lengths = lengths; a.starts = starts; a.tree = tree;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + (size_t)p.splits * total * heads * cache->dim);
    a.pages = cache->pages;
    a.kv_heads = cache->heads; a.share = heads / cache->heads; a.by_share = divider((uint32_t)a.share);
    a.q_whole = !off(q, 16) && q_token_stride % 8 == 0 && q_head_stride % 8 == 0;
    a.page_shift = __builtin_ctz(cache->page); a.capacity = (int)capacity;
    a.total = (int)total; a.max_queries = (int)max_queries; a.row_tiles = p.row_tiles; a.splits = p.splits; a.chunk = p.chunk;
    a.clustered = p.clustered;
    a.tree_words = tree_words;
    a.scale_log2 = scale_log2;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
#define FBSR_ATTEND(d, b) \
    if (cache->dim == d && cache->bits == b) \
        return q_fmt == FBSR_BF16 ? launch_rows<d, b, true>(a, p, *cache, batch, stream) : launch_rows<d, b, false>(a, p, *cache, batch, stream);
    FBSR_ATTEND(128, 8) FBSR_ATTEND(128, 4) FBSR_ATTEND(64, 8) FBSR_ATTEND(64, 4)
#undef FBSR_ATTEND
    return FBSR_ERR_UNSUPPORTED;
}
