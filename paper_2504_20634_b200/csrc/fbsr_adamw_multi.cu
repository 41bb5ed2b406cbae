// fbsr_adamw_multi: one AdamW step over many tensors, with binary32 or 8-bit moments and the stochastically
// rounded low-precision copy of the weights.  The arithmetic is stated in include/fbsr.h.
//
// The tensor table travels as a kernel argument (up to 400 tensors a launch): nothing is uploaded, nothing has to
// outlive the call, and gradients may lie elsewhere at every step.  A warp owns 1024 consecutive elements of one
// tensor and finds the tensor by bisection over the table's running tile counts, so that a tensor of one element
// costs one warp and a tensor of 2^25 elements spreads over the whole GPU.
#include <cmath>

#include "../../include/fbsr.h"
#include "fbsr_internal.h"
#include "fbsr_kernels.cuh"

namespace fbsr {
namespace {

constexpr int TILE = 1024;                       // elements of a warp: 4 rows of 256
constexpr int STATE_BLOCK = 256;                 // elements that share a scale of the 8-bit state: one row
static_assert(STATE_BLOCK == ROW_ELEMS, "a row is a block");
constexpr int DRAW_WORDS = 4 * (TILE / 8 + 1);   // words of the generator calls that cover a tile, at most

struct AdamwHyper {
    float beta1, beta2, eps, neg_c1, c2, a1, a2, decay;
    const float* grad_scale;
    uint32_t k0, k1;
    int variant, k, g_fmt, ieee;
};

template <int CAP> struct AdamwTable {
    fbsr_adamw_tensor t[CAP];
    uint32_t first_tile[CAP + 1];
    uint32_t count;
};

// The k-bit draws of the weights' rounding for one warp tile.  Word w of call c lies at 4 c + w.
struct TileDraws {
    uint32_t* words;
    int k, dpw, base;                            // base: place of the tile's first element in the first call
    uint32_t mask, recip;

    __device__ __forceinline__ void fill(uint64_t g0, const AdamwHyper& h, int lane)
    {
        k = h.k; dpw = 32 / k; mask = (1u << k) - 1u; recip = 65536u / (uint32_t)dpw + 1u;
        const uint32_t e = 4u * (uint32_t)dpw;
        const uint64_t call0 = (dpw & (dpw - 1)) == 0 ? g0 >> (31 - __clz((int)e)) : g0 / e;
        base = (int)(g0 - call0 * e);
        const int calls = (base + TILE + (int)e - 1) / (int)e;
        __syncwarp();
        for (int c = lane; c < calls; c += 32)
            reinterpret_cast<uint4*>(words)[c] = philox_block(call0 + c, h.k0, h.k1);
        __syncwarp();
    }
    // element p of the tile
    __device__ __forceinline__ uint32_t at(int p) const
    {
        const uint32_t pos = (uint32_t)(base + p), q = (pos * recip) >> 16;      // pos / dpw (pos < 2^12)
        return (words[q] >> ((pos - q * (uint32_t)dpw) * (uint32_t)k)) & mask;
    }
};

__device__ __forceinline__ float load_grad(const void* g, int g_fmt, uint64_t i)
{
    if (g_fmt == FBSR_FP32) return static_cast<const float*>(g)[i];
    const uint32_t c = static_cast<const uint16_t*>(g)[i];
    return g_fmt == FBSR_BF16 ? __uint_as_float(c << 16) : __half2float(__ushort_as_half((unsigned short)c));
}

__device__ __forceinline__ void load_grad8(const void* g, int g_fmt, uint64_t i, float (&x)[8])
{
    if (g_fmt == FBSR_FP32) {
        unpack(load_f8_stream(static_cast<const float*>(g) + i), x);
        return;
    }
    const uint4 c = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(g) + i));
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (g_fmt == FBSR_BF16) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
            x[2 * j] = f.x; x[2 * j + 1] = f.y;
        }
    }
}

// Largest finite magnitude of the warp's 256 values, as a binary32 pattern.
__device__ __forceinline__ uint32_t row_amax(const float (&x)[8])
{
    uint32_t m = 0u;
#pragma unroll
    for (int c = 0; c < 8; ++c) m = max(m, __float_as_uint(x[c]) & 0x7FFFFFFFu);
    const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, m);
    if (all < 0x7F800000u) return all;
    m = 0u;                                      // an infinity or a NaN in the row (rare, the same for all lanes)
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint32_t b = __float_as_uint(x[c]) & 0x7FFFFFFFu;
        m = max(m, b < 0x7F800000u ? b : 0u);
    }
    return __reduce_max_sync(0xFFFFFFFFu, m);
}

// Codes of one row of state: scale from the row's maximum, then the few-bit rounding.  POSITIVE: a value above zero
// never takes the zero code (a zero second moment under a non-zero first one would blow the next step up).
template <bool POSITIVE>
__device__ __forceinline__ void round_state(const float (&x)[8], const uint4& draws, int shift, const AdamwHyper& h,
                                            float& scale, uint32_t (&code)[8])
{
    const float amax = __uint_as_float(row_amax(x));
    scale = fmaxf(__fmul_rn(amax, 1.0f / 448.0f), 0x1p-126f);
    const float inv = __fdiv_rn(1.0f, scale);
    const uint32_t w[4] = {draws.x, draws.y, draws.z, draws.w};
    const uint32_t mask = (1u << h.k) - 1u;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint32_t n = (w[c >> 1] >> ((c & 1) * 16 + shift)) & mask;
        code[c] = round_core<E4M3, false>(arith_bits(__fmul_rn(x[c], inv)), n, h.variant, h.k, nullptr);
        if (POSITIVE && x[c] > 0.0f && code[c] == 0u) code[c] = 1u;
    }
}

template <int FMT, int BITS, int CAP>
__global__ void __launch_bounds__(CTA_THREADS, 2)
adamw_multi_kernel(const __grid_constant__ AdamwTable<CAP> tab, const __grid_constant__ AdamwHyper h)
{
    __shared__ __align__(16) uint32_t wordbuf[WARPS_PER_CTA][DRAW_WORDS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t tile = blockIdx.x * WARPS_PER_CTA + warp;
    if (tile >= tab.first_tile[tab.count]) return;

    uint32_t lo = 0, hi = tab.count;             // first_tile[lo] <= tile < first_tile[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (tab.first_tile[mid] <= tile) lo = mid; else hi = mid;
    }
    const fbsr_adamw_tensor& t = tab.t[lo];
    const uint64_t e0 = (uint64_t)(tile - tab.first_tile[lo]) * TILE;
    const uint64_t n = t.n;
    const bool draws = h.variant < RTNE;

    constexpr uintptr_t LP_ALIGN = Format<FMT>::K;                 // bytes of 8 codes
    bool vec = ((reinterpret_cast<uintptr_t>(t.w) % 32) | (reinterpret_cast<uintptr_t>(t.w_lp) % LP_ALIGN) |
                (reinterpret_cast<uintptr_t>(t.g) % (h.g_fmt == FBSR_FP32 ? 32 : 16)) |
                ((reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v)) % (BITS == 32 ? 32 : 8))) == 0;

    TileDraws td;
    td.words = wordbuf[warp];
    if (draws && t.w_lp != nullptr) td.fill(t.offset + e0, h, lane);
    const float gs = h.grad_scale ? __ldg(h.grad_scale) : 1.0f;

    for (int row = 0; row < TILE / ROW_ELEMS; ++row) {
        const uint64_t r0 = e0 + (uint64_t)row * ROW_ELEMS;
        if (r0 >= n) break;
        const uint64_t e = r0 + lane * 8;
        const int valid = e >= n ? 0 : n - e >= 8 ? 8 : (int)(n - e);
        const bool whole = vec && valid == 8;
        float w[8] = {}, g[8] = {}, m[8] = {}, v[8] = {}, r[8];
        if (whole) {
            unpack(load_f8(t.w + e), w);
            load_grad8(t.g, h.g_fmt, e, g);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < valid) { w[c] = t.w[e + c]; g[c] = load_grad(t.g, h.g_fmt, e + c); }
        }
        if constexpr (BITS == 32) {
            float* pm = static_cast<float*>(t.m); float* pv = static_cast<float*>(t.v);
            if (whole) {
                unpack(load_f8(pm + e), m); unpack(load_f8(pv + e), v);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < valid) { m[c] = pm[e + c]; v[c] = pv[e + c]; }
            }
        } else {
            const uint8_t* pm = static_cast<const uint8_t*>(t.m); const uint8_t* pv = static_cast<const uint8_t*>(t.v);
            uint32_t cm[2] = {0u, 0u}, cv[2] = {0u, 0u};
            if (whole) {
                const uint2 a = *reinterpret_cast<const uint2*>(pm + e), b = *reinterpret_cast<const uint2*>(pv + e);
                cm[0] = a.x; cm[1] = a.y; cv[0] = b.x; cv[1] = b.y;
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < valid) {
                        cm[c >> 2] |= (uint32_t)pm[e + c] << (8 * (c & 3));
                        cv[c >> 2] |= (uint32_t)pv[e + c] << (8 * (c & 3));
                    }
            }
            const float sm = t.m_scale[r0 / STATE_BLOCK], sr = t.v_scale[r0 / STATE_BLOCK];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float x[4];
                decode4<E4M3>(cm[q], x);
#pragma unroll
                for (int c = 0; c < 4; ++c) m[4 * q + c] = __fmul_rn(x[c], sm);
                decode4<E4M3>(cv[q], x);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float root = __fmul_rn(x[c], sr);
                    v[4 * q + c] = __fmul_rn(root, root);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float gc = __fmul_rn(g[c], gs);
            if constexpr (BITS == 32) {
                m[c] = __fmaf_rn(h.beta1, m[c], __fmul_rn(h.a1, gc));
                v[c] = __fmaf_rn(h.beta2, v[c], __fmul_rn(__fmul_rn(h.a2, gc), gc));
            } else {
                m[c] = __fadd_rn(__fmul_rn(h.beta1, m[c]), __fmul_rn(h.a1, gc));
                v[c] = __fadd_rn(__fmul_rn(h.beta2, v[c]), __fmul_rn(__fmul_rn(h.a2, gc), gc));
            }
            r[c] = __fsqrt_rn(v[c]);
            const float d = __fadd_rn(__fmul_rn(r[c], h.c2), h.eps);
            w[c] = __fmaf_rn(h.neg_c1, __fdiv_rn(m[c], d), __fmul_rn(w[c], h.decay));
        }
        if (whole) {
            store_f8(t.w + e, w);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < valid) t.w[e + c] = w[c];
        }
        if constexpr (BITS == 32) {
            float* pm = static_cast<float*>(t.m); float* pv = static_cast<float*>(t.v);
            if (whole) {
                store_f8(pm + e, m); store_f8(pv + e, v);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < valid) { pm[e + c] = m[c]; pv[e + c] = v[c]; }
            }
        } else {
            // lanes beyond the tensor's end hold zeros, which no maximum notices
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c >= valid) { m[c] = 0.0f; r[c] = 0.0f; }
            uint4 bits = make_uint4(0u, 0u, 0u, 0u);
            if (draws) {
                const uint64_t i = (t.offset + e) >> 3;
                bits = philox4x32_10((uint32_t)i, (uint32_t)(i >> 32), 1u, 0u, h.k0, h.k1);
            }
            float sm, sr;
            uint32_t cm[8], cr[8];
            round_state<false>(m, bits, 0, h, sm, cm);
            round_state<true>(r, bits, 8, h, sr, cr);
            uint8_t* pm = static_cast<uint8_t*>(t.m); uint8_t* pv = static_cast<uint8_t*>(t.v);
            if (whole) {
                uint32_t a[2], b[2];
                pack_codes8<E4M3>(cm, a); pack_codes8<E4M3>(cr, b);
                *reinterpret_cast<uint2*>(pm + e) = make_uint2(a[0], a[1]);
                *reinterpret_cast<uint2*>(pv + e) = make_uint2(b[0], b[1]);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < valid) { pm[e + c] = (uint8_t)cm[c]; pv[e + c] = (uint8_t)cr[c]; }
            }
            if (lane == 0) { t.m_scale[r0 / STATE_BLOCK] = sm; t.v_scale[r0 / STATE_BLOCK] = sr; }
        }
        if (t.w_lp != nullptr) {
            uint32_t code[8];
#pragma unroll
            for (int c = 0; c < 8; ++c)
                code[c] = round_core<FMT, false>(arith_bits(w[c]), draws ? td.at(row * ROW_ELEMS + lane * 8 + c) : 0u, h.variant,
                                                 h.k, nullptr, h.ieee != 0);
            if (whole) {
                store_codes8<FMT>(t.w_lp, e, code);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < valid) store_code1<FMT>(t.w_lp, e + c, code[c]);
            }
        }
    }
}

template <int FMT, int BITS, int CAP>
int launch_chunk(const fbsr_adamw_tensor* t, size_t count, const AdamwHyper& h, cudaStream_t stream)
{
    AdamwTable<CAP> tab;
    tab.count = 0;
    uint64_t tiles = 0;
    for (size_t i = 0; i < count; ++i) {
        if (t[i].n == 0) continue;
        tab.t[tab.count] = t[i];
        tab.first_tile[tab.count++] = (uint32_t)tiles;
        tiles += (t[i].n + TILE - 1) / TILE;
    }
    tab.first_tile[tab.count] = (uint32_t)tiles;
    if (tiles == 0) return FBSR_OK;
    const unsigned grid = (unsigned)((tiles + WARPS_PER_CTA - 1) / WARPS_PER_CTA);
    adamw_multi_kernel<FMT, BITS, CAP><<<grid, CTA_THREADS, 0, stream>>>(tab, h);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? FBSR_OK : FBSR_ERR_CUDA;
}

constexpr int CAP_MANY = 400;                    // 72 + 4 bytes a tensor: under the 32,764 bytes of kernel arguments
constexpr int CAP_FEW = 48;

template <int FMT, int BITS>
int launch_all(const fbsr_adamw_tensor* t, size_t count, const AdamwHyper& h, cudaStream_t stream)
{
    for (size_t at = 0; at < count; at += CAP_MANY) {
        const size_t len = count - at < (size_t)CAP_MANY ? count - at : (size_t)CAP_MANY;
        const int rc = len <= (size_t)CAP_FEW ? launch_chunk<FMT, BITS, CAP_FEW>(t + at, len, h, stream)
                                              : launch_chunk<FMT, BITS, CAP_MANY>(t + at, len, h, stream);
        if (rc != FBSR_OK) return rc;
    }
    return FBSR_OK;
}

typedef int (*launch_fn)(const fbsr_adamw_tensor*, size_t, const AdamwHyper&, cudaStream_t);
const launch_fn kLaunch[5][2] = {{launch_all<0, 32>, launch_all<0, 8>}, {launch_all<1, 32>, launch_all<1, 8>},
                                 {launch_all<2, 32>, launch_all<2, 8>}, {launch_all<3, 32>, launch_all<3, 8>},
                                 {launch_all<4, 32>, launch_all<4, 8>}};

// beta^step by repeated multiplication, as fbsr_adam_scalars forms it (and stopped where it stops: below 2^-54 the
// difference to one is one).
double power(double b, int step)
{
    double p = 1.0;
    for (int t = 0; t < step; ++t) {
        p *= b;
        if (std::fabs(b) < 1.0 && std::fabs(p) < 0x1p-54) break;
    }
    return p;
}

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
    h.neg_c1 = -(float)(lr / (1.0 - power(beta1, step)));
    h.c2 = (float)(1.0 / std::sqrt(1.0 - power(beta2, step)));
    h.a1 = (float)(1.0 - beta1); h.a2 = (float)(1.0 - beta2);
    h.decay = (float)(1.0 - lr * weight_decay);
    h.grad_scale = grad_scale;
    h.k0 = (uint32_t)seed; h.k1 = (uint32_t)(seed >> 32);
    h.variant = variant; h.k = k_bits; h.g_fmt = g_fmt; h.ieee = ieee;
    return kLaunch[fmt][state_bits == 32 ? 0 : 1](tensors, count, h, static_cast<cudaStream_t>(cuda_stream));
}
