// Host-side plumbing shared by the translation units of libfbsr.so (not part of the public ABI).
#pragma once
#include <algorithm>
#include <atomic>
#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

namespace fbsr {

enum OpKind { OP_ROUND = 0, OP_ROUND_BITS, OP_ROUND_STATS, OP_SGD, OP_ADAM, OP_ACCUM, OP_ROUND_LP, OP_QAT, OP_ROUND_MX, OP_QAT_ADAMW };

// Everything an entry point hands to the per-format dispatcher.  Validated by the caller.
struct CallArgs {
    OpKind op;
    int variant, k;
    int ovf_ieee;                   // finite values beyond M: IEEE nearest-even instead of saturation
    size_t n;
    uint64_t seed, offset;
    cudaStream_t stream;
    void* dst;                      // low-precision codes (w_lp for OP_ACCUM)
    // OP_ROUND*, OP_ACCUM (src = update)
    const float* src;
    float scale;
    const uint32_t* words;          // OP_ROUND_BITS
    uint8_t* scales;                // OP_ROUND_MX: one exponent byte per block of 32
    const void* src_lp;             // OP_ROUND_LP: codes of src_fmt; OP_QAT: the 16-bit updates
    int src_fmt;
    // OP_ROUND_STATS
    size_t group_size;
    double* gsum_e;
    double* gsum_e2;
    void* total;                    // fbsr_stats*
    void* partials;                 // workspace
    // OP_SGD / OP_ADAM
    float* w; const float* g; float* m; float* v;
    float neg_lr, mu;                                   // SGD-momentum
    float beta1, beta2, eps, neg_c1, c2, a1, a2;        // Adam
    float neg_lrwd;                                     // OP_QAT_ADAMW: -(lr * weight_decay)
};

constexpr int MAX_SLOW_GRID = 148 * 8;      // CTAs of the general kernel; also the number of partial slots

// One dispatcher per (format, op group); each lives in its own translation unit
// (dispatch_lp_* and dispatch_qat_adamw_* exist for the 8-bit targets only).
#define FBSR_DECLARE_DISPATCH(fmt) \
    int dispatch_round_##fmt(const CallArgs&); \
    int dispatch_round_words_##fmt(const CallArgs&); \
    int dispatch_stats_##fmt(const CallArgs&); \
    int dispatch_optim_##fmt(const CallArgs&);\
    int dispatch_lp_##fmt(const CallArgs&); \
    int dispatch_qat_##fmt(const CallArgs&); \
    int dispatch_qat_adamw_##fmt(const CallArgs&);
FBSR_DECLARE_DISPATCH(0) FBSR_DECLARE_DISPATCH(1) FBSR_DECLARE_DISPATCH(2) FBSR_DECLARE_DISPATCH(3) FBSR_DECLARE_DISPATCH(4)
#undef FBSR_DECLARE_DISPATCH

// Lets a kernel have `bytes` of dynamic shared memory: asked for once per kernel and device, `done` holding a bit for each
// device that has been asked.  FBSR_OK (0) or FBSR_ERR_CUDA (4).
inline int allow_shared_memory(const void* kernel, int bytes, std::atomic<uint64_t>& done)
{
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return 4;
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return 4;
    done.fetch_or(bit, std::memory_order_relaxed);
    return 0;
}

// Rows of `width` bytes in memory, `outer` times `inner` of them; strides in bytes, the outer one not the smaller.
struct RowSet {
    typedef __int128 Wide;                       // no product of a stride and a count passes it
    Wide base, outer_stride, inner_stride, outer, inner, width;

    RowSet(const void* p, int64_t outer_step, int64_t inner_step, size_t outer_count, size_t inner_count, size_t elements, size_t bytes)
        : base((Wide)reinterpret_cast<uintptr_t>(p)), outer_stride((Wide)outer_step * (int64_t)bytes), inner_stride((Wide)inner_step * (int64_t)bytes),
          outer(outer_count), inner(inner_count), width((Wide)elements * (int64_t)bytes)
    {
        settle(outer_stride, outer);
        settle(inner_stride, inner);
        if (outer_stride < inner_stride) { std::swap(outer_stride, inner_stride); std::swap(outer, inner); }
    }

    Wide reach() const { return (inner - 1) * inner_stride + width; }
    Wide end() const { return base + (outer - 1) * outer_stride + reach(); }

    // Whether a row meets the bytes [x, x + n).
    bool meets(Wide x, Wide n) const
    {
        Wide first, last, low, high;
        steps(x - base, n, reach(), outer_stride, outer, first, last);
        for (; first <= last; ++first) {
            steps(x - base - first * outer_stride, n, width, inner_stride, inner, low, high);
            if (low <= high) return true;
        }
        return false;
    }

private:
    // The same row again, or one alone, is a row without a stride; a negative stride counts from the other end.
    void settle(Wide& stride, Wide& count)
    {
        if (count <= 1 || stride == 0) { count = 1; stride = 0; }
        if (stride < 0) { base += (count - 1) * stride; stride = -stride; }
    }
    static Wide floor_div(Wide a, Wide b) { return a / b - (a % b < 0 ? 1 : 0); }
    // The steps 0 <= i < count for which [i stride, i stride + reach) meets [x, x + n).
    static void steps(Wide x, Wide n, Wide reach, Wide stride, Wide count, Wide& first, Wide& last)
    {
        if (stride == 0) { first = 0; last = x < reach && x + n > 0 ? 0 : -1; return; }
        first = std::max<Wide>(floor_div(x - reach, stride) + 1, 0);
        last = std::min<Wide>(floor_div(x + n - 1, stride), count - 1);
    }
};

// Whether a byte of `read` is one of `written`, whose own rows lie apart.  Apart as a whole, as nearly always: a few comparisons.  Rows of the same
// strides, as those of one buffer are: the rows of both meet as the first of `read` meets the rows of `written` moved by every difference
// of their places.  Otherwise row by row.
inline bool rows_meet(const RowSet& read, const RowSet& written)
{
    if (read.end() <= written.base || written.end() <= read.base) return false;
    if (read.outer_stride == written.outer_stride && read.inner_stride == written.inner_stride) {
        RowSet moved = written;
        moved.base -= (read.outer - 1) * read.outer_stride + (read.inner - 1) * read.inner_stride;
        moved.outer += read.outer - 1;
        moved.inner += read.inner - 1;
        return moved.meets(read.base, read.width);
    }
    for (RowSet::Wide i = 0; i < read.outer; ++i)
        for (RowSet::Wide j = 0; j < read.inner; ++j)
            if (written.meets(read.base + i * read.outer_stride + j * read.inner_stride, read.width)) return true;
    return false;
}

void count_launch();                         // bumps the counter behind fbsr_launch_count()

}  // namespace fbsr
