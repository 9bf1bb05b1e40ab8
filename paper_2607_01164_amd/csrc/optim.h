// Internal declarations of the optimiser step (optim.hip, api.cpp): the
// pieces of a list of tensors, and the launchers' arguments.
#pragma once

#include "../../include/gs_optim.h"
#include "internal.h"

namespace gs {

constexpr int64_t kOptimChunk = 1024;  // elements of an item at most: a multiple of 32 that divides 2^32
// Elements of a NormItem at most: with 4096 the norm of 0.26 to 1 M Gaussians
// takes 0.6 to 1.2 us longer (more sums to leave), that of fewer as long, and
// that of 267 M bfloat16 elements 4 % less.
constexpr int64_t kNormChunk = 16384;
constexpr uint32_t kCarryMost = 4096;  // elements of a workgroup's rows in the carry at most

// Flags of a tensor and its items.
constexpr uint32_t kParamBf16 = 1, kGradBf16 = 2, kMoments8 = 4;

struct OptimTensor {
    void *p;
    const void *g;
    void *m, *v;
    uint8_t *ms, *vs;
    int64_t n;
    uint32_t place, flags;
    float lr, wd;
};

// A piece of a tensor: its arrays from the piece's first element on.
struct alignas(16) OptimItem {
    void *p;
    const void *g;
    void *m, *v;
    uint8_t *ms, *vs;
    int64_t base;     // index of the first element in its tensor
    int32_t count;
    uint32_t place;   // of the tensor in the list
    float lr, wd;
    uint32_t flags, pad;
};

// A piece of a tensor for the norm, longer than an OptimItem.
struct alignas(16) NormItem {
    const void *g;
    int32_t count;
    uint32_t flags;
};

// The norm's workspace: a partial sum for each workgroup, and counters of
// those that are done, each in a line of its own: the root's, then one for
// each group of workgroups.
constexpr int kNormBlocks = 2048;  // workgroups at most
constexpr uint32_t kNormGroup = 32;
constexpr int kNormCounters = 1 + kNormBlocks / (int)kNormGroup;
constexpr int kNormCounter = 32;  // words from one counter to the next
struct NormWork {
    double *part;
    uint32_t *count;
};

struct StepArgs {
    float b1, a1, b2, a2, eps, lr_scale, first, second;
    uint64_t step, seed;
};
struct NormArgs {
    double beta1, beta2, max_norm;
};
struct CarryArray {
    const void *m, *v;
    const uint8_t *m_scale, *v_scale;
    void *m_out, *v_out;
    uint8_t *m_scale_out, *v_scale_out;
    // rows: of a workgroup, a multiple of 32. over, over_parts: x / d = x over
    // >> 20 with over = 2^20 / d, up, for d = width and the (width + 3) / 4
    // parts of a row (x below 2^14 times over's excess, below d <= 64, stays
    // below 2^20).
    uint32_t width, rows, over, over_parts;
    uint32_t moments8, pad;
};
// 8-bit rows: 4 parts of a row a thread (2 M Gaussians take a tenth longer
// with 2 parts, and with 8, which leave fewer workgroups resident; 262144 take
// 0.9 us less with 2); 32-bit rows: one pass of 4 elements a thread.
inline uint32_t carry_rows(uint32_t width, bool moments8) {
    const uint32_t most = moments8 ? (width < 4 ? 1024 * width : kCarryMost) : 1024;
    const uint32_t rows = most / width / 32 * 32;
    return rows ? rows : 32;
}
struct CarryArgs {
    CarryArray rows[GS_ADAMW_ROWS_MAX];
    uint32_t first[GS_ADAMW_ROWS_MAX];  // first workgroup of each array, 2^32 - 1 past the last
    uint32_t block0;                    // the launch's first workgroup
    int64_t n_in, n_out;
};

// Scales of n > 0 elements, for every n of the type (n + 31 need not fit it).
template <typename U>
constexpr U scale_count(U n) {
    return ((n - 1) >> 5) + 1;
}
static_assert(scale_count(1u) == 1 && scale_count(32u) == 1 && scale_count(33u) == 2, "blocks of 32");
static_assert(scale_count(0xFFFFFFE0u) == 0x7FFFFFFu && scale_count(0xFFFFFFE1u) == 0x8000000u &&
                  scale_count(0xFFFFFFFFu) == 0x8000000u,
              "up to the end of 32 bits");

inline int64_t norm_items(int64_t n) { return (n + kNormChunk - 1) / kNormChunk; }
inline int64_t optim_items(int64_t n) { return (n + kOptimChunk - 1) / kOptimChunk; }
inline uint32_t optim_flags(const gs_adamw_tensor &t) {
    uint32_t f = 0;
    if (t.param_type == GS_TYPE_BF16) f |= kParamBf16;
    if (t.grad_type == GS_TYPE_BF16) f |= kGradBf16;
    if (t.moments == GS_MOMENTS_MXFP8) f |= kMoments8;
    return f;
}

hipError_t launch_plan_adamw(const gs_adamw_tensor *tensors, int64_t count, OptimItem *items, NormItem *norms,
                             const NormWork &work, hipStream_t s);
// once: keep nothing in the caches
hipError_t launch_grad_norm(const NormItem *items, int64_t n_items, bool once, const NormWork &work,
                            const NormArgs &a, gs_adamw_control *control, hipStream_t s);
hipError_t launch_adamw(const OptimItem *items, int64_t n_items, bool once, const StepArgs &a,
                        const gs_adamw_control *control, hipStream_t s);
hipError_t launch_adamw_carry(const gs_adamw_rows *arrays, int count, int64_t n_in, const int32_t *source,
                              int64_t n_out, hipStream_t s);

}  // namespace gs
