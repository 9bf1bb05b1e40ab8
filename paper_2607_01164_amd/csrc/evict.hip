// Cutting a set of Gaussians down to those of the largest score, and copies
// that share a Gaussian's weight (include/gs_budget.h).
//
// Eviction is a selection, not a sort: the order is that of a 33-bit key
// (pinned, then the score's bits made monotone), whose budget-th largest value
// three counting passes over the scores find digit by digit; what lies above
// it stays, and as many of its equals, by index, as the budget leaves. Bound
// by the rows of the kept ones, read and written once.
#include "budget.h"

namespace gs {
namespace {

size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

// The score's place in the order as an unsigned number: NaN first, -0 as 0.
__device__ __forceinline__ uint32_t score_key(float s) {
    if (!(s == s)) return 0u;
    const uint32_t b = __float_as_uint(s + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// Digits of the key: pinned and its top 11 bits, the next 11, the last 10.
constexpr uint32_t kBins0 = 4096, kBins1 = 2048, kBins2 = 1024;
constexpr uint32_t kBinsAll = kBins0 + kBins1 + kBins2;
constexpr uint32_t kTile = 1024;        // Gaussians of a tile: 4 a thread
constexpr uint32_t kBlocksMost = 1024;  // workgroups of a pass, each over a stretch of tiles

struct Key {
    uint32_t key, pin;
};
__device__ __forceinline__ Key load_key(const float *score, const uint8_t *pinned, int64_t i) {
    return Key{score_key(score[i]), pinned && pinned[i] ? 1u : 0u};
}

// Where the cut lies so far: the digits found, and how many Gaussians are
// still to be taken among those that have them.
struct Cut {
    uint32_t pin, key;  // of the cut's key, the digits found
    uint32_t need;
};

// The bin of a histogram in which the need-th element from the top lies; need
// becomes its rank in there. For the whole workgroup (kBlock threads); lds:
// kWavesPerBlock + 2 words. need is at least 1 and at most the sum.
template <uint32_t BINS>
__device__ uint32_t find_bin(const uint32_t *__restrict__ hist, uint32_t &need, uint32_t *lds) {
    constexpr uint32_t kEach = BINS / kBlock;
    // thread 0 has the top bins
    const uint32_t top = BINS - 1 - threadIdx.x * kEach;
    uint32_t c[kEach], sum = 0, total;
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) sum += c[j] = hist[top - j];
    uint32_t above = block_excl_scan(sum, lds, &total);
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
        if (above < need && need <= above + c[j]) {
            lds[kWavesPerBlock] = top - j;
            lds[kWavesPerBlock + 1] = need - above;
        }
        above += c[j];
    }
    __syncthreads();
    const uint32_t bin = lds[kWavesPerBlock];
    need = lds[kWavesPerBlock + 1];
    __syncthreads();
    return bin;
}

// The first PASS digits of the cut.
template <int PASS>
__device__ Cut find_cut(const uint32_t *hist, uint32_t keep, uint32_t *lds) {
    Cut c{0, 0, keep};
    if (PASS > 0) {
        const uint32_t b = find_bin<kBins0>(hist, c.need, lds);
        c.pin = b >> 11;
        c.key = b << 21;
    }
    if (PASS > 1) c.key |= find_bin<kBins1>(hist + kBins0, c.need, lds) << 10;
    if (PASS > 2) c.key |= find_bin<kBins2>(hist + kBins0 + kBins1, c.need, lds);
    return c;
}

// Counts of digit PASS over the Gaussians that have the cut's earlier digits.
template <int PASS>
__global__ __launch_bounds__(kBlock) void k_evict_count(int64_t n, int64_t stretch, const float *__restrict__ score,
                                                        const uint8_t *__restrict__ pinned, uint32_t keep,
                                                        uint32_t *__restrict__ hist) {
    constexpr uint32_t kBins = PASS == 0 ? kBins0 : PASS == 1 ? kBins1 : kBins2;
    __shared__ uint32_t s_hist[kBins];
    __shared__ uint32_t lds[kWavesPerBlock + 2];
    for (uint32_t b = threadIdx.x; b < kBins; b += kBlock) s_hist[b] = 0;
    const Cut cut = find_cut<PASS>(hist, keep, lds);
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * stretch, i1 = i0 + stretch < n ? i0 + stretch : n;
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kBlock) {
        const Key k = load_key(score, pinned, i);
        if (PASS == 0) {
            atomicAdd(&s_hist[k.pin << 11 | k.key >> 21], 1u);
        } else if (PASS == 1) {
            if (k.pin == cut.pin && ((k.key ^ cut.key) >> 21) == 0) atomicAdd(&s_hist[k.key >> 10 & 2047u], 1u);
        } else {
            if (k.pin == cut.pin && ((k.key ^ cut.key) >> 10) == 0) atomicAdd(&s_hist[k.key & 1023u], 1u);
        }
    }
    __syncthreads();
    uint32_t *out = hist + (PASS == 0 ? 0u : PASS == 1 ? kBins0 : kBins0 + kBins1);
    for (uint32_t b = threadIdx.x; b < kBins; b += kBlock)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
}

__device__ __forceinline__ bool above_cut(Key k, const Cut &c) {
    return k.pin > c.pin || (k.pin == c.pin && k.key > c.key);
}
__device__ __forceinline__ bool at_cut(Key k, const Cut &c) { return k.pin == c.pin && k.key == c.key; }

// Per stretch, the Gaussians above the cut and at it.
__global__ __launch_bounds__(kBlock) void k_evict_stretch(int64_t n, int64_t stretch,
                                                          const float *__restrict__ score,
                                                          const uint8_t *__restrict__ pinned, uint32_t keep,
                                                          const uint32_t *__restrict__ hist,
                                                          uint2 *__restrict__ sums) {
    __shared__ uint32_t lds[kWavesPerBlock + 2];
    const Cut cut = find_cut<3>(hist, keep, lds);
    const int64_t i0 = (int64_t)blockIdx.x * stretch, i1 = i0 + stretch < n ? i0 + stretch : n;
    uint32_t above = 0, at = 0;
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kBlock) {
        const Key k = load_key(score, pinned, i);
        above += above_cut(k, cut) ? 1u : 0u;
        at += at_cut(k, cut) ? 1u : 0u;
    }
    uint32_t total_above, total_at;
    block_excl_scan(above, lds, &total_above);
    block_excl_scan(at, lds, &total_at);
    if (threadIdx.x == 0) sums[blockIdx.x] = make_uint2(total_above, total_at);
}

// Sources of the kept Gaussians, in the order of their indices.
__global__ __launch_bounds__(kBlock) void k_evict_source(int64_t n, int64_t stretch,
                                                         const float *__restrict__ score,
                                                         const uint8_t *__restrict__ pinned, uint32_t keep,
                                                         const uint32_t *__restrict__ hist,
                                                         const uint2 *__restrict__ sums,
                                                         int32_t *__restrict__ source) {
    __shared__ uint32_t lds[kWavesPerBlock + 2];
    const Cut cut = find_cut<3>(hist, keep, lds);
    uint32_t above = 0, at = 0;
    for (uint32_t b = threadIdx.x; b < blockIdx.x; b += kBlock) {
        above += sums[b].x;
        at += sums[b].y;
    }
    uint32_t before, ties;  // above the cut and at it, in earlier stretches
    block_excl_scan(above, lds, &before);
    block_excl_scan(at, lds, &ties);
    const int64_t i0 = (int64_t)blockIdx.x * stretch, i1 = i0 + stretch < n ? i0 + stretch : n;
    for (int64_t t0 = i0; t0 < i1; t0 += kBlock) {
        const int64_t i = t0 + threadIdx.x;
        const bool in = i < i1;
        const Key k = in ? load_key(score, pinned, i) : Key{0, 0};
        const uint32_t up = in && above_cut(k, cut) ? 1u : 0u, tie = in && at_cut(k, cut) ? 1u : 0u;
        uint32_t ups, more;
        const uint32_t rank = before + block_excl_scan(up, lds, &ups);
        const uint32_t place = ties + block_excl_scan(tie, lds, &more);
        const uint32_t taken = place < cut.need ? place : cut.need;  // equals kept before this one
        if (up || (tie && place < cut.need)) source[rank + taken] = (int32_t)i;
        before += ups;
        ties += more;
    }
}

// The rows of the kept Gaussians.
__global__ __launch_bounds__(kBlock) void k_evict_rows(int64_t keep, gs_params in, const float *__restrict__ score,
                                                       const int32_t *__restrict__ source, gs_params out,
                                                       float *__restrict__ score_out) {
    const int64_t d = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (d >= keep) return;
    const int64_t i = source[d];
#pragma unroll
    for (int a = 0; a < 3; ++a) {
        out.mean[3 * d + a] = in.mean[3 * i + a];
        out.log_scale[3 * d + a] = in.log_scale[3 * i + a];
    }
#pragma unroll
    for (int a = 0; a < 4; ++a) out.rot[4 * d + a] = in.rot[4 * i + a];
    out.value_logit[d] = in.value_logit[i];
    out.weight_logit[d] = in.weight_logit[i];
    if (score_out) score_out[d] = score[i];
}

// Copies. Counting the draws of a Gaussian touches only those drawn: their
// counts are cleared, then raised by integer atomics (any order gives the
// same), then every copy works out the shared weight from the logit that it
// took along; the copies of one Gaussian write the same number to it.
__global__ __launch_bounds__(kBlock) void k_split_clear(int64_t n, const int32_t *__restrict__ ids, int64_t count,
                                                        uint32_t *__restrict__ copies) {
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j >= count) return;
    const int64_t i = ids[j];
    if (i >= 0 && i < n) copies[i] = 1u;
}

__global__ __launch_bounds__(kBlock) void k_split_rows(gs_params set, int64_t n, const int32_t *__restrict__ ids,
                                                       int64_t count, int32_t *__restrict__ source,
                                                       float *__restrict__ score, uint32_t *__restrict__ copies) {
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j >= count) return;
    const int64_t i = ids[j], d = n + j;
    const bool some = i >= 0 && i < n;
    if (some) atomicAdd(&copies[i], 1u);
#pragma unroll
    for (int a = 0; a < 3; ++a) {
        set.mean[3 * d + a] = some ? set.mean[3 * i + a] : __uint_as_float(0x7FC00000u);
        set.log_scale[3 * d + a] = some ? set.log_scale[3 * i + a] : 0.0f;
    }
#pragma unroll
    for (int a = 0; a < 4; ++a) set.rot[4 * d + a] = some ? set.rot[4 * i + a] : (a == 0 ? 1.0f : 0.0f);
    set.value_logit[d] = some ? set.value_logit[i] : 0.0f;
    set.weight_logit[d] = some ? set.weight_logit[i] : -__builtin_inff();
    if (score) score[d] = some ? score[i] : 0.0f;
    if (source) source[d] = i >= 0 ? (int32_t)(-1 - i) : -1;
}

__global__ __launch_bounds__(kBlock) void k_split_weights(gs_params set, int64_t n, const int32_t *__restrict__ ids,
                                                          int64_t count, float *__restrict__ score,
                                                          const uint32_t *__restrict__ copies) {
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j >= count) return;
    const int64_t i = ids[j], d = n + j;
    if (i < 0 || i >= n) return;
    // w / c with w = 1 / (1 + e^-l): -ln(c (1 + e^-l) - 1); far down, where
    // e^-l is all of that, l - ln c
    const double c = (double)copies[i], l = (double)set.weight_logit[d];
    const double shared = l < -30.0 ? l - log(c) : -log((c - 1.0) + c * exp(-l));
    set.weight_logit[d] = (float)shared;
    set.weight_logit[i] = (float)shared;
    if (score) {
        const float s = (float)((double)score[d] / c);
        score[d] = s;
        score[i] = s;
    }
}

struct EvictWork {
    uint32_t *hist;
    uint2 *sums;
    size_t bytes;
};
EvictWork evict_layout(void *base) {
    EvictWork w;
    char *b = (char *)base;
    w.hist = (uint32_t *)b;
    w.sums = (uint2 *)(b + al256(sizeof(uint32_t) * kBinsAll));
    w.bytes = al256(sizeof(uint32_t) * kBinsAll) + al256(sizeof(uint2) * kBlocksMost);
    return w;
}

dim3 blocks_of(int64_t n) { return dim3((uint32_t)((n + kBlock - 1) / kBlock)); }

}  // namespace

size_t evict_work_bytes(int64_t) { return evict_layout(nullptr).bytes; }

hipError_t launch_evict(const gs_params &in, int64_t n, const float *score, const uint8_t *pinned, int64_t keep,
                        const gs_params &out, int32_t *source, float *score_out, void *work, hipStream_t s) {
    if (keep <= 0) return hipSuccess;
    const EvictWork w = evict_layout(work);
    // a stretch of whole tiles for every workgroup
    const int64_t tiles = (n + kTile - 1) / kTile;
    const int64_t each = (tiles + kBlocksMost - 1) / kBlocksMost;
    const int64_t stretch = each * kTile;
    const dim3 nb((uint32_t)((n + stretch - 1) / stretch)), tb(kBlock);
    const uint32_t k = (uint32_t)keep;
    hipError_t e;
    prof_begin("evict_select", s);
    if ((e = fill_u32(w.hist, 0u, kBinsAll, s)) != hipSuccess) return e;
    hipLaunchKernelGGL(k_evict_count<0>, nb, tb, 0, s, n, stretch, score, pinned, k, w.hist);
    hipLaunchKernelGGL(k_evict_count<1>, nb, tb, 0, s, n, stretch, score, pinned, k, w.hist);
    hipLaunchKernelGGL(k_evict_count<2>, nb, tb, 0, s, n, stretch, score, pinned, k, w.hist);
    hipLaunchKernelGGL(k_evict_stretch, nb, tb, 0, s, n, stretch, score, pinned, k, w.hist, w.sums);
    hipLaunchKernelGGL(k_evict_source, nb, tb, 0, s, n, stretch, score, pinned, k, w.hist, w.sums, source);
    prof_end("evict_select", s);
    prof_begin("evict_rows", s);
    hipLaunchKernelGGL(k_evict_rows, blocks_of(keep), tb, 0, s, keep, in, score, source, out, score_out);
    prof_end("evict_rows", s);
    return hipGetLastError();
}

hipError_t launch_split(const gs_params &set, int64_t n, const int32_t *ids, int64_t count, int32_t *source,
                        float *score, uint32_t *copies, hipStream_t s) {
    if (count <= 0) return hipSuccess;
    const dim3 nb = blocks_of(count), tb(kBlock);
    prof_begin("split", s);
    hipLaunchKernelGGL(k_split_clear, nb, tb, 0, s, n, ids, count, copies);
    hipLaunchKernelGGL(k_split_rows, nb, tb, 0, s, set, n, ids, count, source, score, copies);
    hipLaunchKernelGGL(k_split_weights, nb, tb, 0, s, set, n, ids, count, score, copies);
    prof_end("split", s);
    return hipGetLastError();
}

}  // namespace gs
