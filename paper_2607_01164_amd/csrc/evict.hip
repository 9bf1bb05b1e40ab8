// Cutting a set of Gaussians down to those of the largest score, and copies
// that share a Gaussian's weight (include/gs_budget.h).
//
// Eviction is a selection, not a sort: the order is that of a 33-bit key
// (pinned, then the score's bits made monotone), whose budget-th largest value
// three counting passes over the scores find digit by digit; what lies above
// it stays, and as many of its equals, by index, as the budget leaves. Bound
// by the rows of the kept ones, read and written once: half of 2 M Gaussians
// moves 173 MB (lines of which half is kept) in 36 us, after five launches of 5
// to 8 us for the scores and counts; smaller sets by their six launches.
#include <type_traits>

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
constexpr uint32_t kDigits = 3;
constexpr uint32_t kBins0 = 4096, kBins1 = 2048, kBins2 = 1024;
constexpr uint32_t kBinsAll = kBins0 + kBins1 + kBins2;
constexpr uint32_t bins_of(int digit) { return digit == 0 ? kBins0 : digit == 1 ? kBins1 : kBins2; }
constexpr uint32_t bins_before(int digit) { return digit == 0 ? 0 : digit == 1 ? kBins0 : kBins0 + kBins1; }
constexpr uint32_t kEach = 4;                 // Gaussians of a thread in a tile
constexpr uint32_t kTile = kBlock * kEach;
constexpr uint32_t kBlocksMost = 1024;        // workgroups of a pass, each over a stretch of tiles
// The counting passes end with an atomic add for every bin that a workgroup
// met, and those to one address wait for each other (1024 workgroups: 15 us
// of a pass of 20): few, large workgroups, and kCopies of the counts.
constexpr uint32_t kCountThreads = 1024;
constexpr uint32_t kCountBlocks = 256;
constexpr uint32_t kCopies = 4;
constexpr uint32_t kSmallThreads = 1024;
constexpr int64_t kSmall = 16384;             // sets that one workgroup selects from

struct Key {
    uint32_t key, pin;
};

// Where the cut lies so far: the digits found of its key, and how many
// Gaussians are still to be taken among those that have them.
struct Cut {
    uint32_t pin, key, need, pad;
};

template <int DIGIT>
__device__ __forceinline__ uint32_t digit_of(Key k) {
    return DIGIT == 0 ? k.pin << 11 | k.key >> 21 : DIGIT == 1 ? k.key >> 10 & 2047u : k.key & 1023u;
}
template <int DIGIT>
__device__ __forceinline__ bool has_digits(Key k, const Cut &c) {
    if (DIGIT == 0) return true;
    return k.pin == c.pin && ((k.key ^ c.key) >> (DIGIT == 1 ? 21 : 10)) == 0;
}
__device__ __forceinline__ bool above_cut(Key k, const Cut &c) {
    return k.pin > c.pin || (k.pin == c.pin && k.key > c.key);
}
__device__ __forceinline__ bool at_cut(Key k, const Cut &c) { return k.pin == c.pin && k.key == c.key; }

// Keys of Gaussians i .. i + 3, those below i1; returns how many.
__device__ __forceinline__ uint32_t load_keys(const float *score, const uint8_t *pinned, int64_t i, int64_t i1,
                                              Key k[kEach]) {
    typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t m = i + kEach <= i1 ? kEach : i < i1 ? (uint32_t)(i1 - i) : 0u;
    float v[kEach] = {};
    uint32_t pin = 0;
    if (m == kEach) {
        const f4a q = *(const f4a *)(score + i);
        v[0] = q.x;
        v[1] = q.y;
        v[2] = q.z;
        v[3] = q.w;
        if (pinned) __builtin_memcpy(&pin, pinned + i, 4);
    } else {
        for (uint32_t t = 0; t < m; ++t) {
            v[t] = score[i + t];
            if (pinned) pin |= (uint32_t)pinned[i + t] << (8 * t);
        }
    }
#pragma unroll
    for (uint32_t t = 0; t < kEach; ++t) k[t] = Key{score_key(v[t]), (pin >> (8 * t) & 255u) ? 1u : 0u};
    return m;
}

// Adds 1 to a bin for every active lane. Scores repeat (a Gaussian that no
// query reached has none), and lanes that meet in a bin wait for each other:
// the bin of the first lane is counted for all lanes at once. (2 M scores, 0.6
// of them 0: the selection 38 -> 32 us; 262144 different scores: 21.6 -> 22.7.)
__device__ __forceinline__ void hist_add(uint32_t *hist, uint32_t bin, bool active) {
    const uint64_t any = __ballot(active);
    if (any == 0) return;
    const uint32_t leader = (uint32_t)__builtin_ctzll(any);
    const bool meets = active && bin == (uint32_t)__builtin_amdgcn_readlane(bin, leader);
    const uint64_t same = __ballot(meets);
    if (lane_id() == leader) atomicAdd(&hist[bin], (uint32_t)__popcll(same));
    if (active && !meets) atomicAdd(&hist[bin], 1u);
}

// Exclusive sums over a workgroup of NT threads; *total gets the sum.
template <int NT>
__device__ __forceinline__ uint32_t group_scan(uint32_t x, uint32_t *lds, uint32_t *total) {
    constexpr uint32_t kWaves = NT / kWave;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const uint32_t incl = wave_incl_sum(x);
    __syncthreads();
    if (lane == kWave - 1) lds[wave] = incl;
    __syncthreads();
    const uint32_t upto = wave_incl_sum(lane < kWaves ? lds[lane] : 0u);
    *total = __builtin_amdgcn_readlane(upto, kWaves - 1);
    return (wave ? (uint32_t)__builtin_amdgcn_readlane(upto, wave - 1) : 0u) + incl - x;
}

// The cut with its next digit, from that digit's counts: the bin in which
// the need-th Gaussian from the top lies. need is at least 1 and at most the
// sum. lds: NT / kWave + 2 words.
template <int NT, int DIGIT, int COPIES>
__device__ Cut next_digit(Cut cut, const uint32_t *hist, uint32_t *lds) {
    constexpr uint32_t kBins = bins_of(DIGIT), kMine = kBins / NT > 0 ? kBins / NT : 1;
    const uint32_t top = kBins - 1 - threadIdx.x * kMine;  // thread 0 has the top bins
    uint32_t c[kMine], sum = 0, total;
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        c[j] = 0;
        if (threadIdx.x * kMine + j < kBins) {
#pragma unroll
            for (int r = 0; r < COPIES; ++r) c[j] += hist[r * kBinsAll + top - j];
        }
        sum += c[j];
    }
    uint32_t above = group_scan<NT>(sum, lds, &total);
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        if (above < cut.need && cut.need <= above + c[j]) {
            lds[NT / kWave] = top - j;
            lds[NT / kWave + 1] = cut.need - above;
        }
        above += c[j];
    }
    __syncthreads();
    const uint32_t bin = lds[NT / kWave];
    cut.need = lds[NT / kWave + 1];
    if (DIGIT == 0) {
        cut.pin = bin >> 11;
        cut.key = bin << 21;
    } else {
        cut.key |= DIGIT == 1 ? bin << 10 : bin;
    }
    return cut;
}

// The cut after digit DIGIT, given what a pass before kept of the earlier
// ones; the first workgroup keeps it for the passes after.
template <int NT, int DIGIT>
__device__ Cut cut_after(const uint32_t *hist, Cut *cuts, uint32_t keep, uint32_t *lds) {
    Cut c{0, 0, keep, 0};
    if (DIGIT > 0) c = cuts[DIGIT > 0 ? DIGIT - 1 : 0];
    c = next_digit<NT, DIGIT, kCopies>(c, hist + bins_before(DIGIT), lds);
    if (blockIdx.x == 0 && threadIdx.x == 0) cuts[DIGIT] = c;
    return c;
}

// Counts of a digit over the Gaussians that have the cut's earlier digits.
template <int DIGIT>
__global__ __launch_bounds__(kCountThreads) void k_evict_count(int64_t n, int64_t stretch,
                                                               const float *__restrict__ score,
                                                               const uint8_t *__restrict__ pinned, uint32_t keep,
                                                               uint32_t *hist, Cut *cuts) {
    constexpr uint32_t kBins = bins_of(DIGIT);
    __shared__ uint32_t s_hist[kBins];
    __shared__ uint32_t lds[kCountThreads / kWave + 2];
    for (uint32_t b = threadIdx.x; b < kBins; b += kCountThreads) s_hist[b] = 0;
    Cut cut{};
    if (DIGIT > 0) cut = cut_after<kCountThreads, DIGIT ? DIGIT - 1 : 0>(hist, cuts, keep, lds);
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * stretch, i1 = i0 + stretch < n ? i0 + stretch : n;
    for (int64_t t0 = i0; t0 < i1; t0 += kCountThreads * kEach) {
        Key k[kEach];
        const uint32_t m = load_keys(score, pinned, t0 + threadIdx.x * kEach, i1, k);
#pragma unroll
        for (uint32_t t = 0; t < kEach; ++t)
            hist_add(s_hist, digit_of<DIGIT>(k[t]), t < m && has_digits<DIGIT>(k[t], cut));
    }
    __syncthreads();
    uint32_t *out = hist + blockIdx.x % kCopies * kBinsAll + bins_before(DIGIT);
    for (uint32_t b = threadIdx.x; b < kBins; b += kCountThreads)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
}

// Per stretch, the Gaussians above the cut and at it.
__global__ __launch_bounds__(kBlock) void k_evict_stretch(int64_t n, int64_t stretch,
                                                          const float *__restrict__ score,
                                                          const uint8_t *__restrict__ pinned, uint32_t keep,
                                                          const uint32_t *hist, Cut *cuts,
                                                          uint2 *__restrict__ sums) {
    __shared__ uint32_t lds[kWavesPerBlock + 2];
    const Cut cut = cut_after<kBlock, kDigits - 1>(hist, cuts, keep, lds);
    const int64_t i0 = (int64_t)blockIdx.x * stretch, i1 = i0 + stretch < n ? i0 + stretch : n;
    uint32_t above = 0, at = 0;
    for (int64_t t0 = i0; t0 < i1; t0 += kTile) {
        Key k[kEach];
        const uint32_t m = load_keys(score, pinned, t0 + threadIdx.x * kEach, i1, k);
#pragma unroll
        for (uint32_t t = 0; t < kEach; ++t) {
            above += t < m && above_cut(k[t], cut) ? 1u : 0u;
            at += t < m && at_cut(k[t], cut) ? 1u : 0u;
        }
    }
    uint32_t total_above, total_at;
    group_scan<kBlock>(above, lds, &total_above);
    group_scan<kBlock>(at, lds, &total_at);
    if (threadIdx.x == 0) sums[blockIdx.x] = make_uint2(total_above, total_at);
}

// A Gaussian's free parameters: one access an array. (Accesses of 4 bytes to
// a line that is still on its way wait for it one by one: 419430 copies out
// of 2 M Gaussians took 87 us with them.)
typedef float f3a __attribute__((ext_vector_type(3), aligned(4)));
typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
struct Row {
    f3a mean, log_scale;
    f4a rot;
    float value, weight;
};
// (a vector of three floats takes the place of four in C: rows are addressed
// as floats)
__device__ __forceinline__ Row load_row(const gs_params &p, int64_t i) {
    Row r;
    __builtin_memcpy(&r.mean, p.mean + 3 * i, 12);
    __builtin_memcpy(&r.log_scale, p.log_scale + 3 * i, 12);
    r.rot = *(const f4a *)(p.rot + 4 * i);
    r.value = p.value_logit[i];
    r.weight = p.weight_logit[i];
    return r;
}
__device__ __forceinline__ void store_row(const gs_params &p, int64_t d, const Row &r) {
    __builtin_memcpy(p.mean + 3 * d, &r.mean, 12);
    __builtin_memcpy(p.log_scale + 3 * d, &r.log_scale, 12);
    *(f4a *)(p.rot + 4 * d) = r.rot;
    p.value_logit[d] = r.value;
    p.weight_logit[d] = r.weight;
}

// A row of the output.
__device__ __forceinline__ void keep_row(const gs_params &in, const float *score, int64_t i, const gs_params &out,
                                         float *score_out, int64_t d) {
    const Row r = load_row(in, i);
    if (score_out) score_out[d] = score[i];
    store_row(out, d, r);
}

// The kept Gaussians of every stretch, in the order of their indices: a
// tile's go to LDS, then their rows are copied side by side.
__global__ __launch_bounds__(kBlock) void k_evict_keep(int64_t n, int64_t stretch, const float *__restrict__ score,
                                                       const uint8_t *__restrict__ pinned,
                                                       const Cut *__restrict__ cuts, const uint2 *__restrict__ sums,
                                                       gs_params in, gs_params out, int32_t *__restrict__ source,
                                                       float *__restrict__ score_out) {
    __shared__ uint32_t lds[kWavesPerBlock];
    __shared__ uint32_t s_kept[kTile];
    const Cut cut = cuts[kDigits - 1];
    uint32_t above = 0, at = 0;
    for (uint32_t b = threadIdx.x; b < blockIdx.x; b += kBlock) {
        above += sums[b].x;
        at += sums[b].y;
    }
    uint32_t before, ties;  // above the cut and at it, in earlier stretches
    group_scan<kBlock>(above, lds, &before);
    group_scan<kBlock>(at, lds, &ties);
    const int64_t i0 = (int64_t)blockIdx.x * stretch, i1 = i0 + stretch < n ? i0 + stretch : n;
    for (int64_t t0 = i0; t0 < i1; t0 += kTile) {
        const int64_t i = t0 + threadIdx.x * kEach;
        Key k[kEach];
        const uint32_t m = load_keys(score, pinned, i, i1, k);
        uint32_t mine = 0, total;  // above: low half, at: high half
#pragma unroll
        for (uint32_t t = 0; t < kEach; ++t)
            if (t < m) mine += above_cut(k[t], cut) ? 1u : at_cut(k[t], cut) ? 0x10000u : 0u;
        uint32_t run = group_scan<kBlock>(mine, lds, &total);
        const uint32_t taken = ties < cut.need ? ties : cut.need;  // equals kept in earlier tiles
        const uint32_t room = cut.need - taken;                    // and still to be kept
#pragma unroll
        for (uint32_t t = 0; t < kEach; ++t) {
            const bool up = t < m && above_cut(k[t], cut), tie = t < m && at_cut(k[t], cut);
            const uint32_t equals = run >> 16, kept = equals < room ? equals : room;
            if (up || (tie && equals < room)) s_kept[(run & 0xFFFFu) + kept] = (uint32_t)(i + t);
            run += up ? 1u : tie ? 0x10000u : 0u;
        }
        const uint32_t more = total >> 16, ups = total & 0xFFFFu;
        const uint32_t count = ups + (more < room ? more : room);
        const int64_t first = (int64_t)before + taken;
        __syncthreads();
        for (uint32_t r = threadIdx.x; r < count; r += kBlock) {
            const uint32_t from = s_kept[r];
            source[first + r] = (int32_t)from;
            keep_row(in, score, from, out, score_out, first + r);
        }
        before += ups;
        ties += more;
        __syncthreads();
    }
}

// Small sets: the whole selection in one workgroup, its keys in registers.
__global__ __launch_bounds__(kSmallThreads) void k_evict_small(int n, const float *__restrict__ score,
                                                               const uint8_t *__restrict__ pinned, uint32_t keep,
                                                               int32_t *__restrict__ source) {
    constexpr int kTiles = (int)(kSmall / (kSmallThreads * kEach));
    __shared__ uint32_t s_hist[kBins0];
    __shared__ uint32_t lds[kSmallThreads / kWave + 2];
    Key k[kTiles][kEach];
    uint32_t m[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
        m[t] = load_keys(score, pinned, (t * kSmallThreads + threadIdx.x) * kEach, n, k[t]);
    Cut cut{0, 0, keep, 0};
    auto digit = [&](auto which) {
        constexpr int D = decltype(which)::value;
        for (uint32_t b = threadIdx.x; b < bins_of(D); b += kSmallThreads) s_hist[b] = 0;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            if (t * (int)(kSmallThreads * kEach) >= n) continue;
#pragma unroll
            for (uint32_t j = 0; j < kEach; ++j)
                hist_add(s_hist, digit_of<D>(k[t][j]), j < m[t] && has_digits<D>(k[t][j], cut));
        }
        __syncthreads();
        cut = next_digit<kSmallThreads, D, 1>(cut, s_hist, lds);
        __syncthreads();
    };
    digit(std::integral_constant<int, 0>());
    digit(std::integral_constant<int, 1>());
    digit(std::integral_constant<int, 2>());
    uint32_t before = 0, ties = 0;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        if (t * (int)(kSmallThreads * kEach) >= n) continue;
        uint32_t mine = 0, total;
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j)
            if (j < m[t]) mine += above_cut(k[t][j], cut) ? 1u : at_cut(k[t][j], cut) ? 0x10000u : 0u;
        uint32_t run = group_scan<kSmallThreads>(mine, lds, &total) + (ties << 16) + before;
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) {
            const bool up = j < m[t] && above_cut(k[t][j], cut), tie = j < m[t] && at_cut(k[t][j], cut);
            const uint32_t equals = run >> 16, kept = equals < cut.need ? equals : cut.need;
            if (up || (tie && equals < cut.need))
                source[(run & 0xFFFFu) + kept] = (t * (int)kSmallThreads + (int)threadIdx.x) * (int)kEach + (int)j;
            run += up ? 1u : tie ? 0x10000u : 0u;
        }
        before += total & 0xFFFFu;
        ties += total >> 16;
    }
}

__global__ __launch_bounds__(kBlock) void k_evict_rows(int64_t keep, gs_params in, const float *__restrict__ score,
                                                       const int32_t *__restrict__ source, gs_params out,
                                                       float *__restrict__ score_out) {
    const int64_t d = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (d < keep) keep_row(in, score, source[d], out, score_out, d);
}

// Copies. Counting the draws of a Gaussian touches only those drawn: their
// counts are cleared, then raised by integer atomics (any order gives the
// same), then every copy works out the shared weight from the logit that it
// took along; the copies of one Gaussian write the same number to it. Bound by
// the random lines that rows are read from: 419430 copies out of 2 M Gaussians
// read 314 MB for their 20 MB in 53 us, the shared weights take 18.
// Below one draw in so many Gaussians only the drawn ones' counts are cleared
// (2 M Gaussians: all of them 4 us, 419430 draws' one by one 10 us).
constexpr int64_t kClearAll = 16;

__global__ __launch_bounds__(kBlock) void k_split_fill(int64_t n, uint32_t *__restrict__ copies) {
    // the workspace is aligned and its size is a multiple of 256 bytes
    const int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * 4;
    if (i < n) *(uint4 *)(copies + i) = make_uint4(1u, 1u, 1u, 1u);
}

__global__ __launch_bounds__(kBlock) void k_split_clear(int64_t n, const int32_t *__restrict__ ids, int64_t count,
                                                        uint32_t *__restrict__ copies) {
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j >= count) return;
    const int64_t i = ids[j];
    if (i >= 0 && i < n) copies[i] = 1u;
}

// Row n + j, with the logit and the score that the Gaussian had, and its count.
__device__ __forceinline__ void split_row(const gs_params &set, int64_t n, const int32_t *ids, int64_t j,
                                          int32_t *source, float *score, uint32_t *copies) {
    const int64_t i = ids[j], d = n + j;
    Row r;
    float share = 0.0f;
    if (i >= 0 && i < n) {
        r = load_row(set, i);
        if (score) share = score[i];
        atomicAdd(&copies[i], 1u);
    } else {
        const float nan = __uint_as_float(0x7FC00000u);
        r.mean = f3a{nan, nan, nan};
        r.log_scale = f3a{0.0f, 0.0f, 0.0f};
        r.rot = f4a{1.0f, 0.0f, 0.0f, 0.0f};
        r.value = 0.0f;
        r.weight = -__builtin_inff();
    }
    store_row(set, d, r);
    if (score) score[d] = share;
    if (source) source[d] = i >= 0 ? (int32_t)(-1 - i) : -1;
}

// The shared weight of c copies: w / c with w = 1 / (1 + e^-l) is the logit -ln(c
// (1 + e^-l) - 1); far down, where e^-l is all of that, l - ln c.
__device__ __forceinline__ void split_weight(const gs_params &set, int64_t n, int64_t i, int64_t j, float *score,
                                             uint32_t copies) {
    const int64_t d = n + j;
    const double c = (double)copies, l = (double)set.weight_logit[d];
    const double shared = l < -30.0 ? l - log(c) : -log((c - 1.0) + c * exp(-l));
    set.weight_logit[d] = (float)shared;
    set.weight_logit[i] = (float)shared;
    if (score) {
        const float s = (float)((double)score[d] / c);
        score[d] = s;
        score[i] = s;
    }
}

__global__ __launch_bounds__(kBlock) void k_split_rows(gs_params set, int64_t n, const int32_t *__restrict__ ids,
                                                       int64_t count, int32_t *__restrict__ source, float *score,
                                                       uint32_t *__restrict__ copies) {
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j < count) split_row(set, n, ids, j, source, score, copies);
}

__global__ __launch_bounds__(kBlock) void k_split_weights(gs_params set, int64_t n, const int32_t *__restrict__ ids,
                                                          int64_t count, float *score,
                                                          const uint32_t *__restrict__ copies) {
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j >= count) return;
    const int64_t i = ids[j];
    if (i >= 0 && i < n) split_weight(set, n, i, j, score, copies[i]);
}

// Few copies: the three steps in one workgroup (819 copies: 14.9 us by three
// launches, the host's time). A thread takes the same copies in every step, so
// that only the counts pass between threads, by atomics.
constexpr int64_t kSplitSmall = 2048;
__global__ __launch_bounds__(kSmallThreads) void k_split_small(gs_params set, int64_t n, const int32_t *ids,
                                                               int count, int32_t *source, float *score,
                                                               uint32_t *copies) {
    auto own = [&](int j) { return ids[j] >= 0 && ids[j] < n; };
    for (int j = threadIdx.x; j < count; j += kSmallThreads)
        if (own(j)) __hip_atomic_store(&copies[ids[j]], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // (what each wave has sent is carried out)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int j = threadIdx.x; j < count; j += kSmallThreads) split_row(set, n, ids, j, source, score, copies);
    // (what each wave has sent is carried out)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int j = threadIdx.x; j < count; j += kSmallThreads)
        if (own(j))
            split_weight(set, n, ids[j], j, score,
                         __hip_atomic_load(&copies[ids[j]], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

struct EvictWork {
    uint32_t *hist;
    Cut *cuts;
    uint2 *sums;
    size_t bytes;
};
EvictWork evict_layout(void *base) {
    EvictWork w;
    char *b = (char *)base;
    w.hist = (uint32_t *)b;
    w.cuts = (Cut *)(b + sizeof(uint32_t) * kBinsAll * kCopies);
    const size_t head = al256(sizeof(uint32_t) * kBinsAll * kCopies + sizeof(Cut) * kDigits);
    w.sums = (uint2 *)(b + head);
    w.bytes = head + al256(sizeof(uint2) * kBlocksMost);
    return w;
}

dim3 blocks_of(int64_t n) { return dim3((uint32_t)((n + kBlock - 1) / kBlock)); }

}  // namespace

size_t evict_work_bytes(int64_t) { return evict_layout(nullptr).bytes; }

hipError_t launch_evict(const gs_params &in, int64_t n, const float *score, const uint8_t *pinned, int64_t keep,
                        const gs_params &out, int32_t *source, float *score_out, void *work, hipStream_t s) {
    if (keep <= 0) return hipSuccess;
    const EvictWork w = evict_layout(work);
    const dim3 tb(kBlock);
    const uint32_t k = (uint32_t)keep;
    if (n <= kSmall) {
        prof_begin("evict", s);
        hipLaunchKernelGGL(k_evict_small, dim3(1), dim3(kSmallThreads), 0, s, (int)n, score, pinned, k, source);
        hipLaunchKernelGGL(k_evict_rows, blocks_of(keep), tb, 0, s, keep, in, score, source, out, score_out);
        prof_end("evict", s);
        return hipGetLastError();
    }
    // a stretch of whole tiles for every workgroup
    const int64_t tiles = (n + kTile - 1) / kTile;
    const int64_t stretch = (tiles + kBlocksMost - 1) / kBlocksMost * kTile;
    const dim3 nb((uint32_t)((n + stretch - 1) / stretch));
    const int64_t ctiles = (n + kCountThreads * kEach - 1) / (kCountThreads * kEach);
    const int64_t cstretch = (ctiles + kCountBlocks - 1) / kCountBlocks * (kCountThreads * kEach);
    const dim3 cb((uint32_t)((n + cstretch - 1) / cstretch)), ct(kCountThreads);
    hipError_t e;
    prof_begin("evict_select", s);
    if ((e = fill_u32(w.hist, 0u, kBinsAll * kCopies, s)) != hipSuccess) return e;
    hipLaunchKernelGGL(k_evict_count<0>, cb, ct, 0, s, n, cstretch, score, pinned, k, w.hist, w.cuts);
    hipLaunchKernelGGL(k_evict_count<1>, cb, ct, 0, s, n, cstretch, score, pinned, k, w.hist, w.cuts);
    hipLaunchKernelGGL(k_evict_count<2>, cb, ct, 0, s, n, cstretch, score, pinned, k, w.hist, w.cuts);
    hipLaunchKernelGGL(k_evict_stretch, nb, tb, 0, s, n, stretch, score, pinned, k, w.hist, w.cuts, w.sums);
    prof_end("evict_select", s);
    prof_begin("evict_rows", s);
    hipLaunchKernelGGL(k_evict_keep, nb, tb, 0, s, n, stretch, score, pinned, w.cuts, w.sums, in, out, source,
                       score_out);
    prof_end("evict_rows", s);
    return hipGetLastError();
}

hipError_t launch_split(const gs_params &set, int64_t n, const int32_t *ids, int64_t count, int32_t *source,
                        float *score, uint32_t *copies, hipStream_t s) {
    if (count <= 0) return hipSuccess;
    const dim3 nb = blocks_of(count), tb(kBlock);
    prof_begin("split", s);
    if (count <= kSplitSmall) {
        hipLaunchKernelGGL(k_split_small, dim3(1), dim3(kSmallThreads), 0, s, set, n, ids, (int)count, source, score,
                           copies);
        prof_end("split", s);
        return hipGetLastError();
    }
    if (n > 0 && count >= n / kClearAll) {
        hipLaunchKernelGGL(k_split_fill, blocks_of((n + 3) / 4), tb, 0, s, n, copies);
    } else {
        hipLaunchKernelGGL(k_split_clear, nb, tb, 0, s, n, ids, count, copies);
    }
    hipLaunchKernelGGL(k_split_rows, nb, tb, 0, s, set, n, ids, count, source, score, copies);
    hipLaunchKernelGGL(k_split_weights, nb, tb, 0, s, set, n, ids, count, score, copies);
    prof_end("split", s);
    return hipGetLastError();
}

}  // namespace gs
